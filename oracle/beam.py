"""Beam search over the oracle's target, every hypothesis from scratch (no cache is kept)."""
import numpy as np

from .operators import beam_select


def last_logits(target, xkv, tokens, suppress=None):
    left_out = None if suppress is None else np.nonzero(suppress)[0]
    logits, _ = target.forward(target.new_cache(), np.asarray(tokens, np.int64), 0, xkv, left_out)
    return np.asarray(logits[-1], np.float64)


def beam_search(target, xkv, prompt, max_new, beams, length_penalty=1.0, suppress=None):
    """Hypotheses [(tokens, score)], best first by score / len^length_penalty, `beams` at most.

    Each step scores every continuation of every beam; the 2 * beams best are taken in order:
    those that end with the end-of-transcript token finish (up to `beams` of them), the others go
    on, until there are `beams` of these.  Scores are held in 32 bits between steps.  suppress: mask [n_vocab].
    """
    cfg = target.cfg
    prompt = [int(t) for t in prompt]
    live, finished, steps = [([], np.float32(0))], [], 0
    while True:
        rows = np.stack([last_logits(target, xkv, prompt + path, suppress) for path, _ in live])[None]
        got = beam_select(rows, np.array([[s for _, s in live]]), 2 * beams)
        nxt = []
        for score, b, tok in zip(*(x[0] for x in got)):
            if b < 0 or len(nxt) == beams:
                break
            hyp = (live[b][0] + [int(tok)], np.float32(score))
            if tok == cfg.eos_id:
                if len(finished) < beams:
                    finished.append(hyp)
            else:
                nxt.append(hyp)
        live = nxt
        steps += 1
        if len(finished) >= beams or not live or steps >= max_new or len(prompt) - 1 + steps >= cfg.n_ctx:
            break
    hyps = (finished + live)[:beams]
    return sorted(hyps, key=lambda h: -(float(h[1]) / len(h[0]) ** length_penalty))

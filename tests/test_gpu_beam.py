"""Beam search on a handle against the oracle's, which recomputes every hypothesis from scratch."""
import numpy as np
import pytest
import torch

from oracle import OracleOpts, Target
from oracle.beam import beam_search
from wf_fixtures import LARGE_V3, MICRO, full_manifest, make_memory, make_prefix, make_weights
from paper_2609_32869_amd import WfError, WhisperFlash, to_device_storage

pytestmark = pytest.mark.gpu
BF16 = MICRO.with_(name="micro-beam-bf16", dtype="bf16", n_vocab=501, n_frames=45)


def engine(cfg, batch, bits=16):
    W = make_weights(cfg)
    return W, WhisperFlash.from_host(cfg, batch, [W.values[n] for n, _ in W.order], acoustic_bits=bits)


def target(cfg, W):
    return Target(cfg, W.values, OracleOpts(dtype=np.float32, kv_bf16=cfg.dtype == "bf16", exact=cfg.dtype != "bf16"))


def prompts(cfg, lens, first=0):
    rows = [make_prefix(cfg, first + i, n) for i, n in enumerate(lens)]
    toks = np.zeros((len(lens), max(lens)), np.int32)
    for i, p in enumerate(rows):
        toks[i, :len(p)] = p
    return rows, torch.from_numpy(toks).cuda()


def set_memory(eng, cfg, slot0, n):
    eng.encode_memory_set(slot0, torch.stack([to_device_storage(make_memory(cfg, slot0 + i), cfg.dtype) for i in range(n)]))


def hypotheses(out):
    tokens, lens, scores = (t.cpu().numpy() for t in out)
    return [[(list(tokens[r, b, :lens[r, b]]), scores[r, b]) for b in range(lens.shape[1]) if lens[r, b] > 0]
            for r in range(lens.shape[0])]


def check(got, want, tol):
    """The same hypotheses in the same order; two whose scores the logits' tolerance does not tell apart may change
    places, but none does here."""
    assert [h[0] for h in got] == [h[0] for h in want]
    for g, w in zip(got, want):
        assert abs(g[1] - w[1]) <= tol * len(w[0])


# fp32 logits agree to 1e-4 (the parity tests' micro runs: under 1e-5), a token's log-probability to twice that
F32_TOL, BF16_TOL = 2e-4, 2e-2


@pytest.mark.parametrize("beams,lens,max_new", [(1, [5], 8), (3, [11, 16], 12), (5, [17, 3, 30], 20), (16, [9], 6), (4, [1], 20), (11, [12, 7, 20], 10)])
def test_beam_search_matches_the_oracle(beams, lens, max_new):
    cfg = MICRO
    W, eng = engine(cfg, beams * len(lens))
    T = target(cfg, W)
    rows, toks = prompts(cfg, lens)
    set_memory(eng, cfg, 0, len(lens))
    got = hypotheses(eng.beam_search(0, toks, lens, [max_new] * len(lens), beams))
    for r, p in enumerate(rows):
        check(got[r], beam_search(T, T.cross_kv(make_memory(cfg, r)), p, max_new, beams), F32_TOL)
    assert eng.status() == 0
    eng.close()


@pytest.mark.parametrize("penalty", [0.0, 1.0, 2.0])
def test_finished_hypotheses(penalty):
    """A vocabulary of six tokens and the end of transcript: hypotheses finish early, at different steps, and rank by
    the length penalty."""
    cfg, beams, lens = MICRO, 4, [6, 15]
    W, eng = engine(cfg, 8)
    T = target(cfg, W)
    sup = np.ones(cfg.n_vocab, np.uint8)
    sup[[cfg.eos_id, 3, 50, 51, 200, 400, 511]] = 0
    rows, toks = prompts(cfg, lens)
    set_memory(eng, cfg, 0, 2)
    dsup = torch.from_numpy(sup).cuda()
    eng.set_sampling(0.0, suppress=dsup)
    got = hypotheses(eng.beam_search(0, toks, lens, [10, 30], beams, penalty, poll=1))
    for r, p in enumerate(rows):
        want = beam_search(T, T.cross_kv(make_memory(cfg, r)), p, [10, 30][r], beams, penalty, suppress=sup)
        check(got[r], want, F32_TOL)
    assert sum(h[0][-1] == cfg.eos_id for h in want) == 3   # the second request's: at 13, 23 and 28 tokens
    eng.close()


def test_fewer_continuations_than_beams():
    """Three tokens allowed: the first choice fills three of eight beams, the others stay empty until there are more."""
    cfg, beams = MICRO, 8
    W, eng = engine(cfg, 8)
    T = target(cfg, W)
    sup = np.ones(cfg.n_vocab, np.uint8)
    sup[[9, 10, 11]] = 0
    rows, toks = prompts(cfg, [13])
    set_memory(eng, cfg, 0, 1)
    dsup = torch.from_numpy(sup).cuda()
    eng.set_sampling(0.0, suppress=dsup)
    for max_new in (1, 2, 9):
        got = hypotheses(eng.beam_search(0, toks, [13], [max_new], beams))
        check(got[0], beam_search(T, T.cross_kv(make_memory(cfg, 0)), rows[0], max_new, beams, suppress=sup), F32_TOL)
    eng.close()


def test_context_end():
    """Searches that fill the context: the last position is read, the token after it ends the hypothesis."""
    cfg, beams, lens = MICRO, 3, [60, 64]
    W, eng = engine(cfg, 6)
    T = target(cfg, W)
    rows, toks = prompts(cfg, lens)
    set_memory(eng, cfg, 0, 2)
    got = hypotheses(eng.beam_search(0, toks, lens, [50, 50], beams))
    for r, p in enumerate(rows):
        check(got[r], beam_search(T, T.cross_kv(make_memory(cfg, r)), p, 50, beams), F32_TOL)
        assert len(got[r][0][0]) == cfg.n_ctx - lens[r] + 1
    assert eng.status() == 0
    eng.close()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("beams,n", [(5, 1), (3, 4), (9, 2), (10, 2), (16, 3)])
def test_bf16_storage(beams, n, bits):
    """bf16 caches (above nine beams a request's rows are those of two slots on one memory); with the acoustic keys and
    values in 4 bits the first request's hypotheses are read again token by token, as a plain slot's."""
    cfg = BF16
    W, eng = engine(cfg, beams * n, bits)
    lens = [4 + 13 * i for i in range(n)]
    rows, toks = prompts(cfg, lens)
    set_memory(eng, cfg, 0, n)
    out = eng.beam_search(0, toks, lens, [14] * n, beams)
    got = hypotheses(out)
    if bits == 16:
        T = target(cfg, W)
        for r, p in enumerate(rows):
            want = beam_search(T, T.cross_kv(make_memory(cfg, r)), p, 14, beams)
            check(got[r], want, BF16_TOL)
    else:
        eng.set_debug(True)
        for path, score in got[0]:
            seq = np.concatenate([rows[0], np.asarray(path, np.int32)])[None].astype(np.int32)
            total = 0.0
            for i in range(len(path)):
                m = lens[0] + i
                eng.prefill(0, torch.from_numpy(seq[:, :m - 1].copy()).cuda(), [m - 1], [60])
                st = eng.state()
                st[0, 0], st[0, 1] = m - 1, int(seq[0, m - 1])       # the anchor is the hypothesis's own token
                eng.verify_accept(0, torch.zeros((1, 8), dtype=torch.int32, device="cuda"), 0)
                total += float(torch.log_softmax(eng.target_logits()[0, 0].double(), 0)[path[i]])
            # the caches' bf16 rounding of keys and values from other passes moves a log-probability by 1e-3 at most
            assert abs(total - score) <= 2e-3 * len(path)
    assert eng.status() == 0
    eng.close()


@pytest.mark.parametrize("bits", [16, 4])
def test_a_search_after_a_broken_memory(bits):
    """A recording of non-finite features leaves non-finite activation rows behind; once its cache pages hold other
    prompts, a search on the same slots sets no status bit (rows that no beam uses are made anew, not left as they were)."""
    cfg = BF16
    W, eng = engine(cfg, 6, bits)
    rows, toks = prompts(cfg, [8, 8])
    eng.encode_memory_set(0, torch.full((6, cfg.n_frames, cfg.d_model), float("nan"), dtype=torch.bfloat16, device="cuda"))
    eng.prefill(0, toks[:1].expand(6, 8).contiguous(), [8] * 6, [9] * 6)
    eng.step(0, 6)
    assert eng.status() != 0
    set_memory(eng, cfg, 0, 6)
    eng.prefill(0, torch.full((6, cfg.n_ctx), 9, dtype=torch.int32, device="cuda"), [cfg.n_ctx] * 6, [9] * 6)
    eng.status()
    eng.prefill(0, toks, [8, 8], [5, 5])
    assert eng.status() == 0
    eng.beam_begin(0, 3, toks[:, 7].contiguous(), [5, 5])
    for _ in range(5):
        eng.beam_step(0)
    assert eng.status() == 0
    assert eng.beam_end(0)[2].isfinite().all()
    eng.close()


@pytest.mark.parametrize("bits", [16, 4])
def test_large_v3_scores_are_the_hypotheses_own(bits):
    """Large-v3 shapes, three recordings of five beams on 15 slots (page borders crossed, pages shared and copied): each
    hypothesis's score is the sum of its tokens' log-probabilities in one plain verification pass over it.  The passes'
    products sum in other orders and the fused adds vary: a logit moves by 1e-3 (the step's parity tests), a
    log-probability by 2e-3, nine of them by 2e-2."""
    cfg, B, lens = LARGE_V3.with_(eos_id=-1), 5, [30, 41, 16]
    g = torch.Generator("cuda").manual_seed(11)
    weights = []
    for name, shape in full_manifest(cfg):
        w = (0.02 * torch.randn(shape, device="cuda", generator=g)).bfloat16()
        weights.append(w + 1 if name.endswith(".g") else w)
    weights[0] *= 4          # a livelier vocabulary: paths differ, and differ in score
    eng = WhisperFlash(cfg, 15, weights, acoustic_bits=bits)
    eng.encode_memory_set(0, torch.randn((3, cfg.n_frames, cfg.d_model), device="cuda", generator=g).bfloat16())
    toks = torch.randint(0, cfg.n_vocab, (3, 41), dtype=torch.int32, device="cuda", generator=g)
    out, n_tok, scores = eng.beam_search(0, toks, lens, [9] * 3, B)
    assert (n_tok == 9).all() and (scores[:, :-1] >= scores[:, 1:]).all()
    assert len({tuple(p) for p in out[0, :, :9].tolist()}) == B
    eng.set_debug(True)
    for r in range(3):
        for b in range(B):
            eng.prefill(r, toks[r:r + 1, :lens[r] - 1].contiguous(), [lens[r] - 1], [60])
            st = eng.state()
            st[r, 1] = toks[r, lens[r] - 1]     # the anchor is the prompt's own last token
            eng.verify_accept(r, out[r:r + 1, b, :8].contiguous())
            logp = torch.log_softmax(eng.target_logits()[r].double(), -1)
            total = logp.gather(1, out[r, b, :9, None].long()).sum()
            assert abs(float(total - scores[r, b])) <= 2e-2, (r, b)
    assert eng.status() == 0
    eng.close()


def test_one_beam_is_greedy_decoding():
    """One beam without a length choice follows plain greedy decoding, on every path a single slot takes."""
    for cfg, bits in ((MICRO, 16), (BF16, 16), (BF16, 4)):
        W, eng = engine(cfg, 1, bits)
        rows, toks = prompts(cfg, [20])
        set_memory(eng, cfg, 0, 1)
        plain = [int(eng.prefill(0, toks, [20], [13])[0])]
        while len(plain) < 13 and plain[-1] != cfg.eos_id:
            out, n_out, _, _ = eng.step(0, 1, 0)
            plain += out[0, :int(n_out[0])].tolist()
        got = hypotheses(eng.beam_search(0, toks, [20], [13], 1))
        assert got[0][0][0] == plain
        # and the slot decodes as before once the search has given it back
        again = [int(eng.prefill(0, toks, [20], [13])[0])]
        while len(again) < 13 and again[-1] != cfg.eos_id:
            out, n_out, _, _ = eng.step(0, 1, 0)
            again += out[0, :int(n_out[0])].tolist()
        assert again == plain
        eng.close()


@pytest.mark.parametrize("cfg", [MICRO, BF16], ids=["f32", "bf16"])
def test_searches_beside_each_other_and_graphs(cfg):
    """Two searches and a plainly decoded slot on one handle, steps interleaved, graphs and eager: what each gives
    alone; twice, so that graphs are replayed over other memory contents and captured anew for a new search."""
    W, eng = engine(cfg, 11)
    rows, toks = prompts(cfg, [7, 21, 12, 9])
    set_memory(eng, cfg, 0, 11)
    alone = []
    for s0, n, B, first in ((0, 2, 3, 0), (6, 1, 4, 2)):
        alone.append(hypotheses(eng.beam_search(s0, toks[first:first + n].contiguous(), [7, 21, 12, 9][first:first + n], [15] * n, B)))
    eng.prefill(10, toks[3:4, :9].contiguous(), [9], [16])
    plain = []
    for _ in range(15):
        out, n_out, _, _ = eng.step(10, 1, 0)
        plain += out[0, :int(n_out[0])].tolist()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for graph in (False, True, True):
        with torch.cuda.stream(stream):
            eng.prefill(0, toks[:2].contiguous(), [7, 21], [1, 1])
            eng.prefill(6, toks[2:3].contiguous(), [12], [1])
            eng.prefill(10, toks[3:4, :9].contiguous(), [9], [16])
            eng.beam_begin(0, 3, torch.stack([toks[0, 6], toks[1, 20]]), [15, 15])
            eng.beam_begin(6, 4, toks[2, 11:12].contiguous(), [15])
            done = torch.zeros(2, dtype=torch.int32, device="cuda")
            outs, decoded = eng._outs(1), []
            for step in range(15):
                eng.beam_step(0, done, graph)
                eng.step(10, 1, 0, outs=outs, use_graph=graph)
                eng.beam_step(6, None, graph)
                decoded += outs[0][0, :int(outs[1][0])].tolist()
            assert bool(done.all())
            for s0, want in ((6, alone[1]), (0, alone[0])):
                got = hypotheses(eng.beam_end(s0))
                for g, w in zip(got, want):
                    check(g, w, F32_TOL if cfg.dtype == "f32" else BF16_TOL)
            assert decoded == plain
    eng.close()


def test_on_a_given_stream_and_after_a_refused_step():
    cfg = MICRO
    W, eng = engine(cfg, 4)
    rows, toks = prompts(cfg, [10])
    set_memory(eng, cfg, 0, 1)
    whole = eng.beam_search(0, toks, [10], [9], 4)
    last = toks[0, 9:10].contiguous()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        eng.prefill(0, toks, [10], [1])
        torch.cuda.synchronize()
        eng.beam_begin(0, 4, last, [9], stream=stream)
        for _ in range(9):
            eng.beam_step(0, use_graph=True, stream=stream)
        got = eng.beam_end(0, stream=stream)
        stream.synchronize()
        for a, b in zip(got, whole):
            assert torch.equal(a, b)
    with pytest.raises(WfError, match="non-null stream"):       # no graph on the default stream: the slots come back
        eng.beam_search(0, toks, [10], [9], 4, use_graph=True)
    assert eng.searches == {}
    for a, b in zip(eng.beam_search(0, toks, [10], [9], 4), whole):
        assert torch.equal(a, b)
    for wrong in (last.long(), toks[:, :1], toks[0, ::2], last.cpu()):
        with pytest.raises(WfError, match="last_tokens"):
            eng.beam_begin(0, 2, wrong, [9])
    eng.close()


def test_results_cut_and_ended_early():
    cfg = MICRO
    W, eng = engine(cfg, 4)
    rows, toks = prompts(cfg, [10])
    set_memory(eng, cfg, 0, 1)
    whole = eng.beam_search(0, toks, [10], [9], 4)
    eng.prefill(0, toks, [10], [1])
    eng.beam_begin(0, 4, toks[0, 9:10].contiguous(), [9])
    none = eng.beam_end(0)
    assert (none[1] == 0).all() and (none[0] == -1).all() and none[2].isneginf().all()   # ended before a step
    eng.prefill(0, toks, [10], [1])
    eng.beam_begin(0, 4, toks[0, 9:10].contiguous(), [9])
    for _ in range(12):      # steps past the end change nothing
        eng.beam_step(0)
    cut = eng.beam_end(0, len_max=4)
    assert torch.equal(cut[0], whole[0][:, :, :4]) and torch.equal(cut[1], whole[1]) and torch.equal(cut[2], whole[2])
    eng.close()


def test_refusals():
    cfg = MICRO
    W, eng = engine(cfg, 6)
    rows, toks = prompts(cfg, [10, 5])
    last = torch.zeros(2, dtype=torch.int32, device="cuda")

    def refused(f, code):
        with pytest.raises(WfError, match=rf"\({code}\)"):
            f()
    refused(lambda: eng.beam_begin(0, 2, last, [5, 5]), -2)          # no prompt yet
    set_memory(eng, cfg, 0, 2)
    eng.prefill(0, toks, [10, 5], [3, 3])
    refused(lambda: eng.beam_begin(0, 4, last, [5, 5]), -1)          # eight slots of six
    refused(lambda: eng.beam_begin(0, 0, last, [5, 5]), -1)
    refused(lambda: eng.beam_begin(-1, 2, last, [5, 5]), -1)
    refused(lambda: eng.beam_begin(3, 2, last, [5, 5]), -1)
    refused(lambda: eng.beam_begin(0, 2, last, [5, 0]), -1)
    refused(lambda: eng.beam_begin(0, 2, last, [5, 5], float("nan")), -1)
    refused(lambda: eng.beam_step(0), -2)
    refused(lambda: eng.beam_end(0), -2)
    eng.set_sampling(0.7)
    refused(lambda: eng.beam_begin(0, 2, last, [5, 5]), -2)
    eng.set_sampling(0.0)
    eng.beam_begin(0, 2, last, [5, 5])
    refused(lambda: eng.beam_begin(1, 2, last, [5, 5]), -2)
    for f in (lambda: eng.prefill(1, toks[1:2], [5], [3]), lambda: eng.step(0, 1), lambda: eng.draft(3, 1),
              lambda: set_memory(eng, cfg, 1, 1), lambda: eng.step_noalloc(0, 6)):
        refused(f, -2)
    refused(lambda: eng.beam_step(1), -2)
    eng.set_sampling(0.7)
    refused(lambda: eng.beam_step(0), -2)
    eng.set_sampling(0.0)
    s = torch.cuda.current_stream()
    if s.cuda_stream == 0:
        refused(lambda: eng.beam_step(0, use_graph=True), -1)        # graphs need a stream
    eng.beam_step(0)
    eng.beam_end(0)
    refused(lambda: eng.step(0, 1), -2)                              # empty again
    eng.prefill(0, toks, [10, 5], [3, 3])
    eng.step(0, 2)
    eng.close()

"""fp32 attention over packed prompts and the 8-bit cache: every bf16 term of its operands and every product of them that is
kept counts (selfattn_terms: a lost one is off by more than twice the bounds)."""
import numpy as np
import pytest
import torch

import selfattn_terms as st
from test_gpu_selfattn import i32, lib, num, random_tables

pytestmark = pytest.mark.gpu

# rows, heads, sequences at most, rows of a sequence: 32-row blocks, 128-row blocks of one and of two groups of waves.  Of a
# sequence the first and the last key count: the same tile, or the last row's own and an earlier one.
KINDS = [(600, 2, 300, 2), (600, 2, 12, 50), (8192, 4, 4096, 2), (8192, 4, 163, 50), (12000, 3, 40, 2), (12000, 3, 40, 50)]


def layout(T, most, length):
    """Borders: `most` sequences of `length` rows, and one of the rest."""
    n = min(most, T // length)
    return n, [length * i for i in range(n + 1)] + ([T] if n * length < T else [])


def placed(T, H, n, length, first, last, between):
    """[T, H, 64] of n sequences' first and last rows [n * H, 64] and what lies between; zeros in the rest."""
    x = np.zeros((T, H, 64), np.float32)
    y = x[:n * length].reshape(n, length, H, 64)
    y[:, 1:-1] = between.reshape(n, 1, H, 64)
    y[:, 0], y[:, -1] = first.reshape(n, H, 64), last.reshape(n, H, 64)
    return torch.from_numpy(x).cuda()


def last_rows(got, n, length):
    return num(got[:n * length].view(n, length, -1, 64)[:, -1]).reshape(-1, 64)


def keeps(got, want, bound):
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()


@pytest.mark.parametrize("T,H,most,length", KINDS)
def test_prompt_scores_in_three_terms(T, H, most, length):
    rng = np.random.default_rng(T + length)
    n, starts = layout(T, most, length)
    q, k = st.score_case(rng, n * H)
    ones = np.ones((n * H, 64))
    # keys between: their scores lie 120 and more below, a weight of 0 in 32 bits and of e^-120 in 64
    args = (placed(T, H, n, length, q, q, q), placed(T, H, n, length, k[:, 0], k[:, 1], -16 * q), placed(T, H, n, length, ones, -ones, ones))
    got = last_rows(lib().prompt_attention(*args, i32(starts)), n, length)
    keeps(got, st.score_result(q, k)[:, None], st.score_bound(q, k)[:, None])


@pytest.mark.parametrize("T,H,most,length", KINDS)
def test_prompt_values_in_three_terms(T, H, most, length):
    rng = np.random.default_rng(T + length + 1)
    n, starts = layout(T, most, length)
    d, v = st.value_case(rng, n * H)
    one = np.zeros((n * H, 64))
    one[:, 0] = 1
    args = (placed(T, H, n, length, 8 * one, 8 * one, 8 * one), placed(T, H, n, length, 0 * one, d[:, None] * one, -200 * one),
            placed(T, H, n, length, v[:, 0], v[:, 1], v[:, 0]))
    got = last_rows(lib().prompt_attention(*args, i32(starts)), n, length)
    keeps(got, st.value_result(d, v), st.value_bound(d, v))


@pytest.mark.parametrize("n,width,length", [(300, 1, 2), (40, 4, 50), (40, 70, 50), (5, 28, 440), (5, 200, 3000)])
def test_attend8_scores_in_three_terms(n, width, length):
    """One, four and eight waves a block, chunks; keys of one term, exact in 8 bits beside +-16."""
    rng = np.random.default_rng(n + length)
    H = 4
    q, k = st.score_case(rng, n * H, exact_keys=True)
    ones = np.ones((n * H, 64))
    keys, values = (placed(n * length, H, n, length, *x).view(n, length, H, 64)
                    for x in ((k[:, 0], k[:, 1], -16 * np.sign(q)), (ones, -ones, ones)))
    cache, tables = lib().PagedCache8(n * width, H), i32(random_tables(rng, n, width, n * width))
    cache.store(keys, values, tables, i32([0] * n))
    query = torch.from_numpy(q).float().cuda().view(n, 1, H, 64)
    got = num(cache.attend(query, tables, i32([length - 1] * n))).reshape(-1, 64)
    keeps(got, st.score_result(q, k)[:, None], st.score_bound(q, k)[:, None])

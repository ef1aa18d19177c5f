"""The bounds of selfattn_terms: the products in three terms keep them, a lost term or product does not."""
import numpy as np
import pytest

import selfattn_terms as st


def test_terms():
    rng = np.random.default_rng(0)
    for x in (st.operands(rng, 1000), rng.standard_normal(1000).astype(np.float32)):
        t = st.terms(x)
        assert np.array_equal(sum(t), x)
        for part in t:                                       # eight bits each
            m, _ = np.frexp(part)
            assert np.array_equal(np.ldexp(m, 8), np.rint(np.ldexp(m, 8)))
    a = st.operands(rng, 1000)
    h, m, l = st.terms(a)
    assert (np.abs(h) == 1).all() and set(np.abs(m)) == {0, 2.0 ** -8} and set(np.abs(l)) == {0, 2.0 ** -16}


def test_sums_are_exact_in_32_bits():
    """In any order, and from a reference on."""
    rng = np.random.default_rng(1)
    q, k = st.score_case(rng, 300)
    parts = np.concatenate([s * t for i, s in enumerate(st.terms(q[:, None])) for j, t in enumerate(st.terms(k)) if (i, j) in st.KEPT], -1)
    whole = parts.sum(-1)
    for _ in range(5):
        order = rng.permutation(parts.shape[-1])
        for start in (0, -whole[:, :1].astype(np.float32)):
            x = np.zeros(whole.shape, np.float32) + start
            for i in order:
                x = (x + parts[..., i].astype(np.float32)).astype(np.float32)
            assert np.array_equal(x, whole + start)
    assert np.array_equal(st.product(q[:, None], k), whole)


def worst(got, want, bound):
    return (np.abs(got - want) / bound).max()


@pytest.mark.parametrize("pairs", [120, 4000])
def test_score_bound(pairs):
    rng = np.random.default_rng(pairs)
    q, k = st.score_case(rng, pairs)
    want, bound = st.score_result(q, k), st.score_bound(q, k)
    assert worst(st.score_result(q, k, st.product(q[:, None], k)), want, bound) <= 1
    for lost in [dict(n=(2, 3)), dict(n=(3, 2)), dict(n=(2, 2))] + [dict(kept=[x for x in st.KEPT if x != gone]) for gone in st.KEPT]:
        assert worst(st.score_result(q, k, st.product(q[:, None], k, **lost)), want, bound) > 2, lost
    q, k = st.score_case(rng, pairs, exact_keys=True)
    want, bound = st.score_result(q, k), st.score_bound(q, k)
    assert worst(st.score_result(q, k, st.product(q[:, None], k, n=(2, 1))), want, bound) > 2


@pytest.mark.parametrize("pairs", [40, 1000])
def test_value_bound(pairs):
    rng = np.random.default_rng(pairs)
    d, v = st.value_case(rng, pairs)
    want, bound = st.value_result(d, v), st.value_bound(d, v)
    assert worst(st.value_result(d, v, list(st.KEPT)), want, bound) <= 1
    for lost in [dict(n=(2, 3)), dict(n=(3, 2)), dict(n=(2, 2))] + [dict(kept=[x for x in st.KEPT if x != gone]) for gone in st.KEPT]:
        assert worst(st.value_result(d, v, **lost), want, bound) > 2, lost

"""Attention from trees of more than 16 query rows per KV head holds its weights to the 11 bits of f16."""
import numpy as np
import pytest
import torch

from oracle import pace_oracle as O
from test_gpu_kv import Pool, _cu, _f64, _tokens, pace  # noqa: F401
from test_gpu_kv_tree import _ids, tree


def bound(r, see, D):
    """How far the output may be from the oracle's r.

    A weight is off by 2^-11 of itself (f16, half a step) or 2^-24 of the row's largest, and by the error of its score: a sum of D products in
    fp32, off by at most 2^-23 (D + 8) times the sum of their sizes, and 2^-20 for the exponential; the sum that it is divided by carries the
    latter once more.  The sums over n slots are off by n + 8 roundings of 2^-23.  What results is rounded once to bf16: 2^-8 of it."""
    n = see.sum(axis=1)[:, None, None]
    score = (2.0 ** -23 * (D + 8) * r["abs_score"] + 2.0 ** -20)[..., None]
    off = (2.0 ** -11 + 2 * score + 2.0 ** -23 * (n + 8)) * r["abs_out"] + 2.0 ** -24 * np.sqrt(n) * r["peak"][..., None]
    return off + 2.0 ** -8 * (np.abs(r["out"]) + off)


def _rounded(x, bits):
    """To so many significant bits, ties to even."""
    m, e = np.frexp(x)
    return np.ldexp(np.round(np.ldexp(m, bits)), e - bits)


@pytest.mark.parametrize("context,n,shape", [(3, 64, "fours"), (300, 40, "random"), (1500, 17, "forest")])
@pytest.mark.parametrize("dim", [64, 128])
def test_the_bound_tells_8_bits_from_11(context, n, shape, dim):
    rng = np.random.default_rng(context)
    Q, (K, V) = rng.normal(size=(n, 4, dim)), rng.normal(size=(2, context + n, 2, dim))
    see = O.kv_tree_visible(context + n, tree(shape, n))
    r = O.kv_attention_dense(Q, K, V, see, dim ** -0.5)
    far = {}
    for bits in (8, 11):
        got = np.zeros_like(r["out"])
        for h in range(4):
            s = np.where(see, Q[:, h] @ K[:, h // 2].T * dim ** -0.5, -np.inf)
            w = np.exp(s - s.max(axis=1)[:, None])
            got[:, h] = _rounded(w, bits) @ V[:, h // 2] / w.sum(axis=1)[:, None]
        got = torch.from_numpy(got).to(torch.bfloat16).double().numpy()
        far[bits] = (np.abs(got - r["out"]) / bound(r, see, dim)).max()
    assert far[11] <= 1.0
    if context == 3:      # (of the errors of many slots most cancel)
        assert far[8] > 1.0


@pytest.mark.gpu
# short contexts, where a weight counts; more than a row tile; a few-row tree among others; 24 trees on long contexts, shared by the halves of a CTA
@pytest.mark.parametrize("lens,nodes,which", [((67,), (64,), (0,)), ((20,), (20,), (0,)), ((340, 130), (40, 100), (0, 1)), ((603,), (600,), (0,)),
                                              ((5, 70, 9), (2, 64, 1), (0, 1, 2)),
                                              ([1250 + 61 * (i % 9) for i in range(24)], [40 + i % 5 for i in range(24)], (0, 7, 23))])
@pytest.mark.parametrize("shape", ["fours", "forest"])
@pytest.mark.parametrize("hq,hkv,dim", [(16, 8, 128), (8, 8, 64), (14, 2, 64)])
def test_weights(pace, lens, nodes, which, shape, hq, hkv, dim):  # noqa: F811
    pool = Pool(pace, 130, list(lens), hkv, dim, 16)
    parents = [tree(shape, n, b) for b, n in enumerate(nodes)]
    cu, Q = _cu(nodes), _tokens(131, sum(nodes), hq, dim)
    out = pace.pace_kv_tree_attention(pool.cache, Q, cu, _ids(sum(parents, [])), pool.lens, pool.table, max(lens))
    for b in which:
        k, v = pool.read("k", b), pool.read("v", b)
        see = O.kv_tree_visible(lens[b], parents[b])
        r = O.kv_attention_dense(_f64(Q[cu[b]:cu[b + 1]]), k, v, see, dim ** -0.5)
        off = np.abs(_f64(out[cu[b]:cu[b + 1]]) - r["out"]) / bound(r, see, dim)
        assert off.max() <= 1.0, (b, float(off.max()))

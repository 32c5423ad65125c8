"""Norm and rotation of queries and keys against their formulas in 64 bits.

Bound of an element: half a step of its type, and in fp32 the norm's and the weight's products (relative, 8 steps of 2^-24 with
the sum of squares over 128 dims in a tree of 8 + 4 additions and a root), cosine and sine (2 steps each) and the
rotation's two products and sum, all relative to |a| + |b| of the pair."""
import numpy as np
import pytest
import torch

import mts_workloads as W
import paper_2604_22881_amd as mts
import q8_reference as R
from paper_2604_22881_amd import binding as B
from paper_2604_22881_amd.runtime import DeviceBatch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPE = {"f32": (B.MTS_F32, torch.float32), "bf16": (B.MTS_BF16, torch.bfloat16)}


def draw(rng, shape, dtype):
    x = (rng.standard_normal(shape) * 2.0 ** rng.standard_normal(shape[:-1] + (1,))).astype(np.float32)
    return x if dtype == "f32" else W.bf16_bits_to_f32(W.f32_to_bf16_bits(x))


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV).to(TYPE[dtype][1])


def bound(ref, rot, pairs, dtype):
    y = np.abs(ref).copy()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = y[..., b] = np.abs(ref[..., a]) + np.abs(ref[..., b])
    # |a| + |b| of the rotated pair is at least that of the pair it came from over sqrt 2
    return (0.0 if dtype == "f32" else 2.0 ** -8) * np.abs(ref) + 1.5 * 32 * 2.0 ** -24 * y + 1e-37


def run(seed, dtype, Hq, Hk, D, rot, pairs, prefix, new, norm=True, weights=True, packed=False, in_place=False, eps=1e-6, freqs=None):
    rng = np.random.default_rng(seed)
    prefix, new = np.asarray(prefix), np.asarray(new)
    n = int(new.sum())
    freqs = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1)) if freqs is None else freqs
    indptr = np.concatenate([[0], np.cumsum(new)])
    batch = DeviceBatch(np.zeros(len(new) + 1), np.zeros(1), prefix, indptr, DEV)
    qkv = draw(rng, (n, Hq + 2 * Hk, D), dtype)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    w = [draw(rng, (D,), dtype) if weights else None for _ in range(2)]
    wd = [dev(x, dtype) if weights else None for x in w]
    f = torch.from_numpy(np.asarray(freqs, np.float64)).to(DEV)
    stride = (Hq + 2 * Hk) * D if packed else 0
    desc = mts.QkDesc(TYPE[dtype][0], Hq, Hk, D, stride, stride, stride if in_place else 0, stride if in_place else 0,
                      wd[0].data_ptr() if weights else 0, wd[1].data_ptr() if weights else 0, B.MTS_NORM_RMS if norm else B.MTS_NORM_NONE,
                      eps, f.data_ptr() if rot else 0, rot, B.MTS_ROPE_NEIGHBOURS if pairs else B.MTS_ROPE_HALVES)
    t = dev(qkv, dtype)
    src = (t, t[:, Hq:]) if packed else (dev(q, dtype), dev(k, dtype))
    if in_place:
        dst = src
    else:
        dst = tuple(torch.full((n + 1, h, D), -7.0, dtype=TYPE[dtype][1], device=DEV) for h in (Hq, Hk))
    mts.mts_qk_norm_rope(desc, *src, *dst, batch.meta)
    torch.cuda.synchronize()
    pos = np.concatenate([p + np.arange(m) for p, m in zip(prefix, new)])
    if in_place and packed:
        got = t[:, :Hq], t[:, Hq:Hq + Hk]
        assert torch.equal(t[:, Hq + Hk:], dev(qkv[:, Hq + Hk:], dtype))     # V is not touched
    else:
        got = [d[:n] for d in dst]
        if not in_place:
            assert all((d[n:] == -7.0).all() for d in dst)
            assert torch.equal(t, dev(qkv, dtype))
    for g, x, ww in zip(got, (q, k), w):
        ref = R.norm_rope(x, ww, pos, eps, freqs, pairs, norm)
        err = np.abs(g.float().cpu().numpy() - ref)
        b = bound(ref, rot, pairs, dtype)
        assert (err <= b).all(), float((err / b).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("Hq,Hk,D,rot", [(8, 2, 128, 128), (5, 5, 128, 64), (1, 1, 128, 8), (12, 3, 64, 64), (3, 1, 64, 40), (4, 4, 32, 32),
                                         (33, 1, 32, 24), (7, 7, 64, 0)])
def test_against_the_formulas(Hq, Hk, D, rot, pairs, dtype):
    run(1, dtype, Hq, Hk, D, rot, pairs, [0, 5, 0, 777, 131000], [1, 3, 0, 17, 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_strides_and_in_place(packed, in_place, dtype):
    run(2, dtype, 6, 2, 64, 64, False, [9, 0], [4, 30], packed=packed, in_place=in_place)


@pytest.mark.parametrize("norm,weights", [(False, False), (False, True), (True, False)])
def test_without_norm_or_weights(norm, weights):
    run(3, "f32", 4, 2, 128, 96, True, [100], [20], norm=norm, weights=weights)


def test_far_positions():
    """Angles of positions near 2^30, where 32 bits hold none of the turn."""
    run(4, "f32", 2, 1, 64, 64, False, [(1 << 30) - 40, 1 << 24], [33, 1], freqs=np.linspace(1.0, 1e-4, 32))


def test_many_users_and_tokens():
    rng = np.random.default_rng(5)
    run(5, "bf16", 2, 1, 32, 32, True, rng.integers(0, 9000, 4300), rng.integers(0, 3, 4300))
    run(6, "bf16", 16, 8, 128, 128, False, [0, 4000], [900, 3], eps=0.0)


def test_a_row_of_zeros():
    n, D = 3, 64
    batch = DeviceBatch([0, 0], [0], [7], [0, n], DEV)
    f = torch.ones(32, dtype=torch.float64, device=DEV)
    x = torch.zeros(n, 1, D, device=DEV)
    out = [torch.full_like(x, -7.0) for _ in range(2)]
    desc = mts.QkDesc(B.MTS_F32, 1, 1, D, 0, 0, 0, 0, 0, 0, B.MTS_NORM_RMS, 1e-6, f.data_ptr(), D, B.MTS_ROPE_HALVES)
    mts.mts_qk_norm_rope(desc, x, x, *out, batch.meta)
    assert all((o == 0).all() for o in out)

"""The 8-bit pool on the GPU against 64-bit definitions (q8_reference): the quantising writes and the read-back bit for bit,
the attention within the bound that its roundings add up to."""
import numpy as np
import pytest
import torch

import mts_workloads as W
import paper_2604_22881_amd as mts
import q8_reference as R
from paper_2604_22881_amd import binding as B
from paper_2604_22881_amd.runtime import DeviceBatch, PagedKVCache, SegmentList

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPE = {"f32": (B.MTS_F32, torch.float32), "bf16": (B.MTS_BF16, torch.bfloat16)}


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV).to(TYPE[dtype][1])


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def rows(rng, shape, dtype, spread=2.0):
    """Rows of differing size, values of the type."""
    x = rng.standard_normal(shape) * 2.0 ** (rng.standard_normal(shape[:-1] + (1,)) * spread)
    return x.astype(np.float32) if dtype == "f32" else W.bf16_bits_to_f32(W.f32_to_bf16_bits(x.astype(np.float32)))


class Step:
    """A layer of an 8-bit pool filled with a byte, its page tables, and the image that the pool should have."""

    def __init__(self, seed, H, D, S, prefix, new, dtype, fill=0xFF, layers=1, layer=0):
        self.w = W.custom_workload("q8", seed, dtype, 1, H, D, S, prefix, new)
        w = self.w
        self.layer, self.dtype = layer, dtype
        self.cache = PagedKVCache(layers, w.num_pages, S, H, D, "e4m3", DEV, fill_byte=fill)
        self.batch = DeviceBatch.from_workload(w, DEV)
        self.image = np.full((w.num_pages, self.cache.page_bytes), fill, np.uint8)
        self.fill = fill

    def pool(self, layer=None):
        return self.cache.layer_bytes(self.layer if layer is None else layer).cpu().numpy()

    def append(self, k, v, k_stride=0, v_stride=0):
        mts.mts_kv_append_q8(self.cache.desc, self.layer, TYPE[self.dtype][0], k, v, self.batch.meta, k_stride, v_stride)

    def expect_append(self, k, v):
        w = self.w
        for u in range(w.batch):
            a, b = w.new_indptr[u], w.new_indptr[u + 1]
            if b > a:
                R.store(self.image, w.user_pages(u), w.page_size, int(w.prefix_lens[u]), np.stack([k[a:b], v[a:b]]))

    def unpack(self, runs, data):
        segs = SegmentList(*zip(*runs), DEV)
        flat = dev(np.concatenate([d.reshape(-1) for d in data]), self.dtype)
        mts.mts_kv_unpack_q8(self.cache.desc, self.layer, TYPE[self.dtype][0], flat, *segs.args(), self.batch.meta)

    def pack(self, runs, dtype=None):
        w, dtype = self.w, dtype or self.dtype
        segs = SegmentList(*zip(*runs), DEV)
        row = 2 * w.heads * w.head_dim
        out = torch.full((segs.total_tokens * row + 64,), -7.0, dtype=TYPE[dtype][1], device=DEV)
        mts.mts_kv_pack_q8(self.cache.desc, self.layer, TYPE[dtype][0], out, *segs.args(), self.batch.meta)
        assert (out[segs.total_tokens * row:] == -7.0).all()
        ends = segs.host_indptr * row
        return [out[a:b].view(2, -1, w.heads, w.head_dim) for a, b in zip(ends[:-1], ends[1:])]

    def fill_prefixes(self, rng, spread=1.0):
        """Every user's prefix stored, on both sides."""
        w = self.w
        runs = [(u, 0, int(p)) for u, p in enumerate(w.prefix_lens) if p > 0]
        if not runs:
            return
        data = [rows(rng, (2, n, w.heads, w.head_dim), self.dtype, spread) for _, _, n in runs]
        self.unpack(runs, data)
        for (u, p, n), x in zip(runs, data):
            R.store(self.image, w.user_pages(u), w.page_size, p, x)

    def attention(self, q, group, scale=0.0, stream=None):
        w = self.w
        Hq = w.heads * group
        n = mts.mts_attn_q8_workspace_bytes(self.cache.desc, Hq, self.batch.meta)
        ws = torch.full((max(n, 256),), 0xA5, dtype=torch.uint8, device=DEV)
        out = torch.full((max(w.total_new, 1) + 2, Hq, w.head_dim), -7.0, dtype=TYPE[self.dtype][1], device=DEV)
        mts.mts_attn_incremental_q8(self.cache.desc, self.layer, TYPE[self.dtype][0], Hq, q, out, self.batch.meta, scale, ws, n, stream)
        torch.cuda.synchronize()
        assert (out[w.total_new:] == -7.0).all()             # nothing behind the last row is written
        return host(out[:w.total_new])

    def check_attention(self, got, q, group, scale=0.0, users=None):
        w = self.w
        scale = scale or w.head_dim ** -0.5
        worst = 0.0
        for u in range(w.batch) if users is None else users:
            a, b = w.new_indptr[u], w.new_indptr[u + 1]
            if a == b:
                continue
            T = int(w.total_lens[u])
            kv = R.load(self.image, w.user_pages(u), w.page_size, T, w.heads, w.head_dim)
            out, mag, lsum = R.attention(q[a:b], kv, int(w.prefix_lens[u]), scale)
            bound = R.attention_bound(out, mag, lsum, T, w.head_dim, self.dtype == "f32")
            err = np.abs(got[a:b] - out)
            assert np.isfinite(got[a:b]).all(), u
            assert (err <= bound).all(), (u, float((err / bound).max()))
            worst = max(worst, float((err / bound).max()))
        return worst


# ---- writes and read-back ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,S,H", [(32, 16, 3), (32, 64, 1), (64, 32, 5), (64, 16, 4), (128, 16, 2), (128, 64, 3)])
def test_append_writes_exactly_its_rows(D, S, H, dtype):
    # segments of 0, 1, a few and many tokens, from every place of a group and a sub-block on
    prefix = [0, 1, 2, 3, 5, 15, 16, 17, 31, 63, 64, 100, 7, 0]
    new = [1, 1, 3, 17, 0, 2, 16, 1, 33, 1, 64, 5, 130, 0]
    rng = np.random.default_rng(D + S + H)
    s = Step(3, H, D, S, prefix, new, dtype, fill=0xA5)
    k, v = rows(rng, (s.w.total_new, H, D), dtype), rows(rng, (s.w.total_new, H, D), dtype)
    s.append(dev(k, dtype), dev(v, dtype))
    s.expect_append(k, v)
    np.testing.assert_array_equal(s.pool(), s.image)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_takes_rows_from_a_packed_projection(dtype):
    rng = np.random.default_rng(5)
    H, D, Hq = 3, 64, 6
    s = Step(4, H, D, 16, [10, 0, 33], [3, 20, 1], dtype, layers=3, layer=1)
    qkv = rows(rng, (s.w.total_new, Hq + 2 * H, D), dtype)
    t = dev(qkv, dtype)
    stride = (Hq + 2 * H) * D
    s.append(t[:, Hq:], t[:, Hq + H:], stride, stride)
    s.expect_append(qkv[:, Hq:Hq + H], qkv[:, Hq + H:])
    np.testing.assert_array_equal(s.pool(), s.image)
    for other in (0, 2):                                     # the other layers keep every byte
        assert (s.pool(other) == 0xFF).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,S", [(32, 32), (64, 16), (128, 32)])
def test_rows_at_the_type_s_corners(D, S, dtype):
    """Zeros, both signs, ties, subnormal codes, saturation, rows under and over the exponents' range, infinities, NaN."""
    rng = np.random.default_rng(9)
    H = 2
    s = Step(5, H, D, S, [3], [77], dtype)
    x = rows(rng, (2, 77, H, D), dtype, spread=0.0)
    x[:, 0] = 0.0
    x[:, 1] = -0.0
    for i, e in enumerate([-149, -126, -100, -75, -70, -69, -61, -60, 0, 30, 59, 60, 67, 68, 69, 100, 126]):
        x[:, 2 + i] = np.clip(x[:, 2 + i], -1.9, 1.9) * np.float32(2.0 ** max(e, -126)) * np.float32(2.0 ** min(0, e + 126))
    ties = np.concatenate([R.VALUES[:0x7E] + np.diff(R.VALUES[:0x7F]) / 2, R.VALUES[:0x7F], [456.0, 464.0]])
    for i in range(8):
        x[:, 25 + i] = rng.choice(ties, (2, H, D)) * rng.choice([-1.0, 1.0], (2, H, D)) * 2.0 ** (i - 4)
        x[:, 33 + i, :, 0] = [464.0, 464.5, 448.0, 480.0, 465.0, 447.0, 463.0, 256.0][i]
    x[0, 50, 0, 3], x[0, 51, 1, D - 1], x[1, 52, 0, 0], x[1, 53, 1, 7] = np.inf, -np.inf, np.nan, np.inf
    x[:, 54] = np.nan
    x[:, 55] = -np.inf
    x = x.astype(np.float32) if dtype == "f32" else W.bf16_bits_to_f32(W.f32_to_bf16_bits(x.astype(np.float32)))
    s.append(dev(x[0], dtype), dev(x[1], dtype))
    s.expect_append(x[0], x[1])
    np.testing.assert_array_equal(s.pool(), s.image)
    got = host(s.pack([(0, 3, 77)])[0])
    np.testing.assert_array_equal(got, R.quantise(x)[2])     # NaN compare equal here


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,S,H", [(32, 16, 5), (64, 64, 2), (128, 32, 4), (128, 16, 1)])
def test_runs_are_stored_and_read_back(D, S, H, dtype):
    rng = np.random.default_rng(D * S)
    s = Step(6, H, D, S, [300, 41, 9, 260], [0, 0, 0, 0], dtype, fill=0x5A)
    # out of order, neighbours that share a sub-block, an empty run, single tokens
    runs = [(3, 0, 100), (0, 0, 130), (0, 130, 131), (1, 5, 1), (2, 0, 0), (0, 261, 39), (3, 100, 3), (3, 103, 1), (3, 104, 156), (1, 7, 30)]
    data = [rows(rng, (2, n, H, D), dtype) for _, _, n in runs]
    s.unpack(runs, data)
    for (u, p, n), x in zip(runs, data):
        R.store(s.image, s.w.user_pages(u), S, p, x) if n else None
    np.testing.assert_array_equal(s.pool(), s.image)
    for got, x in zip(s.pack(runs), data):
        np.testing.assert_array_equal(host(got), R.quantise(x)[2])
    # the other row type reads the same values, other cuts of a user too
    other = "bf16" if dtype == "f32" else "f32"
    whole = R.load(s.image, s.w.user_pages(0), S, 300, H, D)
    np.testing.assert_array_equal(host(s.pack([(0, 17, 200)], other)[0]), whole[:, 17:217])
    # what was read back is stored again as the same bytes
    back = s.pack(runs)
    s.cache.pool.fill_(0x5A)
    s.unpack(runs, [host(b) for b in back])
    np.testing.assert_array_equal(s.pool(), s.image)


def test_runs_behind_other_rows_of_the_buffer():
    """Offsets that do not begin at 0: the runs of a part of a larger buffer."""
    rng = np.random.default_rng(13)
    H, D, S, skip = 2, 64, 16, 1003
    s = Step(9, H, D, S, [70, 33], [0, 0], "bf16", fill=0x21)
    runs = [(1, 0, 33), (0, 20, 50), (0, 0, 20)]
    data = [rows(rng, (2, n, H, D), "bf16") for _, _, n in runs]
    segs = SegmentList(*zip(*runs), DEV)
    segs.seg_tok_indptr += skip
    row = 2 * H * D
    flat = torch.cat([torch.full((skip * row,), 3.0, dtype=torch.bfloat16, device=DEV), dev(np.concatenate([d.reshape(-1) for d in data]), "bf16")])
    mts.mts_kv_unpack_q8(s.cache.desc, 0, B.MTS_BF16, flat, *segs.args(), s.batch.meta)
    for (u, p, n), x in zip(runs, data):
        R.store(s.image, s.w.user_pages(u), S, p, x)
    np.testing.assert_array_equal(s.pool(), s.image)
    out = torch.full((flat.numel(),), -7.0, dtype=torch.bfloat16, device=DEV)
    mts.mts_kv_pack_q8(s.cache.desc, 0, B.MTS_BF16, out, *segs.args(), s.batch.meta)
    assert (out[:skip * row] == -7.0).all()
    np.testing.assert_array_equal(host(out[skip * row:]), np.concatenate([R.quantise(x)[2].reshape(-1) for x in data]))


def test_many_users_and_runs():
    """More users than a wavefront has lanes, and more than the square of that."""
    rng = np.random.default_rng(11)
    n = 4200
    prefix, new = rng.integers(0, 20, n), rng.integers(0, 3, n)
    s = Step(7, 1, 32, 16, prefix, new, "bf16", fill=0)
    k, v = rows(rng, (s.w.total_new, 1, 32), "bf16"), rows(rng, (s.w.total_new, 1, 32), "bf16")
    s.append(dev(k, "bf16"), dev(v, "bf16"))
    s.expect_append(k, v)
    np.testing.assert_array_equal(s.pool(), s.image)
    runs = [(u, int(prefix[u]), int(new[u])) for u in range(n)]
    got = s.pack(runs)
    for (u, p, m), g in zip(runs, got):
        if m:
            a = s.w.new_indptr[u]
            np.testing.assert_array_equal(host(g), R.quantise(np.stack([k[a:a + m], v[a:a + m]]))[2])


def test_bad_page_ids_are_skipped():
    rng = np.random.default_rng(12)
    s = Step(8, 2, 64, 16, [40], [5], "bf16", fill=0x11)
    s.batch.page_indices[1] = s.w.num_pages + 7
    s.batch.page_indices[2] = -3
    k = rows(rng, (5, 2, 64), "bf16")
    s.append(dev(k, "bf16"), dev(k, "bf16"))                 # tokens 40 .. 44 lie in the third page
    s.unpack([(0, 0, 40)], [rows(rng, (2, 40, 2, 64), "bf16")])
    pool = s.pool()
    touched = (pool != 0x11).any(1)
    assert touched.sum() == 1 and touched[s.w.user_pages(0)[0]]


# ---- attention -------------------------------------------------------------------------------------

def attend(seed, H, G, D, S, prefix, new, dtype, spread=1.0, scale=0.0, users=None, fill=0xFF):
    rng = np.random.default_rng(seed)
    s = Step(seed, H, D, S, prefix, new, dtype, fill=fill)
    s.fill_prefixes(rng, spread)
    n = s.w.total_new
    k, v = rows(rng, (n, H, D), dtype, spread), rows(rng, (n, H, D), dtype, spread)
    s.append(dev(k, dtype), dev(v, dtype))
    s.expect_append(k, v)
    q = rows(rng, (n, H * G, D), dtype, 0.3)
    got = s.attention(dev(q, dtype), G, scale)
    print("share of the bound:", s.check_attention(got, q, G, scale, users))
    return s, q, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,D,S", [(4, 1, 32, 16), (2, 3, 32, 64), (5, 1, 64, 32), (3, 4, 64, 16), (2, 8, 128, 16), (1, 5, 128, 64), (8, 1, 128, 32)])
def test_single_tokens_and_short_segments(H, G, D, S, dtype):
    # one key, lengths about tiles, sub-blocks and pages, users without rows
    prefix = [0, 1, 15, 16, 30, 31, 32, 33, 127, 250, 0, 64, 500]
    new = [1, 1, 1, 1, 1, 1, 2, 1, 3, 7, 12, 0, 5]
    attend(21, H, G, D, S, prefix, new, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,D,S", [(2, 4, 64, 16), (1, 1, 128, 32), (2, 2, 32, 16)])
def test_long_keys_are_cut_and_joined(H, G, D, S, dtype):
    # stretches of unequal users, one that ends on a stretch's edge, one behind it
    s, _, _ = attend(22, H, G, D, S, [4000, 255, 256, 0, 1023, 2047], [1, 1, 1, 1, 2, 1], dtype)
    assert mts.mts_attn_q8_workspace_bytes(s.cache.desc, H * G, s.batch.meta) > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,D,S,new", [(2, 1, 128, 16, [300, 17, 0, 65]), (1, 3, 64, 32, [130, 33, 1, 90]), (3, 2, 32, 64, [64, 31, 200, 2])])
def test_segments_of_many_tiles(H, G, D, S, new, dtype):
    attend(23, H, G, D, S, [0, 100, 40, 333], new, dtype)


@pytest.mark.parametrize("H,G,D,S,prefix,new", [
    (2, 1, 64, 16, [3000, 0, 500, 0, 1200, 7, 900], [1, 300, 20, 0, 2, 64, 65]),     # both kinds cut and joined
    (3, 2, 128, 32, [40, 0, 500, 0, 100], [1, 150, 32, 33, 200]),                    # neither
    (1, 4, 32, 16, [700, 1500], [200, 1]),
    (2, 2, 64, 64, [10, 300], [140, 140]),                                           # no user of few rows: one kernel
    (2, 1, 128, 16, [2000], [129]),
])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_users_of_few_and_of_many_rows_in_one_call(H, G, D, S, prefix, new, dtype):
    attend(36, H, G, D, S, prefix, new, dtype)


def test_tiles_of_rows_and_stretches_of_keys_at_once():
    # some rows of a tile see none of its last stretch's keys
    s, _, _ = attend(24, 1, 2, 64, 16, [1000, 240], [70, 40], "bf16")
    assert mts.mts_attn_q8_workspace_bytes(s.cache.desc, 2, s.batch.meta) > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_very_different_size(dtype):
    """V rows over 2^20 apart in size, K rows that make one logit dominate or all alike."""
    attend(25, 2, 4, 64, 16, [700, 90], [1, 20], dtype, spread=6.0)


@pytest.mark.parametrize("D", [32, 64, 128])
def test_huge_logits(D):
    """One key's logit far above all others: the output is that key's V; equal largest ones share."""
    rng = np.random.default_rng(26)
    H, S, T = 2, 16, 200
    s = Step(26, H, D, S, [T], [1], "f32")
    kv = rows(rng, (2, T, H, D), "f32", 0.0)
    kv[1] *= 2.0 ** rng.integers(-6, 7, (T, H, 1))           # V's exponents differ
    kv[0, 77] = 1.0
    kv[0, 150, 1] = 1.0
    kv[0, :, :, :][np.arange(T) % 50 != 27] *= 0.25
    kv[0, 77], kv[0, 150, 1] = 1.0, 1.0
    for big in (1e4, 1e9, 1e20, 1e30):
        q = np.full((1, H, D), big, np.float32)
        k_new = np.zeros((1, H, D), np.float32)
        v_new = rows(rng, (1, H, D), "f32")
        s.unpack([(0, 0, T)], [kv])
        s.append(dev(k_new, "f32"), dev(v_new, "f32"))
        got = s.attention(dev(q, "f32"), 1, 1.0)
        v = R.quantise(kv[1])[2]
        if big < 1e9:
            # the weight is some 2^8 * 2^f: its two fp16 parts are off by 2^-22 of it (half a step, 2^-11, of a part that is
            # half a step of the other), 1 / l and the product with it by 2^-24 each, the sum l by 2^-24 for each of 4 wavefronts
            np.testing.assert_allclose(got[0, 0], v[77, 0], rtol=2.0 ** -22 + 6 * 2.0 ** -24)
        else:
            np.testing.assert_array_equal(got[0, 0], v[77, 0])   # the weight is a power of two
        np.testing.assert_allclose(got[0, 1], (v[77, 1] + v[150, 1]) / 2, rtol=0,
                                   atol=(2.0 ** -22 + 6 * 2.0 ** -24) * np.abs(v[[77, 150], 1]).max())


def test_small_weights_count():
    """Many keys of small weight beside a large one: 4000 keys at 2^-18 of it together weigh 1.5 %; fp16's normal numbers end
    at 2^-14."""
    H, D, T = 1, 64, 4000
    s = Step(27, H, D, 16, [T], [1], "bf16", fill=0)
    k = np.zeros((T + 1, H, D))
    k[:, 0, 0] = -18.0 * np.log(2.0)
    k[T, 0, 0] = 0.0
    v = np.ones((T + 1, H, D))
    v[T] = 0.0
    k = W.bf16_bits_to_f32(W.f32_to_bf16_bits(k.astype(np.float32)))
    s.unpack([(0, 0, T)], [np.stack([k[:T], v[:T]]).astype(np.float32)])
    s.append(dev(k[T:], "bf16"), dev(v[T:], "bf16"))
    R.store(s.image, s.w.user_pages(0), 16, 0, np.stack([k, v]))
    q = np.zeros((1, H, D), np.float32)
    q[0, 0, 0] = 1.0
    got = s.attention(dev(q, "bf16"), 1, 1.0)
    s.check_attention(got, q, 1, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 128])
def test_nan_and_infinity_reach_only_the_queries_that_see_them(D, dtype):
    rng = np.random.default_rng(28)
    H, G, S = 2, 2, 16
    prefix, new = [50, 20, 0], [40, 9, 33]
    s = Step(28, H, D, S, prefix, new, dtype)
    s.fill_prefixes(rng)
    n = s.w.total_new
    k, v = rows(rng, (n, H, D), dtype), rows(rng, (n, H, D), dtype)
    at = s.w.new_indptr
    k[at[0] + 30, 0, 5] = np.nan                             # user 0: key head 0 from token 30 on
    v[at[0] + 11, 1, 3] = np.inf                             # ... value head 1, dim 3, from token 11 on
    v[at[2] + 32, 0, 0] = np.nan                             # the last token of user 2
    v[at[2] + 4, 1, D - 1] = -np.inf
    s.append(dev(k, dtype), dev(v, dtype))
    s.expect_append(k, v)
    q = rows(rng, (n, H * G, D), dtype, 0.3)
    got = s.attention(dev(q, dtype), G)
    for u in range(3):
        kv = R.load(s.image, s.w.user_pages(u), S, int(s.w.total_lens[u]), H, D)
        ref, mag, lsum = R.attention(q[at[u]:at[u + 1]], kv, prefix[u], D ** -0.5)
        part = got[at[u]:at[u + 1]]
        np.testing.assert_array_equal(np.isnan(part), np.isnan(ref))
        fine = np.isfinite(ref)
        err = np.abs(part - ref)[fine]
        # magnitudes of rows with a NaN key are NaN; the others are bounded
        assert (err <= R.attention_bound(ref, mag, lsum, kv.shape[1], D, dtype == "f32")[fine]).all()


def test_what_lies_behind_a_user_s_last_key_is_not_read_as_data():
    """The same call over pools whose unwritten slots hold NaN codes, zeros and the largest exponents."""
    got = []
    for fill in (0xFF, 0x00, 0x7F, 0x01):
        _, _, g = attend(29, 2, 2, 64, 32, [5, 37, 1000], [1, 3, 1], "bf16", fill=fill)
        got.append(g)
    for g in got[1:]:
        np.testing.assert_array_equal(g, got[0])


def test_many_users_attend():
    rng = np.random.default_rng(30)
    n = 4500
    attend(30, 1, 1, 32, 16, rng.integers(0, 40, n), rng.integers(0, 3, n), "bf16", users=rng.choice(n, 150, replace=False))


def test_bad_page_ids_and_short_page_lists_do_not_fault():
    rng = np.random.default_rng(31)
    s = Step(31, 2, 64, 16, [400, 100], [1, 2], "bf16", fill=0)
    s.fill_prefixes(rng)
    s.batch.page_indices[3] = 1 << 30
    s.batch.page_indices[4] = -1
    s.batch.prefix_lens[1] = 5000                            # more than its pages hold
    q = dev(rows(rng, (3, 4, 64), "bf16"), "bf16")
    assert np.isfinite(s.attention(q, 2)[0]).all()


@pytest.mark.parametrize("scale", [0.0, 0.03, 1.0])
def test_scales(scale):
    attend(32, 2, 2, 64, 16, [100], [3], "bf16", scale=scale)


def test_calls_repeat_bit_for_bit_on_another_stream():
    s, q, got = attend(33, 4, 4, 128, 16, [3000, 800, 1], [1, 1, 1], "bf16")
    side = torch.cuda.Stream()
    t = dev(q, "bf16")
    torch.cuda.synchronize()
    for _ in range(3):
        np.testing.assert_array_equal(s.attention(t, 4, stream=side), got)


def test_a_step_of_all_calls_replays_from_a_graph():
    """norm + rotation, append, attention and read-back captured together; replays with new inputs in the same buffers against
    the same calls made eagerly."""
    rng = np.random.default_rng(34)
    H, G, D, S = 2, 4, 64, 16
    prefix, new = [1200, 30, 0], [1, 2, 5]
    s = Step(34, H, D, S, prefix, new, "bf16", fill=0)
    s.fill_prefixes(rng)
    n, Hq = s.w.total_new, H * G
    qkv = torch.zeros(n, Hq + 2 * H, D, dtype=torch.bfloat16, device=DEV)
    q, k = torch.empty(n, Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, H, D, dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(q)
    freqs = torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D / 2))).to(DEV)
    stride = (Hq + 2 * H) * D
    desc = mts.QkDesc(B.MTS_BF16, Hq, H, D, stride, stride, 0, 0, 0, 0, B.MTS_NORM_RMS, 1e-6, freqs.data_ptr(), D, B.MTS_ROPE_HALVES)
    nb = mts.mts_attn_q8_workspace_bytes(s.cache.desc, Hq, s.batch.meta)
    ws = torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV)
    segs = SegmentList([0, 1, 2], prefix, new, DEV)
    back = torch.empty(n * 2 * H * D, dtype=torch.bfloat16, device=DEV)

    def step():
        mts.mts_qk_norm_rope(desc, qkv, qkv[:, Hq:], q, k, s.batch.meta)
        mts.mts_kv_append_q8(s.cache.desc, 0, B.MTS_BF16, k, qkv[:, Hq + H:], s.batch.meta, 0, stride)
        mts.mts_attn_incremental_q8(s.cache.desc, 0, B.MTS_BF16, Hq, q, out, s.batch.meta, 0.0, ws, nb)
        mts.mts_kv_pack_q8(s.cache.desc, 0, B.MTS_BF16, back, *segs.args(), s.batch.meta)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        x = dev(rows(rng, qkv.shape, "bf16"), "bf16")
        qkv.copy_(x)
        step()
        eager = [t.clone() for t in (q, k, out, back, s.cache.pool)]
        torch.cuda.synchronize()
        for t in (q, k, out, back, ws):
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip((q, k, out, back, s.cache.pool), eager):
            assert torch.equal(t, e)


def test_decode_steps_of_a_serving_loop():
    """Users grow over several steps through norm + rotation, append and attention; each step against 64 bits over the rows that
    were stored so far, and the history read back at the end."""
    rng = np.random.default_rng(35)
    H, G, D, S, steps = 2, 3, 64, 16, 6
    Hq = H * G
    grown = [np.zeros((2, 0, H, D)) for _ in range(3)]
    total = [[40, 1, 5, 1, 1, 2], [0, 3, 1, 1, 0, 1], [17, 1, 1, 1, 30, 1]]
    pages_of = [list(range(u, 60, 3)) for u in range(3)]
    cache = PagedKVCache(1, 60, S, H, D, "e4m3", DEV, fill_byte=0xFF)
    freqs = 10000.0 ** (-np.arange(D // 2) / (D / 2))
    f = torch.from_numpy(freqs).to(DEV)
    w = [rows(rng, (D,), "bf16", 0.0) for _ in range(2)]
    wd = [dev(x, "bf16") for x in w]
    desc = mts.QkDesc(B.MTS_BF16, Hq, H, D, 0, 0, 0, 0, wd[0].data_ptr(), wd[1].data_ptr(), B.MTS_NORM_RMS, 1e-6, f.data_ptr(), D,
                      B.MTS_ROPE_NEIGHBOURS)
    for step in range(steps):
        new = [t[step] for t in total]
        prefix = [g.shape[1] for g in grown]
        held = [-(-(p + n) // S) for p, n in zip(prefix, new)]
        batch = DeviceBatch(np.concatenate([[0], np.cumsum(held)]), np.concatenate([pages_of[u][:held[u]] for u in range(3)]).astype(np.int32),
                            prefix, np.concatenate([[0], np.cumsum(new)]), DEV)
        n = sum(new)
        q, k, v = (rows(rng, (n, h, D), "bf16", 0.5) for h in (Hq, H, H))
        qo, ko = (torch.empty(n, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hq, H))
        out = torch.empty_like(qo)
        mts.mts_qk_norm_rope(desc, dev(q, "bf16"), dev(k, "bf16"), qo, ko, batch.meta)
        mts.mts_kv_append_q8(cache.desc, 0, B.MTS_BF16, ko, dev(v, "bf16"), batch.meta)
        nb = mts.mts_attn_q8_workspace_bytes(cache.desc, Hq, batch.meta)
        ws = torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV)
        mts.mts_attn_incremental_q8(cache.desc, 0, B.MTS_BF16, Hq, qo, out, batch.meta, 0.0, ws, nb)
        qh, kh, got = host(qo), host(ko), host(out)
        at = np.concatenate([[0], np.cumsum(new)])
        for u in range(3):
            a, b = at[u], at[u + 1]
            pos = prefix[u] + np.arange(b - a)
            for x, y, ww in ((q, qh, w[0]), (k, kh, w[1])):
                ref = R.norm_rope(x[a:b], ww, pos, 1e-6, freqs, True)
                size = np.abs(ref[..., 0::2]) + np.abs(ref[..., 1::2])
                assert (np.abs(y[a:b] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * np.repeat(size, 2, -1) + 1e-30).all()
            grown[u] = np.concatenate([grown[u], R.quantise(np.stack([kh[a:b], v[a:b].astype(np.float64)]))[2]], 1)
            if b > a:
                ref, mag, lsum = R.attention(qh[a:b], grown[u], prefix[u], D ** -0.5)
                assert (np.abs(got[a:b] - ref) <= R.attention_bound(ref, mag, lsum, grown[u].shape[1], D, False)).all()
    held = [-(-g.shape[1] // S) for g in grown]
    batch = DeviceBatch(np.concatenate([[0], np.cumsum(held)]), np.concatenate([pages_of[u][:held[u]] for u in range(3)]).astype(np.int32),
                        [g.shape[1] for g in grown], [0, 0, 0, 0], DEV)
    segs = SegmentList([0, 1, 2], [0, 0, 0], [g.shape[1] for g in grown], DEV)
    out = torch.empty(segs.total_tokens * 2 * H * D, dtype=torch.float32, device=DEV)
    mts.mts_kv_pack_q8(cache.desc, 0, B.MTS_F32, out, *segs.args(), batch.meta)
    np.testing.assert_array_equal(host(out), np.concatenate([g.reshape(-1) for g in grown]))


# ---- many rows: the keys shared by a workgroup's wavefronts -----------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,prefix,new", [(64, [300, 0, 64], [1, 1, 1]), (128, [3000], [2]), (32, [300, 20], [140, 3]), (128, [40], [150]),
                                          (64, [1500], [130])])
def test_large_rows_of_v_without_weight_leave_the_others_theirs(D, prefix, new, dtype):
    """Rows of V at 2^50 whose logits lie 400 below the others': the outputs are those of the other keys, each with all bits."""
    rng = np.random.default_rng(40)
    H, G, S = 2, 1, 16
    s = Step(40, H, D, S, prefix, new, dtype)
    s.fill_prefixes(rng, 0.5)
    q = rows(rng, (s.w.total_new, H * G, D), dtype, 0.0) * 0.25
    q[..., 0] = 1.0

    def with_large(n):
        x = rows(rng, (2, n, H, D), dtype, 0.5)
        x[0, ..., 0] = 0.0
        far = rng.random((n, H)) < 0.3
        x[0][far] = 0.0
        x[0, ..., 0][far] = -400.0
        x[1][far] *= 2.0 ** 50
        return x
    runs = [(u, 0, p) for u, p in enumerate(prefix) if p > 0]
    data = [with_large(n) for _, _, n in runs]
    s.unpack(runs, data)
    for (u, p, n), x in zip(runs, data):
        R.store(s.image, s.w.user_pages(u), S, p, x)
    x = with_large(s.w.total_new)
    for u in range(len(new)):                                # every query has a key of its own size
        if prefix[u] == 0:
            x[:, s.w.new_indptr[u]] = 0.5
    s.append(dev(x[0], dtype), dev(x[1], dtype))
    s.expect_append(x[0], x[1])
    got = s.attention(dev(q, dtype), G, 1.0)
    assert s.check_attention(got, q, G, 1.0) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 130])
def test_weights_that_are_subnormal_in_fp16_count(n, dtype):
    """4000 keys at 2^-27 of the largest weight, which alone make up half of the dims: 2^-19 where the largest is 2^8."""
    H, D, T = 1, 64, 4000
    s = Step(41, H, D, 16, [T], [n], dtype, fill=0)
    k, v = np.zeros((T + n, H, D)), np.ones((T + n, H, D))
    k[:T, 0, 0] = -27.0 * np.log(2.0)
    v[T:, :, :32] = 0.0
    k = W.bf16_bits_to_f32(W.f32_to_bf16_bits(k.astype(np.float32))).astype(np.float64)
    s.unpack([(0, 0, T)], [np.stack([k[:T], v[:T]]).astype(np.float32)])
    s.append(dev(k[T:], dtype), dev(v[T:], dtype))
    R.store(s.image, s.w.user_pages(0), 16, 0, np.stack([k, v]))
    q = np.zeros((n, H, D), np.float32)
    q[:, 0, 0] = 1.0
    got = s.attention(dev(q, dtype), 1, 1.0)
    kv = R.load(s.image, s.w.user_pages(0), 16, T + n, H, D)
    out, mag, lsum = R.attention(q, kv, T, 1.0)
    # a weight is off by 2^-33 of the largest product of a weight and its row's 2^e at most (half of fp16's least step, 2^-25, where
    # that product is 2^8 or more; all rows of V have one e here): over all keys 4130 * 2^-33 of p <= 1, times the values' 1
    bound = R.attention_bound(out, mag, lsum, T + n, D, dtype == "f32") + (T + n) * 2.0 ** -33
    assert out[0, 0, 0] > 1e-5
    assert (np.abs(got - out) <= bound).all()
    assert (np.abs(got - out)[..., :32] <= 2.0 ** -5 * out[..., :32]).all()    # 2^-25 of 2^-19, and a rounding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_very_different_size_under_many_rows(dtype):
    attend(42, 2, 4, 64, 16, [700, 90], [40, 70], dtype, spread=6.0)
    attend(43, 1, 1, 128, 32, [1500], [140], dtype, spread=6.0)


@pytest.mark.parametrize("D", [32, 64, 128])
def test_huge_logits_under_many_rows(D):
    rng = np.random.default_rng(44)
    H, S, T, n = 2, 16, 200, 130
    s = Step(44, H, D, S, [T], [n], "f32")
    kv = rows(rng, (2, T, H, D), "f32", 0.0)
    kv[1] *= 2.0 ** rng.integers(-6, 7, (T, H, 1))
    kv[0] *= 0.25
    kv[0, 77], kv[0, 150, 1] = 1.0, 1.0
    k_new, v_new = np.zeros((n, H, D), np.float32), rows(rng, (n, H, D), "f32")
    s.unpack([(0, 0, T)], [kv])
    s.append(dev(k_new, "f32"), dev(v_new, "f32"))
    v = R.quantise(kv[1])[2]
    for big in (1e9, 1e20, 1e30):
        got = s.attention(dev(np.full((n, H, D), big, np.float32), "f32"), 1, 1.0)
        np.testing.assert_array_equal(got[:, 0], np.broadcast_to(v[77, 0], (n, D)))       # the weight is a power of two
        np.testing.assert_allclose(got[:, 1], np.broadcast_to((v[77, 1] + v[150, 1]) / 2, (n, D)), rtol=0,
                                   atol=(2.0 ** -22 + 6 * 2.0 ** -24) * np.abs(v[[77, 150], 1]).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,prefix,new", [(32, [50, 20, 0], [140, 9, 150]), (128, [50, 20, 0], [140, 9, 150]), (64, [1100, 1000], [140, 130])])
def test_nan_and_infinity_under_many_rows(D, prefix, new, dtype):
    """Uncut and in stretches: NaN among a user's own new keys reaches the queries from it on, and no other."""
    rng = np.random.default_rng(45)
    H, G, S = 2, 2, 16
    s = Step(45, H, D, S, prefix, new, dtype)
    s.fill_prefixes(rng)
    n, at = s.w.total_new, s.w.new_indptr
    k, v = rows(rng, (n, H, D), dtype), rows(rng, (n, H, D), dtype)
    k[at[0] + 100, 0, 5] = np.nan
    v[at[0] + 11, 1, 3] = np.inf
    v[at[0] + 63, 1, D - 1] = np.nan
    v[at[0] + 64, 1, 0] = np.nan
    v[at[-1] - 1, 0, 0] = np.nan                             # the last token of the last user
    v[at[-2] + 4, 1, D - 1] = -np.inf
    k[at[-2] + 127, 1, 0] = np.nan
    s.append(dev(k, dtype), dev(v, dtype))
    s.expect_append(k, v)
    q = rows(rng, (n, H * G, D), dtype, 0.3)
    got = s.attention(dev(q, dtype), G)
    for u in range(len(new)):
        kv = R.load(s.image, s.w.user_pages(u), S, int(s.w.total_lens[u]), H, D)
        ref, mag, lsum = R.attention(q[at[u]:at[u + 1]], kv, prefix[u], D ** -0.5)
        part = got[at[u]:at[u + 1]]
        np.testing.assert_array_equal(np.isnan(part), np.isnan(ref))
        fine = np.isfinite(ref)
        assert (np.abs(part - ref)[fine] <= R.attention_bound(ref, mag, lsum, kv.shape[1], D, dtype == "f32")[fine]).all()


def test_what_lies_behind_the_last_key_under_many_rows():
    for prefix, new in (([5, 37, 0], [130, 3, 200]), ([1100], [131])):
        got = [attend(46, 2, 2, 64, 32, prefix, new, "bf16", fill=fill, users=[0])[2] for fill in (0xFF, 0x00, 0x7F, 0x01)]
        for g in got[1:]:
            np.testing.assert_array_equal(g, got[0])


def test_bad_page_ids_and_short_page_lists_under_many_rows():
    rng = np.random.default_rng(47)
    s = Step(47, 2, 64, 16, [400, 1200], [130, 140], "bf16", fill=0)
    s.fill_prefixes(rng)
    k = dev(rows(rng, (270, 2, 64), "bf16"), "bf16")
    s.append(k, k)
    s.batch.page_indices[3] = 1 << 30
    s.batch.page_indices[4] = -1
    s.batch.prefix_lens[1] = 500000                          # more than its pages hold
    q = dev(rows(rng, (270, 4, 64), "bf16"), "bf16")
    assert np.isfinite(s.attention(q, 2)[:130]).all()


@pytest.mark.parametrize("prefix,new", [([900, 0], [140, 200]), ([3000, 1200, 40], [140, 1, 200])])
def test_many_rows_repeat_on_another_stream_and_from_a_graph(prefix, new):
    """Uncut; and cut, with users of few rows in a launch of their own."""
    s, q, got = attend(48, 2, 4, 64, 16, prefix, new, "bf16", users=[0])
    t = dev(q, "bf16")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(s.attention(t, 4, stream=side), got)
    n = mts.mts_attn_q8_workspace_bytes(s.cache.desc, 8, s.batch.meta)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mts.mts_attn_incremental_q8(s.cache.desc, 0, B.MTS_BF16, 8, t, out, s.batch.meta, 0.0, ws, n)
    rng = np.random.default_rng(49)
    for i in range(4):
        t.copy_(dev(rows(rng, q.shape, "bf16", 0.3), "bf16"))
        eager = s.attention(t, 4)
        ws.fill_(77)
        out.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(host(out), eager)


@pytest.mark.parametrize("prefix,new,used", [([40, 9, 100], [3, 2, 4], [1, 0, 2]), ([2000, 100], [40, 60], [1, 37]),
                                             ([300, 20, 0], [140, 150, 3], [130, 0, 1]), ([3000, 40], [200, 200], [129, 1])])
def test_a_padded_step(prefix, new, used):
    """Sizes that are bounds, as a captured step has them: the device's tables end earlier, and the rows behind them stay as they are.
    Norm + rotation, append and attention against the same calls of the step's own size, bit for bit in the pool."""
    rng = np.random.default_rng(50)
    H, G, D, S = 2, 2, 64, 16
    Hq, n_used, dtype = H * G, sum(used), "bf16"
    freqs = torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D / 2))).to(DEV)
    desc = mts.QkDesc(B.MTS_BF16, Hq, H, D, 0, 0, 0, 0, 0, 0, B.MTS_NORM_RMS, 1e-6, freqs.data_ptr(), D, B.MTS_ROPE_HALVES)
    q, k, v = (rows(rng, (sum(new), h, D), dtype, 0.5) for h in (Hq, H, H))
    hist = [rows(rng, (2, p, H, D), dtype) for p in prefix]
    got = []
    for lengths in (used, new):
        s = Step(50, H, D, S, prefix, new, dtype, fill=0x22)
        s.unpack([(u, 0, p) for u, p in enumerate(prefix) if p], [x for x in hist if x.size])
        b = s.batch
        if lengths is used:                                  # the step's own sizes, the same pages
            b = DeviceBatch(s.w.page_indptr, s.w.page_indices, prefix, np.concatenate([[0], np.cumsum(used)]), DEV)
        else:
            b.new_indptr.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(used)]).astype(np.int32)))
        n = sum(lengths)
        qo, out = (torch.full((n, Hq, D), -7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ko = torch.full((n, H, D), -7.0, dtype=torch.bfloat16, device=DEV)
        mts.mts_qk_norm_rope(desc, dev(q[:n], dtype), dev(k[:n], dtype), qo, ko, b.meta)
        mts.mts_kv_append_q8(s.cache.desc, 0, B.MTS_BF16, ko, dev(v[:n], dtype), b.meta)
        nb = mts.mts_attn_q8_workspace_bytes(s.cache.desc, Hq, b.meta)
        ws = torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV)
        mts.mts_attn_incremental_q8(s.cache.desc, 0, B.MTS_BF16, Hq, qo, out, b.meta, 0.0, ws, nb)
        torch.cuda.synchronize()
        for t in (qo, ko, out):
            assert (t[n_used:] == -7.0).all()
        got.append([host(t[:n_used]) for t in (qo, ko, out)] + [s.pool()])
    for a, b in zip(got[0][:2], got[1][:2]):
        np.testing.assert_array_equal(a, b)
    np.testing.assert_array_equal(got[0][3], got[1][3])
    # the keys may be cut otherwise: each is within its bound of the same value
    s = Step(50, H, D, S, prefix, used, dtype)
    for u in range(len(used)):
        a, b = sum(used[:u]), sum(used[:u + 1])
        if b == a:
            continue
        kv = np.concatenate([R.quantise(hist[u])[2], R.quantise(np.stack([got[0][1][a:b], v[a:b].astype(np.float64)]))[2]], 1)
        ref, mag, lsum = R.attention(got[0][0][a:b], kv, prefix[u], D ** -0.5)
        bound = R.attention_bound(ref, mag, lsum, kv.shape[1], D, False)
        for g in got:
            assert (np.abs(g[2][a:b] - ref) <= bound).all()


def test_pools_and_strides_beyond_32_bits():
    """A layer of 5.3 GB and tokens 2 GB apart: the same bytes and results as in a small pool from rows that follow one another."""
    rng = np.random.default_rng(51)
    H, G, D, S, prefix, new = 8, 2, 128, 64, [300, 70, 1500], [1, 2, 1]
    Hq, n, dtype = H * G, sum(new), "bf16"
    small = Step(51, H, D, S, prefix, new, dtype, fill=0x33)
    w = small.w
    pages = 40000
    cache = PagedKVCache(1, pages, S, H, D, "e4m3", DEV, fill_byte=0x33)
    assert cache.page_bytes * pages > 1 << 32
    ids = np.asarray(w.page_indices)
    far = pages - 1 - ids                                    # the last pages of the pool, backwards
    batch = DeviceBatch(w.page_indptr, far, prefix, w.new_indptr, DEV)
    q, k, v = (rows(rng, (n, h, D), dtype, 0.5) for h in (Hq, H, H))
    hist = [rows(rng, (2, p, H, D), dtype) for p in prefix]
    runs = [(u, 0, p) for u, p in enumerate(prefix)]
    stride = 1 << 30
    apart = torch.empty((n - 1) * stride + (Hq + 2 * H) * D, dtype=torch.bfloat16, device=DEV)
    qkv = apart.as_strided((n, Hq + 2 * H, D), (stride, D, 1))
    qkv.copy_(dev(np.concatenate([q, k, v], 1), dtype))
    freqs = torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D / 2))).to(DEV)
    got = []
    for c, b, s in ((small.cache, small.batch, 0), (cache, batch, stride)):
        segs = SegmentList(*zip(*runs), DEV)
        mts.mts_kv_unpack_q8(c.desc, 0, B.MTS_BF16, dev(np.concatenate([x.reshape(-1) for x in hist]), dtype), *segs.args(), b.meta)
        qi, ki, vi = (qkv, qkv[:, Hq:], qkv[:, Hq + H:]) if s else (dev(q, dtype), dev(k, dtype), dev(v, dtype))
        qo = torch.empty(n, Hq, D, dtype=torch.bfloat16, device=DEV)
        ko = ki if s else torch.empty(n, H, D, dtype=torch.bfloat16, device=DEV)      # in place where they lie apart
        desc = mts.QkDesc(B.MTS_BF16, Hq, H, D, s, s, 0, s, 0, 0, B.MTS_NORM_RMS, 1e-6, freqs.data_ptr(), D, B.MTS_ROPE_HALVES)
        mts.mts_qk_norm_rope(desc, qi, ki, qo, ko, b.meta)
        mts.mts_kv_append_q8(c.desc, 0, B.MTS_BF16, ko, vi, b.meta, s, s)
        out = torch.empty_like(qo)
        nb = mts.mts_attn_q8_workspace_bytes(c.desc, Hq, b.meta)
        ws = torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV)
        mts.mts_attn_incremental_q8(c.desc, 0, B.MTS_BF16, Hq, qo, out, b.meta, 0.0, ws, nb)
        back = torch.empty(segs.total_tokens * 2 * H * D, dtype=torch.bfloat16, device=DEV)
        mts.mts_kv_pack_q8(c.desc, 0, B.MTS_BF16, back, *segs.args(), b.meta)
        torch.cuda.synchronize()
        image = c.layer_bytes(0)[torch.from_numpy(ids if c is small.cache else far).long().to(DEV)]
        got.append([host(qo), host(out), host(back), image.cpu().numpy()])
    for a, b in zip(*got):
        np.testing.assert_array_equal(a, b)


def test_the_same_run_twice_and_calls_side_by_side():
    rng = np.random.default_rng(52)
    H, G, D, S = 2, 2, 64, 16
    s = Step(52, H, D, S, [45, 200], [1, 1], "bf16")
    a, b = rows(rng, (2, 45, H, D), "bf16"), rows(rng, (2, 200, H, D), "bf16")
    runs, data = [(0, 0, 45), (1, 0, 200), (0, 0, 45), (1, 10, 33)], [a, b, a, b[:, 10:43]]
    s.unpack(runs, data)
    R.store(s.image, s.w.user_pages(0), S, 0, a)
    R.store(s.image, s.w.user_pages(1), S, 0, b)
    np.testing.assert_array_equal(s.pool(), s.image)
    for got, x in zip(s.pack(runs), data):
        np.testing.assert_array_equal(host(got), R.quantise(x)[2])
    # calls of two pools on two streams at once, each with a workspace of its own
    steps = [Step(53 + i, H, D, S, p, n, "bf16") for i, (p, n) in enumerate((([5000, 30], [1, 2]), ([300, 2000], [150, 1])))]
    work = []
    for t in steps:
        t.fill_prefixes(rng)
        k, v, q = (dev(rows(rng, (t.w.total_new, h, D), "bf16"), "bf16") for h in (H, H, H * G))
        t.append(k, v)
        nb = mts.mts_attn_q8_workspace_bytes(t.cache.desc, H * G, t.batch.meta)
        work.append((q, torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV), nb, torch.cuda.Stream(), t.attention(q, G)))
    outs = [torch.zeros_like(w[0]) for w in work]
    torch.cuda.synchronize()
    for _ in range(20):
        for t, (q, ws, nb, stream, _), out in zip(steps, work, outs):
            mts.mts_attn_incremental_q8(t.cache.desc, 0, B.MTS_BF16, H * G, q, out, t.batch.meta, 0.0, ws, nb, stream)
    torch.cuda.synchronize()
    for (_, _, _, _, alone), out in zip(work, outs):
        np.testing.assert_array_equal(host(out), alone)

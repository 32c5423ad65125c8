"""The 8-bit pool and the norm + rotation on the host: layout, workspace query, refusals; no GPU needed, every refused call
fails before anything is launched."""
import numpy as np
import pytest

import paper_2604_22881_amd as mts
import q8_reference as R
from paper_2604_22881_amd import binding as B

FAKE = 0x10000          # aligned, never dereferenced: validation fails first
ANY = dict(stream=0)


def _desc(**kw):
    d = dict(pool=FAKE, layer_stride_bytes=1 << 20, dtype=B.MTS_E4M3, num_layers=2, num_pages=8, page_size=16, num_heads=4, head_dim=64)
    d.update(kw)
    return B.CacheDesc(**d)


def _meta(**kw):
    d = dict(batch=2, page_indptr=FAKE, page_indices=FAKE, prefix_lens=FAKE, new_indptr=FAKE, total_new=10, max_new=8,
             max_total_len=100, total_pages=8)
    d.update(kw)
    return B.BatchMeta(**d)


def _qk(**kw):
    d = dict(dtype=B.MTS_BF16, num_q_heads=8, num_k_heads=4, head_dim=64, q_token_stride=0, k_token_stride=0, q_out_token_stride=0,
             k_out_token_stride=0, q_weight=FAKE, k_weight=FAKE, norm=B.MTS_NORM_RMS, eps=1e-6, freqs=FAKE, rot_dim=64,
             pairs=B.MTS_ROPE_HALVES)
    d.update(kw)
    return B.QkDesc(**d)


def _code(fn, *args, **kw):
    with pytest.raises(mts.MtsError) as e:
        fn(*args, **kw)
    assert str(e.value)
    return e.value.code


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("S", [16, 32, 64])
def test_layout_is_the_stated_one_and_a_bijection(D, S):
    H = 3
    d = _desc(page_size=S, num_heads=H, head_dim=D)
    assert mts.mts_page_bytes(d) == 2 * H * S * (D + 1)
    seen = []
    for kv in (0, 1):
        for h in range(H):
            for s in range(S):
                row = [mts.mts_elem_offset(d, kv, h, s, x) for x in range(D)]
                assert row == [R.code_offset(kv, h, s, x, S, D) for x in range(D)]
                e = mts.mts_q8_exp_offset(d, kv, h, s)
                assert e == R.exp_offset(kv, h, s, S, D)
                seen += row + [e]
    assert sorted(seen) == list(range(2 * H * S * (D + 1)))


def test_offsets_are_refused_out_of_range():
    d = _desc()
    for args in [(2, 0, 0, 0), (0, 4, 0, 0), (0, 0, 16, 0), (0, 0, 0, 64), (-1, 0, 0, 0)]:
        assert _code(mts.mts_elem_offset, d, *args) == B.MTS_ERR_INVALID_ARG
    for args in [(2, 0, 0), (0, 4, 0), (0, 0, 16), (0, -1, 0)]:
        assert _code(mts.mts_q8_exp_offset, d, *args) == B.MTS_ERR_INVALID_ARG
    assert _code(mts.mts_q8_exp_offset, _desc(dtype=B.MTS_BF16), 0, 0, 0) == B.MTS_ERR_UNSUPPORTED


def _calls(d, m, t=B.MTS_BF16, ptr=FAKE, layer=0):
    return [
        lambda: mts.mts_kv_append_q8(d, layer, t, ptr, ptr, m, **ANY),
        lambda: mts.mts_kv_unpack_q8(d, layer, t, ptr, 2, FAKE, FAKE, FAKE, 4, m, **ANY),
        lambda: mts.mts_kv_pack_q8(d, layer, t, ptr, 2, FAKE, FAKE, FAKE, 4, m, **ANY),
        lambda: mts.mts_attn_incremental_q8(d, layer, t, 8, ptr, ptr, m, workspace=FAKE, workspace_bytes=1 << 40, **ANY),
    ]


@pytest.mark.parametrize("change,code", [
    (dict(dtype=B.MTS_BF16), B.MTS_ERR_UNSUPPORTED), (dict(dtype=7), B.MTS_ERR_UNSUPPORTED), (dict(head_dim=96), B.MTS_ERR_UNSUPPORTED),
    (dict(page_size=48), B.MTS_ERR_UNSUPPORTED), (dict(num_heads=0), B.MTS_ERR_INVALID_ARG), (dict(pool=0), B.MTS_ERR_INVALID_ARG),
    (dict(pool=FAKE + 16), B.MTS_ERR_INVALID_ARG), (dict(layer_stride_bytes=8 * 2 * 4 * 16 * 65 - 256), B.MTS_ERR_SHAPE),
    (dict(layer_stride_bytes=(1 << 20) + 16), B.MTS_ERR_INVALID_ARG), (dict(num_pages=0), B.MTS_ERR_INVALID_ARG)])
def test_bad_descriptors_are_refused(change, code):
    for call in _calls(_desc(**change), _meta()):
        assert _code(call) == code


def test_bad_arguments_are_refused():
    d = _desc()
    for call in _calls(d, _meta(), layer=2) + _calls(d, _meta(), ptr=None) + _calls(d, _meta(), ptr=FAKE + 8) + _calls(d, _meta(batch=-1)):
        assert _code(call) == B.MTS_ERR_INVALID_ARG
    for call in _calls(d, _meta(), t=B.MTS_E4M3) + _calls(d, _meta(), t=9):
        assert _code(call) == B.MTS_ERR_UNSUPPORTED
    for call in _calls(d, _meta(page_indices=0)):
        assert _code(call) == B.MTS_ERR_INVALID_ARG
    # rows that overlap, or whose stride is no multiple of 16 bytes
    append = lambda **kw: _code(mts.mts_kv_append_q8, d, 0, B.MTS_BF16, FAKE, FAKE, _meta(), **ANY, **kw)
    assert append(k_token_stride=4 * 64 - 8) == B.MTS_ERR_SHAPE
    assert append(v_token_stride=-4 * 64) == B.MTS_ERR_SHAPE
    assert append(v_token_stride=4 * 64 + 4) == B.MTS_ERR_INVALID_ARG
    attn = lambda heads=8, **kw: _code(mts.mts_attn_incremental_q8, d, 0, B.MTS_BF16, heads, FAKE, FAKE, _meta(), **ANY, **kw)
    assert attn(heads=6) == B.MTS_ERR_SHAPE and attn(heads=0) == B.MTS_ERR_INVALID_ARG and attn(heads=1 << 16) == B.MTS_ERR_INVALID_ARG
    for s in (-1.0, float("nan"), float("inf")):
        assert attn(sm_scale=s) == B.MTS_ERR_INVALID_ARG
    assert _code(mts.mts_kv_unpack_q8, d, 0, B.MTS_BF16, FAKE, 1, FAKE, FAKE, FAKE, 4, _meta(batch=0, total_new=0, max_new=0), **ANY) == B.MTS_ERR_SHAPE


def test_the_other_calls_refuse_the_8_bit_pool():
    d, m = _desc(), _meta()
    assert _code(mts.mts_kv_append, d, 0, FAKE, FAKE, m, stream=0) == B.MTS_ERR_UNSUPPORTED
    assert _code(mts.mts_attn_workspace_bytes, d, m) == B.MTS_ERR_UNSUPPORTED
    assert _code(mts.mts_attn_incremental, d, 0, FAKE, FAKE, m, workspace=FAKE, workspace_bytes=1 << 40, stream=0) == B.MTS_ERR_UNSUPPORTED
    assert _code(mts.mts_kv_pack, d, 0, FAKE, 2, FAKE, FAKE, FAKE, 4, m, stream=0) == B.MTS_ERR_UNSUPPORTED


def test_empty_calls_do_nothing():
    d, none = _desc(), _meta(batch=0, total_new=0, max_new=0, total_pages=0)
    no_rows = _meta(total_new=0, max_new=0)
    for m in (none, no_rows):
        assert mts.mts_kv_append_q8(d, 0, B.MTS_F32, None, None, m, **ANY) == 0
        assert mts.mts_attn_incremental_q8(d, 0, B.MTS_F32, 4, None, None, m, **ANY) == 0
        assert mts.mts_attn_q8_workspace_bytes(d, 4, m) == 0
        assert mts.mts_qk_norm_rope(_qk(), None, None, None, None, m, **ANY) == 0
    assert mts.mts_kv_pack_q8(d, 0, B.MTS_F32, None, 0, None, None, None, 4, _meta(), **ANY) == 0
    assert mts.mts_kv_unpack_q8(d, 0, B.MTS_F32, None, 3, FAKE, FAKE, FAKE, 0, _meta(), **ANY) == 0


def test_workspace_is_asked_for_where_the_keys_are_cut_and_insisted_on():
    d = _desc(num_heads=8, head_dim=128)
    whole = _meta(batch=2, total_new=2, max_new=1, max_total_len=200, total_pages=20)
    assert mts.mts_attn_q8_workspace_bytes(d, 32, whole) == 0
    cut = _meta(batch=1, total_new=1, max_new=1, max_total_len=100000, total_pages=6300)
    need = mts.mts_attn_q8_workspace_bytes(d, 32, cut)
    assert 0 < need < 1 << 30
    call = lambda ws, n: _code(mts.mts_attn_incremental_q8, d, 0, B.MTS_BF16, 32, FAKE, FAKE, cut, workspace=ws, workspace_bytes=n, **ANY)
    assert call(None, 0) == call(FAKE, need - 1) == call(FAKE + 16, need) == B.MTS_ERR_WORKSPACE


def test_calls_beyond_the_launch_are_refused():
    d = _desc(num_heads=8)
    huge = _meta(batch=65535, total_new=1 << 30, max_new=1 << 20, max_total_len=1 << 20, total_pages=1 << 26)
    assert _code(mts.mts_attn_q8_workspace_bytes, d, 8, huge) == B.MTS_ERR_UNSUPPORTED
    assert _code(mts.mts_attn_q8_workspace_bytes, d, 8, _meta(max_total_len=(1 << 30) + 1)) == B.MTS_ERR_UNSUPPORTED
    assert _code(mts.mts_qk_norm_rope, _qk(num_q_heads=64), FAKE, FAKE, FAKE, FAKE,
                 _meta(batch=1, total_new=1 << 27, max_new=1 << 27, max_total_len=1 << 27), **ANY) == B.MTS_ERR_UNSUPPORTED


@pytest.mark.parametrize("change,code", [
    (dict(dtype=B.MTS_E4M3), B.MTS_ERR_UNSUPPORTED), (dict(head_dim=80), B.MTS_ERR_UNSUPPORTED), (dict(num_q_heads=0), B.MTS_ERR_INVALID_ARG),
    (dict(num_k_heads=70000), B.MTS_ERR_INVALID_ARG), (dict(norm=2), B.MTS_ERR_UNSUPPORTED), (dict(pairs=2), B.MTS_ERR_UNSUPPORTED),
    (dict(eps=-1.0), B.MTS_ERR_INVALID_ARG), (dict(eps=float("nan")), B.MTS_ERR_INVALID_ARG), (dict(rot_dim=72), B.MTS_ERR_SHAPE),
    (dict(rot_dim=12), B.MTS_ERR_SHAPE), (dict(rot_dim=-8), B.MTS_ERR_SHAPE), (dict(freqs=0), B.MTS_ERR_INVALID_ARG),
    (dict(freqs=FAKE + 4), B.MTS_ERR_INVALID_ARG), (dict(q_weight=FAKE + 8), B.MTS_ERR_INVALID_ARG),
    (dict(q_token_stride=500), B.MTS_ERR_SHAPE), (dict(k_out_token_stride=260), B.MTS_ERR_INVALID_ARG)])
def test_bad_norm_rope_descriptors_are_refused(change, code):
    assert _code(mts.mts_qk_norm_rope, _qk(**change), FAKE, FAKE, FAKE, FAKE, _meta(), **ANY) == code


def test_bad_norm_rope_pointers_are_refused():
    for at in range(4):
        for bad in (None, FAKE + 8):
            ptrs = [FAKE] * 4
            ptrs[at] = bad
            assert _code(mts.mts_qk_norm_rope, _qk(), *ptrs, _meta(), **ANY) == B.MTS_ERR_INVALID_ARG
    assert _code(mts.mts_qk_norm_rope, _qk(), FAKE, FAKE, FAKE, FAKE, _meta(new_indptr=0), **ANY) == B.MTS_ERR_INVALID_ARG
    with pytest.raises(mts.MtsError):
        mts.mts_qk_norm_rope(None, FAKE, FAKE, FAKE, FAKE, _meta(), **ANY)


def test_reference_rounding_on_known_rows():
    """The stored form's corners, by hand: 464 rounds to the code 448, what lies above takes the next exponent; ties go to even."""
    row = lambda *v: np.array(list(v) + [0.0] * (32 - len(v)))
    code, e, val = R.quantise(row(448.0, 1.0))
    assert e == 0 and val[0] == 448.0 and code[0] == 0x7E
    code, e, val = R.quantise(row(464.0, 1.0))
    assert e == 0 and val[0] == 448.0
    code, e, val = R.quantise(row(465.0, 1.0))
    assert e == 1 and val[0] == 480.0                # 232.5 * 2: rounds to 240
    code, e, val = R.quantise(row(256.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -5.0))
    assert e == 0 and val[1] == 16.0 and val[2] == 20.0 and val[3] == 0.0 and val[4] == 2.0 ** -8 and val[5] == -5.0
    code, e, val = R.quantise(row(np.inf, 3.0, np.nan))
    assert code[0] == code[2] == 0x7F and e == -7 and val[1] == 3.0
    code, e, val = R.quantise(row(1e30, 1.0))
    assert e == 60 and val[0] == 448.0 * 2.0 ** 60 and val[1] == 0.0
    code, e, val = R.quantise(row(1e-25))
    assert e == -60 and val[0] == 0.0
    x = np.random.default_rng(0).standard_normal((500, 64)) * 2.0 ** np.random.default_rng(1).integers(-50, 50, (500, 1))
    _, e, val = R.quantise(x)
    again = R.quantise(val)
    assert (again[1] == e).all() and (again[0] == R.quantise(x)[0]).all() and (again[2] == val).all()
    assert (np.abs(val - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** (e[:, None] - 10.0))).all()

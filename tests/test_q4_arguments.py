"""Host-side refusals of the calls over a cache in 4 bits and of the rotating append: nothing reaches a GPU."""
import ctypes as C

import pytest
import torch

BIG = 1 << 40


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _params(csp, **kw):
    args = dict(batch=2, n_q_heads=8, n_kv_heads=4, head_dim=128, window=1, recent=0, max_len=512, out_capacity=512)
    args.update(kw)
    return csp.Params(**args)


def _tensor(csp, ptr=4096, rows=512, heads=4, d=128):
    return csp.CTensor(ptr, heads * rows * d, rows * d, d)


def _cache(csp, d=128, H=4, R=128, codes=None, scales=None):
    return csp.CQ4Cache(codes or csp.CTensor(4096, H * R * d // 2, R * d // 2, d // 2), scales or csp.CTensor(8192, H * R * 2, R * 2, 2))


def _rope(csp, **kw):
    args = dict(cos_sin=4096, row_stride=128, table_rows=100, rope_dim=128, interleaved=0, positions=None, pos_stride_b=0)
    args.update(kw)
    return csp.CRope(**args)


# of codes and scales: what no kernel is written for (wrong addresses, strides that are no multiple of 16 bytes, rows with gaps) ...
ODD = [dict(codes=(4104, 32768, 8192, 64)), dict(codes=(4096, 32776, 8192, 64)), dict(codes=(4096, 32768, 8200, 64)), dict(codes=(4096, 32768, 8192, 128)),
       dict(scales=(8196, 1024, 256, 2)), dict(scales=(8192, 1020, 256, 2)), dict(scales=(8192, 1024, 260, 2)), dict(scales=(8192, 1024, 256, 4)),
       dict(codes=(4096, -32768, 8192, 64)), dict(scales=(8192, 1024, -256, 2))]
# ... and, where they are written, rows that share memory
SHARED = [dict(codes=(4096, 32768, 4096, 64)), dict(codes=(4096, 0, 8192, 64)), dict(scales=(8192, 1024, 128, 2)), dict(scales=(8192, 0, 256, 2))]


def _edited(csp, edit):
    return _cache(csp, **{k: csp.CTensor(*v) for k, v in edit.items()})


def test_struct_layouts_match_the_header(csp):
    assert C.sizeof(csp.CRope) == 8 + 8 + 3 * 4 + 4 + 8 + 8
    assert C.sizeof(csp.CQ4Cache) == 64


def _ref(x):
    return None if x is None else C.byref(x)


def _attn(csp, p, max_new=4, q=None, K=0, V=0, out=None, pages=0, rows=256, mods=None, ws=256, n=BIG):
    cp = p.c()
    K, V = (_cache(csp, d=p.head_dim) if x == 0 else x for x in (K, V))
    pages = csp.CPages(256, 4, 128, 9) if pages == 0 else pages
    q, out = q or _tensor(csp, rows=4, heads=8), out or _tensor(csp, rows=4, heads=8)
    return csp.lib().csp_chunk_attn_q4_paged(C.byref(cp), max_new, q, _ref(K), _ref(V), _ref(pages), rows, None, _ref(mods), out, None, ws, n, None)


def _append(csp, p, max_new=1, kn=None, vn=None, rope=0, q=None, q_out=None, K=0, V=0, pages=0, rows=256, out=256, ws=256, n=BIG, four=True):
    cp, t, none = p.c(), _tensor(csp, rows=max(max_new, 1), d=p.head_dim), csp.CTensor(None, 0, 0, 0)
    rope = _rope(csp) if rope == 0 else rope
    pages = csp.CPages(256, 4, 128, 9) if pages == 0 else pages
    front = (C.byref(cp), max_new, kn or t, vn or t, None, 0, _ref(rope), q or none, q_out or none)
    back = (_ref(pages), rows, out, ws, n, None)
    if four:
        K, V = (_cache(csp, d=p.head_dim) if x == 0 else x for x in (K, V))
        return csp.lib().csp_append_q4_paged(*front, _ref(K), _ref(V), *back)
    K, V = (_tensor(csp, rows=128, d=p.head_dim) if x == 0 else x for x in (K, V))
    return csp.lib().csp_append_rope_paged(*front, K, V, *back)


def _load(csp, p, max_rows=4, K=0, V=0, pages=0, rows=256, k_out=None, v_out=None, ws=256, n=BIG):
    cp, t = p.c(), _tensor(csp, rows=4, d=p.head_dim)
    K, V = (_cache(csp, d=p.head_dim) if x == 0 else x for x in (K, V))
    pages = csp.CPages(256, 4, 128, 9) if pages == 0 else pages
    return csp.lib().csp_load_q4_paged(C.byref(cp), _ref(K), _ref(V), _ref(pages), None, rows, max_rows, k_out or t, v_out or t, ws, n, None)


def test_attention_refusals(csp):
    p = _params(csp)
    null, odd = csp.CTensor(None, 1, 1, 1), _tensor(csp, ptr=4098)
    assert _attn(csp, p, max_new=-1) == csp.ERR_INVALID_ARG
    for name in ("q", "out"):
        assert _attn(csp, p, **{name: null}) == csp.ERR_INVALID_ARG
        assert _attn(csp, p, **{name: odd}) == csp.ERR_UNSUPPORTED
    for name in ("K", "V"):
        assert _attn(csp, p, **{name: None}) == csp.ERR_INVALID_ARG
        for part in ("codes", "scales"):
            assert _attn(csp, p, **{name: _cache(csp, **{part: null})}) == csp.ERR_INVALID_ARG
        for edit in ODD:
            assert _attn(csp, p, **{name: _edited(csp, edit)}) == csp.ERR_UNSUPPORTED, edit
    assert _attn(csp, p, rows=None) == csp.ERR_INVALID_ARG and _attn(csp, p, pages=None) == csp.ERR_INVALID_ARG
    for pages in ((256, 4, 64, 9), (256, 4, 128, 0), (256, 0, 128, 9), (None, 4, 128, 9), (256, 3, 128, 9)):
        assert _attn(csp, p, pages=csp.CPages(*pages)) == csp.ERR_INVALID_ARG
    for cap in (-1.0, float("nan"), 1e-7, 1001.0):
        assert _attn(csp, p, mods=csp.CScoreMods(softcap=cap)) == csp.ERR_INVALID_ARG
    need = csp.lib().csp_chunk_q4_workspace_bytes(C.byref(p.c()), 4)
    assert need >= 256 and _attn(csp, p, n=need - 1) == csp.ERR_WORKSPACE
    assert _attn(csp, p, ws=None) == csp.ERR_WORKSPACE and _attn(csp, p, ws=264) == csp.ERR_WORKSPACE
    assert _attn(csp, p, out=csp.CTensor(4096, 8 * 4 * 128, 4 * 128, 0)) == csp.ERR_UNSUPPORTED       # outputs that share memory


@pytest.mark.parametrize("kw,max_new", [(dict(dtype=1, head_dim=64), 4), (dict(head_dim=256), 4), (dict(n_q_heads=64), 4), (dict(out_capacity=(1 << 30) + 1), 4),
                                        (dict(), 1 << 24), (dict(batch=16383, out_capacity=1 << 30), 1), (dict(), -1)])
def test_shapes_that_are_refused_have_no_workspace(csp, kw, max_new):
    if "dtype" in kw:
        kw = dict(kw, dtype=csp.F32)
    p = _params(csp, **kw)
    assert csp.lib().csp_chunk_q4_workspace_bytes(C.byref(p.c()), max_new) == 0
    with pytest.raises(csp.CspError):
        csp.new_chunk_q4_workspace(p, max_new, device="cpu")
    assert _attn(csp, p, max_new=max_new, K=_cache(csp), V=_cache(csp), pages=csp.CPages(256, 1 << 23, 128, 9)) in (csp.ERR_UNSUPPORTED, csp.ERR_INVALID_ARG)


@pytest.mark.parametrize("batch,n_kv,cap", [(1, 1, 512), (1, 4, 1024), (1, 8, 33), (3, 2, 700), (2, 4, 20000), (64, 8, 300)])
def test_a_workspace_for_longer_chunks_is_enough_for_shorter_ones(csp, batch, n_kv, cap):
    for G in range(1, 9):
        p = _params(csp, batch=batch, n_q_heads=n_kv * G, n_kv_heads=n_kv, max_len=cap, out_capacity=cap)
        cp = p.c()
        sizes = [csp.lib().csp_chunk_q4_workspace_bytes(C.byref(cp), T) for T in list(range(0, 200)) + [511, 1024, 5000]]
        assert min(sizes) >= 256 and sizes == sorted(sizes), G


def test_append_refusals(csp):
    p = _params(csp)
    null, odd = csp.CTensor(None, 1, 1, 1), _tensor(csp, ptr=4104)
    q = _tensor(csp, rows=1, heads=8)
    for four in (True, False):
        def call(**kw):
            return _append(csp, p, four=four, **kw)
        assert call(max_new=-1) == csp.ERR_INVALID_ARG
        for name in ("kn", "vn"):
            assert call(**{name: null}) == csp.ERR_INVALID_ARG
            assert call(**{name: odd}) == csp.ERR_UNSUPPORTED
        assert call(rows=None) == csp.ERR_INVALID_ARG and call(out=None) == csp.ERR_INVALID_ARG and call(pages=None) == csp.ERR_INVALID_ARG
        assert call(pages=csp.CPages(256, 4, 64, 9)) == csp.ERR_INVALID_ARG
        assert call(ws=None) == csp.ERR_WORKSPACE and call(n=255) == csp.ERR_WORKSPACE
        assert call(q=q) == csp.ERR_INVALID_ARG                                          # queries that go nowhere
        assert call(q=q, q_out=odd) == csp.ERR_UNSUPPORTED and call(q=odd, q_out=q) == csp.ERR_UNSUPPORTED
        assert call(q=q, q_out=csp.CTensor(4096, 0, 128, 128)) == csp.ERR_UNSUPPORTED   # outputs that share memory
        for kw in (dict(cos_sin=None), dict(table_rows=0), dict(rope_dim=0), dict(rope_dim=24), dict(interleaved=2), dict(row_stride=64)):
            assert call(rope=_rope(csp, **kw)) == csp.ERR_INVALID_ARG, kw
        for kw in (dict(rope_dim=144, row_stride=144), dict(cos_sin=4100), dict(row_stride=130)):
            assert call(rope=_rope(csp, **kw)) == csp.ERR_UNSUPPORTED, kw
    assert _append(csp, p, rope=None, four=False) == csp.ERR_INVALID_ARG
    assert _append(csp, p, rope=None, q=q, q_out=q) == csp.ERR_INVALID_ARG              # nothing to rotate the queries by
    for name in ("K", "V"):
        assert _append(csp, p, **{name: None}) == csp.ERR_INVALID_ARG
        assert _append(csp, p, four=False, **{name: null}) == csp.ERR_INVALID_ARG
        assert _append(csp, p, four=False, **{name: odd}) == csp.ERR_UNSUPPORTED
        for part in ("codes", "scales"):
            assert _append(csp, p, **{name: _cache(csp, **{part: null})}) == csp.ERR_INVALID_ARG
        for edit in ODD + SHARED:
            assert _append(csp, p, **{name: _edited(csp, edit)}) == csp.ERR_UNSUPPORTED, edit
    assert _append(csp, _params(csp, dtype=csp.F32, head_dim=64)) == csp.ERR_UNSUPPORTED
    assert _append(csp, _params(csp, head_dim=256)) == csp.ERR_UNSUPPORTED


def test_load_refusals(csp):
    p = _params(csp)
    null, odd = csp.CTensor(None, 1, 1, 1), _tensor(csp, ptr=4104)
    assert _load(csp, p, max_rows=-1) == csp.ERR_INVALID_ARG and _load(csp, p, rows=None) == csp.ERR_INVALID_ARG
    assert _load(csp, p, K=None) == csp.ERR_INVALID_ARG and _load(csp, p, pages=None) == csp.ERR_INVALID_ARG
    for name in ("k_out", "v_out"):
        assert _load(csp, p, **{name: null}) == csp.ERR_INVALID_ARG
        assert _load(csp, p, **{name: odd}) == csp.ERR_UNSUPPORTED
        assert _load(csp, p, **{name: csp.CTensor(4096, 4 * 128, 128, 64)}) == csp.ERR_UNSUPPORTED
    for name in ("K", "V"):
        for part in ("codes", "scales"):
            assert _load(csp, p, **{name: _cache(csp, **{part: null})}) == csp.ERR_INVALID_ARG
        for edit in ODD:
            assert _load(csp, p, **{name: _edited(csp, edit)}) == csp.ERR_UNSUPPORTED, edit
    assert _load(csp, p, ws=None) == csp.ERR_WORKSPACE and _load(csp, p, n=255) == csp.ERR_WORKSPACE
    assert _load(csp, _params(csp, head_dim=256)) == csp.ERR_UNSUPPORTED


def test_empty_tensors_are_no_missing_ones(csp):
    null = csp.CTensor(None, 1, 1, 1)
    fine = (csp.OK,) if torch.cuda.is_available() else (csp.ERR_CUDA, csp.ERR_ARCH)
    none = _params(csp, batch=0)
    assert _attn(csp, _params(csp), max_new=0, q=null, out=null) in fine
    assert _attn(csp, none, q=null, out=null, rows=None, pages=csp.CPages(None, 4, 128, 9)) in fine
    assert _load(csp, _params(csp), max_rows=0, k_out=null, v_out=null) in fine
    assert _load(csp, none, k_out=null, v_out=null, rows=None, pages=csp.CPages(None, 4, 128, 9)) in fine
    for four in (True, False):
        assert _append(csp, none, kn=null, vn=null, rows=None, out=None, pages=csp.CPages(None, 4, 128, 9), four=four) in fine


def test_descriptors_check_their_tensors(csp):
    f = torch.zeros(10, 64)
    for bad in (f.double(), f[0], f.t()):
        with pytest.raises(AssertionError):
            csp.Rope(bad)
    for bad in (torch.zeros(2, 4), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32).t()):
        with pytest.raises(AssertionError):
            csp.Rope(f, positions=bad)
    codes, scales = torch.zeros(3, 2, 128, 32, dtype=torch.uint8), torch.zeros(3, 2, 128, 2, dtype=torch.bfloat16)
    csp.Q4Cache(codes, scales)
    for bad in ((codes.char(), scales), (codes, scales.half()), (codes[0], scales), (codes, scales[:2]), (codes, scales[..., :1])):
        with pytest.raises(AssertionError):
            csp.Q4Cache(*bad)

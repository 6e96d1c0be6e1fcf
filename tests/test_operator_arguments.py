"""Host-side refusals of chunk attention, appending and the page calls: nothing reaches a GPU, so they are the same with
and without one."""
import ctypes as C

import pytest
import torch


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


BIG = 1 << 40


def _chunk(csp, p, max_new=4, q=None, k=None, v=None, out=None, pages=None, paged=False, rows=256, mods=None, ws=256, ws_bytes=BIG, lse=None):
    cp = p.c()
    q = q or _tensor(csp, rows=4, heads=8)
    k, v, out = k or _tensor(csp), v or _tensor(csp), out or _tensor(csp, rows=4, heads=8)
    m = C.byref(mods) if mods is not None else None
    if paged:
        return csp.lib().csp_chunk_attn_paged(C.byref(cp), max_new, q, k, v, C.byref(pages) if pages else None, rows, None, m, out, lse, ws, ws_bytes, None)
    return csp.lib().csp_chunk_attn(C.byref(cp), max_new, q, k, v, rows, None, m, out, lse, ws, ws_bytes, None)


def test_struct_layouts_match_the_header(csp):
    assert C.sizeof(csp.CScoreMods) == 8 + 8 + 3 * 24
    assert C.sizeof(csp.CPageState) == 4 * 8 + 5 * 4 + 4


def test_chunk_attention_refusals(csp):
    p = _params(csp)
    null, odd = csp.CTensor(None, 1, 1, 1), _tensor(csp, ptr=4098)
    assert _chunk(csp, p, max_new=-1) == csp.ERR_INVALID_ARG
    for name in ("q", "k", "v", "out"):
        assert _chunk(csp, p, **{name: null}) == csp.ERR_INVALID_ARG
        assert _chunk(csp, p, **{name: odd}) == csp.ERR_UNSUPPORTED
    assert _chunk(csp, p, rows=None) == csp.ERR_INVALID_ARG
    assert _chunk(csp, p, ws=None) == csp.ERR_WORKSPACE
    assert _chunk(csp, p, ws=264) == csp.ERR_WORKSPACE
    assert _chunk(csp, p, ws_bytes=csp.chunk_workspace_bytes(p, 4) - 1) == csp.ERR_WORKSPACE
    assert _chunk(csp, _params(csp, dtype=csp.F32, head_dim=64)) == csp.ERR_UNSUPPORTED
    assert _chunk(csp, _params(csp, head_dim=256)) == csp.ERR_UNSUPPORTED
    assert _chunk(csp, _params(csp, n_q_heads=64)) == csp.ERR_UNSUPPORTED
    assert _chunk(csp, _params(csp, n_q_heads=9)) == csp.ERR_INVALID_ARG
    assert _chunk(csp, _params(csp, n=-1.0)) == csp.ERR_INVALID_ARG
    assert _chunk(csp, p, max_new=1 << 24) == csp.ERR_UNSUPPORTED        # tokens times heads are counted in 32 bits


def test_outputs_that_share_memory_are_refused(csp):
    p = _params(csp)
    for bad in (csp.CTensor(4096, 8 * 4 * 128, 4 * 128, 0), csp.CTensor(4096, 8 * 4 * 128, 0, 128), csp.CTensor(4096, 0, 4 * 128, 128),
                csp.CTensor(4096, 8 * 4 * 128, 4 * 128, 64)):
        assert _chunk(csp, p, out=bad) == csp.ERR_UNSUPPORTED


@pytest.mark.parametrize("cap", [-1.0, float("nan"), float("inf")])
def test_caps_that_are_no_cap_are_refused(csp, cap):
    assert _chunk(csp, _params(csp), mods=csp.CScoreMods(softcap=cap)) == csp.ERR_INVALID_ARG


@pytest.mark.parametrize("pages", [None, (256, 4, 64, 9), (256, 4, 128, 0), (256, 0, 128, 9), (None, 4, 128, 9), (256, 3, 128, 9), (256, 4, 0, 9)])
def test_page_tables_that_do_not_fit_are_refused(csp, pages):
    """No table, pages of half tiles, no pool, no entries, a table shorter than the capacity."""
    p = _params(csp)
    pg = csp.CPages(*pages) if pages else None
    assert _chunk(csp, p, paged=True, pages=pg) == csp.ERR_INVALID_ARG
    cp, t = p.c(), _tensor(csp)
    rc = csp.lib().csp_append_paged(C.byref(cp), 1, t, t, None, t, t, C.byref(pg) if pg else None, 256, 256, 256, BIG, None)
    assert rc == csp.ERR_INVALID_ARG


def test_append_refusals(csp):
    p = _params(csp)
    cp, t, odd, null = p.c(), _tensor(csp), _tensor(csp, ptr=4104), csp.CTensor(None, 1, 1, 1)
    pg = csp.CPages(256, 4, 128, 9)

    def call(max_new=1, kn=t, vn=t, k=t, v=t, rows=256, out=256, ws=256, n=BIG):
        return csp.lib().csp_append_paged(C.byref(cp), max_new, kn, vn, None, k, v, C.byref(pg), rows, out, ws, n, None)
    assert call(max_new=-1) == csp.ERR_INVALID_ARG
    for name in ("kn", "vn", "k", "v"):
        assert call(**{name: null}) == csp.ERR_INVALID_ARG
        assert call(**{name: odd}) == csp.ERR_UNSUPPORTED
    assert call(rows=None) == csp.ERR_INVALID_ARG and call(out=None) == csp.ERR_INVALID_ARG
    assert call(ws=None) == csp.ERR_WORKSPACE and call(n=255) == csp.ERR_WORKSPACE
    assert call(k=csp.CTensor(4096, 0, 512 * 128, 128)) == csp.ERR_UNSUPPORTED      # every page the same memory


def _state(csp, **kw):
    args = dict(page_table=256, held=256, refs=256, n_rows=256, batch=2, n_heads=4, max_pages=3, page_rows=128, n_pages=20)
    args.update(kw)
    return csp.CPageState(**args)


def test_page_call_refusals(csp):
    lib = csp.lib()
    calls = {
        "fork": lambda s, ws=256, n=BIG: lib.csp_pages_fork(C.byref(s), 256, 256, 1, ws, n, None),
        "reserve": lambda s, ws=256, n=BIG: lib.csp_pages_reserve(C.byref(s), None, 0, 256, 4, 256, ws, n, None),
        "free": lambda s, ws=256, n=BIG: lib.csp_pages_free(C.byref(s), ws, n, None),
        "compact": lambda s, ws=256, n=BIG: lib.csp_pages_compact(C.byref(s), 256, 4, 256, ws, n, None),
    }
    for name, call in calls.items():
        for field, value in (("batch", -1), ("n_heads", 0), ("max_pages", 0), ("page_rows", 0), ("n_pages", 0),
                             ("page_table", None), ("held", None), ("refs", None), ("n_rows", None)):
            assert call(_state(csp, **{field: value})) == csp.ERR_INVALID_ARG, (name, field)
        assert call(_state(csp, batch=1 << 20, max_pages=1 << 12)) == csp.ERR_UNSUPPORTED, name
        s = _state(csp)
        need = lib.csp_pages_workspace_bytes(C.byref(s))
        assert need >= 256 and call(s, n=need - 1) == csp.ERR_WORKSPACE and call(s, ws=None) == csp.ERR_WORKSPACE, name
        assert call(s, ws=300) == csp.ERR_WORKSPACE, name
    s = _state(csp)
    assert lib.csp_pages_fork(C.byref(s), None, 256, 1, 256, BIG, None) == csp.ERR_INVALID_ARG
    assert lib.csp_pages_fork(C.byref(s), 256, 256, -1, 256, BIG, None) == csp.ERR_INVALID_ARG
    assert lib.csp_pages_reserve(C.byref(s), None, 0, None, 4, 256, 256, BIG, None) == csp.ERR_INVALID_ARG
    assert lib.csp_pages_reserve(C.byref(s), None, 0, 256, 4, None, 256, BIG, None) == csp.ERR_INVALID_ARG
    assert lib.csp_pages_reserve(C.byref(s), None, 0, 260, 4, 256, 256, BIG, None) == csp.ERR_UNSUPPORTED
    assert lib.csp_pages_compact(C.byref(s), 256, -1, 256, 256, BIG, None) == csp.ERR_INVALID_ARG
    assert lib.csp_pages_workspace_bytes(C.byref(_state(csp, n_pages=0))) == 0


def test_page_copy_refusals(csp):
    p = _params(csp)
    cp, t, odd, null = p.c(), _tensor(csp), _tensor(csp, ptr=4104), csp.CTensor(None, 1, 1, 1)

    def call(k=t, v=t, n_pages=9, R=128, moves=256, most=4, n=256, ws=256, size=BIG):
        return csp.lib().csp_pages_copy(C.byref(cp), k, v, n_pages, R, moves, most, n, ws, size, None)
    assert call(k=null) == csp.ERR_INVALID_ARG and call(v=odd) == csp.ERR_UNSUPPORTED
    assert call(n_pages=0) == csp.ERR_INVALID_ARG and call(R=0) == csp.ERR_INVALID_ARG
    assert call(moves=None) == csp.ERR_INVALID_ARG and call(most=-1) == csp.ERR_INVALID_ARG and call(n=None) == csp.ERR_INVALID_ARG
    assert call(ws=None) == csp.ERR_WORKSPACE and call(size=255) == csp.ERR_WORKSPACE and call(moves=260) == csp.ERR_UNSUPPORTED
    assert call(k=csp.CTensor(4096, 1 << 20, 64, 128)) == csp.ERR_UNSUPPORTED        # heads overlap


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-GPU failure mode")
def test_without_a_gpu_the_calls_fail_loudly(csp):
    p = _params(csp)
    assert _chunk(csp, p) in (csp.ERR_CUDA, csp.ERR_ARCH)
    s = _state(csp)
    assert csp.lib().csp_pages_free(C.byref(s), 256, BIG, None) in (csp.ERR_CUDA, csp.ERR_ARCH)


def test_unsupported_sizes_have_no_workspace(csp):
    assert csp.chunk_workspace_bytes(_params(csp, n_q_heads=64), 4) == 0
    assert csp.chunk_workspace_bytes(_params(csp), -1) == 0
    assert csp.chunk_workspace_bytes(_params(csp), 4) >= 256


@pytest.mark.parametrize("cap", [1e-7, 1001.0, 1e30])
def test_caps_outside_the_accurate_range_are_refused(csp, cap):
    assert _chunk(csp, _params(csp), mods=csp.CScoreMods(softcap=cap)) == csp.ERR_INVALID_ARG


def test_capacities_past_the_row_index_are_refused(csp):
    p = _params(csp, out_capacity=(1 << 30) + 1)
    assert _chunk(csp, p) == csp.ERR_UNSUPPORTED
    assert _chunk(csp, p, paged=True, pages=csp.CPages(256, 1 << 23 | 1, 128, 9)) == csp.ERR_UNSUPPORTED


@pytest.mark.parametrize("batch,n_kv,cap", [(1, 1, 512), (1, 4, 1024), (1, 4, 4096), (1, 8, 1024), (3, 2, 700), (2, 4, 20000)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_workspace_for_longer_chunks_is_enough_for_shorter_ones(csp, batch, n_kv, cap, d):
    """Also where fewer tokens take another kernel with smaller tiles, whose work is cut into more parts."""
    for G in range(1, 9):
        p = _params(csp, batch=batch, n_q_heads=n_kv * G, n_kv_heads=n_kv, head_dim=d, max_len=cap, out_capacity=cap)
        sizes = [csp.chunk_workspace_bytes(p, T) for T in list(range(0, 300)) + [511, 1024, 5000]]
        falls = [(T, a, b) for T, (a, b) in enumerate(zip(sizes, sizes[1:])) if b < a]
        assert not falls, (G, falls[0])


@pytest.mark.parametrize("kw,max_new", [
    (dict(dtype="F32", head_dim=64), 4),
    (dict(head_dim=256), 4),
    (dict(out_capacity=(1 << 30) + 1), 4),
    (dict(), 1 << 24), (dict(), (1 << 31) - 1), (dict(n_q_heads=4), (1 << 24) + 1),
    (dict(batch=16383, out_capacity=1 << 30), 1),        # more key tiles than are counted in 30 bits
    (dict(batch=4000, out_capacity=1 << 20), 5000),
])
def test_shapes_that_the_attention_refuses_have_no_workspace(csp, kw, max_new):
    if "dtype" in kw:
        kw = dict(kw, dtype=csp.F32)
    p = _params(csp, **kw)
    assert csp.chunk_workspace_bytes(p, max_new) == 0
    with pytest.raises(csp.CspError):
        csp.new_chunk_workspace(p, max_new, device="cpu")
    assert _chunk(csp, p, max_new=max_new) == csp.ERR_UNSUPPORTED


def test_the_longest_chunk_has_a_workspace(csp):
    assert csp.chunk_workspace_bytes(_params(csp, n_q_heads=4), 1 << 24) >= csp.chunk_workspace_bytes(_params(csp, n_q_heads=4), 1 << 23) > 0


def test_empty_tensors_are_no_missing_ones(csp):
    """A chunk without tokens and a batch without sequences have no addresses to pass; what is needed still is."""
    null = csp.CTensor(None, 1, 1, 1)
    fine = (csp.OK,) if torch.cuda.is_available() else (csp.ERR_CUDA, csp.ERR_ARCH)
    assert _chunk(csp, _params(csp), max_new=0, q=null, out=null) in fine
    assert _chunk(csp, _params(csp, batch=0), q=null, k=null, v=null, out=null, rows=None) in fine
    assert _chunk(csp, _params(csp), max_new=0, q=null, out=null, ws=None) == csp.ERR_WORKSPACE
    assert _chunk(csp, _params(csp), q=null) == csp.ERR_INVALID_ARG
    lib, p = csp.lib(), _params(csp)
    cp, t, pg = p.c(), _tensor(csp), csp.CPages(256, 4, 128, 9)
    append = lambda cp, new, max_new, pool, rows: lib.csp_append_paged(  # noqa: E731
        C.byref(cp), max_new, new, new, None, pool, pool, C.byref(pg), rows, rows, 256, BIG, None)
    assert append(cp, null, 0, null, 256) == csp.ERR_INVALID_ARG
    assert append(cp, null, 0, t, None) == csp.ERR_INVALID_ARG
    assert append(cp, null, 1, t, 256) == csp.ERR_INVALID_ARG
    assert append(_params(csp, batch=0).c(), null, 1, t, None) in fine
    s = _state(csp, batch=0, page_table=None, held=None, n_rows=None)
    assert lib.csp_pages_free(C.byref(s), 256, BIG, None) in fine
    s = _state(csp, batch=0, page_table=None, held=None, n_rows=None, refs=None)
    assert lib.csp_pages_free(C.byref(s), 256, BIG, None) == csp.ERR_INVALID_ARG


def test_parameters_stay_plain_after_a_call(csp):
    """What a call keeps beside them is no attribute that a copy through __dict__ would hand to the constructor."""
    import copy
    import dataclasses
    import pickle
    p = _params(csp, n=2.0)
    fields = {f.name for f in dataclasses.fields(p)}
    first, size = bytes(p.c()), csp.chunk_workspace_bytes(p, 3)
    assert set(vars(p)) == fields
    own = p.c()
    own.head_dim = 64                                   # a caller's struct is the caller's
    assert bytes(p.c()) == first and csp.chunk_workspace_bytes(p, 3) == size
    for q in (csp.Params(**{**p.__dict__, "batch": 7}), dataclasses.replace(p, batch=7), copy.copy(p), copy.deepcopy(p), pickle.loads(pickle.dumps(p))):
        q.batch = 7
        csp.chunk_workspace_bytes(q, 3)
        assert q.c().batch == 7 and q.c().n == 2.0 and set(vars(q)) == fields
    assert bytes(p.c()) == first and p == _params(csp, n=2.0)
    p.n_q_heads = 4
    assert csp.chunk_workspace_bytes(p, 3) == csp.chunk_workspace_bytes(_params(csp, n_q_heads=4), 3) != size

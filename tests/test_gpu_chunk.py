"""csp_chunk_attn and csp_chunk_attn_paged against the definition in 64 bits: group sizes, head widths, chunk lengths from
one token to several tiles, ragged caches and chunks, score modifiers, hostile memory behind the rows, strides,
streams, graphs, and the chain prefill - prune - decode."""
import math

import numpy as np
import pytest
import torch

from chunk_util import assert_chunk_close, paged_copy, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def _case(seed, B, Hq, Hkv, d, cap, rows, new, gain=1.0, T=None):
    g = torch.Generator().manual_seed(seed)
    T = T or max(1, max(new))
    q = (torch.randn(B, T, Hq, d, generator=g) * gain).to(torch.bfloat16).transpose(1, 2)
    k = torch.randn(B, Hkv, cap, d, generator=g).to(torch.bfloat16)
    v = torch.randn(B, Hkv, cap, d, generator=g).to(torch.bfloat16)
    rows = torch.as_tensor(rows, dtype=torch.int32).reshape(B, Hkv)
    return q, k, v, rows, torch.as_tensor(new, dtype=torch.int32)


def _cuda(t):
    return None if t is None else t.cuda()


def _run(csp, case, page_rows=0, n=1.0, scale=0.0, status=0, want_rows=None, want_new=None, poison=True, lse=True,
         seed=0, check=True, what="", **mods):
    """One call, dense or paged, compared with the definition; returns (out, lse)."""
    q, k, v, rows, new = case
    B, Hq, T, d = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    p = csp.Params(B, Hq, Hkv, d, 1, 0, cap, cap, n=n, scale=scale)
    ws = csp.new_chunk_workspace(p, T)
    ws[256:] = 0xff                                     # scratch may hold anything (NaN as floats)
    m = None
    if mods:
        m = csp.ScoreMods(**{key: _cuda(x) if isinstance(x, torch.Tensor) else x for key, x in mods.items()})
    out = torch.full((B, T, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    z = torch.full((B, Hq, T), 7.0, device="cuda") if lse else None
    if page_rows:
        kp, vp, table = paged_copy(k.cuda(), v.cuda(), rows.clamp(0, cap), page_rows, seed)
        csp.chunk_attn_paged(p, q.cuda(), kp, vp, table, rows.cuda(), out, ws, n_new=new.cuda(), mods=m, lse=z)
    else:
        kd, vd = k.cuda(), v.cuda()
        if poison:
            for b in range(B):
                for h in range(Hkv):
                    kd[b, h, max(0, int(rows[b, h])):] = float("nan")
                    vd[b, h, max(0, int(rows[b, h])):] = float("inf")
        csp.chunk_attn(p, q.cuda(), kd, vd, rows.cuda(), out, ws, n_new=new.cuda(), mods=m, lse=z)
    assert csp.device_status(ws) == status
    used_rows = rows if want_rows is None else torch.as_tensor(want_rows).reshape(B, Hkv)
    used_new = new if want_new is None else torch.as_tensor(want_new)
    if check:
        assert_chunk_close(out, z, reference(q, k, v, used_rows, used_new, n, scale, **mods), used_new, what)
    for b in range(B):                                  # behind the last token nothing is written
        N = int(used_new[b])
        assert (out[b, :, N:] == 7.0).all() and (z is None or (z[b, :, N:] == 7.0).all())
    return out, z


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page_rows", [0, 128])
def test_one_token(csp, G, d, page_rows):
    _run(csp, _case(G + d, 2, 2 * G, 2, d, 333, [333, 200, 129, 1], [1, 1]), page_rows)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("d,page_rows", [(64, 0), (128, 128)])
def test_groups_fill_the_row_tiles(csp, G, d, page_rows):
    """Chunks around the number of tokens whose G heads fill one or two tiles of 128 rows."""
    per_tile = 128 // G
    for T in (per_tile - 1, per_tile, per_tile + 1, 2 * per_tile, 2 * per_tile + 3):
        T = max(T, 1)
        _run(csp, _case(T, 1, G, 1, d, 310, [310], [T], gain=1.5), page_rows, what=f"T={T}")


@pytest.mark.parametrize("rows,new", [((1, 1), (1, 1)), ((127, 128), (127, 128)), ((129, 130), (129, 1)), ((257, 640), (256, 255)),
                                      ((511, 385), (300, 17)), ((300, 0), (1, 0))])
@pytest.mark.parametrize("page_rows", [0, 128, 256])
def test_edges_of_tiles_and_ragged_chunks(csp, rows, new, page_rows):
    H = 2
    r = [[rows[0]] * H, [rows[1]] * H]
    r[0][1] = max(new[0], rows[0] - 3)                  # a pruned cache: heads keep different numbers of rows
    _run(csp, _case(sum(rows), 2, 2 * H, H, 128, 640, r, new), page_rows)


@pytest.mark.parametrize("n", [0.0, 1.0, 50.0])
@pytest.mark.parametrize("gain", [0.05, 1.0, 8.0])
def test_n_scale_and_peaked_rows(csp, n, gain):
    case = _case(5, 2, 4, 2, 64, 400, [400, 399, 130, 5], [33, 5], gain=gain)
    _run(csp, case, 0, n=n, scale=0.31)


@pytest.mark.parametrize("splits_case", [(1, 1, 1, 128, 8192, 1), (1, 4, 1, 64, 9000, 3), (1, 7, 1, 128, 5000, 40), (2, 2, 2, 128, 2500, 130)])
def test_long_caches_are_split_and_joined(csp, splits_case):
    B, Hq, Hkv, d, cap, T = splits_case
    rows = [[cap - 37 * (b + h) for h in range(Hkv)] for b in range(B)]
    _run(csp, _case(T, B, Hq, Hkv, d, cap, rows, [T] * B, gain=2.0), 128)


def test_many_short_units(csp):
    g = np.random.RandomState(3)
    rows = g.randint(1, 300, size=(24, 8))
    new = np.minimum(g.randint(1, 4, size=24), rows.min(1))
    _run(csp, _case(11, 24, 16, 8, 64, 300, rows, list(new)), 128)


# ---- score modifiers

def _slopes(Hq):
    return torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq)


@pytest.mark.parametrize("T,page_rows", [(1, 0), (5, 128), (200, 0), (150, 128)])
@pytest.mark.parametrize("cap_at", [5.0, 30.0, 50.0])
def test_cap(csp, T, page_rows, cap_at):
    # gain 20 drives the logits far beyond the cap, where its tanh is flat
    for gain in (1.0, 20.0):
        _run(csp, _case(T, 2, 4, 2, 128, 333, [333, 332, 250, 251], [T, T], gain=gain), page_rows, softcap=cap_at, what=f"gain {gain}")


@pytest.mark.parametrize("T,page_rows", [(1, 128), (9, 0), (140, 128)])
@pytest.mark.parametrize("positions", ["rows", "shared", "per head", "far"])
def test_distance_bias(csp, T, page_rows, positions):
    Hq, Hkv, cap = 6, 2, 700
    case = _case(T + 1, 2, Hq, Hkv, 64, cap, [700, 690, 300, 299], [T, T])
    g = torch.Generator().manual_seed(T)
    pos = None
    if positions == "shared":
        pos = torch.randint(1, 9, (2, cap), generator=g).cumsum(1).int()
    elif positions == "per head":
        pos = torch.randint(1, 9, (2, Hkv, cap), generator=g).cumsum(2).int()
    elif positions == "far":                            # positions that need all of 31 bits
        pos = (torch.randint(1, 3, (2, Hkv, cap), generator=g).cumsum(2) + (2 ** 31 - 1 - 2 * cap)).int()
    kw = {} if pos is None else {"positions": pos}
    _run(csp, case, page_rows, slopes=_slopes(Hq), **kw)


@pytest.mark.parametrize("page_rows", [0, 128])
@pytest.mark.parametrize("per_head", [False, True])
def test_documents(csp, page_rows, per_head):
    rows = [600, 580, 513, 400]
    case = _case(4, 2, 4, 2, 128, 600, rows, [300, 150])
    g = torch.Generator().manual_seed(9)
    doc = torch.sort(torch.randint(0, 5, (2, 2, 600) if per_head else (2, 600), generator=g), -1).values.int()
    _run(csp, case, page_rows, documents=doc, what="packed")
    mixed = torch.randint(-2, 3, doc.shape, generator=g).int()      # any order, any numbers
    _run(csp, case, page_rows, documents=mixed, what="mixed")
    alone = torch.arange(600).expand(doc.shape).contiguous().int()   # every row a document: each token sees itself
    _run(csp, case, page_rows, documents=alone, what="alone")


@pytest.mark.parametrize("prefix", [[[0, 0], [1, 1]], [[700, 700], [700, 700]], [[130, 129], [260, 5]], [[-5, 2000], [399, 400]]])
def test_prefix(csp, prefix):
    case = _case(6, 2, 4, 2, 64, 400, [400, 390, 260, 250], [260, 250])
    want = torch.tensor(prefix)
    for page_rows in (0, 128):
        _run(csp, case, page_rows, prefix=want.int())
    shared = want[:, :1].int().contiguous()
    _run(csp, case, 0, prefix=shared)


def test_all_modifiers_together(csp):
    Hq, Hkv, cap = 14, 2, 500
    g = torch.Generator().manual_seed(2)
    pos = torch.randint(1, 4, (2, Hkv, cap), generator=g).cumsum(2).int()
    doc = torch.sort(torch.randint(0, 3, (2, cap), generator=g), -1).values.int()
    pre = torch.tensor([[200, 10], [0, 333]]).int()
    for T in (1, 30, 170):
        case = _case(T, 2, Hq, Hkv, 128, cap, [500, 480, 333, 334], [T, min(T, 77)], gain=3.0)
        for page_rows in (0, 128):
            _run(csp, case, page_rows, n=2.0, softcap=15.0, slopes=_slopes(Hq), positions=pos, documents=doc, prefix=pre, what=f"T={T}")


# ---- what the device flags

def test_bad_counts_are_clamped_and_flagged(csp):
    case = _case(8, 2, 4, 2, 64, 200, [250, 200, -3, 40], [30, 99], T=50)
    _run(csp, case, 0, status=csp.DEV_BAD_LEN, want_rows=[200, 200, 0, 40], want_new=[30, 50], poison=False)


def test_more_new_tokens_than_rows_see_nothing(csp):
    """Tokens whose own row would be negative get zeros and a lse of -infinity, and the call is flagged; also with a
    prefix, which makes rows visible only to tokens that have one."""
    case = _case(9, 1, 2, 2, 64, 100, [5, 0], [9])
    _run(csp, case, 0, status=csp.DEV_BAD_LEN)
    _run(csp, case, 0, status=csp.DEV_BAD_LEN, prefix=torch.tensor([[3]]).int())


def test_a_page_outside_the_pool_reads_as_zeros(csp):
    q, k, v, rows, new = _case(10, 1, 2, 1, 128, 384, [384], [2])
    kp, vp, table = paged_copy(k.cuda(), v.cuda(), rows, 128, 1)
    p = csp.Params(1, 2, 1, 128, 1, 0, 384, 384)
    ws = csp.new_chunk_workspace(p, 2)
    for bad in (-1, kp.shape[0], 2 ** 31 - 1):
        t = table.clone()
        t[0, 1] = bad
        out = torch.zeros(1, 2, 2, 128, dtype=torch.bfloat16, device="cuda")
        csp.chunk_attn_paged(p, q.cuda(), kp, vp, t, rows.cuda(), out, ws)
        assert csp.device_status(ws) == csp.DEV_BAD_LEN
        k0, v0 = k.clone(), v.clone()
        k0[0, 0, 128:256] = 0
        v0[0, 0, 128:256] = 0
        assert_chunk_close(out, None, reference(q, k0, v0, rows, new), new)
    csp.chunk_attn_paged(p, q.cuda(), kp, vp, table, rows.cuda(), out, ws)
    assert csp.device_status(ws) == 0


# ---- how it is called

def test_strided_inputs_and_outputs(csp):
    """Caches in [B, rows, H, d] order, a query that is a slice of a wider projection, an output with gaps."""
    q, k, v, rows, new = _case(12, 2, 4, 2, 64, 150, [150, 140, 99, 98], [20, 7])
    p = csp.Params(2, 4, 2, 64, 1, 0, 150, 150)
    ws = csp.new_chunk_workspace(p, 20)
    qkv = torch.full((2, 20, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    qkv[:, :, :4] = q.transpose(1, 2).cuda()
    kv = torch.stack([k, v]).transpose(2, 3).contiguous().cuda()                 # [2, B, rows, H, d]
    wide = torch.full((2, 20, 4, 72), 3.0, dtype=torch.bfloat16, device="cuda")
    out = wide[..., :64].transpose(1, 2)
    csp.chunk_attn(p, qkv[:, :, :4].transpose(1, 2), kv[0].transpose(1, 2), kv[1].transpose(1, 2), rows.cuda(), out, ws,
                   n_new=new.cuda())
    assert csp.device_status(ws) == 0
    assert_chunk_close(out, None, reference(q, k, v, rows, new), new)
    assert (wide[..., 64:] == 3.0).all() and (wide[1, 7:] == 3.0).all()


def test_no_new_counts_means_all_of_them(csp):
    case = _case(13, 2, 2, 2, 64, 100, [100, 90, 80, 70], [11, 11])
    q, k, v, rows, new = case
    p = csp.Params(2, 2, 2, 64, 1, 0, 100, 100)
    ws = csp.new_chunk_workspace(p, 11)
    out = torch.zeros(2, 2, 11, 64, dtype=torch.bfloat16, device="cuda")
    csp.chunk_attn(p, q.cuda(), k.cuda(), v.cuda(), rows.cuda(), out, ws)
    assert_chunk_close(out, None, reference(q, k, v, rows, new), new)


def test_offsets_past_32_bits(csp):
    """A pool of more than 2^32 bytes and 2^31 elements per tensor, the sequence on its last pages."""
    H, d, R = 8, 128, 128
    n_pages = (2 ** 31) // (H * R * d) + 40
    q, k, v, rows, new = _case(14, 1, H, H, d, 300, [300] * H, [5])
    kp = torch.empty(n_pages, H, R, d, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty_like(kp)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3]], dtype=torch.int32, device="cuda")
    for i in range(3):
        rows_i = min(128, 300 - 128 * i)
        kp[int(table[0, i]), :, :rows_i] = k[0, :, 128 * i:128 * i + rows_i].cuda()
        vp[int(table[0, i]), :, :rows_i] = v[0, :, 128 * i:128 * i + rows_i].cuda()
    p = csp.Params(1, H, H, d, 1, 0, 300, 300)
    ws = csp.new_chunk_workspace(p, 5)
    out = torch.zeros(1, H, 5, d, dtype=torch.bfloat16, device="cuda")
    csp.chunk_attn_paged(p, q.cuda(), kp, vp, table, rows.cuda(), out, ws)
    assert csp.device_status(ws) == 0
    assert_chunk_close(out, None, reference(q, k, v, rows, new), new)


def test_results_repeat_exactly_and_do_not_depend_on_what_ran_before(csp):
    """The same call gives the same bits, also on a workspace that calls of other shapes have used."""
    case = _case(15, 3, 8, 2, 128, 3000, [[3000, 2900], [64, 1], [1500, 700]], [1, 1, 1])
    other = _case(16, 1, 8, 2, 128, 900, [[900, 880]], [200])
    q, k, v, rows, new = case
    p = csp.Params(3, 8, 2, 128, 1, 0, 3000, 3000)
    po = csp.Params(1, 8, 2, 128, 1, 0, 900, 900)
    ws = torch.zeros(max(csp.chunk_workspace_bytes(p, 1), csp.chunk_workspace_bytes(po, 200)), dtype=torch.uint8, device="cuda")
    dev = [t.cuda() for t in case]
    odev = [t.cuda() for t in other]
    outs = []
    for _ in range(4):
        out = torch.zeros(3, 8, 1, 128, dtype=torch.bfloat16, device="cuda")
        csp.chunk_attn(p, dev[0], dev[1], dev[2], dev[3], out, ws)
        outs.append(out)
        oo = torch.zeros(1, 8, 200, 128, dtype=torch.bfloat16, device="cuda")
        csp.chunk_attn(po, odev[0], odev[1], odev[2], odev[3], oo, ws)
    assert csp.device_status(ws) == 0
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    assert_chunk_close(outs[0], None, reference(q, k, v, rows, new), new)


def test_two_streams_and_a_graph(csp):
    """Calls on two streams at once with a workspace each; the same call captured and replayed on new inputs."""
    cases = [_case(20 + i, 2, 8, 4, 128, 1200, [[1200 - 100 * i, 900, 30, 1100], [7, 8, 9, 1000]], [3, 2]) for i in range(2)]
    p = csp.Params(2, 8, 4, 128, 1, 0, 1200, 1200)
    want = [reference(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for c in cases:
        work.append(([t.cuda() for t in c], csp.new_chunk_workspace(p, 3), torch.zeros(2, 8, 3, 128, dtype=torch.bfloat16, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(3):
        for st, (dev, ws, out) in zip(streams, work):
            with torch.cuda.stream(st):
                csp.chunk_attn(p, *dev[:4], out, ws, n_new=dev[4])
    torch.cuda.synchronize()
    for c, w, (dev, ws, out) in zip(cases, want, work):
        assert csp.device_status(ws) == 0
        assert_chunk_close(out, None, w, c[4])
    dev, ws, out = work[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        csp.chunk_attn(p, *dev[:4], out, ws, n_new=dev[4])
    for c, w in zip(cases[::-1], want[::-1]):
        for d, s in zip(dev, c):
            d.copy_(s)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert csp.device_status(ws) == 0
        assert_chunk_close(out, None, w, c[4])


def test_single_token_agrees_with_the_decode_call(csp):
    """One token per sequence is csp_decode_attn, up to the rounding of weights and result to bf16."""
    case = _case(30, 3, 14, 2, 128, 900, [[900, 850], [3, 700], [129, 128]], [1, 1, 1])
    q, k, v, rows, new = case
    out, _ = _run(csp, case)
    p = csp.Params(3, 14, 2, 128, 1, 0, 900, 900)
    ws = csp.new_decode_workspace(p)
    dec = torch.zeros(3, 14, 128, device="cuda")
    csp.decode_attn(p, q[:, :, 0].contiguous().cuda(), k.cuda(), v.cuda(), rows.cuda(), dec, ws)
    ref = reference(q, k, v, rows, new)
    tol = 2.0 ** -8 * ref[0].abs() + 2.0 ** -7 * ref[2]
    assert ((out.cpu().double() - dec[:, :, None].cpu().double()).abs() <= tol).all()


def test_log_sum_exp_feeds_the_prune(csp, oracle):
    """A prompt's last chunk leaves the log-sum-exp of its window rows; csp_prune_layer with it keeps what it keeps
    without (scores within their tolerance, index sets up to ties within it)."""
    import csp_synth as synth
    from parity_util import GpuRun, assert_index_sets_match, assert_scores_close, gpu_params, orc_params
    lay = [synth.interleaved_layout([30, 45, 200], 100), synth.interleaved_layout([60, 100], 150)]
    cfg = synth.small_config("chain", lay, 8, 2, 128, 32, 32, seed=3)
    q, k, v = synth.make_layer(cfg, 0, "cuda")
    lens = torch.from_numpy(cfg.seq_lens).cuda()
    T = 64                                              # the chunk: the window and the 32 tokens in front of it
    gen = torch.Generator(device="cuda").manual_seed(1)
    qc = torch.randn(2, 8, T, 128, device="cuda", generator=gen).to(torch.bfloat16)
    qc[:, :, T - 32:] = q
    pc = csp.Params(2, 8, 2, 128, 1, 0, cfg.max_len, cfg.max_len)
    rows = lens[:, None].expand(2, 2).contiguous()
    out = torch.zeros(2, 8, T, 128, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(2, 8, T, device="cuda")
    ws = csp.new_chunk_workspace(pc, T)
    csp.chunk_attn(pc, qc, k, v, rows, out, ws, lse=lse)
    assert csp.device_status(ws) == 0
    p = gpu_params(csp, cfg)
    run = GpuRun(csp, p, q, k, v, cfg.modality(), cfg.seq_lens, cfg.budgets)
    window = lse[:, :, T - 32:].contiguous()
    csp.prune_layer(p, run.q, k, v, run.mod, run.lens, run.bud, run.k_out, run.v_out, run.mod_out, run.n_out, run.ws, lse=window,
                    score_self=run.ss, score_cross=run.sc, keep_idx=run.idx)
    assert run.status() == 0
    ref = oracle.prune_layer(orc_params(oracle, cfg), q.cpu(), k.cpu(), v.cpu(), cfg.modality(), cfg.seq_lens, cfg.budgets)
    assert_scores_close(run.ss.cpu().numpy(), ref["score_self"], cfg.seq_lens, 32, "self")
    assert_scores_close(run.sc.cpu().numpy(), ref["score_cross"], cfg.seq_lens, 32, "cross")
    assert_index_sets_match(run.idx.cpu().numpy(), run.n_out.cpu().numpy(), ref, cfg.modality(), cfg.seq_lens, 32)


def test_random_launches(csp):
    """Seeded shapes over the whole range, dense and paged."""
    rng = np.random.RandomState(77)
    for trial in range(24):
        d = int(rng.choice([64, 128]))
        Hkv, G, B = int(rng.choice([1, 2, 3])), int(rng.randint(1, 9)), int(rng.randint(1, 4))
        cap = int(rng.randint(1, 900))
        rows = rng.randint(0, cap + 1, size=(B, Hkv))
        T = int(rng.choice([1, 2, 8, 40, 130]))
        new = [int(rng.randint(0, min(T, int(r.min())) + 1)) for r in rows]
        mods = {}
        if rng.rand() < 0.4:
            mods["softcap"] = float(rng.uniform(2, 60))
        if rng.rand() < 0.4:
            mods["slopes"] = _slopes(G * Hkv)
            if rng.rand() < 0.5:
                mods["positions"] = torch.from_numpy(np.cumsum(rng.randint(1, 5, size=(B, Hkv, cap)), 2).astype(np.int32))
        if rng.rand() < 0.4:
            mods["documents"] = torch.from_numpy(np.sort(rng.randint(0, 4, size=(B, cap)), 1).astype(np.int32))
        if rng.rand() < 0.4:
            mods["prefix"] = torch.from_numpy(rng.randint(0, cap + 1, size=(B, Hkv)).astype(np.int32))
        case = _case(trial, B, G * Hkv, Hkv, d, cap, rows, new, gain=float(rng.choice([0.5, 1.5, 4.0])), T=T)
        _run(csp, case, int(rng.choice([0, 128, 256])), n=float(rng.choice([0.0, 1.0])), seed=trial, what=f"trial {trial}", **mods)


# ---- logits far below zero

@pytest.mark.parametrize("T,rows,page_rows", [(1, 333, 0), (1, 6000, 128), (40, 6000, 0), (150, 333, 128)])
@pytest.mark.parametrize("n", [0.0, 1.0])
def test_logits_far_below_zero(csp, T, rows, page_rows, n):
    """Near -362 e^-o is not a float any more: without n the weights are still those of a softmax, with n they are zeros."""
    g = torch.Generator().manual_seed(T + rows)
    q = torch.full((1, T, 4, 128), 4.0).to(torch.bfloat16).transpose(1, 2)
    k = (-8.0 + torch.randint(-4, 5, (1, 2, rows, 128), generator=g) / 16.0).to(torch.bfloat16)
    v = torch.randn(1, 2, rows, 128, generator=g).to(torch.bfloat16)
    case = q, k, v, torch.full((1, 2), rows, dtype=torch.int32), torch.tensor([T], dtype=torch.int32)
    out, _ = _run(csp, case, page_rows, n=n)
    assert (out != 0).any() == (n == 0.0)


# ---- documents: items that are drawn one by one, and shares without any of the tokens' documents

@pytest.mark.parametrize("T", [20, 150])
def test_documents_of_many_units(csp, T):
    B, H, cap = 4, 160 if T == 20 else 80, 260
    g = np.random.RandomState(T)
    new = [T, 1, 0, T - 3]
    rows = np.maximum(g.randint(1, cap + 1, size=(B, H)), np.array(new)[:, None])
    case = _case(T, B, H, H, 64, cap, rows, new)
    doc = torch.from_numpy((np.arange(cap)[None, :] * 5 // cap + np.arange(B)[:, None]).astype(np.int32))
    first = _run(csp, case, 0, documents=doc)
    again = _run(csp, case, 0, check=False, documents=doc)
    for x, y in zip(first, again):
        assert torch.equal(x, y)


@pytest.mark.parametrize("T", [4, 200])
def test_shares_without_the_tokens_documents(csp, T):
    cap = 6000
    case = _case(T, 1, 4, 1, 128, cap, [cap - 1], [T])
    doc = (torch.arange(cap, dtype=torch.int32) // 1200)[None, :].contiguous()
    _run(csp, case, 128, documents=doc, what="the last of five")
    _run(csp, case, 0, documents=(doc == 4).int() * torch.tensor(7, dtype=torch.int32) + (doc == 1).int() * torch.tensor(7, dtype=torch.int32),
         what="the second and the last are one")


def test_documents_of_one_long_unit_among_many(csp):
    """More items than are shared out as a rule, one of them longer than everybody's share: it is cut all the same."""
    B, H, cap, T = 80, 4, 5000, 20
    rows = np.full((B, H), T, dtype=np.int64)
    rows[3, 1] = cap
    case = _case(T, B, H, H, 64, cap, rows, [T] * B)
    doc = (torch.arange(cap, dtype=torch.int32) % 3)[None, :].expand(B, cap).contiguous()
    _run(csp, case, 0, documents=doc)


@pytest.mark.parametrize("page_rows", [0, 256])
def test_ends_of_caches_under_load(csp, page_rows):
    """Tiles that end behind the last row, in many units at once and call after call: every call gives the first one's bits."""
    B, H, T, cap = 6, 32, 60, 1103
    g = np.random.RandomState(8)
    rows = g.randint(900, cap + 1, size=(B, H))
    new = [60, 41, 59, 18, 33, 60]
    q, k, v, rows, new = _case(T, B, H, H, 128, cap, rows, new)
    p = csp.Params(B, H, H, 128, 1, 0, cap, cap)
    ws, first = csp.new_chunk_workspace(p, T), None
    q, k, v, rows, new = (x.cuda() for x in (q, k, v, rows, new))
    kp, vp, table = paged_copy(k, v, rows, page_rows, 1) if page_rows else (None, None, None)
    for _ in range(60):
        out = torch.zeros(B, T, H, 128, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        if page_rows:
            csp.chunk_attn_paged(p, q, kp, vp, table, rows, out, ws, n_new=new)
        else:
            csp.chunk_attn(p, q, k, v, rows, out, ws, n_new=new)
        first = out if first is None else first
        assert torch.equal(out, first)
    few = slice(0, 2)                                   # (the definition is slow: two heads of it)
    ref = reference(q[:, few].cpu(), k[:, few].cpu(), v[:, few].cpu(), rows[:, few].cpu(), new.cpu())
    assert_chunk_close(first[:, few], None, ref, new.cpu())


# ---- where the tensors live, and what is captured

def test_tensors_on_another_device_are_refused(csp):
    q, k, v, rows, new = _case(40, 1, 4, 2, 64, 100, [100, 90], [3])
    p = csp.Params(1, 4, 2, 64, 1, 0, 100, 100)
    ws, out = csp.new_chunk_workspace(p, 3), torch.zeros(1, 4, 3, 64, dtype=torch.bfloat16, device="cuda")
    good = dict(q=q.cuda(), k=k.cuda(), v=v.cuda(), n_rows=rows.cuda(), out=out, ws=ws, n_new=new.cuda())
    for name in good:
        bad = dict(good, **{name: good[name].cpu()})
        with pytest.raises(ValueError):
            csp.chunk_attn(p, bad["q"], bad["k"], bad["v"], bad["n_rows"], bad["out"], bad["ws"], n_new=bad["n_new"])
    for m in (csp.ScoreMods(slopes=torch.ones(4)), csp.ScoreMods(documents=torch.zeros(1, 100, dtype=torch.int32)),
              csp.ScoreMods(prefix=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            csp.chunk_attn(p, good["q"], good["k"], good["v"], good["n_rows"], out, ws, n_new=good["n_new"], mods=m)


@pytest.mark.parametrize("T,B,H,cap", [(2, 2, 2, 6000), (40, 1, 2, 6000), (20, 4, 80, 260)])
def test_captured_calls_replay_on_new_inputs(csp, T, B, H, cap):
    """Cut items and their joining, few rows and many, and items drawn from a counter, each replayed twice."""
    doc = (torch.arange(cap, dtype=torch.int32) * 4 // cap)[None, :].expand(B, cap).contiguous().cuda()
    cases = [_case(50 + i, B, H, H, 64, cap, np.full((B, H), cap - 7 * i), [T] * B) for i in range(2)]
    p, dev = csp.Params(B, H, H, 64, 1, 0, cap, cap), [t.cuda() for t in cases[0]]
    ws, out = csp.new_chunk_workspace(p, T), torch.zeros(B, H, T, 64, dtype=torch.bfloat16, device="cuda")
    mods = csp.ScoreMods(documents=doc)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        csp.chunk_attn(p, *dev[:4], out, ws, n_new=dev[4], mods=mods)
    for c in cases[::-1]:
        for d, s in zip(dev, c):
            d.copy_(s)
        seen = []
        for _ in range(2):
            out.zero_()
            graph.replay()
            seen.append(out.clone())
        csp.chunk_attn(p, *dev[:4], out, ws, n_new=dev[4], mods=mods)
        assert csp.device_status(ws) == 0
        assert torch.equal(seen[0], out) and torch.equal(seen[1], out)
        two = slice(0, 2)
        ref = reference(c[0][:1, two], c[1][:1, two], c[2][:1, two], c[3][:1, two], c[4][:1], documents=doc[:1].cpu())
        assert_chunk_close(out[:1, two], None, ref, c[4][:1])


def test_one_workspace_for_chunks_of_all_lengths(csp):
    """Made for the longest chunk, used for that one, for the lengths around a change of kernel and for single tokens."""
    for Hq, Hkv, longest in ((28, 4, 3), (4, 4, 40), (16, 2, 300)):
        cap = 2000
        ws = csp.new_chunk_workspace(csp.Params(1, Hq, Hkv, 128, 1, 0, cap, cap), longest)
        for T in sorted({longest, 1, 2, min(longest, 17), min(longest, 16), min(longest, 11)}, reverse=True):
            q, k, v, rows, new = _case(T, 1, Hq, Hkv, 128, cap, [cap - 3 * h for h in range(Hkv)], [T])
            p = csp.Params(1, Hq, Hkv, 128, 1, 0, cap, cap)
            out = torch.zeros(1, Hq, T, 128, dtype=torch.bfloat16, device="cuda")
            csp.chunk_attn(p, q.cuda(), k.cuda(), v.cuda(), rows.cuda(), out, ws)
            assert csp.device_status(ws) == 0
            if T <= 17:
                assert_chunk_close(out, None, reference(q, k, v, rows, new), new, f"T={T}")


@pytest.mark.parametrize("B,T", [(2, 0), (0, 3), (0, 0)])
def test_nothing_to_do(csp, B, T):
    """Chunks without tokens and batches without sequences: empty tensors, which have no address."""
    p = csp.Params(B, 4, 2, 64, 1, 0, 256, 256)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    q, k, pool = torch.zeros(B, 4, T, 64, **bf), torch.zeros(B, 2, 256, 64, **bf), torch.zeros(5, 2, 128, 64, **bf)
    rows, new = torch.full((B, 2), 7, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    table = torch.zeros(B, 2, dtype=torch.int32, device="cuda")
    out, lse, ws = torch.zeros_like(q), torch.zeros(B, 4, T, device="cuda"), csp.new_chunk_workspace(p, T)
    csp.chunk_attn(p, q, k, k, rows, out, ws, lse=lse)
    csp.chunk_attn(p, q, k, k, rows, out, ws, n_new=new, mods=csp.ScoreMods(prefix=new))
    csp.chunk_attn_paged(p, q, pool, pool, table, rows, out, ws, n_new=new)
    assert csp.device_status(ws) == 0


# ---- positions far apart

@pytest.mark.parametrize("T,page_rows", [(3, 0), (3, 128), (200, 0), (200, 128)])
@pytest.mark.parametrize("gap", [2 ** 23 - 400, 2 ** 24, 2 ** 30])
def test_tokens_far_apart(csp, T, page_rows, gap):
    """A chunk whose first tokens lie `gap` positions in front of the others: exact distances up to 2^23, flagged beyond."""
    cap, Hq, Hkv = 300, 4, 2
    case = _case(T, 1, Hq, Hkv, 64, cap, [300, 299], [T])
    pos = torch.arange(cap, dtype=torch.int32)[None, :].repeat(1, 1)
    pos[:, cap - T // 2 - 2:] += gap
    fine = gap < 2 ** 23
    _run(csp, case, page_rows, status=0 if fine else csp.DEV_BAD_LEN, check=fine, slopes=_slopes(Hq), positions=pos)


@pytest.mark.parametrize("T", [1, 3, 200])
def test_cached_rows_far_from_the_tokens(csp, T):
    """Rows of a cache up to 2^30 positions in front of the chunk, and slopes so small that they still have a weight."""
    cap, Hq, Hkv = 400, 4, 2
    case = _case(T, 1, Hq, Hkv, 64, cap, [400, 399], [T])
    pos = torch.arange(cap, dtype=torch.int32)[None, :].repeat(1, 1)
    pos[:, 60:] += 2 ** 25 + 1
    pos[:, 130:] += 2 ** 30 - 3
    _run(csp, case, 0, slopes=torch.tensor([2.0 ** -30, 2.0 ** -29, 0.5, 0.01]), positions=pos)

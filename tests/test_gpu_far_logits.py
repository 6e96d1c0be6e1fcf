"""Without n (n = 0) the weights are those of a softmax, however far below zero the logits lie: near -362, where e^-o is not a float
any more, in the decode calls and in the three scoring kernels, with and without the rows' log-sum-exp supplied."""
import numpy as np
import pytest
import torch

import csp_synth as synth
from parity_util import GpuRun, assert_scores_close, gpu_params, orc_params

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def csp():
    from paper_2412_04652_b200 import binding
    binding.lib()
    return binding


def _keys(shape, seed, d):
    """Keys whose product with queries of sixteen and less lies around -362 after the scaling by 1 / sqrt(d)."""
    g = torch.Generator().manual_seed(seed)
    return (-362.0 / (4.0 * np.sqrt(d)) + torch.randint(-4, 5, shape, generator=g) / 16.0).to(torch.bfloat16)


# The decode tolerance (test_gpu_decode.py) plus what a logit of 362 adds in fp32: 524 in base 2, rounded a few times, an
# exponent error of 524 2^-23 and a relative one of 4.4e-5 in weight and normaliser: covered by the 2e-3.
def _close(got, want, v):
    got = got.cpu().numpy().astype(np.float64)
    return (np.abs(got - want) <= 2e-3 * np.abs(want) + 1e-5 * float(v.float().abs().max())).all()


@pytest.mark.parametrize("G,d,rows", [(1, 128, (333, 64)), (4, 64, (2000, 1))])
def test_decode(csp, oracle, G, d, rows):
    cap = max(rows)
    q = torch.full((1, 2 * G, d), 4.0).to(torch.bfloat16)
    k, g = _keys((1, 2, cap, d), cap, d), torch.Generator().manual_seed(1)
    v = torch.randn(1, 2, cap, d, generator=g).to(torch.bfloat16)
    n_rows = torch.tensor([rows], dtype=torch.int32)
    p = csp.Params(1, 2 * G, 2, d, 1, 0, cap, cap, n=0.0)
    po = oracle.Params(1, 2 * G, 2, d, 1, 0, cap, cap, dtype=oracle.BF16, n=0.0)
    want = oracle.decode_attn(po, q, k, v, n_rows.numpy())
    assert np.abs(want).max() > 0.01
    out, ws = torch.full((1, 2 * G, d), 7.0, device="cuda"), csp.new_decode_workspace(p)
    csp.decode_attn(p, q.cuda(), k.cuda(), v.cuda(), n_rows.cuda(), out, ws)
    assert csp.device_status(ws) == 0 and _close(out, want, v)
    # the carried sums of one step
    mod = torch.zeros(1, 2, cap, dtype=torch.uint8)
    mod[:, :, ::3] = 1
    lab = torch.zeros(1, dtype=torch.uint8)
    acc = [torch.full((1, 2, cap), 9.0, device="cuda") for _ in range(2)]
    want_acc = [np.full((1, 2, cap), 9.0) for _ in range(2)]
    ws = csp.new_decode_step_workspace(p)
    csp.decode_step(p, q.cuda(), k.cuda(), v.cuda(), n_rows.cuda(), mod.cuda(), lab.cuda(), True, out, *acc, ws)
    want = oracle.decode_step(po, q, k, v, n_rows.numpy(), mod.numpy(), lab.numpy(), *want_acc, True)
    assert csp.device_status(ws) == 0 and _close(out, want, v)
    for a, w in zip(acc, want_acc):
        np.testing.assert_allclose(a.cpu().numpy(), w, rtol=2e-3, atol=1e-6 * np.abs(w).max())


@pytest.mark.parametrize("lens,heads,d,dtype", [((300, 517), (4, 2), 128, torch.bfloat16), ((300,), (2, 2), 128, torch.float32),
                                                ((900,), (7, 1), 64, torch.bfloat16), (tuple(range(90, 1000, 23)), (8, 8), 128, torch.bfloat16)])
@pytest.mark.parametrize("supplied", [False, True])
def test_scores(csp, oracle, lens, heads, d, dtype, supplied):
    lays = [synth.interleaved_layout([L // 2, L - L // 2 - 40], 40) for L in lens]
    cfg = synth.small_config("far", lays, heads[0], heads[1], d, 32, 32, dtype=dtype, seed=3)
    B, G = len(lens), heads[0] // heads[1]
    q = torch.full((B, heads[0], 32, d), 4.0).to(dtype)
    k = _keys((B, heads[1], cfg.max_len, d), 5, d).to(dtype)
    lse = None
    if supplied:
        lse = np.zeros((B, heads[0], 32))
        for b, L in enumerate(lens):
            o = torch.einsum("hwd,htd->hwt", q[b].double(), k[b, :, :L].double().repeat_interleave(G, 0)) / np.sqrt(d)
            late = torch.arange(L)[None, :] > (L - 32 + torch.arange(32))[:, None]
            lse[b] = torch.logsumexp(o.masked_fill(late[None], float("-inf")), 2).numpy()
    run = GpuRun(csp, gpu_params(csp, cfg, n=0.0), q, k, k, cfg.modality(), cfg.seq_lens, cfg.budgets, lse=lse).score()
    assert run.status() == 0
    s, c = oracle.score(orc_params(oracle, cfg, n=0.0), q, k, cfg.modality(), cfg.seq_lens)
    assert s.max() > 0 and np.isfinite(s).all()
    for b, L in enumerate(lens):                        # (a NaN is close to everything below)
        assert torch.isfinite(run.ss[b, :, :L - 32]).all() and torch.isfinite(run.sc[b, :, :L - 32]).all()
    assert_scores_close(run.ss.cpu().numpy(), s, cfg.seq_lens, 32, "self")
    assert_scores_close(run.sc.cpu().numpy(), c, cfg.seq_lens, 32, "cross")

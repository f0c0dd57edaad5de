"""kvec_prefill_attention on the GPU: the kernels, split and in one piece, and the joins of
few and many splits that the cases of test_gpu_prefill.py leave out (test_prefill_plan.py
holds all of them together to the plan)."""
import pytest

from test_gpu_prefill import _check, _run, _tensors

pytestmark = pytest.mark.gpu

PLANS = [  # b, H, G, d, q rows, keys, dtype, window, sinks, q_lens, kv_lens, kernel, splits
    (1, 1, 2, 128, 5546, 5546, "bf16", 0, 0, None, None, "rows32_half", 8),
    (2, 1, 1, 128, 20, 576, "bf16", 473, 5, [20, 7], [576, 300], "rows32_half", 9),
    (1, 1, 3, 64, 3, 1024, "bf16", 0, 0, None, [900], "rows32_half", 16),
    (1, 8, 4, 64, 589, 59994, "bf16", 0, 0, None, None, "rows32_half", 3),
    (1, 1, 5, 64, 1270, 2805, "bf16", 0, 0, None, None, "rows32_keys4", 2),
    (1, 1, 4, 64, 159, 6188, "f32", 0, 0, None, None, "rows16_keys", 25),
    (1, 4, 1, 64, 41, 25003, "f32", 0, 0, None, None, "rows16_keys", 56),
    (1, 1, 1, 64, 3, 163, "f32", 37, 70, None, None, "rows16", 2),
    (1, 1, 1, 64, 1, 192, "f32", 104, 70, None, None, "rows16", 3),
    (1, 1, 1, 128, 1, 128, "f32", 0, 0, None, None, "rows16_keys", 2),
    (1, 1, 7, 128, 1, 320, "f32", 0, 0, None, None, "rows16_keys", 5),
]


@pytest.mark.parametrize("b,H,G,d,nq,nk,dt,window,sinks,q_lens,kv_lens,kernel,splits", PLANS)
def test_prefill_plans(gpu_lib, b, H, G, d, nq, nk, dt, window, sinks, q_lens, kv_lens, kernel, splits):
    q, k, v = _tensors(b, H, G, d, nq, nk, dt, seed=splits)
    out, lse = _run(gpu_lib, q, k, v, window, sinks, q_lens, kv_lens)
    rows = sorted({r for r in (0, 1, 31, 32, 63, 64, 127, 128, nq // 2, nq - 2, nq - 1) if 0 <= r < nq})
    if nk > 50000:
        rows = [0, nq - 1]
    _check(q, k, v, out, lse, window, sinks, q_lens, kv_lens, rows=rows)


@pytest.mark.parametrize("b,H,G,d,nq,nk,dt,window,sinks", [c[:9] for c in PLANS] + [
    (1, 8, 4, 128, 8, 16384, "bf16", 0, 0), (1, 8, 4, 128, 8192, 8192, "bf16", 0, 0), (1, 4, 7, 128, 2048, 32768, "bf16", 4096, 4),
    (2, 4, 2, 64, 509, 509, "f32", 0, 0), (1, 8, 4, 128, 1000, 1000, "bf16", 0, 0), (1, 16, 1, 64, 1500, 1500, "bf16", 0, 0)])
def test_prefill_same_bits_twice(gpu_lib, b, H, G, d, nq, nk, dt, window, sinks):
    """The same call gives the same bits whatever its workspace held."""
    import torch
    kv = gpu_lib
    q, k, v = _tensors(b, H, G, d, nq, nk, dt, seed=1)
    cfg = kv.AttentionConfig(b, H, H * G, d, nq, nk, window, sinks, kv.KVEC_BF16 if dt == "bf16" else kv.KVEC_F32)
    n = kv.kvec_prefill_workspace_size(cfg)
    got = []
    for fill in (0, 255, 63):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda") if n else None
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        kv.kvec_prefill_attention(cfg, q, k, v, out, ws, lse=lse)
        got.append((out.view(torch.int16 if dt == "bf16" else torch.int32), lse.view(torch.int32)))
    assert all(x.equal(y) for g in got[1:] for x, y in zip(got[0], g))

"""One token's attention over a long cache in eight bits whose sequences are not split, against
its float64 definition: a wave's page entries are looked up more than once."""
import pytest

from device_testlib import check_attention
from q8_testlib import Cache8
from test_gpu_q8 import _decode, _dt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("G,d,dt,window,sinks", [(2, 64, "bf16", 0, 0), (1, 128, "bf16", 4800, 9), (1, 64, "f32", 0, 0), (2, 128, "f32", 4700, 100)])
def test_waves_beyond_a_lookup(gpu_lib, G, d, dt, window, sinks, fmt):
    """One sequence of 5000 slots among 63 short ones of 8 heads: more than the 32 steps of 32
    slots that a wave's lookup is for, with pages that are none behind them."""
    lens = [5000] + [i % 4 for i in range(63)]
    c = Cache8(gpu_lib, lens, 8, G, d, 16, dt, fmt, seed=d + G).cuda()
    for s in (300, 4200, 4990):
        c.table[0, s // 16] = -1
    q = c.rand(len(lens), 8 * G, d).mul_(2).to(_dt(dt)).cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks)
    k, v = (x.double() * z.double()[..., None] for x, z in ((c.k, c.ks), (c.v, c.vs)))
    check_attention(k, v, q, out, lse, [c.slots(i, n) for i, n in enumerate(lens)], G, window, sinks, c.acc, acc0, more=2, terms=2.0 ** -23)
    o2, l2 = _decode(c, q, window, sinks, acc=False)
    assert o2.equal(out) and l2.equal(lse)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("power", [10, 14, 20, 35, 50])
def test_huge_logits_of_bf16_queries(gpu_lib, fmt, power):
    """Logits from 2^20 to 2^100: the largest of three is above the others by far more than a step,
    so its value is the output and its weight 1."""
    import torch
    form, code, top = (gpu_lib.KVEC_Q8_INT8, torch.int8, 127.0) if fmt == "int8" else (gpu_lib.KVEC_Q8_E4M3, torch.float8_e4m3fn, 448.0)
    cfg = gpu_lib.PagedQ8Config(1, 1, 1, 64, 64, 2, 1, gpu_lib.KVEC_BF16, form)
    at = [(3, -3.0), (7, 1.37), (40, 0.61)]  # in two groups of 16, one of which is not whole
    codes, kz = torch.zeros((2, 1, 64, 64), device="cuda"), torch.full((2, 1, 64), 2.0 ** -126, device="cuda")
    for s, x in at:
        codes[1, 0, s], kz[1, 0, s] = top * (1 if x > 0 else -1), abs(x) * 2.0 ** power / top
    g = torch.Generator().manual_seed(power)
    v, vz = torch.randint(-100, 101, (2, 1, 64, 64), generator=g).cuda().float().to(code), torch.full((2, 1, 64), 0.01, device="cuda")
    q = torch.full((1, 1, 64), 1.1 * 2.0 ** power, device="cuda").bfloat16()
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    out, lse, acc = torch.empty((1, 1, 64), device="cuda"), torch.empty((1, 1), device="cuda"), torch.zeros((2, 1, 64), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_q8_workspace_size(cfg, None, True), dtype=torch.uint8, device="cuda")
    gpu_lib.kvec_paged_decode_q8(cfg, q, codes.to(code), v, kz, vz, one.view(1, 1), 60 * one, out, ws, lse=lse, acc=acc)
    want = v[1, 0, 7].float() * 0.01
    assert torch.all((out[0, 0] - want).abs() <= 2.0 ** -21 * want.abs())
    assert acc[1, 0, 7] == 1 and acc.sum() == 1
    x = 64 * q[0, 0, 0].double().item() * top * kz[1, 0, 7].double().item() / 8
    assert abs(lse.item() - x) <= 35 * 2.0 ** -24 * x

"""How float32 logits are summed, seen in the log-sum-exp of one visible slot, which is its logit.

All d products are the same number v = 1 + 2^-19 + 2^-23.  A running sum of d = 64 of them is
rounded the same way in every step from 32 on, where its step is 2^-18: off by 32 * (2^-19 -
2^-23), 2^-14 of 64.  Eight sums of eight take at most half a step an addition, 2 * 2^-23 + 4 *
2^-22 + 2^-21 = 7 * 2^-22 each; added in pairs, 4 * 2^-20 at 16, 2 * 2^-19 at 32 and 2^-18 at
64: 6.5 * 2^-18 in all.  The logit is an eighth of it, 0.82 * 2^-18; its scaling and the
log-sum-exp's own roundings are three half steps at 8 to 16, 2^-21 each.  1.25 * 2^-18 holds
all of it; an eighth of 2^-14, 2^-17, does not pass."""
import pytest

pytestmark = pytest.mark.gpu

V = 1 + 2.0 ** -19 + 2.0 ** -23
BOUND = 1.25 * 2.0 ** -18


def _table(n):
    import torch
    return torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("where", ["prefix", "own"])
def test_shared(gpu_lib, where):
    import torch
    cfg = gpu_lib.PagedConfig(1, 1, 1, 64, 16, 2, 1, gpu_lib.KVEC_F32)
    k = torch.ones((2, 1, 16, 64), device="cuda")
    q = torch.full((1, 1, 64), V, device="cuda")
    table, lens = _table(int(where == "own"))
    pages, plen = torch.ones(1, dtype=torch.int32, device="cuda"), torch.tensor([int(where == "prefix")], dtype=torch.int32, device="cuda")
    out, lse, acc = torch.empty_like(q), torch.empty((1, 1), device="cuda"), torch.zeros((2, 1, 16), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_shared_workspace_size(cfg, 16, 16, True), dtype=torch.uint8, device="cuda")
    gpu_lib.kvec_paged_decode_shared(cfg, q, k, k, pages, plen, table, lens, out, ws, lse=lse, acc=acc)
    assert abs(lse.item() - 64 * V / 8) <= BOUND
    assert torch.all(out == 1)
    # the weight, made of the same logit again: off by the two logits' bounds at most
    assert abs(acc.sum().item() - 1) <= 2 * BOUND


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_decode_q8(gpu_lib, fmt):
    """The codes are the format's largest, the scale its inverse: a product is M times as large,
    and so are its steps; z M is off from 1 by what `held` says."""
    import torch
    form, code, top = (gpu_lib.KVEC_Q8_INT8, torch.int8, 127.0) if fmt == "int8" else (gpu_lib.KVEC_Q8_E4M3, torch.float8_e4m3fn, 448.0)
    cfg = gpu_lib.PagedQ8Config(1, 1, 1, 64, 16, 1, 1, gpu_lib.KVEC_F32, form)
    k = torch.full((1, 1, 16, 64), top, device="cuda").to(code)
    z = torch.full((1, 1, 16), 1 / top, device="cuda")
    held = z[0, 0, 0].double().item() * top
    q = torch.full((1, 1, 64), V, device="cuda")
    table, lens = _table(1)
    out, lse = torch.empty_like(q), torch.empty((1, 1), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_q8_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    gpu_lib.kvec_paged_decode_q8(cfg, q, k, k, z, z, table, lens, out, ws, lse=lse)
    assert abs(lse.item() - 64 * V * held / 8) <= BOUND
    assert abs(out - held).max().item() <= 2.0 ** -23


# Logits from 2^20 to 2^100 and more, whose steps are up to 2^76: the largest of three is above
# the others by far more than a step, so its value is the output, exactly, and it the log-sum-exp
# to three half steps (sum, scaling, logarithm: d / 2 + 3 with sums of equal signs).
HUGE = [10, 14, 20, 35, 50]


def _huge(power):
    import torch
    k = torch.zeros((2, 1, 16, 64), device="cuda")
    v = torch.randn((2, 1, 16, 64), generator=torch.Generator().manual_seed(power)).cuda()
    for slot, x in enumerate((-3.0, 1.37, 0.61)):
        k[1, 0, slot] = x * 2.0 ** power
    q = torch.full((1, 1, 64), 1.1 * 2.0 ** power, device="cuda")
    return q, k, v, 64 * q[0, 0, 0].double().item() * k[1, 0, 1, 0].double().item() / 8


@pytest.mark.parametrize("power", HUGE)
@pytest.mark.parametrize("where", ["prefix", "own"])
def test_huge_logits_shared(gpu_lib, where, power):
    import torch
    cfg = gpu_lib.PagedConfig(1, 1, 1, 64, 16, 2, 1, gpu_lib.KVEC_F32)
    q, k, v, x = _huge(power)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    n = [3 * one, 0 * one] if where == "prefix" else [0 * one, 3 * one]
    out, lse, acc = torch.empty_like(q), torch.empty((1, 1), device="cuda"), torch.zeros((2, 1, 16), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_shared_workspace_size(cfg, 16, 16, True), dtype=torch.uint8, device="cuda")
    gpu_lib.kvec_paged_decode_shared(cfg, q, k, v, one, n[0], one.view(1, 1), n[1], out, ws, lse=lse, acc=acc)
    assert acc[1, 0, 1] == 1 and acc.sum() == 1
    # (the weight cancels but for the rounding of its product and quotient)
    assert torch.all((out[0, 0] - v[1, 0, 1]).abs() <= 2.0 ** -22 * v[1, 0, 1].abs())
    assert abs(lse.item() - x) <= 35 * 2.0 ** -24 * x


@pytest.mark.parametrize("power", HUGE)
@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("b", [1, 70])
def test_huge_logits_shared_bf16(gpu_lib, b, where, power):
    """(Three bf16 terms of a weight are 2^-24 relative.)"""
    import torch
    cfg = gpu_lib.PagedConfig(b, 1, 1, 64, 16, 2, 1, gpu_lib.KVEC_BF16)
    q, k, v, _ = _huge(power)
    q, k, v = q.bfloat16().repeat(b, 1, 1), k.bfloat16(), v.bfloat16()
    x = 64 * q[0, 0, 0].double().item() * k[1, 0, 1, 0].double().item() / 8
    one, all_ = torch.ones(1, dtype=torch.int32, device="cuda"), torch.ones(b, dtype=torch.int32, device="cuda")
    n = [3 * one, 0 * all_] if where == "prefix" else [0 * one, 3 * all_]
    out, lse, acc = torch.empty((b, 1, 64), device="cuda"), torch.empty((b, 1), device="cuda"), torch.zeros((2, 1, 16), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_shared_workspace_size(cfg, 16, 16, True), dtype=torch.uint8, device="cuda")
    # (with the own slots of several sequences in one page, there is no acc)
    gpu_lib.kvec_paged_decode_shared(cfg, q, k, v, one, n[0], all_.view(b, 1), n[1], out, ws, lse=lse,
                                     acc=acc if where == "prefix" or b == 1 else None)
    # the prefix's weights are made of logits that are added up in another order: a step of them may
    # be all of the weight
    assert torch.all((acc >= 0) & (acc <= b)) and acc.sum() == acc[1, 0, 1]
    assert torch.all((out[:, 0] - v[1, 0, 1].float()).abs() <= 2.0 ** -22 * v[1, 0, 1].float().abs())
    assert torch.all((lse.double() - x).abs() <= 35 * 2.0 ** -24 * x)


@pytest.mark.parametrize("power", HUGE)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_huge_logits_q8(gpu_lib, fmt, power):
    import torch
    form, code, top = (gpu_lib.KVEC_Q8_INT8, torch.int8, 127.0) if fmt == "int8" else (gpu_lib.KVEC_Q8_E4M3, torch.float8_e4m3fn, 448.0)
    cfg = gpu_lib.PagedQ8Config(1, 1, 1, 64, 16, 2, 1, gpu_lib.KVEC_F32, form)
    q, k, v, _ = _huge(power)
    kz = (k.abs().amax(-1) / top).clamp(min=2.0 ** -126)
    kc = (torch.sign(k) * top).to(code)
    vc, vz = torch.round(v.clamp(-1, 1) * 100).to(code), torch.full((2, 1, 16), 0.01, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, 1), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_q8_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    gpu_lib.kvec_paged_decode_q8(cfg, q, kc, vc, kz, vz, one.view(1, 1), 3 * one, out, ws, lse=lse)
    want = vc[1, 0, 1].float() * 0.01
    assert torch.all((out[0, 0] - want).abs() <= 2.0 ** -21 * want.abs())
    x = 64 * q[0, 0, 0].double().item() * top * kz[1, 0, 1].double().item() / 8
    assert abs(lse.item() - x) <= 35 * 2.0 ** -24 * x

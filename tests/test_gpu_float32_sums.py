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

"""Attention behind a shared prefix where logits are beyond 2^24 in base 2, a step of float32
there being 2 or more: equal logits weigh the same wherever their slots lie, and the columns
beside such a one are as exact as without it."""
import math

import pytest

pytestmark = pytest.mark.gpu

# A query of 1.1 * 2^power and keys of k * 2^power, all elements alike: 64 equal products of
# bfloat16 numbers, whose sums float32 holds exactly.  k chooses how far the base-2 logit is
# from the nearest float32: -0.28, 0.48, -45, 12 and -2 * 10^5.
FAR = [(10, 1.55), (10, 1.9), (14, 1.37), (14, 1.21), (20, 1.37)]
EQUAL = [5, 40, 100, 600]  # in the first and second block of 32, in another tile, in another split


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _call(kv, cfg, q, k, v, pages, P, table, lens, acc=None, window=0, sinks=0):
    import torch
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    b, hq = q.shape[:2]
    out, lse = torch.empty(q.shape, device="cuda"), torch.empty((b, hq), device="cuda")
    n = len(pages) * cfg.page_size
    ws = torch.empty(kv.kvec_paged_decode_shared_workspace_size(cfg, n, None, acc is not None), dtype=torch.uint8, device="cuda")
    kv.kvec_paged_decode_shared(cfg, q, k, v, i32(pages), i32([P]), i32(table), i32(lens), out, ws, window=window, n_sinks=sinks, lse=lse, acc=acc)
    return out, lse


@pytest.mark.parametrize("power,kk", FAR)
@pytest.mark.parametrize("dt,b", [("bf16", 1), ("bf16", 70), ("f32", 1)])
@pytest.mark.parametrize("where", ["prefix", "own", "both"])
def test_equal_logits_weigh_the_same(gpu_lib, where, dt, b, power, kk):
    """Four slots with the same key, others far below: the output is the mean of their values.
    Every weight is the same float32 number, in three bf16 terms: a weight's 2^-24, the sums' and
    the quotient's roundings are less than 2^-21 of the largest value together."""
    import torch
    n, page = 640, 640
    cfg = gpu_lib.PagedConfig(b, 1, 1, 64, page, 2, 1, gpu_lib.KVEC_BF16 if dt == "bf16" else gpu_lib.KVEC_F32)
    q = torch.full((b, 1, 64), 1.1 * 2.0 ** power, device="cuda").to(_dt(dt))
    k = torch.zeros((2, 1, page, 64), device="cuda")
    v = torch.randn((2, 1, page, 64), generator=torch.Generator().manual_seed(power)).cuda().to(_dt(dt))
    at = {"prefix": [(1, s) for s in EQUAL], "own": [(0, s) for s in EQUAL], "both": [(1, 5), (1, 600), (0, 40), (0, 100)]}[where]
    for p, s in at:
        k[p, 0, s] = kk * 2.0 ** power
    out, lse = _call(gpu_lib, cfg, q, k.to(_dt(dt)), v, [1], 0 if where == "own" else n, [[0]] * b, [0 if where == "prefix" else n] * b)
    want = sum(v[p, 0, s].double() for p, s in at) / 4
    assert torch.all((out[:, 0].double() - want).abs() <= 2.0 ** -21 * v.float().abs().max())
    x = 64 * q[0, 0, 0].double().item() * k.to(_dt(dt)).max().double().item() / 8
    assert torch.all((lse.double() - x).abs() <= 35 * 2.0 ** -24 * x)


@pytest.mark.parametrize("b", [2, 20, 70])
@pytest.mark.parametrize("c,t", [(360, 3), (386, 3), (498, 1)])
def test_a_far_column_leaves_its_neighbours_exact(gpu_lib, b, c, t):
    """Two keys of 64 c and 64 c - 2 t against queries of ones: base-2 logits of 4000 to 5800,
    whose roundings, 2^-12 each, would move a weight by 2^-14; the difference to the largest one
    is exact to 2^-25.  The first sequence's query is 2^14 times as large, and so are its logits."""
    import torch
    cfg = gpu_lib.PagedConfig(b, 1, 1, 64, 16, 2, 1, gpu_lib.KVEC_BF16)
    k, v = (torch.zeros((2, 1, 16, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    k[1, 0, :2] = c
    k[1, 0, 1, 0] = c - 2 * t
    v[1, 0, 0] = 1
    q = torch.ones((b, 1, 64), device="cuda", dtype=torch.bfloat16)
    assert torch.all(k[1, 0, 0] == c) and k[1, 0, 1, 0] == c - 2 * t
    q[0] = 2.0 ** 14
    out, _ = _call(gpu_lib, cfg, q, k, v, [1], 2, [[0]] * b, [0] * b)
    assert torch.all((out[0] - 1).abs() <= 2.0 ** -22)
    assert torch.all((out[1:].double() - 1 / (1 + math.exp(-2 * t / 8))).abs() <= 2.0 ** -19)

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


def _winners(b, G, H, P, d, size, window, seed, page=16):
    """Queries of b sequences, keys of a prefix of P slots, in which each sequence's own key
    beats all others: key i is query i, of the length that makes its base-2 logit about `size`.
    With a window, a key that would beat all of them lies before it."""
    import torch
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((b, 1, d), generator=g)
    q = q / q.norm(dim=-1, keepdim=True) * math.sqrt(size * math.sqrt(d) / 1.4426950408889634)
    slots = [P - 1 - i for i in range(b)]
    pages = (P + page - 1) // page
    k = torch.randn((pages * page, d), generator=g)
    k[slots] = q[:, 0]
    if window:
        k[10] = 4 * q.sum((0, 1))
    k = k.view(pages, 1, page, d).expand(pages, H, page, d).contiguous()
    v = torch.randn(k.shape, generator=g)
    return q.repeat(1, H * G, 1).bfloat16().cuda(), k.bfloat16().cuda(), v.bfloat16().cuda(), slots


WEIGHTS = [  # sequences, G, H, P: few and many columns, keys of 32 and of 128 slots a work-group
    (3, 2, 1, 150), (70, 1, 1, 150), (20, 3, 2, 170), (3, 2, 32, 1100), (70, 1, 33, 1001)]


@pytest.mark.parametrize("size", [2.0 ** 16.4, 2.0 ** 18.4, 2.0 ** 20.4, 2.0 ** 22.4, 2.0 ** 23.4, 2.0 ** 26, 2.0 ** 40, 2.0 ** 90])
@pytest.mark.parametrize("window", [0, 120])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,G,H,P", WEIGHTS)
def test_weights_of_far_columns(gpu_lib, b, G, H, P, d, window, size):
    """Every sequence gives its whole weight to its own key of the prefix, however large its
    logits are: 2^(logit - normaliser), which is the logit rounded to float32, so off by half a
    step of it and the exponential's rounding, and never more than 1; from 2^24 on the logits
    are rounded too and the weight is 1.  All other slots get nothing: their logits are lower
    by thousands and more."""
    import torch
    q, k, v, slots = _winners(b, G, H, P, d, size, window, b + P)
    cfg = gpu_lib.PagedConfig(b, H, H * G, d, 16, k.shape[0], 1, gpu_lib.KVEC_BF16)
    acc = torch.zeros(k.shape[:3], device="cuda")
    out, lse = _call(gpu_lib, cfg, q, k, v, list(range(k.shape[0])), P, [[-1]] * b, [0] * b, acc, window, 4 if window else 0)
    flat = acc.transpose(1, 2).reshape(-1, H)
    own = flat[slots]
    top = (lse.double() / math.log(2)).max().item()
    step = 0.0 if top > 1.01 * 2.0 ** 24 else 2.0 ** (math.floor(math.log2(top * 1.0001)) - 23)
    assert top > 2.0 ** 16
    assert torch.all((own <= 1) & (own >= 2.0 ** (-step / 2) - 2.0 ** -22)), (own.min(), own.max(), step)
    flat[slots] = 0
    assert torch.all(flat == 0)
    want = v.transpose(1, 2).reshape(-1, H, d)[slots].float()
    assert torch.all((out.view(b, H, G, d) - want[:, :, None]).abs() <= 2.0 ** -22 * want[:, :, None].abs())


@pytest.mark.parametrize("power,kk", FAR + [(35, 1.37), (50, 1.37)])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_far_own_slots(gpu_lib, d, power, kk):
    """bf16: own slots' weights come from the logits that the normaliser was made of: the largest
    one's is 1, exactly, and the others, 2^-4 of it below, have none."""
    import torch
    cfg = gpu_lib.PagedConfig(1, 1, 2, d, 16, 4, 3, gpu_lib.KVEC_BF16)
    q = torch.full((1, 2, d), 1.1 * 2.0 ** power, device="cuda").bfloat16()
    k = torch.zeros((4, 1, 16, d), device="cuda")
    k[0, 0, 7], k[1, 0, 3], k[2, 0, 1] = kk * 2.0 ** power * 15 / 16, kk * 2.0 ** power, -kk * 2.0 ** power
    v = torch.randn(k.shape, generator=torch.Generator().manual_seed(power)).cuda().bfloat16()
    for P, pages in ((0, [3]), (9, [3])):  # alone, and behind a prefix whose keys are zeros
        acc = torch.zeros((4, 1, 16), device="cuda")
        out, _ = _call(gpu_lib, cfg, q, k.bfloat16(), v, pages, P, [[0, 1, 2]], [40], acc)
        assert acc[1, 0, 3] == 1 and acc.sum() == 1
        assert torch.all((out - v[1, 0, 3].float()).abs() <= 2.0 ** -22 * v[1, 0, 3].float().abs())


def test_weights_of_far_columns_and_others(gpu_lib):
    """Far columns among ordinary ones, padding rows and missing pages: the ordinary ones' weights
    are those of the same batch without the far ones' (bounds of two sums of the same terms)."""
    import torch
    b, G, H, P, d = 70, 1, 32, 1100, 64
    q, k, v, slots = _winners(b, G, H, P, d, 2.0 ** 30, 0, 3)
    near = torch.randn((b, H, d), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    near *= 2.0 ** -12  # (logits of the far keys to a few)
    far = torch.zeros(b, dtype=torch.bool)
    far[[0, 17, 33, 40, 69]] = True
    lens = torch.zeros(b, dtype=torch.int32)
    lens[[5, 17, 60]] = -1  # one of the far ones is none
    mixed = torch.where(far[:, None, None].cuda(), q, near)
    cfg = gpu_lib.PagedConfig(b, H, H, d, 16, k.shape[0], 1, gpu_lib.KVEC_BF16)
    pages = list(range(k.shape[0]))
    pages[20] = -1
    accs = [torch.zeros(k.shape[:3], device="cuda") for _ in range(2)]
    _call(gpu_lib, cfg, mixed, k, v, pages, P, [[-1]] * b, lens.tolist(), accs[0])
    _call(gpu_lib, cfg, near, k, v, pages, P, [[-1]] * b, torch.where(far, -1, lens).tolist(), accs[1])
    got = (accs[0].double() - accs[1].double()).transpose(1, 2).reshape(-1, H)
    want = torch.zeros_like(got)
    want[[s for i, s in enumerate(slots) if far[i] and lens[i] >= 0]] = 1
    # 62 weights of at most 1, each off by 2^-15 in either batch
    assert torch.all((got - want).abs() <= 62 * 2.0 ** -14)
    assert torch.all(accs[0][20] == 0)

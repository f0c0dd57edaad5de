"""The largest batch, the longest sequence and the most slots that the serving calls take,
against their definitions in float64 on the GPU, all sequences at once."""
import math

import pytest

import serve_testlib as ref

pytestmark = pytest.mark.gpu


def _softmax(q, k, v, live):
    """q [b][d], k and v [b][n][d], live [b][n]; float64: out, lse, weights."""
    import torch
    x = (k.double() * q.double()[:, None]).sum(-1) / math.sqrt(q.shape[-1])
    x = x.masked_fill(~live, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[:, None]).nan_to_num(0)
    return (p[..., None] * v.double()).sum(1), lse, p


def _bound(q, k):
    """Bound of a logit's error (serve_testlib)."""
    d = q.shape[-1]
    return (d + 2) * ref.U24 * float((k.abs().double() * q.abs().double()[:, None]).sum(-1).max()) / math.sqrt(d)


def test_the_largest_batch(gpu_lib):
    """65535 sequences of 0 to 16 slots: a page and a head each."""
    import torch
    kv, b, d, page = gpu_lib, 65535, 64, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    q, k, v = rand(b, 1, d), rand(b, 1, page, d), rand(b, 1, page, d)
    lens = torch.randint(0, page + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    live = torch.arange(page, device="cuda") < lens[:, None]
    out64, lse64, p = _softmax(q[:, 0], k[:, 0], v[:, 0], live)
    off = 2 * _bound(q[:, 0], k[:, 0]) + ref.EXP
    size = v.abs().max().item()

    cfg = kv.PagedConfig(b, 1, 1, d, page, b, 1)
    table = torch.randperm(b, generator=g, device="cuda", dtype=torch.int32).view(b, 1)
    at = table[:, 0].long()
    kp, vp, acc = torch.empty_like(k), torch.empty_like(v), torch.zeros((b, 1, page), device="cuda")
    pos = torch.zeros((b, 1, page), dtype=torch.int32, device="cuda")
    # every token but the first of a sequence is there; the first comes by an append
    kp[at], vp[at] = k, v
    kp[at, :, 0], vp[at, :, 0] = math.nan, math.nan
    q_out, zero = torch.empty_like(q), torch.zeros(b, dtype=torch.int32, device="cuda")
    kv.kvec_paged_append(cfg, q, k[:, :, 0], v[:, :, 0], zero, at * page, q_out, kp, vp, acc=acc, pos=pos)
    assert q_out.equal(q) and kp[at].equal(k) and vp[at].equal(v)
    pos[at] = torch.arange(page, dtype=torch.int32, device="cuda")
    out, lse = torch.empty((b, 1, d), device="cuda"), torch.empty((b, 1), device="cuda")
    ws = torch.empty(kv.kvec_paged_decode_workspace_size(cfg, None, True), dtype=torch.uint8, device="cuda")
    kv.kvec_paged_decode(cfg, q_out, kp, vp, table, lens, out, ws, lse=lse, acc=acc)
    assert (out[:, 0] - out64).abs().max().item() <= off * size
    assert torch.equal(lse[:, 0] == -math.inf, lens == 0) and (lse[:, 0] - lse64).nan_to_num(0).abs().max().item() <= off + ref.EXP * 8
    assert (acc[at][:, 0] - p).abs().max().item() <= off

    budget = 5
    weight = acc[at][:, 0].masked_fill(~live, -1.0)
    kept64 = torch.zeros_like(live).scatter_(1, weight.sort(dim=-1, descending=True, stable=True).indices[:, :budget], True) & live
    want = torch.where(kept64, pos[at][:, 0], 99).sort(-1).values[:, :budget]
    we = torch.empty(kv.kvec_paged_evict_workspace_size(cfg, None, budget), dtype=torch.uint8, device="cuda")
    kept, lens_out = torch.empty((b, 1, budget), dtype=torch.int32, device="cuda"), torch.empty_like(lens)
    k0 = kp[at][:, 0].clone()
    kv.kvec_paged_evict(cfg, budget, kp, vp, table, lens, lens, acc, pos, lens_out, we, kept=kept)
    assert torch.equal(lens_out, lens.clamp(max=budget))
    assert torch.equal(torch.where(kept[:, 0] < 0, 99, kept[:, 0]).sort(-1).values, want)
    there = kept[:, 0] >= 0
    moved = k0.gather(1, kept[:, 0].clamp(min=0).long()[..., None].expand(-1, -1, d))
    assert torch.equal(kp[at][:, 0, :budget][there], moved[there])

    o2, l2 = torch.empty((b, 1, 1, d), dtype=torch.bfloat16, device="cuda"), torch.empty((b, 1, 1), device="cuda")
    attn = kv.AttentionConfig(b, 1, 1, d, 1, page)
    n = kv.kvec_prefill_workspace_size(attn)
    kv.kvec_prefill_attention(attn, q[:, :, None], k, v, o2, torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), lse=l2, kv_lens=lens)
    assert (o2[:, 0, 0].double() - out64).abs().max().item() <= (off + 2 * ref.U_BF16) * size
    assert (l2[:, 0, 0] - lse64).nan_to_num(0).abs().max().item() <= off + ref.EXP * 8


def test_the_longest_sequence(gpu_lib):
    """2^20 slots of one head: decoded over, evicted to half of them, and as a prompt's keys."""
    import torch
    kv, n, d, page = gpu_lib, 1 << 20, 64, 4096
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((1, 2, d), (n // page, 1, page, d), (n // page, 1, page, d)))
    q[:, 1] *= 3
    cfg = kv.PagedConfig(1, 1, 2, d, page, n // page, n // page)
    table, lens = torch.arange(n // page, dtype=torch.int32, device="cuda").view(1, -1), torch.tensor([n], dtype=torch.int32, device="cuda")
    acc = torch.zeros((n // page, 1, page), device="cuda")
    out, lse = torch.empty((1, 2, d), device="cuda"), torch.empty((1, 2), device="cuda")
    ws = torch.empty(kv.kvec_paged_decode_workspace_size(cfg, None, True), dtype=torch.uint8, device="cuda")
    kv.kvec_paged_decode(cfg, q, k, v, table, lens, out, ws, lse=lse, acc=acc)
    live = torch.ones((1, n), dtype=torch.bool, device="cuda")
    mean, wants = 0, []
    for j in range(2):
        o, l, p = _softmax(q[:, j], k.view(1, n, d), v.view(1, n, d), live)
        off = 2 * _bound(q[:, j], k.view(1, n, d)) + ref.EXP
        assert (out[:, j] - o).abs().max().item() <= off * v.abs().max().item()
        assert abs(lse[0, j].item() - l.item()) <= off + ref.EXP * l.item()
        mean = mean + p / 2
        wants.append((o, l, off))
    assert ((acc.view(1, n) - mean).abs() <= off * mean + 1e-30).all()

    attn = kv.AttentionConfig(1, 1, 2, d, 1, n)
    o2, l2 = torch.empty((1, 2, 1, d), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 2, 1), device="cuda")
    wp = torch.empty(kv.kvec_prefill_workspace_size(attn), dtype=torch.uint8, device="cuda")
    kv.kvec_prefill_attention(attn, q[:, :, None], k.view(1, 1, n, d), v.view(1, 1, n, d), o2, wp, lse=l2)
    for j, (o, l, off) in enumerate(wants):
        assert (o2[0, j, 0] - o[0]).abs().max().item() <= (off + 2 * ref.U_BF16) * v.abs().max().item()
        assert abs(l2[0, j, 0].item() - l.item()) <= off + ref.EXP * l.item()

    budget = n // 2
    pos = torch.arange(n, dtype=torch.int32, device="cuda").view(n // page, 1, page).clone()
    order = acc.view(-1).sort(descending=True, stable=True).indices[:budget]
    kept64 = torch.zeros(n, dtype=torch.bool, device="cuda")
    kept64[order] = True
    late, holes = torch.nonzero(kept64[budget:])[:, 0] + budget, torch.nonzero(~kept64[:budget])[:, 0]
    want = torch.arange(budget, device="cuda")
    want[holes] = late
    k0 = k.view(n, d).clone()
    kept, lens_out = torch.empty((1, 1, budget), dtype=torch.int32, device="cuda"), torch.empty_like(lens)
    we = torch.empty(kv.kvec_paged_evict_workspace_size(cfg, None, budget), dtype=torch.uint8, device="cuda")
    kv.kvec_paged_evict(cfg, budget, k, v, table, lens, lens, acc, pos, lens_out, we, kept=kept)
    assert lens_out.item() == budget and torch.equal(kept.view(-1).long(), want)
    assert torch.equal(k.view(n, d)[:budget], k0[want]) and torch.equal(pos.view(-1)[:budget].long(), want)

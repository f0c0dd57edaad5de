"""The largest batches, bounds far above the lengths, and addresses aligned to one element only:
attention behind a shared prefix and over a cache in eight bits."""
import numpy as np
import pytest

from device_testlib import check_attention
from q8_testlib import Cache8
from test_gpu_q8 import _decode as decode_q8
from test_gpu_shared import Shared, _decode, _dt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,H,G,d", [("bf16", 1, 15, 64), ("f32", 1, 15, 64), ("bf16", 5, 3, 128)])
def test_the_largest_batch(gpu_lib, dt, H, G, d):
    """65535 sequences, 983025 query heads, behind one prefix: a few queries in turn, so that the
    outputs of the first ones are everyone's, and the weights are sums of theirs.  Rows 5, 20, 35, ...
    of the batch are none; one sequence has own slots."""
    import torch
    b, P, n_q = 65535, 90, 15
    c = Shared(gpu_lib, P, [3] + [0] * (n_q - 1), H, G, d, 16, dt, seed=G).cuda()
    few = c.rand(n_q, H * G, d).mul_(2).to(_dt(dt)).cuda()
    few[5] = float("nan")
    q = few.repeat(b // n_q, 1, 1)
    lens = torch.zeros(b, dtype=torch.int32, device="cuda")
    lens[5::n_q] = -1
    lens[0] = 3
    table = torch.full((b, 1), -1, dtype=torch.int32, device="cuda")
    table[0] = c.table[0]
    cfg = gpu_lib.PagedConfig(b, H, H * G, d, 16, c.cfg.n_pages, 1, c.cfg.dtype)
    out, lse = torch.full((b, H * G, d), float("nan"), device="cuda"), torch.full((b, H * G), float("nan"), device="cuda")
    ws = torch.empty(gpu_lib.kvec_paged_decode_shared_workspace_size(cfg, P, None, True), dtype=torch.uint8, device="cuda").fill_(255)
    acc0 = c.acc.clone()
    gpu_lib.kvec_paged_decode_shared(cfg, q, c.k, c.v, c.pages, c.plen, table, lens, out, ws, max_prefix=P, lse=lse, acc=c.acc)
    # everyone's results are those of the first fifteen without own slots
    assert out.view(-1, n_q, H * G, d)[1:].eq(out[n_q:2 * n_q]).all() and lse.view(-1, n_q, H * G)[1:].eq(lse[n_q:2 * n_q]).all()
    assert out[1:n_q].equal(out[n_q + 1:2 * n_q]) and lse[1:n_q].equal(lse[n_q + 1:2 * n_q])
    first = c._rows(c.pages, P)
    rows = [[np.concatenate(x) for x in zip(first, c._rows(c.table[0], 3))]] + [None if i % n_q == 5 else first for i in range(1, 2 * n_q)]
    k, v = c.k.double(), c.v.double()
    check_attention(k, v, q, out, lse, rows, G)
    # the weights that one call of the thirty gives, each but the first as often as its query occurs
    alone = torch.zeros_like(acc0)
    for i in range(2 * n_q):
        if rows[i] is None or 0 < i < n_q:
            continue
        page, row = (torch.from_numpy(x).long().cuda() for x in rows[i])
        x = torch.einsum("hgd,nhd->hgn", q[i].double().view(H, G, d), k[page, :, row]) / d ** 0.5
        alone[page, :, row] += (torch.softmax(x, -1).mean(1).T * (1 if i == 0 else b // n_q - (i == n_q))).float()
    want = acc0 + alone
    ok = ~want.isnan()
    # sums of 10^6 terms in chains of b G / 64, rounded at each: half a step of the sum each
    assert torch.equal(c.acc.isnan(), ~ok)
    assert torch.all((c.acc - want).abs()[ok] <= want[ok] * (b * G / 64 + 100) * 2.0 ** -24)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f32", 64)])
def test_bounds_far_above_the_lengths(gpu_lib, dt, d):
    """As a captured call has them: 2^20 slots of a prefix and of a sequence allowed, hundreds there."""
    import torch
    c = Shared(gpu_lib, 700, [333, 0], 2, 2, d, 16, dt, seed=3).cuda()
    page, most = 16, 1 << 20
    c.table = torch.cat([c.table, torch.full((2, most // page - c.table.shape[1]), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
    pages = c.pages
    c.pages = torch.cat([pages, torch.full((most // page - len(pages),), -1, dtype=torch.int32, device="cuda")])
    c.cfg = gpu_lib.PagedConfig(2, 2, 4, d, page, c.cfg.n_pages, most // page, c.cfg.dtype)
    q = c.rand(2, 4, d).mul_(2).to(_dt(dt)).cuda()
    for window, sinks in ((0, 0), (400, 9)):
        acc0 = c.acc.clone()
        out, lse = _decode(c, q, window, sinks)
        first = c._rows(c.pages, 700)
        rows = [[np.concatenate(x) for x in zip(first, c._rows(c.table[i], n))] for i, n in enumerate(c.lens_l)]
        check_attention(c.k.double(), c.v.double(), q, out, lse, rows, 2, window, sinks, c.acc, acc0, columns=4)
    e = Cache8(gpu_lib, [700, 0, 45], 2, 2, d, 16, dt, "e4m3", seed=4, max_pages=most // page).cuda()
    q = e.rand(3, 4, d).mul_(2).to(_dt(dt)).cuda()
    k, v = (x.double() * z.double()[..., None] for x, z in ((e.k, e.ks), (e.v, e.vs)))
    for window, sinks in ((0, 0), (400, 9)):
        acc0 = e.acc.clone()
        out, lse = decode_q8(e, q, window, sinks)
        check_attention(k, v, q, out, lse, [e.slots(i, n) for i, n in enumerate(e.lens_l)], 2, window, sinks, e.acc, acc0, more=2, terms=2.0 ** -23)


def _shifted(t, by=1):
    """The same values `by` elements behind the start of an allocation."""
    import torch
    out = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)[by:].view(t.shape)
    return out.copy_(t)


def test_addresses_aligned_to_an_element(gpu_lib):
    """Weights, scales, lengths, tables and outputs may start at any element: the same bits."""
    import torch
    c = Shared(gpu_lib, 300, [70, 5, 33], 2, 4, 64, 48, "bf16", seed=8).cuda()
    q = c.rand(3, 8, 64).bfloat16().cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q)
    acc, c.acc = c.acc, _shifted(acc0, 3)
    for name in ("pages", "plen", "table", "lens"):
        setattr(c, name, _shifted(getattr(c, name)))
    ws = torch.empty(gpu_lib.kvec_paged_decode_shared_workspace_size(c.cfg, len(c.pages) * 48, None, True) + 16, dtype=torch.uint8, device="cuda")[16:]
    o2, l2 = _shifted(out), _shifted(lse, 3)
    o2.fill_(7)
    gpu_lib.kvec_paged_decode_shared(c.cfg, q, c.k, c.v, c.pages, c.plen, c.table, c.lens, o2, ws, lse=l2, acc=c.acc)
    assert o2.equal(out) and l2.equal(lse) and c.acc.nan_to_num(3).equal(acc.nan_to_num(3))
    for fmt in ("int8", "e4m3"):
        e = Cache8(gpu_lib, [300, 70, 5], 2, 4, 128, 48, "bf16", fmt, seed=8).cuda()
        q = e.rand(3, 8, 128).bfloat16().cuda()
        acc0 = e.acc.clone()
        out, lse = decode_q8(e, q)
        acc, e.acc = e.acc, _shifted(acc0, 1)
        e.ks, e.vs, e.table, e.lens, e.pos = _shifted(e.ks, 1), _shifted(e.vs, 2), _shifted(e.table), _shifted(e.lens), _shifted(e.pos, 3)
        o2, l2 = decode_q8(e, q)
        assert o2.equal(out) and l2.equal(lse) and e.acc.nan_to_num(3).equal(acc.nan_to_num(3))

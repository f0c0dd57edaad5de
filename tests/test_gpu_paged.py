"""The paged cache on the GPU: append, decode and evict against their definitions in
float64 (serve_testlib), through the binding."""
import math

import numpy as np
import pytest

import serve_testlib as ref

pytestmark = pytest.mark.gpu


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


class Cache:
    """A pool whose unused slots hold NaN, with its page table: pages in no order, -1
    or ids beyond the pool behind a sequence's last page."""

    def __init__(self, kv, lens, H, G, d, page, dt, seed=0, rows_first=False, spare_pages=2, max_pages=None, full=False):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.kv, self.lens_l, self.H, self.G, self.d, self.page, self.dt = kv, lens, H, G, d, page, dt
        used = [(n + page - 1) // page for n in lens]
        mp = max_pages or max(max(used), 1)
        n_pages = sum(used) + spare_pages
        ids = torch.randperm(n_pages, generator=g)[: sum(used)]
        self.table = torch.tensor([-1, n_pages, 2**31 - 1, -2**31]).repeat(len(lens) * mp)[: len(lens) * mp].view(len(lens), mp).int().clone()
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = ids[at:at + u].int()
            at += u
        self.cfg = kv.PagedConfig(len(lens), H, H * G, d, page, n_pages, mp, kv.KVEC_BF16 if dt == "bf16" else kv.KVEC_F32)
        shape = (n_pages, page, H, d) if rows_first else (n_pages, H, page, d)
        self.k, self.v = (torch.full(shape, float("nan")).to(_dt(dt)) for _ in range(2))
        if rows_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.acc = torch.full((n_pages, H, page), float("nan"))
        self.pos = torch.full((n_pages, H, page), -7, dtype=torch.int32)
        for i, n in enumerate(lens):
            p, r = ref.rows_of(self.table[i].numpy(), used[i] * page if full else n, page, n_pages)
            p, r = torch.from_numpy(p), torch.from_numpy(r)
            m = len(p)
            self.k[p, :, r] = (torch.randn((m, H, d), generator=g) * 1.5).to(_dt(dt))
            self.v[p, :, r] = torch.randn((m, H, d), generator=g).to(_dt(dt))
            self.acc[p, :, r] = torch.rand((m, H), generator=g) ** 3 * 4
            self.pos[p, :, r] = torch.arange(m, dtype=torch.int32)[:, None]
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.rand = lambda *s: torch.randn(s, generator=g)
        self.gen = g

    def cuda(self):
        for n in ("table", "k", "v", "acc", "pos", "lens"):
            t = getattr(self, n)
            if n in ("k", "v") and not t.is_contiguous():
                setattr(self, n, t.transpose(1, 2).cuda().transpose(1, 2))
            else:
                setattr(self, n, t.cuda())
        return self

    def slots(self, i, n):
        return ref.rows_of(self.table[i].cpu().numpy(), n, self.page, self.cfg.n_pages)


def _decode(c, q, window=0, sinks=0, acc=True, max_len=None, stream=None):
    import torch
    kv, b = c.kv, len(c.lens_l)
    ws = torch.empty(kv.kvec_paged_decode_workspace_size(c.cfg, max_len, acc), dtype=torch.uint8, device="cuda").fill_(255)
    out = torch.full((b, c.H * c.G, c.d), float("nan"), device="cuda")
    lse = torch.full((b, c.H * c.G), float("nan"), device="cuda")
    kv.kvec_paged_decode(c.cfg, q, c.k, c.v, c.table, c.lens, out, ws, max_len=max_len, window=window, n_sinks=sinks, lse=lse,
                         acc=c.acc if acc else None, stream=stream)
    return out, lse


def _check_decode(c, q, out, lse, acc0, window=0, sinks=0, max_len=None):
    """out, lse and the accumulated weights of every slot of the pool."""
    kn, vn, qn = ref.f64(c.k), ref.f64(c.v), ref.f64(q)
    got, got_lse = ref.f64(out), ref.f64(lse)
    want_acc = None if acc0 is None else ref.f64(acc0)
    slack = None if acc0 is None else np.zeros_like(want_acc)
    for i, n in enumerate(c.lens_l):
        n = max(0, min(n, max_len or c.cfg.max_pages * c.page))
        page, row = c.slots(i, n)
        seen = ref.visible(n, n, n - 1, window, sinks) & (page >= 0)
        for h in range(c.H):
            k, v = kn[page, h, row], vn[page, h, row]
            k[~seen], v[~seen] = 0, 0
            for g in range(c.G):
                o, l, w, dx = ref.attend(qn[i, h * c.G + g], k, v, seen)
                tol = (2 * dx + ref.EXP) * max(np.abs(v).max(initial=0), 1e-30)
                assert np.abs(got[i, h * c.G + g] - o).max() <= tol, (i, h, g, np.abs(got[i, h * c.G + g] - o).max(), tol)
                gl = got_lse[i, h * c.G + g]
                assert gl == l or abs(gl - l) <= dx + ref.EXP * (1 + abs(l)), (i, h, g, gl, l)
                if acc0 is not None:
                    want_acc[page[seen], h, row[seen]] += w[seen] / c.G
                    slack[page[seen], h, row[seen]] += w[seen] / c.G * (2 * dx + ref.EXP)
    if acc0 is not None:
        a = ref.f64(c.acc)
        assert np.array_equal(np.isnan(a), np.isnan(want_acc))
        ok = ~np.isnan(a)
        assert np.all(np.abs(a - want_acc)[ok] <= slack[ok] + np.abs(want_acc[ok]) * 2 * ref.U24)


DECODE = [  # lens, H, G, d, page, dtype, window, sinks, rows first
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 100], 2, 4, 128, 16, "bf16", 0, 0, False),
    ([129, 1, 1000, 64], 8, 4, 128, 64, "bf16", 0, 0, False),
    ([700, 0, 333], 4, 7, 128, 48, "bf16", 0, 0, True),
    ([260, 511], 1, 16, 64, 128, "bf16", 0, 0, False),
    ([77, 78], 3, 1, 64, 80, "bf16", 0, 0, True),
    ([5, 130], 2, 5, 128, 16, "f32", 0, 0, False),
    ([1, 300, 64], 4, 2, 64, 32, "f32", 0, 0, True),
    ([40, 3], 1, 16, 128, 16, "f32", 0, 0, False),
    ([500, 20, 65, 0], 2, 4, 128, 16, "bf16", 64, 4, False),
    ([500, 70, 90], 2, 3, 64, 64, "bf16", 50, 37, True),
    ([333, 18], 2, 2, 128, 16, "f32", 1, 0, False),
    ([333, 18], 2, 2, 128, 16, "bf16", 17, 300, False),
    ([9000], 1, 2, 64, 256, "bf16", 0, 0, False),
    # more sequences and heads than it takes work-groups: not split
    ([1100, 0, 5, 290] + [3] * 124, 8, 2, 64, 64, "bf16", 0, 0, False),
    ([1300, 17, 450] + [20] * 125, 8, 5, 64, 16, "f32", 400, 5, False),
    # many sequences, many heads, a page that holds a whole sequence
    ([i % 40 for i in range(500)], 1, 1, 64, 16, "bf16", 0, 0, False),
    ([33, 290], 256, 1, 64, 16, "bf16", 0, 0, False),
    ([1999, 2048], 2, 3, 128, 2048, "bf16", 0, 0, False),
]


@pytest.mark.parametrize("lens,H,G,d,page,dt,window,sinks,rows_first", DECODE)
def test_decode(gpu_lib, lens, H, G, d, page, dt, window, sinks, rows_first):
    c = Cache(gpu_lib, lens, H, G, d, page, dt, seed=len(lens) + G, rows_first=rows_first).cuda()
    q = c.rand(len(lens), H * G, d).mul_(2).to(_dt(dt)).cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks)
    _check_decode(c, q, out, lse, acc0, window, sinks)
    # without the weights: the same bits
    o2, l2 = _decode(c, q, window, sinks, acc=False)
    assert o2.equal(out) and l2.equal(lse)


def test_decode_lengths_are_clamped_and_pages_checked(gpu_lib):
    """Lengths beyond max_len or below 0, and table entries that are no pages inside a
    sequence: their slots are not there."""
    import torch
    c = Cache(gpu_lib, [200, 200, 90], 2, 4, 64, 16, "bf16", seed=3).cuda()
    c.lens_l = [200, 5000, -3]
    c.lens.copy_(torch.tensor(c.lens_l))
    c.table[0, 2], c.table[0, 7], c.table[1, 0] = -1, c.cfg.n_pages, 2**31 - 1
    q = c.rand(3, 8, 64).bfloat16().cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, max_len=150)
    _check_decode(c, q, out, lse, acc0, max_len=150)
    assert torch.all(out[2] == 0) and torch.all(lse[2] == -math.inf)


def test_decode_strided_queries_and_shared_pages(gpu_lib):
    """Queries inside a larger projection; two sequences that share a prefix's pages."""
    c = Cache(gpu_lib, [128, 128], 2, 4, 128, 64, "bf16", seed=4)
    c.table[1, 0] = c.table[0, 0]
    c.cuda()
    wide = c.rand(2, 12, 128).bfloat16().cuda()
    q = wide[:, 2:10]
    out, lse = _decode(c, q, acc=False)
    _check_decode(c, q, out, lse, None)


def test_decode_extreme_logits(gpu_lib):
    """Logits of thousands, of both signs, and equal ones."""
    c = Cache(gpu_lib, [600, 100], 1, 2, 64, 16, "f32", seed=5).cuda()
    page, row = c.slots(0, 600)
    c.k[page[300], 0, row[300]] = 400.0
    c.k[page[:200], 0, row[:200]] = -300.0
    page, row = c.slots(1, 100)
    c.k[page, :, row] = c.k[page[0], 0, row[0]].clone()
    q = c.rand(2, 2, 64).abs().cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q)
    _check_decode(c, q, out, lse, acc0)


def test_decode_far_offsets(gpu_lib):
    """Rows behind 2^31 elements and 2^32 bytes of the pool."""
    import torch
    kv = gpu_lib
    H, page, d, n_pages = 2, 1024, 128, 8300  # 2.2e9 elements: 4.4 GB a pool
    cfg = kv.PagedConfig(1, H, 2 * H, d, page, n_pages, 2)
    c = Cache(kv, [1500], H, 2, d, page, "bf16", seed=6)
    k, v = (torch.empty((n_pages, H, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    where = [n_pages - 1, 4100]
    for j, p in enumerate(where):
        k[p], v[p] = c.k[c.table[0, j]].cuda(), c.v[c.table[0, j]].cuda()
    small = Cache(kv, [1500], H, 2, d, page, "bf16", seed=6).cuda()
    q = c.rand(1, 2 * H, d).bfloat16().cuda()
    acc = torch.zeros((n_pages, H, page), device="cuda")
    small.acc.zero_()
    out, lse = torch.empty(1, 2 * H, d, device="cuda"), torch.empty(1, 2 * H, device="cuda")
    ws = torch.empty(kv.kvec_paged_decode_workspace_size(cfg, None, True), dtype=torch.uint8, device="cuda")
    kv.kvec_paged_decode(cfg, q, k, v, torch.tensor([where], dtype=torch.int32, device="cuda"), small.lens, out, ws, lse=lse, acc=acc)
    o2, l2 = _decode(small, q)
    assert out.equal(o2) and lse.equal(l2)
    for j, p in enumerate(where):
        assert acc[p].equal(small.acc[small.table[0, j].item()])


def test_append_and_evict_far_offsets(gpu_lib):
    """The same rows in the last pages of a pool of 4.4 GB and in a small one."""
    import torch
    kv, H, page, d, n_pages = gpu_lib, 2, 1024, 128, 8300
    small = Cache(kv, [2000], H, 2, d, page, "bf16", seed=41)
    where = [n_pages - 1, n_pages - 7]
    big = {}
    for name, like in (("k", small.k), ("v", small.v), ("acc", small.acc), ("pos", small.pos)):
        big[name] = torch.empty((n_pages, *like.shape[1:]), dtype=like.dtype, device="cuda")
        for j, p in enumerate(where):
            big[name][p] = like[small.table[0, j]].cuda()
    small.cuda()
    cfg = kv.PagedConfig(1, H, 2 * H, d, page, n_pages, 2)
    table, lens = torch.tensor([where], dtype=torch.int32, device="cuda"), small.lens
    q, k, v = (small.rand(9, h, d).bfloat16().cuda() for h in (2 * H, H, H))
    fr = torch.rand(d // 2, dtype=torch.float64, device="cuda")
    at = torch.arange(1500, 1509)
    pos = at.int().cuda()
    outs = []
    for c, tb, t in ((cfg, table, big), (small.cfg, small.table, dict(k=small.k, v=small.v, acc=small.acc, pos=small.pos))):
        slots = (tb[0].long()[(at // page).cuda()] * page + (at % page).cuda())
        q_out = torch.empty_like(q)
        kv.kvec_paged_append(c, q, k, v, pos, slots, q_out, t["k"], t["v"], inv_freq=fr, acc=t["acc"], pos=t["pos"])
        ws = torch.empty(kv.kvec_paged_evict_workspace_size(c, None, 900), dtype=torch.uint8, device="cuda")
        kept, out = torch.empty((1, H, 900), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        kv.kvec_paged_evict(c, 900, t["k"], t["v"], tb, lens, lens, t["acc"], t["pos"], out, ws, window=50, n_sinks=4, kept=kept)
        outs.append((q_out, kept, out, *(t[n][tb[0].long()].nan_to_num(9) for n in ("k", "v", "acc")), t["pos"][tb[0].long()]))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_two_streams_at_once(gpu_lib):
    """Calls on two streams, each with a workspace of its own, over one pool."""
    import torch
    c = Cache(gpu_lib, [3000, 2500, 100], 4, 4, 128, 64, "bf16", seed=42).cuda()
    qs = [c.rand(3, 16, 128).bfloat16().cuda() for _ in range(2)]
    wants = [_decode(c, q, acc=False) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    size = gpu_lib.kvec_paged_decode_workspace_size(c.cfg)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [[torch.empty(3, 16, 128, device="cuda") for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for j, s in enumerate(streams):
            gpu_lib.kvec_paged_decode(c.cfg, qs[j], c.k, c.v, c.table, c.lens, outs[j][i], ws[j], stream=s)
    torch.cuda.synchronize()
    for j in range(2):
        assert all(o.equal(wants[j][0]) for o in outs[j])


APPEND = [  # tokens, H, G, d, page, dtype, rot, norm, start
    (1, 8, 4, 128, 64, "bf16", 128, True, 130000),
    (5, 4, 7, 128, 16, "bf16", 64, False, 7),
    (37, 2, 2, 64, 48, "bf16", 64, True, 0),
    (37, 1, 16, 64, 16, "f32", 16, True, 1000000),
    (1030, 2, 1, 128, 256, "f32", 128, False, 5),
    (1031, 1, 3, 64, 16, "bf16", 48, True, 100),
    # several tokens a work-group, the last one with fewer
    (1537, 2, 1, 128, 256, "f32", 128, False, 5),
    (1551, 1, 3, 64, 16, "bf16", 48, True, 100),
    (3, 2, 2, 128, 16, "f32", 112, True, -5),
    (4, 2, 2, 64, 16, "bf16", 0, True, 0),
    (4, 2, 2, 64, 16, "f32", 0, False, 0),
]


@pytest.mark.parametrize("n,H,G,d,page,dt,rot,norm,start", APPEND)
def test_append(gpu_lib, n, H, G, d, page, dt, rot, norm, start):
    """Every row of q_out and of the pools, those that no token takes included; every
    fifth token is padding (slot -1, or one beyond the pool)."""
    import torch
    c = Cache(gpu_lib, [n + 20], H, G, d, page, dt, seed=n).cuda()
    qkv = c.rand(n, H * G + 2 * H, d).mul_(3).to(_dt(dt)).cuda()
    q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
    wq, wk = ((1 + 0.2 * c.rand(d)).to(_dt(dt)).cuda() if norm else None for _ in range(2))
    inv_freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None
    positions = (torch.arange(n) * 3 + start).int().cuda()
    page_i, row_i = c.slots(0, n + 20)
    order = torch.randperm(n + 20, generator=c.gen)[:n].numpy()
    slots = torch.from_numpy(page_i[order].astype(np.int64) * page + row_i[order])
    total = c.cfg.n_pages * page
    slots[::5] = torch.tensor([-1, total, -2**62, 2**62]).repeat(n)[: len(slots[::5])]
    q_out = torch.full((n, H * G, d), float("nan"), dtype=_dt(dt), device="cuda")
    k0, v0, acc0, pos0 = (ref.f64(t) for t in (c.k, c.v, c.acc, c.pos))
    gpu_lib.kvec_paged_append(c.cfg, q, k, v, positions, slots.cuda(), q_out, c.k, c.v, q_weight=wq, k_weight=wk, eps=1e-5, inv_freq=inv_freq,
                              acc=c.acc, pos=c.pos)
    u = ref.half_step(_dt(dt))
    fr = None if inv_freq is None else ref.f64(inv_freq)
    got_q, got_k = ref.f64(q_out), ref.f64(c.k)
    want_k, off_k = k0.copy(), np.zeros_like(k0)
    for t in range(n):
        at = int(positions[t])
        if t % 7 == 0 or n < 50:  # queries: every row of the small cases
            for j in range(H * G):
                y, off = ref.rotated(ref.f64(q[t, j]), None if wq is None else ref.f64(wq), 1e-5, at, fr)
                assert np.all(np.abs(got_q[t, j] - y) <= off * (1 + u) + u * np.abs(y)), (t, j)
        s = int(slots[t])
        if 0 <= s < total:
            for h in range(H):
                y, off = ref.rotated(ref.f64(k[t, h]), None if wk is None else ref.f64(wk), 1e-5, at, fr)
                want_k[s // page, h, s % page], off_k[s // page, h, s % page] = y, off * (1 + u) + u * np.abs(y)
            v0[s // page, :, s % page] = ref.f64(v[t])
            acc0[s // page, :, s % page] = 0
            pos0[s // page, :, s % page] = at
    nan = np.isnan(want_k)
    assert np.array_equal(nan, np.isnan(got_k))
    assert np.all((np.abs(got_k - want_k) <= off_k) | nan)
    for got, want in ((c.v, v0), (c.acc, acc0), (c.pos, pos0)):
        assert np.array_equal(ref.f64(got), want, equal_nan=True)
    assert not torch.isnan(q_out).any()


def test_append_in_place_and_rows_first(gpu_lib):
    """q_out may be q; a pool of [page][row][head] order; no acc, no pos, no norm of one side."""
    import torch
    a, b = (Cache(gpu_lib, [64], 2, 4, 128, 32, "bf16", seed=9, rows_first=f).cuda() for f in (False, True))
    q, k, v = (a.rand(64, h, 128).bfloat16().cuda() for h in (8, 2, 2))
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    page, row = a.slots(0, 64)
    slots = torch.from_numpy(page.astype(np.int64) * 32 + row).cuda()
    fr = torch.rand(64, dtype=torch.float64, device="cuda")
    pos = torch.arange(64, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    gpu_lib.kvec_paged_append(a.cfg, q, k, v, pos, slots, out, a.k, a.v, k_weight=w, inv_freq=fr)
    gpu_lib.kvec_paged_append(b.cfg, q, k, v, pos, slots, q, b.k, b.v, k_weight=w, inv_freq=fr)
    assert q.equal(out)
    assert torch.equal(a.k.nan_to_num(9), b.k.nan_to_num(9)) and torch.equal(a.v.nan_to_num(9), b.v.nan_to_num(9))


def test_append_of_nothing(gpu_lib):
    import torch
    c = Cache(gpu_lib, [10], 2, 2, 64, 16, "f32").cuda()
    e = lambda h: torch.empty((0, h, 64), device="cuda")  # noqa: E731
    before = c.k.clone()
    gpu_lib.kvec_paged_append(c.cfg, e(4), e(2), e(2), torch.empty(0, dtype=torch.int32, device="cuda"),
                              torch.empty(0, dtype=torch.int64, device="cuda"), e(4), c.k, c.v)
    assert torch.equal(before.nan_to_num(3), c.k.nan_to_num(3))


def _evict(c, budget, window, sinks, seen, max_len=None, in_place=False):
    import torch
    kv, b = c.kv, len(c.lens_l)
    ws = torch.full((kv.kvec_paged_evict_workspace_size(c.cfg, max_len, budget),), 255, dtype=torch.uint8, device="cuda")
    kept = torch.full((b, c.H, budget), -9, dtype=torch.int32, device="cuda")
    out = c.lens if in_place else torch.full((b,), -9, dtype=torch.int32, device="cuda")
    kv.kvec_paged_evict(c.cfg, budget, c.k, c.v, c.table, c.lens, seen, c.acc, c.pos, out, ws, window=window, n_sinks=sinks, kept=kept,
                        max_len=max_len)
    return kept, out


def _check_evict(c, before, kept, out, budget, window, sinks, seen, max_len=None):
    """Bit for bit: kept slots, lengths, and the whole pools."""
    import torch
    k0, v0, acc0, pos0 = (t.cpu().clone() for t in before)
    kept, out, seen = kept.cpu().numpy(), out.cpu().numpy(), seen.cpu().numpy()
    for i, n in enumerate(c.lens_l):
        n = max(0, min(n, max_len or c.cfg.max_pages * c.page))
        page, row = c.slots(i, max(n, budget) if (max(n, budget) + c.page - 1) // c.page <= c.cfg.max_pages else n)
        for h in range(c.H):
            p, r = page[:n], row[:n]
            ok = p >= 0
            want, m = ref.evict(before[2].cpu().numpy()[p, h, r], before[3].cpu().numpy()[p, h, r], ok, n, budget, window, sinks, seen[i])
            assert np.array_equal(kept[i, h], want), (i, h)
            assert out[i] == m
            d = np.arange(m)
            d = d[(want[:m] != d) & ok[:m]]
            d = d[ok[want[d]]]
            for t, o in ((k0, before[0]), (v0, before[1]), (acc0, before[2]), (pos0, before[3])):
                t[p[d], h, r[d]] = o.cpu()[p[want[d]], h, r[want[d]]]
    for got, want in ((c.k, k0), (c.v, v0), (c.acc, acc0), (c.pos, pos0)):
        got = got.cpu()
        bits = torch.int16 if got.element_size() == 2 else torch.int32
        assert torch.equal(got.contiguous().view(bits), want.contiguous().view(bits))


EVICT = [  # lens, H, d, page, dtype, budget, window, sinks, rows first
    ([0, 1, 16, 17, 40, 33], 2, 64, 16, "bf16", 16, 3, 2, False),
    ([300, 128, 129, 250], 8, 128, 64, "bf16", 128, 32, 4, False),
    ([1000, 77], 1, 128, 48, "f32", 64, 0, 0, True),
    ([500, 900], 4, 64, 16, "f32", 400, 400, 0, True),
    ([4096, 4095], 2, 64, 256, "bf16", 1, 0, 1, False),
    ([5000, 3000, 10], 2, 64, 128, "bf16", 2999, 100, 16, False),
    ([33000], 1, 64, 1024, "bf16", 3001, 8, 8, False),
    ([i % 50 for i in range(400)], 2, 64, 16, "bf16", 20, 5, 3, False),
    ([60, 41], 200, 64, 16, "f32", 40, 40, 0, True),
    ([4097, 4096, 4099], 1, 128, 2048, "bf16", 4096, 10, 10, False),
]


@pytest.mark.parametrize("lens,H,d,page,dt,budget,window,sinks,rows_first", EVICT)
def test_evict(gpu_lib, lens, H, d, page, dt, budget, window, sinks, rows_first):
    import torch
    c = Cache(gpu_lib, lens, H, 1, d, page, dt, seed=budget, rows_first=rows_first).cuda()
    before = [t.clone() for t in (c.k, c.v, c.acc, c.pos)]
    seen = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kept, out = _evict(c, budget, window, sinks, seen)
    _check_evict(c, before, kept, out, budget, window, sinks, seen)
    assert c.lens.tolist() == lens


@pytest.mark.parametrize("kind", ["equal", "few values", "nan and inf", "zeros of both signs", "shuffled positions"])
def test_evict_ties_and_special_weights(gpu_lib, kind):
    import torch
    c = Cache(gpu_lib, [700, 1300], 2, 1, 64, 16, "bf16", seed=11)
    g = torch.Generator().manual_seed(12)
    x = c.acc
    if kind == "equal":
        x.fill_(0.25)
    elif kind == "few values":
        x.copy_(torch.randint(0, 3, x.shape, generator=g).float())
    elif kind == "nan and inf":
        x.copy_(torch.tensor([math.nan, -math.nan, math.inf, -math.inf, 1.0, -1.0, 3e38, 1e-45])[torch.randint(0, 8, x.shape, generator=g)])
    elif kind == "zeros of both signs":
        x.copy_(torch.tensor([0.0, -0.0])[torch.randint(0, 2, x.shape, generator=g)])
    else:
        c.pos = torch.randint(-5, 2000, c.pos.shape, generator=g, dtype=torch.int32)
    c.cuda()
    before = [t.clone() for t in (c.k, c.v, c.acc, c.pos)]
    seen = torch.tensor([1990, 1700], dtype=torch.int32, device="cuda")
    kept, out = _evict(c, 500, 300, 100, seen)
    _check_evict(c, before, kept, out, 500, 300, 100, seen)


@pytest.mark.parametrize("lens,budget", [([32768, 32769, 40000], 20000), ([65537], 33000), ([4096, 4097], 1500)])
def test_evict_few_values_at_the_ends_of_key_tiles(gpu_lib, lens, budget):
    """Ties, kept and evicted slots on both sides of the 4096 and 32768 keys held at a time."""
    import torch
    c = Cache(gpu_lib, lens, 1, 1, 64, 256, "bf16", seed=15)
    c.acc.copy_(torch.randint(0, 4, c.acc.shape, generator=c.gen).float())
    c.cuda()
    before = [t.clone() for t in (c.k, c.v, c.acc, c.pos)]
    seen = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kept, out = _evict(c, budget, 700, 5, seen)
    _check_evict(c, before, kept, out, budget, 700, 5, seen)


@pytest.mark.parametrize("lens,d,dt,budget", [([300, 257, 256, 5], 64, "bf16", 256), ([290, 500, 0], 128, "bf16", 256), ([200, 129], 128, "f32", 128),
                                              ([90, 64, 77], 64, "f32", 60), ([40, 60], 128, "bf16", 3)])
def test_evict_few_rows_with_lengths_apart_and_in_place(gpu_lib, lens, d, dt, budget):
    """Few rows to move: the same results whether the lengths are replaced in place or not."""
    import torch
    seen = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for in_place in (False, True):
        c = Cache(gpu_lib, lens, 3, 1, d, 32, dt, seed=budget).cuda()
        before = [t.clone() for t in (c.k, c.v, c.acc, c.pos)]
        kept, out = _evict(c, budget, 1, 1, seen, in_place=in_place)
        _check_evict(c, before, kept, out, budget, 1, 1, seen)


def test_evict_in_place_lengths_bad_pages_and_clamped_lengths(gpu_lib):
    """lens_out = lens = n_seen; slots without a page rank last and do not move."""
    import torch
    c = Cache(gpu_lib, [200, 200, 90], 2, 1, 64, 16, "f32", seed=13).cuda()
    c.lens_l = [200, 5000, -3]
    c.lens.copy_(torch.tensor(c.lens_l))
    c.table[0, 2], c.table[0, 11], c.table[1, 0] = -1, c.cfg.n_pages, 2**31 - 1
    before = [t.clone() for t in (c.k, c.v, c.acc, c.pos)]
    seen = c.lens.clone()
    ws = torch.empty(c.kv.kvec_paged_evict_workspace_size(c.cfg, 190, 100), dtype=torch.uint8, device="cuda")
    kept = torch.full((3, 2, 100), -9, dtype=torch.int32, device="cuda")
    c.kv.kvec_paged_evict(c.cfg, 100, c.k, c.v, c.table, c.lens, c.lens, c.acc, c.pos, c.lens, ws, window=20, n_sinks=4, kept=kept, max_len=190)
    _check_evict(c, before, kept, c.lens, 100, 20, 4, seen, max_len=190)
    assert c.lens.tolist() == [100, 100, 0]


def test_evict_budget_above_every_length(gpu_lib):
    """max_len <= budget: nothing moves, kept and lengths are still written."""
    import torch
    c = Cache(gpu_lib, [30, 0, 17], 2, 1, 64, 16, "bf16", seed=14).cuda()
    before = [t.clone() for t in (c.k, c.v, c.acc, c.pos)]
    kept, out = _evict(c, 600, 5, 5, c.lens)
    _check_evict(c, before, kept, out, 600, 5, 5, c.lens)


def test_serving_loop(gpu_lib):
    """Tokens appended one by one, each attending over what the cache then holds, the
    cache evicted whenever it is over its budget; against the same loop in float64 on
    lists of slots (picks follow the GPU's weights, which are held to theirs)."""
    import torch
    kv, H, G, d, page, budget = gpu_lib, 2, 3, 64, 16, 40
    steps, b = 90, 2
    cap = 64
    cfg = kv.PagedConfig(b, H, H * G, d, page, b * cap // page, cap // page)
    g = torch.Generator().manual_seed(21)
    table = torch.randperm(cfg.n_pages, generator=g).view(b, -1).int().cuda()
    k_pool, v_pool = (torch.full((cfg.n_pages, H, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    acc = torch.full((cfg.n_pages, H, page), float("nan"), device="cuda")
    pos = torch.full((cfg.n_pages, H, page), -1, dtype=torch.int32, device="cuda")
    fr = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    lens, seen = torch.zeros(b, dtype=torch.int32, device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")
    wd = torch.empty(kv.kvec_paged_decode_workspace_size(cfg, None, True), dtype=torch.uint8, device="cuda")
    we = torch.empty(kv.kvec_paged_evict_workspace_size(cfg, None, budget), dtype=torch.uint8, device="cuda")
    out, q_out = torch.empty(b, H * G, d, device="cuda"), torch.empty(b, H * G, d, dtype=torch.bfloat16, device="cuda")
    mirror = [[[] for _ in range(H)] for _ in range(b)]  # per head: [k, v, weight, position] of every slot
    evictions = 0
    for t in range(steps):
        q, k, v = (torch.randn((b, h, d), generator=g).bfloat16() for h in (H * G, H, H))
        at = lens.long()
        slots = table[torch.arange(b, device="cuda"), at // page].long() * page + at % page
        kv.kvec_paged_append(cfg, q.cuda(), k.cuda(), v.cuda(), seen, slots, q_out, k_pool, v_pool, inv_freq=fr.cuda(), acc=acc, pos=pos)
        lens += 1
        seen += 1
        kv.kvec_paged_decode(cfg, q_out, k_pool, v_pool, table, lens, out, wd, acc=acc)
        qn, got = ref.f64(q_out), ref.f64(out)
        kn, an = ref.f64(k_pool), ref.f64(acc)
        for i in range(b):
            n = int(lens[i])
            p, r = ref.rows_of(table[i].cpu().numpy(), n, page, cfg.n_pages)
            for h in range(H):
                m = mirror[i][h]
                want, off = ref.rotated(ref.f64(k[i, h]), None, 0, t, fr.numpy())
                row = kn[p[-1], h, r[-1]]
                assert np.all(np.abs(row - want) <= off * 1.01 + ref.U_BF16 * np.abs(want))
                m.append([row, ref.f64(v[i, h]), 0.0, t])
                ks, vs = np.stack([x[0] for x in m]), np.stack([x[1] for x in m])
                for gq in range(G):
                    o, _, w, dx = ref.attend(qn[i, h * G + gq], ks, vs, np.ones(n, bool))
                    assert np.abs(got[i, h * G + gq] - o).max() <= (2 * dx + ref.EXP) * np.abs(vs).max()
                    for x, y in zip(m, w):
                        x[2] += y / G
                have = an[p, h, r]
                assert np.allclose([x[2] for x in m], have, rtol=(t + 1) * (2 * dx + ref.EXP), atol=0)
                for x, y in zip(m, have):
                    x[2] = y
        if t % 11 == 10:
            kept = torch.empty((b, H, budget), dtype=torch.int32, device="cuda")
            over = int(lens.max()) > budget
            kv.kvec_paged_evict(cfg, budget, k_pool, v_pool, table, lens, seen, acc, pos, lens, we, window=8, n_sinks=2, kept=kept)
            for i in range(b):
                for h in range(H):
                    m = mirror[i][h]
                    want, n = ref.evict([x[2] for x in m], [x[3] for x in m], np.ones(len(m), bool), len(m), budget, 8, 2, t + 1)
                    assert np.array_equal(kept[i, h].cpu().numpy(), want)
                    mirror[i][h] = [list(m[s]) for s in want[:n]]
                    assert {x[3] for x in mirror[i][h]} >= {0, 1} | set(range(max(0, t - 7), t + 1))
            evictions += over
    assert evictions >= 3
    assert lens.tolist() == [len(mirror[i][0]) for i in range(b)]


def test_streams_and_graph(gpu_lib):
    """A decode step (append, decode with weights, evict) captured once and replayed,
    with eager work between, equals the eager steps; on a stream of its own."""
    import torch
    kv, H, G, d, page, budget, b = gpu_lib, 2, 4, 128, 16, 60, 2

    def state():
        c = Cache(kv, [60, 55], H, G, d, page, "bf16", seed=31, max_pages=6).cuda()
        need = [(70 + page - 1) // page] * b
        ids = torch.arange(sum(need), dtype=torch.int32).view(b, -1)
        n_pages = sum(need) + 1
        k, v = (torch.zeros((n_pages, H, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        acc, pos = torch.zeros((n_pages, H, page), device="cuda"), torch.zeros((n_pages, H, page), dtype=torch.int32, device="cuda")
        for i, n in enumerate(c.lens_l):
            p, r = c.slots(i, n)
            for s in range(n):
                at = (int(ids[i, s // page]), slice(None), s % page)
                for dst, src in ((k, c.k), (v, c.v), (acc, c.acc), (pos, c.pos)):
                    dst[at] = src[p[s], :, r[s]]
        cfg = kv.PagedConfig(b, H, H * G, d, page, n_pages, need[0])
        s = dict(cfg=cfg, k=k, v=v, acc=acc, pos=pos, table=ids.cuda(), lens=c.lens.clone(), seen=c.lens.clone(),
                 q=torch.zeros(b, H * G, d, dtype=torch.bfloat16, device="cuda"), nk=torch.zeros(b, H, d, dtype=torch.bfloat16, device="cuda"),
                 out=torch.zeros(b, H * G, d, device="cuda"), q_out=torch.zeros(b, H * G, d, dtype=torch.bfloat16, device="cuda"),
                 fr=torch.rand(d // 2, dtype=torch.float64, generator=torch.Generator().manual_seed(1)).cuda())
        s["wd"] = torch.empty(kv.kvec_paged_decode_workspace_size(cfg, None, True), dtype=torch.uint8, device="cuda")
        s["we"] = torch.empty(kv.kvec_paged_evict_workspace_size(cfg, None, budget), dtype=torch.uint8, device="cuda")
        return s

    def step(s):
        at = s["lens"].long()
        slots = s["table"].gather(1, (at // page)[:, None])[:, 0].long() * page + at % page
        kv.kvec_paged_append(s["cfg"], s["q"], s["nk"], s["nk"], s["seen"], slots, s["q_out"], s["k"], s["v"], inv_freq=s["fr"], acc=s["acc"],
                             pos=s["pos"])
        s["lens"] += 1
        s["seen"] += 1
        kv.kvec_paged_decode(s["cfg"], s["q_out"], s["k"], s["v"], s["table"], s["lens"], s["out"], s["wd"], acc=s["acc"])
        kv.kvec_paged_evict(s["cfg"], budget, s["k"], s["v"], s["table"], s["lens"], s["seen"], s["acc"], s["pos"], s["lens"], s["we"], window=8)

    gen = torch.Generator().manual_seed(33)
    inputs = [(torch.randn((b, H * G, d), generator=gen).bfloat16().cuda(), torch.randn((b, H, d), generator=gen).bfloat16().cuda()) for _ in range(12)]
    eager, graphed = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    warm = state()
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    for q, nk in inputs:
        for s in (eager, graphed):
            s["q"].copy_(q)
            s["nk"].copy_(nk)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step(eager)
        side.synchronize()
        graph.replay()
        (torch.randn(512, 512, device="cuda") @ torch.randn(512, 512, device="cuda")).sum().item()
        for name in ("out", "q_out", "k", "v", "acc", "pos", "lens", "seen"):
            assert torch.equal(eager[name], graphed[name]), name
    assert eager["lens"].tolist() == [60, 60]


@pytest.mark.parametrize("dt,G,n", [("bf16", 4, 1500), ("f32", 5, 700)])
def test_same_bits_twice(gpu_lib, dt, G, n):
    """A decode step gives the same bits whatever its workspace held."""
    import torch
    got = []
    for fill in (0, 255):
        c = Cache(gpu_lib, [n, 3, n // 2], 2, G, 64, 32, dt, seed=8).cuda()
        q = c.rand(3, 2 * G, 64).to(_dt(dt)).cuda()
        ws = torch.full((gpu_lib.kvec_paged_decode_workspace_size(c.cfg, None, True),), fill, dtype=torch.uint8, device="cuda")
        out, lse = torch.empty(3, 2 * G, 64, device="cuda"), torch.empty(3, 2 * G, device="cuda")
        gpu_lib.kvec_paged_decode(c.cfg, q, c.k, c.v, c.table, c.lens, out, ws, lse=lse, acc=c.acc)
        got.append([x.view(torch.int32) for x in (out, lse, c.acc)])
    assert all(x.equal(y) for x, y in zip(*got))


def test_binding_refuses_on_the_gpu(gpu_lib):
    """Tensors that do not fit the configuration, and values that the C interface refuses:
    the error is raised and nothing is written."""
    import torch
    kv, b, H, HQ, d, page = gpu_lib, 2, 2, 8, 64, 16
    cfg = kv.PagedConfig(b, H, HQ, d, page, 6, 3)
    zeros = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    i32 = torch.int32
    pools = dict(k_pool=zeros(6, H, page, d), v_pool=zeros(6, H, page, d))
    seq = dict(page_table=torch.arange(6, dtype=i32, device="cuda").view(b, 3), lens=zeros(b, t=i32) + 5)
    meta = dict(acc=zeros(6, H, page, t=torch.float32), pos=zeros(6, H, page, t=i32))
    ws = zeros(1 << 20, t=torch.uint8)
    tok = dict(q=zeros(3, HQ, d) + 1, k=zeros(3, H, d) + 1, v=zeros(3, H, d) + 1, positions=zeros(3, t=i32),
               slots=torch.arange(3, device="cuda"), q_out=zeros(3, HQ, d))
    wide, rows = zeros(6, H, page, 2 * d), zeros(6, page, H, d).transpose(1, 2)
    f32 = torch.float32
    attn = kv.AttentionConfig(b, H, HQ, d, 7, 40)
    prompt = dict(q=zeros(b, HQ, 7, d) + 1, k=zeros(b, H, 40, d) + 1, v=zeros(b, H, 40, d) + 1, out=zeros(b, HQ, 7, d), ws=ws)
    step = dict(q=zeros(b, HQ, d) + 1, out=zeros(b, HQ, d, t=f32), ws=ws)
    off = lambda t: torch.cat([t.flatten(), t.flatten()])[1:1 + t.numel()].view(t.shape)  # noqa: E731  (2 or 4 bytes off)
    cases = [
        (lambda **k: kv.kvec_paged_append(cfg, **k), {**tok, **pools, **meta},
         [dict(q=tok["q"][:, :7]), dict(k=tok["k"].float()), dict(v=tok["v"][:2]), dict(positions=tok["positions"].long()),
          dict(slots=tok["slots"].int()), dict(q_out=zeros(3, d, HQ).transpose(1, 2)), dict(k_pool=rows), dict(v_pool=pools["v_pool"].cpu()),
          dict(v_pool=wide[..., ::2]), dict(q_weight=zeros(d + 8)), dict(k_weight=zeros(d, t=f32)), dict(inv_freq=zeros(d // 2, t=f32)),
          dict(acc=meta["acc"].half()), dict(pos=meta["pos"][:5])],
         [dict(q=off(tok["q"])), dict(inv_freq=zeros(d // 2 + 8, t=torch.float64)), dict(inv_freq=zeros(3, t=torch.float64)), dict(eps=-1.0),
          dict(q_weight=off(zeros(d)))]),
        (lambda **k: kv.kvec_paged_decode(cfg, **k), {**step, **pools, **seq, "acc": meta["acc"]},
         [dict(q=step["q"][:1]), dict(out=step["out"].bfloat16()), dict(out=zeros(HQ, b, d, t=f32).transpose(0, 1)), dict(lens=seq["lens"].cpu()),
          dict(page_table=seq["page_table"][:, :2]), dict(lse=zeros(b, H, t=f32)), dict(acc=zeros(6, page, H, t=f32)), dict(ws=ws[::2]),
          dict(ws=ws.cpu()), dict(k_pool=wide[..., :d])],
         [dict(ws=None), dict(ws=ws[:64]), dict(ws=ws[1:]), dict(max_len=0), dict(max_len=49), dict(window=-1), dict(n_sinks=-1), dict(q=off(step["q"]))]),
        (lambda **k: kv.kvec_paged_evict(cfg, **{**dict(budget=4), **k}), {**pools, **seq, **meta, "n_seen": seq["lens"], "lens_out": zeros(b, t=i32), "ws": ws},
         [dict(n_seen=zeros(b + 1, t=i32)), dict(lens_out=zeros(b, t=f32)), dict(acc=None), dict(kept=zeros(b, H, 5, t=i32)),
          dict(kept=zeros(b, 4, H, t=i32).transpose(1, 2)), dict(pos=meta["pos"].cpu())],
         [dict(budget=0), dict(budget=(1 << 20) + 1), dict(window=4, n_sinks=1), dict(window=-1), dict(ws=None), dict(max_len=49)]),
        (lambda **k: kv.kvec_prefill_attention(attn, **k), prompt,
         [dict(q=prompt["q"][:, :, :6]), dict(k=prompt["k"][:, :1]), dict(v=prompt["v"].float()), dict(out=prompt["out"].cpu()),
          dict(lse=zeros(b, HQ, 7)), dict(lse=zeros(b, 7, HQ, t=f32).transpose(1, 2)), dict(q_lens=zeros(b, t=torch.int64)), dict(kv_lens=zeros(1, t=i32)),
          dict(k=prompt["k"].transpose(2, 3).contiguous().transpose(2, 3))],
         [dict(q=off(prompt["q"])), dict(out=zeros(b, HQ, 7, d + 4)[..., :d])]),
    ]
    before = [t.clone() for t in (*pools.values(), *meta.values(), tok["q_out"], step["out"], prompt["out"])]
    for call, good, misfits, invalid in cases:
        for bad in misfits:
            with pytest.raises(AssertionError):
                call(**{**good, **bad})
        for bad in invalid:
            with pytest.raises(kv.KvecError):
                call(**{**good, **bad})
    torch.cuda.synchronize()
    for x, t in zip(before, (*pools.values(), *meta.values(), tok["q_out"], step["out"], prompt["out"])):
        assert x.equal(t)
    for call, good, _, _ in cases:
        call(**good)  # and without a fault they run
    torch.cuda.synchronize()
    assert pools["k_pool"].any() and step["out"].any() and prompt["out"].any()

"""One token's attention of a batch behind a shared prefix on the GPU, against its float64
definition (serve_testlib) and the attention of single sequences."""
import math

import numpy as np
import pytest

import serve_testlib as ref

pytestmark = pytest.mark.gpu


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


class Shared:
    """A pool whose unused slots hold NaN: a prefix's pages and those of every sequence, in no
    order; no pages behind a sequence's last."""

    def __init__(self, kv, prefix, lens, H, G, d, page, dt, seed=0, rows_first=False, spare_pages=2):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.kv, self.P, self.lens_l, self.H, self.G, self.d, self.page, self.dt = kv, prefix, list(lens), H, G, d, page, dt
        used = [(max(n, 0) + page - 1) // page for n in (prefix, *lens)]
        mp = max(max(used[1:]), 1)
        n_pages = sum(used) + spare_pages
        ids = torch.randperm(n_pages, generator=g)[: sum(used)].int()
        bad = torch.tensor([-1, n_pages, 2**31 - 1, -2**31]).int()
        self.pages = torch.cat([ids[: used[0]], bad[:1]])  # one entry more than the prefix needs
        self.table = bad.repeat(len(lens) * mp)[: len(lens) * mp].view(len(lens), mp).clone()
        at = used[0]
        for i, u in enumerate(used[1:]):
            self.table[i, :u] = ids[at:at + u]
            at += u
        self.cfg = kv.PagedConfig(len(lens), H, H * G, d, page, n_pages, mp, kv.KVEC_BF16 if dt == "bf16" else kv.KVEC_F32)
        shape = (n_pages, page, H, d) if rows_first else (n_pages, H, page, d)
        self.k, self.v = (torch.full(shape, float("nan")).to(_dt(dt)) for _ in range(2))
        if rows_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.acc = torch.full((n_pages, H, page), float("nan"))
        for i, n in enumerate((prefix, *lens)):
            p, r = self._rows(self.pages if i == 0 else self.table[i - 1], max(n, 0))
            m = len(p)
            self.k[p, :, r] = (torch.randn((m, H, d), generator=g) * 1.5).to(_dt(dt))
            self.v[p, :, r] = torch.randn((m, H, d), generator=g).to(_dt(dt))
            self.acc[p, :, r] = torch.rand((m, H), generator=g) ** 3 * 4
        self.lens = torch.tensor(list(lens), dtype=torch.int32)
        self.plen = torch.tensor([prefix], dtype=torch.int32)
        self.rand = lambda *s: torch.randn(s, generator=g)
        self.gen = g

    def _rows(self, table, n):
        return ref.rows_of(table.cpu().numpy(), n, self.page, self.cfg.n_pages)

    def cuda(self):
        for n in ("pages", "table", "k", "v", "acc", "lens", "plen"):
            t = getattr(self, n)
            strided = n in ("k", "v") and not t.is_contiguous()
            setattr(self, n, t.transpose(1, 2).cuda().transpose(1, 2) if strided else t.cuda())
        return self


def _decode(c, q, window=0, sinks=0, acc=True, max_prefix=None, max_len=None, stream=None):
    import torch
    kv, b = c.kv, len(c.lens_l)
    most = len(c.pages) * c.page if max_prefix is None else max_prefix
    ws = torch.empty(kv.kvec_paged_decode_shared_workspace_size(c.cfg, most, max_len, acc), dtype=torch.uint8, device="cuda").fill_(255)
    out = torch.full((b, c.H * c.G, c.d), float("nan"), device="cuda")
    lse = torch.full((b, c.H * c.G), float("nan"), device="cuda")
    kv.kvec_paged_decode_shared(c.cfg, q, c.k, c.v, c.pages, c.plen, c.table, c.lens, out, ws, max_prefix=max_prefix, max_len=max_len,
                                window=window, n_sinks=sinks, lse=lse, acc=c.acc if acc else None, stream=stream)
    return out, lse


def _check(c, q, out, lse, acc0, window=0, sinks=0, max_prefix=None, max_len=None, heads=None):
    """out, lse and the accumulated weights of every slot of the pool.  Bounds as for a single
    sequence, with probabilities in three bf16 terms (2^-24); a prefix slot's weight is a sum
    of as many terms as there are columns."""
    kn, vn, qn = ref.f64(c.k), ref.f64(c.v), ref.f64(q)
    got, got_lse = ref.f64(out), ref.f64(lse)
    terms = 2.0 ** -24
    want_acc = None if acc0 is None else ref.f64(acc0)
    slack = None if acc0 is None else np.zeros_like(want_acc)
    P = max(0, min(c.P, max_prefix or len(c.pages) * c.page))
    first = c._rows(c.pages, P)
    columns = len(c.lens_l) * c.G
    for i, n in enumerate(c.lens_l):
        n = min(n, max_len or c.cfg.max_pages * c.page)
        own = c._rows(c.table[i], max(n, 0))
        page, row = (np.concatenate(x) for x in zip(first, own))
        N = P + max(n, 0)
        seen = ref.visible(N, N, N - 1, window, sinks) & (page >= 0) & (n >= 0)
        for h in range(c.H):
            k, v = kn[page, h, row], vn[page, h, row]
            k[~seen], v[~seen] = 0, 0
            for g in range(c.G):
                j = h * c.G + g
                if heads is not None and (i, j) not in heads and acc0 is None:
                    continue
                o, l, w, dx = ref.attend(qn[i, j], k, v, seen)
                tol = (2 * dx + ref.EXP + terms) * max(np.abs(v).max(initial=0), 1e-30)
                assert np.abs(got[i, j] - o).max() <= tol, (i, h, g, np.abs(got[i, j] - o).max(), tol)
                gl = got_lse[i, j]
                assert gl == l or abs(gl - l) <= dx + ref.EXP * (1 + abs(l)), (i, h, g, gl, l)
                if acc0 is not None:
                    want_acc[page[seen], h, row[seen]] += w[seen] / c.G
                    slack[page[seen], h, row[seen]] += w[seen] / c.G * (2 * dx + ref.EXP + (columns + 2) * ref.U24)
    if acc0 is not None:
        a = ref.f64(c.acc)
        assert np.array_equal(np.isnan(a), np.isnan(want_acc))
        ok = ~np.isnan(a)
        assert np.all(np.abs(a - want_acc)[ok] <= slack[ok] + np.abs(want_acc[ok]) * 2 * ref.U24)


CASES = [  # prefix, lens, H, G, d, page, dtype, window, sinks, rows first
    (100, [5, 0, 17], 2, 4, 128, 16, "bf16", 0, 0, False),
    (1, [1], 1, 1, 64, 16, "bf16", 0, 0, False),
    (16, [0, 0], 2, 2, 64, 16, "bf16", 0, 0, True),
    (0, [40, 3, 0], 2, 2, 128, 16, "bf16", 0, 0, False),
    (1000, [33, 1, 64, 5, -1, 100, 7, 8], 2, 4, 128, 64, "bf16", 0, 0, False),       # 32 columns
    (777, [9] * 5 + [-1, 40], 3, 7, 128, 48, "bf16", 0, 0, True),                    # 49
    (515, [i % 37 for i in range(30)], 2, 4, 128, 16, "bf16", 0, 0, False),          # 120
    (300, [i % 21 - 1 for i in range(75)], 1, 7, 128, 128, "bf16", 0, 0, False),     # 525: five tiles of columns
    (2049, [70, 3], 8, 4, 64, 64, "bf16", 0, 0, False),
    (640, [12] * 20, 2, 3, 64, 32, "bf16", 0, 0, True),                              # 60
    (333, [5, 6, 7] * 12, 2, 5, 64, 16, "bf16", 0, 0, False),                        # 180
    (130, [20, 0, -1, 3], 2, 5, 128, 16, "f32", 0, 0, False),
    (600, [41] * 9, 4, 2, 64, 32, "f32", 0, 0, True),
    (70, [2] * 40, 1, 4, 128, 16, "f32", 0, 0, False),                               # 160: three tiles
    # windows that end in the prefix, behind it, and both
    (500, [3, 60, 0, 200], 2, 4, 128, 16, "bf16", 64, 4, False),
    (500, [20, 10, 30, 40] * 4, 2, 4, 128, 64, "bf16", 100, 37, True),
    (257, [1, 300, 70] * 14, 1, 3, 64, 16, "bf16", 90, 0, False),
    (300, [10] * 3, 2, 2, 64, 16, "bf16", 1, 0, False),
    (90, [5, 33], 2, 2, 128, 16, "bf16", 17, 110, False),                            # sinks beyond the prefix
    (333, [18, 2, -1, 150], 2, 2, 128, 16, "f32", 60, 5, False),
    (200, [30] * 20, 1, 4, 64, 64, "f32", 45, 100, True),
]


@pytest.mark.parametrize("prefix,lens,H,G,d,page,dt,window,sinks,rows_first", CASES)
def test_shared(gpu_lib, prefix, lens, H, G, d, page, dt, window, sinks, rows_first):
    import torch
    c = Shared(gpu_lib, prefix, lens, H, G, d, page, dt, seed=len(lens) + G + prefix, rows_first=rows_first).cuda()
    q = c.rand(len(lens), H * G, d).mul_(2).to(_dt(dt)).cuda()
    for i, n in enumerate(lens):
        if n < 0:
            q[i] = float("nan")
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks)
    _check(c, q, out, lse, acc0, window, sinks)
    for i, n in enumerate(lens):
        if n < 0:
            assert torch.all(out[i] == 0) and torch.all(lse[i] == -math.inf)
    # without the weights: the same bits; again: the same bits
    o2, l2 = _decode(c, q, window, sinks, acc=False)
    assert o2.equal(out) and l2.equal(lse)
    a1 = c.acc.clone()
    c.acc.copy_(acc0)
    o3, l3 = _decode(c, q, window, sinks)
    assert o3.equal(out) and l3.equal(lse) and c.acc.nan_to_num(3).equal(a1.nan_to_num(3))


@pytest.mark.parametrize("dt,b,window", [("bf16", 3, 0), ("bf16", 12, 0), ("bf16", 40, 0), ("bf16", 40, 150), ("f32", 7, 0), ("f32", 7, 150)])
def test_lengths_are_clamped_and_pages_checked(gpu_lib, dt, b, window):
    """Lengths beyond their bounds, and table entries that are no pages inside the prefix and
    inside a sequence: their slots are not there."""
    import torch
    c = Shared(gpu_lib, 400, [60] * b, 2, 4, 64, 16, dt, seed=b).cuda()
    c.P = 2**31 - 1
    c.plen.fill_(c.P)
    c.lens_l[1] = 5000
    c.lens.copy_(torch.tensor(c.lens_l))
    c.pages[3], c.pages[20], c.pages[21], c.table[0, 1] = -1, c.cfg.n_pages, 2**31 - 1, -2**31
    q = c.rand(b, 8, 64).to(_dt(dt)).cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, max_prefix=390, max_len=50)
    _check(c, q, out, lse, acc0, window, 0, max_prefix=390, max_len=50)
    # a prefix of negative length is none
    c.P = -7
    c.plen.fill_(-7)
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, max_prefix=390, max_len=50)
    _check(c, q, out, lse, acc0, window, 0, max_prefix=390, max_len=50)


def test_as_single_sequences(gpu_lib):
    """A prefix of whole pages, that every sequence's table begins with: the attention of
    kvec_paged_decode, and the sums of its weights."""
    import torch
    kv = gpu_lib
    c = Shared(kv, 1024, [100, 1, 0, 77, 250, 31], 4, 4, 128, 64, "bf16", seed=5).cuda()
    q = c.rand(6, 16, 128).bfloat16().cuda()
    c.acc.zero_()
    out, lse = _decode(c, q)
    table = torch.cat([c.pages[None, :16].expand(6, -1), c.table], 1).contiguous()
    total = torch.zeros_like(c.acc)
    for i in range(6):
        one = kv.PagedConfig(1, 4, 16, 128, 64, c.cfg.n_pages, table.shape[1], kv.KVEC_BF16)
        acc = torch.zeros_like(c.acc)
        o, l = torch.empty((1, 16, 128), device="cuda"), torch.empty((1, 16), device="cuda")
        ws = torch.empty(kv.kvec_paged_decode_workspace_size(one, None, True), dtype=torch.uint8, device="cuda")
        kv.kvec_paged_decode(one, q[i:i + 1], c.k, c.v, table[i:i + 1], c.lens[i:i + 1] + 1024, o, ws, lse=l, acc=acc)
        total += acc
        # two sums of the same terms in other orders, each within the bounds of its float64 one
        assert torch.all((o[0] - out[i]).abs() <= 2.0 ** -14 * c.v.float().nan_to_num().abs().max())
        assert torch.all((l[0] - lse[i]).abs() <= 2.0 ** -14 * (1 + lse[i].abs()))
    assert torch.all((total - c.acc).abs() <= 2.0 ** -14 * total + 1e-12)


@pytest.mark.parametrize("dt,b", [("bf16", 3), ("bf16", 14), ("bf16", 40), ("f32", 5)])
def test_rows_that_are_no_numbers(gpu_lib, dt, b):
    """NaN and infinities in slots that some sequences see and others do not, in keys and in
    values: they reach the outputs of those that see them and of no other."""
    import torch
    lens = [200, 20, 150] + [120] * (b - 3)
    c = Shared(gpu_lib, 300, lens, 2, 2, 64, 16, dt, seed=9).cuda()
    q = c.rand(b, 4, 64).to(_dt(dt)).cuda()
    window, sinks = 180, 4
    p, r = c._rows(c.pages, 300)
    # from P + n - 180 on: sequence 0 from 320, 1 from 140, 2 from 270, the others from 240
    c.v[p[150], 0, r[150], 5] = float("nan")   # of sequence 1 alone
    c.v[p[250], 1, r[250], 7] = float("inf")   # of 1 and the others, not of 2
    c.v[p[100], :, r[100]] = float("nan")      # of none
    c.k[p[60], :, r[60]] = float("nan")        # of none
    out, lse = _decode(c, q, window, sinks, acc=False)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[1, :2, 5] = True
    want[1, 2:, 7] = True
    want[3:, 2:, 7] = True
    assert torch.equal(~torch.isfinite(out), want)
    assert torch.isfinite(lse).all()
    # the finite ones are those of a pool without them
    clean = Shared(gpu_lib, 300, lens, 2, 2, 64, 16, dt, seed=9).cuda()
    ref_out, ref_lse = _decode(clean, q, window, sinks, acc=False)
    tol = 2.0 ** -14 * clean.v.float().nan_to_num().abs().max()
    assert torch.all(((out - ref_out).abs() <= tol) | want)
    assert lse.equal(ref_lse)
    # a key: the logits of those that see it
    c = Shared(gpu_lib, 300, lens, 2, 2, 64, 16, dt, seed=9).cuda()
    c.k[p[260], 1, r[260]] = float("nan")
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks)
    sees = torch.tensor([300 + n - window <= 260 for n in lens])
    assert torch.equal(lse.isnan().cpu(), sees[:, None] & torch.tensor([False, False, True, True]))
    assert torch.equal(out.isnan().all(-1), lse.isnan()) and torch.equal(out.isnan().any(-1), lse.isnan())
    # weights: NaN for the slots of head 1 that one of these sees
    low = min(300 + n - window for n in lens if 300 + n - window <= 260)
    nan = c.acc[p, 1, r].isnan().cpu()
    assert nan[low:].all() and nan[:sinks].all() and not nan[sinks:low].any()
    assert not c.acc[p, 0, r].isnan().any() and c.acc[p[sinks:low], 1, r[sinks:low]].equal(acc0[p[sinks:low], 1, r[sinks:low]])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 50])
def test_rows_that_are_none_do_not_matter(gpu_lib, dt, window):
    """Padding rows: neither what their queries hold nor keys that are no numbers, which no
    sequence sees, reach the weights; a batch of padding alone leaves everything as it is."""
    import torch
    c = Shared(gpu_lib, 300, [20, -1, 30, -5, -2**31], 2, 4, 64, 16, dt, seed=23).cuda()
    q = c.rand(5, 8, 64).to(_dt(dt)).cuda()
    q[1], q[3], q[4] = float("nan"), float("inf"), 1e30
    p, r = c._rows(c.pages, 300)
    if window:
        c.k[p[100], :, r[100]] = float("nan")  # behind every window
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window)
    _check(c, q.nan_to_num(0, 0, 0), out, lse, acc0, window)
    assert torch.all(out[[1, 3, 4]] == 0) and torch.all(lse[[1, 3, 4]] == -math.inf)
    c.lens.fill_(-1)
    c.k[p[200], :, r[200]] = float("nan")
    before = c.acc.clone()
    out, lse = _decode(c, q, window)
    assert torch.all(out == 0) and torch.all(lse == -math.inf) and c.acc.nan_to_num(7).equal(before.nan_to_num(7))


@pytest.mark.parametrize("H,b,G", [(1, 300, 16), (3, 200, 8), (4, 400, 7), (2, 700, 3)])
def test_many_columns(gpu_lib, H, b, G):
    """More column tiles than compute units have work-groups, on few KV heads: every column and
    tile, against single sequences' attention of the same rows."""
    import torch
    kv = gpu_lib
    lens = [(7 * i) % 23 for i in range(b)]
    c = Shared(kv, 256, lens, H, G, 64, 16, "bf16", seed=b).cuda()
    q = c.rand(b, H * G, 64).bfloat16().cuda()
    out, lse = _decode(c, q, acc=False)
    table = torch.cat([c.pages[None, :16].expand(b, -1), c.table], 1).contiguous()
    one = kv.PagedConfig(b, H, H * G, 64, 16, c.cfg.n_pages, table.shape[1], kv.KVEC_BF16)
    o, l = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty(kv.kvec_paged_decode_workspace_size(one), dtype=torch.uint8, device="cuda")
    kv.kvec_paged_decode(one, q, c.k, c.v, table, c.lens + 256, o, ws, lse=l)
    # sums of the same terms in other orders, each within its bounds
    assert torch.all((o - out).abs() <= 2.0 ** -14 * c.v.float().nan_to_num().abs().max())
    assert torch.all((l - lse).abs() <= 2.0 ** -14 * (1 + lse.abs()))


def test_extreme_logits(gpu_lib):
    """Logits of thousands in the prefix or behind it, and a column that all of them overflow."""
    import torch
    for dt in ("bf16", "f32"):
        c = Shared(gpu_lib, 600, [100, 40, 0], 1, 2, 64, 16, dt, seed=6).cuda()
        p, r = c._rows(c.pages, 600)
        c.k[p[300], 0, r[300]] = 400.0
        c.k[p[:200], 0, r[:200]] = -300.0
        p, r = c._rows(c.table[1], 40)
        c.k[p[30], 0, r[30]] = 900.0
        q = c.rand(3, 2, 64).abs().to(_dt(dt)).cuda()
        acc0 = c.acc.clone()
        out, lse = _decode(c, q)
        _check(c, q, out, lse, acc0)


@pytest.mark.parametrize("dt,columns", [("bf16", 8), ("bf16", 60), ("bf16", 130), ("f32", 20)])
def test_far_offsets(gpu_lib, dt, columns):
    """A prefix in the last pages of a pool of more than 2^32 bytes, and in a small one."""
    import torch
    kv, H, page, d, b = gpu_lib, 2, 1024, 128, columns // 2
    n_pages = 8300 if dt == "bf16" else 4200
    small = Shared(kv, 1500, [30] * b, H, 2, d, page, dt, seed=31, spare_pages=1)
    used = [*small.pages[:2].tolist(), *small.table[:, 0].tolist()]
    where = [n_pages - 1 - 7 * i for i in range(len(used))]
    big = {}
    for name in ("k", "v", "acc"):
        like = getattr(small, name)
        big[name] = torch.empty((n_pages, *like.shape[1:]), dtype=like.dtype, device="cuda")
        for p, u in zip(where, used):
            big[name][p] = like[u].cuda()
    small.cuda()
    q = small.rand(b, 2 * H, d).to(_dt(dt)).cuda()
    out, lse = _decode(small, q)
    cfg = kv.PagedConfig(b, H, 2 * H, d, page, n_pages, 1, small.cfg.dtype)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty(kv.kvec_paged_decode_shared_workspace_size(cfg, 3 * page, None, True), dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv.kvec_paged_decode_shared(cfg, q, big["k"], big["v"], i32(where[:2] + [-1]), small.plen, i32(where[2:])[:, None].contiguous(), small.lens, o2, ws,
                                lse=l2, acc=big["acc"])
    assert o2.equal(out) and l2.equal(lse)
    for p, u in zip(where, used):
        assert big["acc"][p].nan_to_num(3).equal(small.acc[u].nan_to_num(3))


def test_serving_loop_evicts_the_prefix(gpu_lib):
    """As a program serves: tokens appended behind the prefix and attended, then the prefix cut
    by the weights that all sequences gave it, with the calls of a single sequence."""
    import torch
    kv, H, G, d, page = gpu_lib, 2, 4, 128, 16
    c = Shared(kv, 200, [30, 12, 0, 5], H, G, d, page, "bf16", seed=14, spare_pages=20).cuda()
    c.acc.zero_()
    grown = torch.full((4, 4), -1, dtype=torch.int32, device="cuda")
    free = sorted(set(range(c.cfg.n_pages)) - set(c.pages.tolist()) - set(c.table.flatten().tolist()))
    grown[:, :c.table.shape[1]] = c.table
    for i, n in enumerate(c.lens_l):
        for j in range((n + page - 1) // page, 4):
            grown[i, j] = free.pop()
    c.table = grown
    c.cfg = kv.PagedConfig(4, H, H * G, d, page, c.cfg.n_pages, 4)
    pos = torch.zeros((c.cfg.n_pages, H, page), dtype=torch.int32, device="cuda")
    p, r = c._rows(c.pages, 200)
    pos[p, :, r] = torch.arange(200, dtype=torch.int32, device="cuda")[:, None]
    one = kv.PagedConfig(1, H, H * G, d, page, c.cfg.n_pages, len(c.pages))
    ws = torch.empty(kv.kvec_paged_evict_workspace_size(one, None, 120), dtype=torch.uint8, device="cuda")
    for step in range(6):
        q, k, v = (c.rand(4, h, d).bfloat16().cuda() for h in (H * G, H, H))
        at = c.lens.long()
        slots = c.table.long().gather(1, at[:, None] // page)[:, 0] * page + at % page
        kv.kvec_paged_append(c.cfg, q, k, v, (at + 200).int(), slots, q, c.k, c.v, acc=c.acc, pos=pos)
        c.lens += 1
        c.lens_l = [n + 1 for n in c.lens_l]
        acc0 = c.acc.clone()
        out, lse = _decode(c, q)
        _check(c, q, out, lse, acc0)
        if step == 3:
            weights = c.acc[c._rows(c.pages, 200)[0], 0, c._rows(c.pages, 200)[1]]
            kv.kvec_paged_evict(one, 120, c.k, c.v, c.pages[None], c.plen, c.plen, c.acc, pos, c.plen, ws, window=16, n_sinks=4)
            c.P = 120
            assert c.plen.tolist() == [120]
            kept = c.acc[c._rows(c.pages, 120)[0], 0, c._rows(c.pages, 120)[1]]
            assert kept.sum() >= weights.topk(100).values.sum()


def test_streams_and_graph(gpu_lib):
    """A captured call replayed between eager ones, with lengths and prefix that grow on the
    device; a call on another stream than the current one; two streams at once."""
    import torch
    c = Shared(gpu_lib, 900, [50] * 10, 4, 4, 128, 64, "bf16", seed=17).cuda()
    q = c.rand(10, 16, 128).bfloat16().cuda()
    acc0 = c.acc.nan_to_num(0)
    ws = [torch.empty(gpu_lib.kvec_paged_decode_shared_workspace_size(c.cfg, 960, None, True), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.empty((10, 16, 128), device="cuda") for _ in range(2)]
    accs = [acc0.clone() for _ in range(2)]

    def call(i, stream=None):
        gpu_lib.kvec_paged_decode_shared(c.cfg, q, c.k, c.v, c.pages, c.plen, c.table, c.lens, outs[i], ws[i], max_prefix=960, acc=accs[i], stream=stream)

    def eager(P, n):
        c.plen.fill_(P)
        c.lens.fill_(n)
        accs[0].copy_(acc0)
        call(0)
        return outs[0].clone(), accs[0].clone()

    wants = {(P, n): eager(P, n) for P, n in ((900, 50), (700, 3), (0, 9), (333, 0))}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        accs[1].copy_(acc0)
        call(1)
    for P, n in [*wants, *wants]:
        o, a = eager(P, n)
        graph.replay()
        assert o.equal(wants[P, n][0]) and a.equal(wants[P, n][1])
        assert outs[1].equal(o) and accs[1].equal(a)
        torch.cuda.synchronize()
    c.plen.fill_(900)
    c.lens.fill_(50)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                accs[i].copy_(acc0)
            call(i, s)
    torch.cuda.synchronize()
    for i in range(2):
        assert outs[i].equal(wants[900, 50][0]) and accs[i].equal(wants[900, 50][1])


def test_strided_queries_and_many_heads(gpu_lib):
    """Queries inside a larger projection; more KV heads than a launch has work-groups."""
    import torch
    c = Shared(gpu_lib, 130, [7, 30], 300, 1, 64, 16, "bf16", seed=19).cuda()
    wide = c.rand(2, 304, 64).bfloat16().cuda()
    out, lse = _decode(c, wide[:, 2:302], acc=False)
    _check(c, wide[:, 2:302], out, lse, None)


def test_every_misfit_is_named(gpu_lib):
    import torch
    c = Shared(gpu_lib, 60, [20], 2, 2, 64, 16, "bf16").cuda()
    args = dict(q=c.rand(1, 4, 64).bfloat16().cuda(), k_pool=c.k, v_pool=c.v, prefix_pages=c.pages, prefix_len=c.plen, page_table=c.table, lens=c.lens,
                out=torch.empty((1, 4, 64), device="cuda"), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    gpu_lib.kvec_paged_decode_shared(c.cfg, **args)
    for name in args:
        if name not in ("q", "ws"):
            with pytest.raises(AssertionError, match=f"{name} must be on the GPU"):
                gpu_lib.kvec_paged_decode_shared(c.cfg, **{**args, name: args[name].cpu()})
    with pytest.raises(gpu_lib.KvecError):
        gpu_lib.kvec_paged_decode_shared(c.cfg, **{**args, "ws": args["ws"][:16]})
    with pytest.raises(gpu_lib.KvecError):
        gpu_lib.kvec_paged_decode_shared(c.cfg, **args, max_prefix=10000)

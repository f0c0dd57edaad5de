"""The paged cache in eight bits on the GPU: append, read, decode and evict against their
definitions (q8_testlib, serve_testlib), through the binding."""
import math

import numpy as np
import pytest

import q8_testlib as q8
import serve_testlib as ref
from q8_testlib import Cache8

pytestmark = pytest.mark.gpu


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _bits(c):
    """Copies of everything that the cache holds."""
    import torch
    return [t.clone() for t in (c.k.view(torch.int8), c.v.view(torch.int8), c.ks.view(torch.int32), c.vs.view(torch.int32), c.acc.view(torch.int32), c.pos)]


APPEND = [  # tokens, H, G, d, page, dtype, format, rot, norm, start
    (1, 8, 4, 128, 64, "bf16", "int8", 128, True, 130000),
    (5, 4, 7, 128, 16, "bf16", "e4m3", 64, False, 7),
    (37, 2, 2, 64, 48, "bf16", "int8", 64, True, 0),
    (37, 1, 16, 64, 16, "f32", "e4m3", 16, True, 1000000),
    (300, 2, 1, 128, 256, "f32", "int8", 128, False, 5),
    # several tokens a work-group, the last one with fewer
    (1537, 2, 1, 128, 256, "f32", "e4m3", 128, False, 5),
    (1551, 1, 3, 64, 16, "bf16", "int8", 48, True, 100),
    (3, 2, 2, 128, 16, "f32", "int8", 112, True, -5),
    (4, 2, 2, 64, 16, "bf16", "e4m3", 0, True, 0),
    (40, 3, 2, 64, 16, "f32", "int8", 0, False, 0),
    (40, 3, 2, 128, 16, "bf16", "e4m3", 0, False, 0),
]


@pytest.mark.parametrize("n,H,G,d,page,dt,fmt,rot,norm,start", APPEND)
def test_append(gpu_lib, n, H, G, d, page, dt, fmt, rot, norm, start):
    """Every row of the pools, those that no token takes included: values have the codes and
    scales of the definition, bit for bit, and so have keys that are neither normed nor
    rotated; others are within half a step of the row in 64 bits."""
    import torch
    c = Cache8(gpu_lib, [n + 20], H, G, d, page, dt, fmt, seed=n).cuda()
    qkv = c.rand(n, H * G + 2 * H, d).mul_(3).to(_dt(dt)).cuda()
    q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
    wq, wk = ((1 + 0.2 * c.rand(d)).to(_dt(dt)).cuda() if norm else None for _ in range(2))
    inv_freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None
    positions = (torch.arange(n) * 3 + start).int().cuda()
    page_i, row_i = c.slots(0, n + 20)
    order = torch.randperm(n + 20, generator=c.gen)[:n].numpy()
    slots = torch.from_numpy(page_i[order].astype(np.int64) * page + row_i[order])
    total = c.cfg.n_pages * page
    if n > 1:
        slots[::5] = torch.tensor([-1, total, -2**62, 2**62]).repeat(n)[: len(slots[::5])]
    q_out = torch.full((n, H * G, d), float("nan"), dtype=_dt(dt), device="cuda")
    want = [ref.f64(t) for t in (c.ks, c.vs, c.acc, c.pos)]
    num = [q8.numbers(c.k), q8.numbers(c.v)]
    gpu_lib.kvec_paged_append_q8(c.cfg, q, k, v, positions, slots.cuda(), q_out, *c.pools, q_weight=wq, k_weight=wk, eps=1e-5, inv_freq=inv_freq,
                                 acc=c.acc, pos=c.pos)
    # the queries are those of the plain append
    plain = gpu_lib.PagedConfig(1, H, H * G, d, page, c.cfg.n_pages, c.cfg.max_pages, c.cfg.dtype)
    pools = [torch.empty(plain.pool_shape, dtype=_dt(dt), device="cuda") for _ in range(2)]
    q_plain = torch.empty_like(q_out)
    gpu_lib.kvec_paged_append(plain, q, k, v, positions, slots.cuda(), q_plain, *pools, q_weight=wq, k_weight=wk, eps=1e-5, inv_freq=inv_freq)
    assert q_out.equal(q_plain)
    fr = None if inv_freq is None else ref.f64(inv_freq)
    got_k, got_ks = q8.numbers(c.k), ref.f64(c.ks)
    for t in range(n):
        s = int(slots[t])
        if not 0 <= s < total:
            continue
        p, r = s // page, s % page
        num[1][p, :, r], want[1][p, :, r] = q8.quantised(v[t].float().cpu().numpy(), fmt)
        want[2][p, :, r], want[3][p, :, r] = 0, int(positions[t])
        exact, z = q8.quantised(k[t].float().cpu().numpy(), fmt)
        for h in range(H):
            if norm or rot:
                y, off = ref.rotated(ref.f64(k[t, h]), None if wk is None else ref.f64(wk), 1e-5, int(positions[t]), fr)
                gz = got_ks[p, h, r]
                assert abs(gz - np.abs(y).max() / q8.TOP[fmt]) <= off.max() / q8.TOP[fmt] + gz * 2.0 ** -22
                # the float32 row is off by `off`, its quotient and the bound by a rounding each
                tol = off * (1 + 2.0 ** -3) + q8.half_step(y, gz, fmt) * (1 + 2.0 ** -20) + 2.0 ** -22 * np.abs(y)
                assert np.all(np.abs(got_k[p, h, r] * gz - y) <= tol), (t, h)
                num[0][p, h, r], want[0][p, h, r] = got_k[p, h, r], gz
            else:
                num[0][p, h, r], want[0][p, h, r] = exact[h], z[h]
    for got, w in zip((c.ks, c.vs, c.acc, c.pos), want):
        assert np.array_equal(ref.f64(got), w, equal_nan=True)
    for got, w in zip((c.k, c.v), num):
        assert np.array_equal(q8.numbers(got), w, equal_nan=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_special_rows(gpu_lib, dt, fmt, d):
    """Rows of zeros of both signs, of the smallest and largest numbers, with ties, NaN and
    infinities: codes and scales of the definition; and they read back as its values."""
    import torch
    rows = torch.zeros((12, d))
    rows[1] = -0.0
    rows[2, 3] = 1e-45
    rows[3] = torch.linspace(-1e-38, 1e-38, d)
    rows[4] = torch.linspace(-3e38, 3e38, d)
    rows[5, :5] = torch.tensor([1.0, 0.5, -0.5, 0.25, 63.5 / 127])
    rows[6] = torch.arange(d) + 0.5
    rows[7, d - 1] = float("nan")
    rows[8, 0] = float("inf")
    rows[9, 9] = -float("inf")
    rows[10] = 448.0
    rows[10, : d // 2] = torch.arange(d // 2) * 2.0 ** -9
    rows[11] = -127.0
    rows[11, ::2] = torch.arange(d // 2) / 2
    rows = rows.to(_dt(dt))
    c = Cache8(gpu_lib, [12], 1, 1, d, 16, dt, fmt, seed=3).cuda()
    k = rows[:, None].cuda()
    v = rows.flip(0)[:, None].contiguous().cuda()
    page, row = c.slots(0, 12)
    slots = torch.from_numpy(page.astype(np.int64) * 16 + row).cuda()
    q_out = torch.empty_like(k)
    gpu_lib.kvec_paged_append_q8(c.cfg, k, k, v, torch.zeros(12, dtype=torch.int32, device="cuda"), slots, q_out, *c.pools)
    out = [torch.empty((1, 1, 12, d), dtype=_dt(dt), device="cuda") for _ in range(2)]
    gpu_lib.kvec_paged_read_q8(c.cfg, *c.pools, c.table, c.lens, *out)
    for pool, scale, x, back in ((c.k, c.ks, k, out[0]), (c.v, c.vs, v, out[1])):
        n, z = q8.quantised(x[:, 0].float().cpu().numpy(), fmt)
        assert np.array_equal(q8.numbers(pool)[page, 0, row], n)
        assert np.array_equal(scale.cpu().numpy()[page, 0, row], z, equal_nan=True)
        want = (torch.from_numpy(n).float() * torch.from_numpy(z)[:, None]).to(_dt(dt))
        assert torch.equal(back[0, 0].cpu().nan_to_num(7), want.nan_to_num(7)) and torch.equal(back[0, 0].cpu().isnan(), want.isnan())


def test_append_of_nothing(gpu_lib):
    import torch
    c = Cache8(gpu_lib, [20], 2, 2, 64, 16, "bf16", "int8").cuda()
    before = _bits(c)
    e = lambda h: torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    gpu_lib.kvec_paged_append_q8(c.cfg, e(4), e(2), e(2), torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"),
                                 e(4), *c.pools, acc=c.acc, pos=c.pos)
    assert all(a.equal(b) for a, b in zip(before, _bits(c)))


READ = [  # lens, H, d, page, dtype, format, rows first, rows of the outputs
    ([0, 1, 15, 16, 17, 100], 2, 128, 16, "bf16", "int8", False, 100),
    ([700, 3, 333], 4, 64, 48, "f32", "e4m3", True, 720),
    ([64, 65], 1, 64, 64, "bf16", "e4m3", False, 65),
    ([1000], 3, 128, 128, "f32", "int8", True, 1024),
    ([5] * 300, 1, 64, 16, "bf16", "int8", False, 16),
]


@pytest.mark.parametrize("lens,H,d,page,dt,fmt,rows_first,n", READ)
def test_read(gpu_lib, lens, H, d, page, dt, fmt, rows_first, n):
    """The product of code and scale, rounded once; rows behind a sequence's last and between
    the strided outputs' rows as they were; zeros for a slot without a page."""
    import torch
    c = Cache8(gpu_lib, lens, H, 1, d, page, dt, fmt, seed=len(lens), rows_first=rows_first, max_pages=(n + page - 1) // page).cuda()
    if len(lens) < 10 and c.table.shape[1] > 1:
        c.table[-1, 1] = -1
    b = len(lens)
    wide = [torch.full((b, n, H + 1, d), 7.0, dtype=_dt(dt), device="cuda") for _ in range(2)]
    out = [w[:, :, :H].transpose(1, 2) for w in wide]
    gpu_lib.kvec_paged_read_q8(c.cfg, *c.pools, c.table, c.lens, *out)
    for o, codes, scale in zip(out, (c.k, c.v), (c.ks, c.vs)):
        x = (codes.float() * scale[..., None]).to(_dt(dt))
        for i, m in enumerate(lens):
            p, r = c.slots(i, m)
            want = torch.where(torch.from_numpy(p >= 0).cuda()[:, None, None], x[p, :, r], torch.zeros((), dtype=_dt(dt), device="cuda"))
            assert o[i, :, :m].transpose(0, 1).equal(want)
            assert torch.all(o[i, :, m:] == 7)
    assert all(torch.all(w[:, :, H] == 7) for w in wide)


def test_read_lengths_are_clamped(gpu_lib):
    import torch
    c = Cache8(gpu_lib, [90, 90, 90], 2, 1, 64, 16, "bf16", "int8", seed=5).cuda()
    c.lens.copy_(torch.tensor([-4, 2**31 - 1, 50]))
    out = [torch.full((3, 2, 60, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    gpu_lib.kvec_paged_read_q8(c.cfg, *c.pools, c.table, c.lens, *out)
    for o, x in zip(out, c.values()):
        assert torch.all(o[0] == 7) and torch.all(o[2, :, 50:] == 7)
        p, r = c.slots(1, 60)
        assert o[1].transpose(0, 1).equal(torch.from_numpy(x[p, :, r]).bfloat16().cuda())


def _decode(c, q, window=0, sinks=0, acc=True, max_len=None, stream=None):
    import torch
    kv, b = c.kv, len(c.lens_l)
    ws = torch.empty(kv.kvec_paged_decode_q8_workspace_size(c.cfg, max_len, acc), dtype=torch.uint8, device="cuda").fill_(255)
    out = torch.full((b, c.H * c.G, c.d), float("nan"), device="cuda")
    lse = torch.full((b, c.H * c.G), float("nan"), device="cuda")
    kv.kvec_paged_decode_q8(c.cfg, q, *c.pools, c.table, c.lens, out, ws, max_len=max_len, window=window, n_sinks=sinks, lse=lse,
                            acc=c.acc if acc else None, stream=stream)
    return out, lse


def _check_decode(c, q, out, lse, acc0, window=0, sinks=0, max_len=None):
    """out, lse and the accumulated weights of every slot of the pool.  A logit has two more
    roundings than a plain dot product (the scales' products), so d + 4 of them; queries in
    float32 and probabilities enter the products as three bf16 terms, 2^-24 relative each."""
    (kn, vn), qn = c.values(), ref.f64(q)
    got, got_lse = ref.f64(out), ref.f64(lse)
    terms = 2.0 ** -23
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
                dx *= (c.d + 4) / (c.d + 2)
                tol = (2 * dx + ref.EXP + terms) * max(np.abs(v).max(initial=0), 1e-30)
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


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,H,G,d,page,dt,window,sinks,rows_first", DECODE)
def test_decode(gpu_lib, lens, H, G, d, page, dt, window, sinks, rows_first, fmt):
    c = Cache8(gpu_lib, lens, H, G, d, page, dt, fmt, seed=len(lens) + G, rows_first=rows_first).cuda()
    q = c.rand(len(lens), H * G, d).mul_(2).to(_dt(dt)).cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks)
    _check_decode(c, q, out, lse, acc0, window, sinks)
    # without the weights: the same bits
    o2, l2 = _decode(c, q, window, sinks, acc=False)
    assert o2.equal(out) and l2.equal(lse)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_decode_lengths_are_clamped_and_pages_checked(gpu_lib, fmt):
    """Lengths beyond max_len or below 0, and table entries that are no pages inside a
    sequence: their slots are not there."""
    import torch
    c = Cache8(gpu_lib, [200, 200, 90], 2, 4, 64, 16, "bf16", fmt, seed=3).cuda()
    c.lens_l = [200, 5000, -3]
    c.lens.copy_(torch.tensor(c.lens_l))
    c.table[0, 2], c.table[0, 7], c.table[1, 0] = -1, c.cfg.n_pages, 2**31 - 1
    q = c.rand(3, 8, 64).bfloat16().cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, max_len=150)
    _check_decode(c, q, out, lse, acc0, max_len=150)
    assert torch.all(out[2] == 0) and torch.all(lse[2] == -math.inf)


@pytest.mark.parametrize("dt,fmt", [("bf16", "int8"), ("f32", "e4m3")])
def test_decode_rows_that_are_no_numbers(gpu_lib, dt, fmt):
    """A visible key that reads as NaN makes out, lse and the weights of its KV head NaN, a
    visible value its outputs; other heads and sequences, and masked rows, do not matter."""
    import torch
    c = Cache8(gpu_lib, [300, 200, 150], 2, 2, 128, 16, dt, fmt, seed=8).cuda()
    q = c.rand(3, 4, 128).to(_dt(dt)).cuda()
    p, r = c.slots(0, 300)
    c.ks[p[250], 0, r[250]] = float("nan")
    p, r = c.slots(1, 200)
    c.vs[p[190], 1, r[190]] = float("nan")
    p, r = c.slots(2, 150)
    c.vs[p[20], :, r[20]] = float("nan")  # before the window
    c.ks[p[30], :, r[30]] = float("nan")
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window=100, sinks=4)
    assert out[0, :2].isnan().all() and lse[0, :2].isnan().all() and not out[0, 2:].isnan().any() and not lse[0, 2:].isnan().any()
    assert out[1, 2:].isnan().all() and not out[1, :2].isnan().any() and not lse[1].isnan().any()
    assert not out[2].isnan().any() and not lse[2].isnan().any()
    seen = ref.visible(300, 300, 299, 100, 4)
    p, r = c.slots(0, 300)
    assert c.acc[p[seen], 0, r[seen]].isnan().all() and c.acc[p[~seen], 0, r[~seen]].equal(acc0[p[~seen], 0, r[~seen]])
    assert not c.acc[p, 1, r].isnan().any()


def test_decode_extreme_logits(gpu_lib):
    """Logits of thousands, of both signs, and equal ones; scales of very different rows."""
    import torch
    c = Cache8(gpu_lib, [600, 100], 1, 2, 64, 16, "f32", "int8", seed=5).cuda()
    page, row = c.slots(0, 600)
    c.ks[page[300], 0, row[300]] = 4.0
    c.ks[page[:200], 0, row[:200]] = 3.0
    c.vs[page[100:250], 0, row[100:250]] *= 1e-6
    page, row = c.slots(1, 100)
    c.k[page, :, row] = c.k[page[0], 0, row[0]].clone()
    c.ks[page, :, row] = 0.01
    q = c.rand(2, 2, 64).abs().cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q)
    _check_decode(c, q, out, lse, acc0)


def test_far_offsets(gpu_lib):
    """Rows behind 2^32 bytes of the pool: append, decode, read and evict as in a small one."""
    import torch
    kv, H, page, d, n_pages = gpu_lib, 4, 1024, 128, 8300  # 4.4 GB a pool
    small = Cache8(kv, [2000], H, 2, d, page, "bf16", "int8", seed=41, full=True)
    where = [n_pages - 1, n_pages - 7]
    big = {}
    for name in ("k", "v", "ks", "vs", "acc", "pos"):
        like = getattr(small, name)
        big[name] = torch.empty((n_pages, *like.shape[1:]), dtype=like.dtype, device="cuda")
        for j, p in enumerate(where):
            big[name][p] = like[small.table[0, j]].cuda()
    small.cuda()
    cfg = kv.PagedQ8Config(1, H, 2 * H, d, page, n_pages, 2)
    table = torch.tensor([where], dtype=torch.int32, device="cuda")
    q, k, v = (small.rand(9, h, d).bfloat16().cuda() for h in (2 * H, H, H))
    fr = torch.rand(d // 2, dtype=torch.float64, device="cuda")
    at = torch.arange(1500, 1509)
    pos = at.int().cuda()
    outs = []
    for c, tb, t in ((cfg, table, big), (small.cfg, small.table, {n: getattr(small, n) for n in big})):
        pools = [t[n] for n in ("k", "v", "ks", "vs")]
        slots = (tb[0].long()[(at // page).cuda()] * page + (at % page).cuda())
        q_out = torch.empty_like(q)
        kv.kvec_paged_append_q8(c, q, k, v, pos, slots, q_out, *pools, inv_freq=fr, acc=t["acc"], pos=t["pos"])
        out, lse = torch.empty((1, 2 * H, d), device="cuda"), torch.empty((1, 2 * H), device="cuda")
        ws = torch.empty(kv.kvec_paged_decode_q8_workspace_size(c, None, True), dtype=torch.uint8, device="cuda")
        kv.kvec_paged_decode_q8(c, q[:1], *pools, tb, small.lens, out, ws, lse=lse, acc=t["acc"])
        ws = torch.empty(kv.kvec_paged_evict_q8_workspace_size(c, None, 900), dtype=torch.uint8, device="cuda")
        kept, left = torch.empty((1, H, 900), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        kv.kvec_paged_evict_q8(c, 900, *pools, tb, small.lens, small.lens, t["acc"], t["pos"], left, ws, window=50, n_sinks=4, kept=kept)
        rows = [torch.zeros((1, H, 900, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        kv.kvec_paged_read_q8(c, *pools, tb, left, *rows)
        outs.append((q_out, out, lse, kept, left, *rows, *(t[n][tb[0].long()].nan_to_num(9) for n in ("ks", "vs", "acc")), t["pos"][tb[0].long()],
                     *(t[n][tb[0].long()] for n in ("k", "v"))))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


EVICT = [  # lens, H, d, page, dtype, format, budget, window, sinks, rows first
    ([100, 64, 65, 10, 0], 2, 128, 16, "bf16", "int8", 64, 16, 4, False),
    ([300, 257, 256, 5], 3, 64, 48, "f32", "e4m3", 256, 0, 0, True),
    ([1088], 8, 128, 64, "bf16", "e4m3", 1024, 32, 4, False),
    ([5000, 4100, 3000], 2, 64, 128, "bf16", "int8", 1000, 200, 16, True),
    ([9000], 2, 128, 256, "f32", "int8", 4000, 1, 0, False),
]


@pytest.mark.parametrize("lens,H,d,page,dt,fmt,budget,window,sinks,rows_first", EVICT)
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(gpu_lib, lens, H, d, page, dt, fmt, budget, window, sinks, rows_first, in_place):
    """Codes, scales, weights and positions of every slot; what is not moved stays."""
    import torch
    c = Cache8(gpu_lib, lens, H, 1, d, page, dt, fmt, seed=budget, rows_first=rows_first).cuda()
    before = [t.cpu().numpy() for t in _bits(c)]
    seen = torch.tensor([n + 3 for n in lens], dtype=torch.int32, device="cuda")
    acc, pos = c.acc.cpu().numpy(), c.pos.cpu().numpy()
    ws = torch.empty(gpu_lib.kvec_paged_evict_q8_workspace_size(c.cfg, None, budget), dtype=torch.uint8, device="cuda").fill_(255)
    kept = torch.full((len(lens), H, budget), -9, dtype=torch.int32, device="cuda")
    out = c.lens if in_place else torch.empty_like(c.lens)
    gpu_lib.kvec_paged_evict_q8(c.cfg, budget, *c.pools, c.table, c.lens, seen, c.acc, c.pos, out, ws, window=window, n_sinks=sinks, kept=kept)
    want = [b.copy() for b in before]
    for i, n in enumerate(lens):
        page_i, row_i = c.slots(i, n)
        for h in range(H):
            source, left = ref.evict(acc[page_i, h, row_i], pos[page_i, h, row_i], page_i >= 0, n, budget, window, sinks, n + 3)
            assert np.array_equal(kept[i, h].cpu().numpy(), source)
            at = np.arange(min(n, budget))
            for w, b in zip(want, before):
                w[page_i[at], h, row_i[at]] = b[page_i[source[at]], h, row_i[source[at]]]
            assert int(out[i]) == left
    for got, w in zip(_bits(c), want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_chunked_prompt_and_serving_loop(gpu_lib):
    """As a program serves: a prompt in two chunks, the second one's attention over rows read
    back; then tokens appended, attended and evicted.  The attention of each token is that of
    the definition over what the cache stands for."""
    import torch
    kv, H, G, d, page, dt = gpu_lib, 2, 4, 128, 16, "bf16"
    c = Cache8(kv, [0, 0], H, G, d, page, dt, "e4m3", seed=77, spare_pages=40, max_pages=16).cuda()
    c.table.copy_(torch.randperm(c.cfg.n_pages, generator=c.gen)[:32].view(2, 16).int())
    c.acc.zero_()
    fr = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    seen = torch.zeros(2, dtype=torch.int32, device="cuda")

    def append(n):
        q, k, v = (c.rand(2 * n, h, d).bfloat16().cuda() for h in (H * G, H, H))
        at = (c.lens[:, None] + torch.arange(n, device="cuda")).long()
        slots = (c.table.long().gather(1, at // page) * page + at % page).flatten()
        positions = (seen[:, None] + torch.arange(n, device="cuda")).int().flatten()
        q_out = torch.empty_like(q)
        kv.kvec_paged_append_q8(c.cfg, q, k, v, positions, slots, q_out, *c.pools, inv_freq=fr, acc=c.acc, pos=c.pos)
        c.lens += n
        seen.add_(n)
        c.lens_l = [x + n for x in c.lens_l]
        return q_out.view(2, n, H * G, d).transpose(1, 2)

    for n, total in ((70, 70), (50, 120)):
        q = append(n)
        k, v = (torch.empty((2, H, total, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        kv.kvec_paged_read_q8(c.cfg, *c.pools, c.table, c.lens, k, v)
        attn = kv.AttentionConfig(2, H, H * G, d, n, total)
        out, lse = torch.empty((2, H * G, n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, H * G, n), device="cuda")
        ws = torch.empty(max(16, kv.kvec_prefill_workspace_size(attn)), dtype=torch.uint8, device="cuda")
        kv.kvec_prefill_attention(attn, q.contiguous(), k, v, out, ws, lse=lse)
        kn, vn, qn, on = ref.f64(k), ref.f64(v), ref.f64(q), ref.f64(out)
        for i, j, r in ((0, 0, 0), (1, 5, n - 1), (0, 7, n // 2)):
            p = total - n + r
            o, l, _, dx = ref.attend(qn[i, j, r], kn[i, j // G], vn[i, j // G], np.arange(total) <= p)
            # probabilities and the output are rounded to bf16
            tol = (2 * dx + ref.EXP + ref.U_BF16) * np.abs(vn[i, j // G, :p + 1]).max() + ref.U_BF16 * np.abs(o)
            assert np.all(np.abs(on[i, j, r] - o) <= tol)
    budget = 100
    ws_e = torch.empty(kv.kvec_paged_evict_q8_workspace_size(c.cfg, None, budget), dtype=torch.uint8, device="cuda")
    for step in range(12):
        q = append(1)[:, :, 0].contiguous()
        acc0 = c.acc.clone()
        out, lse = _decode(c, q)
        _check_decode(c, q, out, lse, acc0)
        if step % 4 == 3:
            kv.kvec_paged_evict_q8(c.cfg, budget, *c.pools, c.table, c.lens, seen, c.acc, c.pos, c.lens, ws_e, window=16, n_sinks=4)
            c.lens_l = [min(n, budget) for n in c.lens_l]
            assert c.lens.tolist() == c.lens_l
            for i in range(2):  # the protected ones are there
                p, r = c.slots(i, budget)
                held = set(c.pos[p, 0, r].tolist())
                assert set(range(4)) <= held and set(range(int(seen[i]) - 16, int(seen[i]))) <= held


def test_streams_and_graph(gpu_lib):
    """A captured token (append, decode, evict, read) replayed between eager calls gives the
    eager results every time; a call on another stream than the current one."""
    import torch
    kv, H, G, d, page = gpu_lib, 2, 4, 128, 16
    base = Cache8(kv, [300, 250], H, G, d, page, "bf16", "int8", seed=12, full=True).cuda()
    q, k, v = (base.rand(2, h, d).bfloat16().cuda() for h in (H * G, H, H))
    names = ("k", "v", "ks", "vs", "acc", "pos", "lens")
    start = {n: getattr(base, n).clone() for n in names}
    budget = 200
    bufs = dict(q_out=torch.empty_like(q), out=torch.empty((2, H * G, d), device="cuda"), left=torch.empty_like(base.lens),
                rows=[torch.zeros((2, H, budget, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                ws=torch.empty(max(kv.kvec_paged_decode_q8_workspace_size(base.cfg, None, True), kv.kvec_paged_evict_q8_workspace_size(base.cfg, None, budget)),
                               dtype=torch.uint8, device="cuda"))
    at = torch.tensor([299, 249], device="cuda")
    slots = base.table.long().gather(1, at[:, None] // page)[:, 0] * page + at % page
    positions = at.int()

    def token(stream=None):
        for n in names:
            getattr(base, n).copy_(start[n]) if n not in ("k", "v") else getattr(base, n).view(torch.int8).copy_(start[n].view(torch.int8))
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        kv.kvec_paged_append_q8(base.cfg, q, k, v, positions, slots, bufs["q_out"], *base.pools, acc=base.acc, pos=base.pos, stream=stream)
        kv.kvec_paged_decode_q8(base.cfg, bufs["q_out"], *base.pools, base.table, base.lens, bufs["out"], bufs["ws"], acc=base.acc, stream=stream)
        kv.kvec_paged_evict_q8(base.cfg, budget, *base.pools, base.table, base.lens, base.lens, base.acc, base.pos, bufs["left"], bufs["ws"], stream=stream)
        kv.kvec_paged_read_q8(base.cfg, *base.pools, base.table, bufs["left"], *bufs["rows"], stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)

    def state():
        return [t.clone() for t in (bufs["q_out"], bufs["out"], bufs["left"], *bufs["rows"], *_bits(base))]

    token()
    want = state()
    side = torch.cuda.Stream()
    token(side)
    assert all(a.equal(b) for a, b in zip(state(), want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    for i in range(4):
        for t in bufs["rows"]:
            t.zero_()
        bufs["out"].fill_(float("nan"))
        graph.replay()
        assert all(a.equal(b) for a, b in zip(state(), want))
        if i % 2:
            token()
            torch.cuda.synchronize()
            assert all(a.equal(b) for a, b in zip(state(), want))


def test_same_bits_twice(gpu_lib):
    import torch
    c = Cache8(gpu_lib, [1500, 900, 1], 4, 4, 128, 64, "bf16", "e4m3", seed=21).cuda()
    q = c.rand(3, 16, 128).bfloat16().cuda()
    acc0 = c.acc.clone()
    a = _decode(c, q) + (c.acc.nan_to_num(5),)
    c.acc.copy_(acc0)
    b = _decode(c, q) + (c.acc.nan_to_num(5),)
    assert all(x.equal(y) for x, y in zip(a, b))


def test_every_misfit_is_named(gpu_lib):
    """Pools and scales on the CPU, K and V pools with strides of their own."""
    import torch
    c = Cache8(gpu_lib, [40], 2, 2, 64, 16, "bf16", "int8").cuda()
    args = dict(q=c.rand(1, 4, 64).bfloat16().cuda(), k_pool=c.k, v_pool=c.v, k_scale=c.ks, v_scale=c.vs, page_table=c.table, lens=c.lens,
                out=torch.empty((1, 4, 64), device="cuda"), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    gpu_lib.kvec_paged_decode_q8(c.cfg, **args)
    for name in args:
        if name not in ("q", "ws"):
            with pytest.raises(AssertionError, match=f"{name} must be on the GPU"):
                gpu_lib.kvec_paged_decode_q8(c.cfg, **{**args, name: args[name].cpu()})
    with pytest.raises(AssertionError, match="same strides"):
        gpu_lib.kvec_paged_decode_q8(c.cfg, **{**args, "v_pool": c.v.transpose(1, 2).contiguous().transpose(1, 2)})
    with pytest.raises(gpu_lib.KvecError):
        gpu_lib.kvec_paged_decode_q8(c.cfg, **{**args, "ws": args["ws"][:16]})

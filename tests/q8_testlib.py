"""Definitions of the paged cache in eight bits, in the arithmetic that its header states,
and caches of random rows for the GPU tests."""
import numpy as np

import serve_testlib as ref

TOP = {"int8": 127.0, "e4m3": 448.0}
TINIEST = np.float32(2.0 ** -126)


def e4m3(x):
    """Nearest number of 1 + 4 + 3 bits (bias 7, no infinity), ties to even, |x| below 464."""
    a = np.abs(x.astype(np.float64))
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.copysign(np.rint(a / step) * step, x)  # (rint: to even)


def quantised(y, fmt):
    """Rows y (float32 [..., d]): the numbers that the codes are (float64), the scales
    (float32)."""
    y = np.asarray(y, dtype=np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(y).max(-1)
        z = np.maximum(top / np.float32(TOP[fmt]), TINIEST).astype(np.float32)
        q = (y / z[..., None]).astype(np.float32)
    bad = ~np.isfinite(y).all(-1)
    z[bad] = np.nan
    q[bad] = 0
    return (np.rint(q.astype(np.float64)) if fmt == "int8" else e4m3(q)), z


def half_step(v, z, fmt):
    """How far a code times z may be from the row's value v."""
    return 0.5 * z if fmt == "int8" else np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * z)


def codes(x, fmt):
    """Numbers as a tensor of codes."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).float()
    return t.to(torch.int8) if fmt == "int8" else t.to(torch.float8_e4m3fn)


def numbers(t):
    return t.detach().cpu().float().double().numpy()


def flags(n, n_pages):
    """Table entries that are no pages."""
    import torch
    return torch.tensor([-1, n_pages, 2**31 - 1, -2**31]).repeat(n)[:n].int()


class Cache8:
    """A pool in eight bits whose unused slots read as NaN, with its page table: pages in no
    order, no pages behind a sequence's last."""

    def __init__(self, kv, lens, H, G, d, page, dt, fmt, seed=0, rows_first=False, spare_pages=2, max_pages=None, full=False):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.kv, self.lens_l, self.H, self.G, self.d, self.page, self.dt, self.fmt = kv, lens, H, G, d, page, dt, fmt
        used = [(n + page - 1) // page for n in lens]
        mp = max_pages or max(max(used), 1)
        n_pages = sum(used) + spare_pages
        ids = torch.randperm(n_pages, generator=g)[: sum(used)]
        self.table = flags(len(lens) * mp, n_pages).view(len(lens), mp).clone()
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = ids[at:at + u].int()
            at += u
        self.cfg = kv.PagedQ8Config(len(lens), H, H * G, d, page, n_pages, mp, kv.KVEC_BF16 if dt == "bf16" else kv.KVEC_F32,
                                    kv.KVEC_Q8_INT8 if fmt == "int8" else kv.KVEC_Q8_E4M3)
        shape = (n_pages, page, H, d) if rows_first else (n_pages, H, page, d)
        self.k, self.v = (torch.full(shape, 127, dtype=torch.int8).view(self.cfg.code) for _ in range(2))  # (e4m3: NaN)
        if rows_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.ks, self.vs = (torch.full((n_pages, H, page), float("nan")) for _ in range(2))
        self.acc = torch.full((n_pages, H, page), float("nan"))
        self.pos = torch.full((n_pages, H, page), -7, dtype=torch.int32)
        for i, n in enumerate(lens):
            p, r = ref.rows_of(self.table[i].numpy(), used[i] * page if full else n, page, n_pages)
            p, r = torch.from_numpy(p), torch.from_numpy(r)
            m = len(p)
            for pool, scale, spread in ((self.k, self.ks, 1.5), (self.v, self.vs, 1.0)):
                c, z = quantised((torch.randn((m, H, d), generator=g) * spread).numpy(), fmt)
                pool.view(torch.int8)[p, :, r] = codes(c, fmt).view(torch.int8)
                scale[p, :, r] = torch.from_numpy(z)
            self.acc[p, :, r] = torch.rand((m, H), generator=g) ** 3 * 4
            self.pos[p, :, r] = torch.arange(m, dtype=torch.int32)[:, None]
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.rand = lambda *s: torch.randn(s, generator=g)
        self.gen = g

    def cuda(self):
        for n in ("table", "k", "v", "ks", "vs", "acc", "pos", "lens"):
            t = getattr(self, n)
            if n in ("k", "v") and not t.is_contiguous():
                setattr(self, n, t.transpose(1, 2).cuda().transpose(1, 2))
            else:
                setattr(self, n, t.cuda())
        return self

    @property
    def pools(self):
        return self.k, self.v, self.ks, self.vs

    def values(self):
        """What the rows stand for, float64: K, V."""
        return [numbers(c) * ref.f64(z)[..., None] for c, z in ((self.k, self.ks), (self.v, self.vs))]

    def slots(self, i, n):
        return ref.rows_of(self.table[i].cpu().numpy(), n, self.page, self.cfg.n_pages)

"""Performance cases of the serving operators around the eviction: writing new tokens
into a paged KV cache (`append`), one token's attention over it (`decode`), its
eviction by accumulated attention weight (`evict`) and the prompt's attention with a
sliding window and sinks (`prefill`), each in its plain form and as the library's call.

A case is a dict of plain values:
  op       "append", "decode", "evict" or "prefill"
  batch, kv, q, d, dtype   sequences, KV and query heads, head dimension, type
  page     (paged cache) tokens per page
  T        append: new tokens in all; decode, evict: slots of the longest sequence
           (sequence i holds T - i * T // (2 * batch)); prefill: keys
  rot      (append) leading dimensions that the position rotates
  norm     (append) whether queries and keys are normed
  start    (append) position of the first new token
  acc      (decode) whether the weights of every slot are accumulated
  window, sinks   visible or protected tokens; window 0: everything is visible
  budget   (evict) slots kept per KV head
  rows     (prefill) query rows, the last of the T positions
  ragged   (prefill) whether sequence i is T - i * T // (2 * batch) keys long, padded to T
"""
from __future__ import annotations

import math

import torch

own = False

LLAMA = dict(kv=8, q=32, d=128, dtype="bf16")  # Llama-3.1-8B heads
QWEN = dict(kv=4, q=28, d=128, dtype="bf16")   # Qwen2.5-7B heads
SMALL = dict(kv=8, q=16, d=64, dtype="bf16")
TINY = dict(kv=4, q=8, d=64, dtype="f32")      # the float32 workload's heads


def listed():
    cases = {
        # one generated token of one sequence, far into a long context: latency
        "append-1": dict(op="append", batch=1, T=1, page=64, rot=128, norm=True, start=130001, **LLAMA),
        # a float32 model's prompts, half of each head rotated
        "append-777-f32": dict(op="append", batch=3, T=777, page=16, rot=32, norm=False, start=0, **TINY),
        # a 16k prompt with normed heads
        "append-16k": dict(op="append", batch=1, T=16384, page=64, rot=128, norm=True, start=0, **LLAMA),
        # one sequence over the slots that a 1024-token eviction left and 37 new tokens
        "decode-1k": dict(op="decode", batch=1, T=1061, page=64, acc=True, window=0, sinks=0, **LLAMA),
        # sixteen sequences of 8k to 16k slots
        "decode-16k-b16": dict(op="decode", batch=16, T=16384, page=64, acc=True, window=0, sinks=0, **LLAMA),
        # a sliding-window layer at 32k, seven query heads per KV head
        "decode-window-b8": dict(op="decode", batch=8, T=32011, page=128, acc=False, window=4096, sinks=4, **QWEN),
        # one sequence, 64 tokens over its budget
        "evict-1k": dict(op="evict", batch=1, T=1088, page=64, budget=1024, window=32, sinks=4, **LLAMA),
        # a served batch, cut from 24k slots to 4096
        "evict-24k-b4": dict(op="evict", batch=4, T=24571, page=64, budget=4096, window=64, sinks=64, **LLAMA),
        # two short float32 prompts of odd length
        "prefill-500-f32": dict(op="prefill", batch=2, T=509, rows=509, window=0, sinks=0, ragged=True, **TINY),
        # eight drafted tokens of one sequence at 16k: few rows, many keys
        "prefill-8-rows": dict(op="prefill", batch=1, T=16384, rows=8, window=0, sinks=0, ragged=False, **LLAMA),
        # an 8k prompt, causal, whose normalisers go to the eviction
        "prefill-8k": dict(op="prefill", batch=1, T=8192, rows=8192, window=0, sinks=0, ragged=False, **LLAMA),
        # a chunk of a 32k prompt in a sliding-window layer
        "prefill-window-32k": dict(op="prefill", batch=1, T=32768, rows=2048, window=4096, sinks=4, ragged=False, **QWEN),
    }
    return [dict(name=n, **c) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "evict", "prefill"])
    heads = rng.choice([LLAMA, LLAMA, QWEN, SMALL, TINY])
    page = rng.choice([16, 48, 64, 128, 256])
    if op == "append":
        return dict(op=op, batch=rng.choice([1, 2, 5]), T=_log_int(rng, 5, 12000), page=page, rot=heads["d"] // rng.choice([1, 1, 2]),
                    norm=rng.random() < 0.5, start=_log_int(rng, 1, 200000), **heads)
    if op == "decode":
        batch = _log_int(rng, 1, 32)
        T = _log_int(rng, 20, min(32000, 200000 // batch))
        window = rng.choice([0, 0, 0, max(1, T // 5)])
        return dict(op=op, batch=batch, T=T, page=page, acc=rng.random() < 0.6, window=window, sinks=rng.choice([0, 4, 17]) if window else 0, **heads)
    if op == "evict":
        batch = _log_int(rng, 1, 24)
        budget = _log_int(rng, 64, min(8000, 60000 // batch))
        T = budget + _log_int(rng, 1, min(4 * budget, 80000 // batch - budget))
        return dict(op=op, batch=batch, T=T, page=page, budget=budget, window=rng.randrange(0, budget // 2), sinks=rng.choice([0, 4, 16]), **heads)
    batch = rng.choice([1, 1, 2, 3])
    T = _log_int(rng, 10, 2000 if heads is TINY else 6000 // batch)
    rows = rng.choice([T, T, max(1, T // 3), min(T, rng.randrange(1, 40))])
    window = rng.choice([0, 0, max(1, T // rng.choice([3, 9]))])
    return dict(op=op, batch=batch, T=T, rows=rows, window=window, sinks=rng.choice([0, 4, 70]) if window else 0, ragged=batch > 1, **heads)


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lens(c):
    """Slots (or keys) of every sequence: the first is the longest."""
    T, b = c["T"], c["batch"]
    if c["op"] == "append":
        return [T // b + (i < T % b) for i in range(b)]
    if c["op"] == "prefill" and not c["ragged"]:
        return [T] * b
    return [T - i * T // (2 * b) for i in range(b)]


def _pages(c, g):
    """A pool's page table: every sequence's pages in no order, -1 behind them."""
    used = [(n + c["page"] - 1) // c["page"] for n in _lens(c)]
    ids = torch.randperm(sum(used) + 3, generator=g, device="cuda")[: sum(used)].int()
    table = torch.full((c["batch"], max(used)), -1, dtype=torch.int32, device="cuda")
    for i, n in enumerate(used):
        table[i, :n] = ids[sum(used[:i]): sum(used[:i]) + n]
    return table, sum(used) + 3


def _pool_keys(c, n_pages, g):
    """Keys as a cache holds them: unit normal, a few heavy hitters per head."""
    shape = (n_pages, c["kv"], c["page"])
    k = torch.randn((*shape, c["d"]), generator=g, device="cuda")
    u = torch.randn((1, c["kv"], 1, c["d"]), generator=g, device="cuda")
    hit = 4.0 * (torch.rand((*shape, 1), generator=g, device="cuda") < 0.01)
    return k.addcmul_(hit * math.sqrt(c["d"]), u / u.norm(dim=-1, keepdim=True)).to(_dtype(c))


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(seed)
    b, H, HQ, d, dt = c["batch"], c["kv"], c["q"], c["d"], _dtype(c)
    rand = lambda *shape, dtype=dt: torch.randn(shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    s = dict(case=c)
    if c["op"] == "prefill":
        s.update(q=rand(b, HQ, c["rows"], d), k=rand(b, H, c["T"], d), v=rand(b, H, c["T"], d))
        s["k"][:, :, ::97] *= 2  # a few keys that draw more weight
        s["kv_lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
        s["q_lens"] = s["kv_lens"].clamp(max=c["rows"]) if c["ragged"] else None
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((b, HQ, c["rows"]), device="cuda")
        return s
    table, n_pages = _pages(c, g)
    s.update(table=table, k=_pool_keys(c, n_pages, g), v=rand(n_pages, H, c["page"], d), lens=torch.tensor(_lens(c), dtype=torch.int32, device="cuda"))
    if c["op"] == "append":
        at = torch.cat([torch.arange(n, device="cuda") for n in _lens(c)])
        seq = torch.repeat_interleave(torch.arange(b, device="cuda"), s["lens"])
        s["positions"] = (at + c["start"]).int()
        s["slots"] = table[seq, at // c["page"]].long() * c["page"] + at % c["page"]
        qkv = rand(c["T"], HQ + 2 * H, d)  # one projection's output, as a model holds it
        s["new"] = [qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:]]
        s["weights"] = [(1 + 0.1 * rand(d, dtype=torch.float32)).to(dt) if c["norm"] else None for _ in range(2)]
        s["inv_freq"] = 500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
        s["q_out"] = torch.empty((c["T"], HQ, d), dtype=dt, device="cuda")
        s["acc"] = torch.rand((n_pages, H, c["page"]), generator=g, device="cuda")
        s["pos"] = torch.full((n_pages, H, c["page"]), -1, dtype=torch.int32, device="cuda")
        return s
    # weights with the heavy tail that accumulated attention has
    acc = torch.exp(2 * rand(n_pages, H, c["page"], dtype=torch.float32))
    if c["op"] == "decode":
        s.update(q=2 * rand(b, HQ, d), out=torch.empty((b, HQ, d), device="cuda"), lse=torch.empty((b, HQ), device="cuda"), acc0=acc, acc=acc.clone())
        return s
    # a cache in order: slot s holds token s
    pos = torch.zeros((n_pages, 1, c["page"]), dtype=torch.int32, device="cuda")
    slot = torch.arange(table.shape[1] * c["page"], device="cuda").view(1, -1, 1, c["page"]).expand(b, -1, -1, -1)
    pos[table[table >= 0].long()] = slot[table >= 0].int()
    s["meta0"] = torch.stack([acc, pos.expand_as(acc).contiguous().view(torch.float32)])  # one copy restores both
    s["meta"] = s["meta0"].clone()
    s.update(lens_out=torch.empty_like(s["lens"]), kept=torch.empty((b, H, c["budget"]), dtype=torch.int32, device="cuda"))
    return s


def _plain_append(c, s):
    half = c["rot"] // 2
    angle = torch.remainder(s["positions"].double()[:, None, None] * s["inv_freq"], 2 * math.pi)
    cos, sin = angle.cos().float(), angle.sin().float()

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        lo, hi = x[..., :half], x[..., half:2 * half]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, x[..., 2 * half:]], -1)

    (q, k, v), (wq, wk), (page, row) = s["new"], s["weights"], (s["slots"] // c["page"], s["slots"] % c["page"])
    s["q_out"].copy_(turned(q, wq))
    s["k"][page, :, row] = turned(k, wk).to(k.dtype)
    s["v"][page, :, row] = v
    s["acc"][page, :, row] = 0.0
    s["pos"][page, :, row] = s["positions"][:, None]


def _rows(c, s):
    """Row of the flat pool [pages * heads * page] that holds each slot, and the slots that exist: [b][H][slots], [b][1][slots]."""
    slot = torch.arange(s["table"].shape[1] * c["page"], device="cuda")
    page = s["table"].long().clamp(min=0).repeat_interleave(c["page"], 1)
    rows = (page[:, None] * c["kv"] + torch.arange(c["kv"], device="cuda")[:, None]) * c["page"] + slot % c["page"]
    return rows, (slot < s["lens"][:, None])[:, None]


def _plain_decode(c, s):
    b, H, d, G = c["batch"], c["kv"], c["d"], c["q"] // c["kv"]
    rows, live = _rows(c, s)
    if c["window"]:
        slot, n = torch.arange(rows.shape[-1], device="cuda"), s["lens"][:, None, None]
        live = live & ((slot >= n - c["window"]) | (slot < c["sinks"]))
    k, v = s["k"].view(-1, d)[rows].float(), s["v"].view(-1, d)[rows].float()
    x = torch.matmul(s["q"].float().view(b, H, G, d), k.transpose(-1, -2)) / math.sqrt(d)
    x = x.masked_fill(~live[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    p = e / total
    s["out"].copy_(torch.matmul(p, v).view(b, H * G, d))
    s["lse"].copy_((top + total.log()).view(b, H * G))
    if c["acc"]:
        s["acc"].view(-1).scatter_add_(0, rows.flatten(), p.mean(2).flatten())


def _plain_evict(c, s):
    B, d = c["budget"], c["d"]
    rows, live = _rows(c, s)
    acc, pos = s["meta"][0].view(-1), s["meta"][1].view(torch.int32).view(-1)
    at = pos[rows]
    safe = (at < c["sinks"]) | (at >= s["lens"][:, None, None] - c["window"])
    weight = torch.where(safe, math.inf, acc[rows]).masked_fill(~live, -math.inf)
    order = torch.sort(weight, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(rows, dtype=torch.bool).scatter_(-1, order[..., :B], True) & live
    slot = torch.arange(rows.shape[-1], device="cuda").expand_as(rows)
    late = torch.where(kept & (slot >= B), slot, rows.shape[-1]).sort(-1).values[..., :B]
    hole = ~kept[..., :B]
    source = torch.where(hole, late.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), slot[..., :B])
    exists = slot[..., :B] < s["lens"][:, None, None]
    s["kept"].copy_(torch.where(exists, source, -1))
    s["lens_out"].copy_(s["lens"].clamp(max=B))
    # rows that do not exist repeat what slot 0 gets
    source, target = torch.where(exists, source, source[..., :1]), torch.where(exists, slot[..., :B], 0)
    source, target = rows.gather(-1, source.clamp(max=rows.shape[-1] - 1)).flatten(), rows.gather(-1, target).flatten()
    for flat in (s["k"].view(-1, d), s["v"].view(-1, d), acc, pos):
        flat[target] = flat[source]


def _hidden(c, s):
    """Keys that each row does not see: [b or 1][rows][T]; rows of negative position see none."""
    t, r = torch.arange(c["T"], device="cuda"), torch.arange(c["rows"], device="cuda")[:, None]
    last = r + c["T"] - c["rows"] if s["kv_lens"] is None else r + (s["kv_lens"] - s["q_lens"])[:, None, None]
    hidden = t > last
    if c["window"]:
        hidden = hidden | ((t <= last - c["window"]) & (t >= c["sinks"]))
    return hidden.view(-1, 1, 1, c["rows"], c["T"])


def _plain_prefill(c, s):
    b, H, d, G, R = c["batch"], c["kv"], c["d"], c["q"] // c["kv"], c["rows"]
    q, k, v = s["q"].float().view(b, H, G * R, d), s["k"].float(), s["v"].float()
    x = torch.matmul(q, k.transpose(-1, -2)).view(b, H, G, R, -1).div_(math.sqrt(d)).masked_fill_(_hidden(c, s), -math.inf)
    top = x.amax(-1, keepdim=True)
    e = x.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e.view(b, H, G * R, -1), v).view(b, H, G, R, d) / total
    lse = (top + total.log()).squeeze(-1)
    if s["q_lens"] is not None:  # rows behind a sequence's last are left as they were
        real = (torch.arange(R, device="cuda") < s["q_lens"][:, None])[:, None, None]
        out, lse = torch.where(real[..., None], out, s["out"].view_as(out)), torch.where(real, lse, s["lse"].view_as(lse))
    s["out"].copy_(out.view(b, H * G, R, d))
    s["lse"].copy_(lse.view(b, H * G, R))


def _handle(c, s):
    """What a program sets up once for its shapes: the configuration and a workspace."""
    from paper_2606_29563_amd import kvec
    dt = kvec.KVEC_BF16 if c["dtype"] == "bf16" else kvec.KVEC_F32
    if c["op"] == "prefill":
        cfg = kvec.AttentionConfig(batch=c["batch"], n_kv_heads=c["kv"], n_q_heads=c["q"], head_dim=c["d"], q_len=c["rows"], kv_len=c["T"],
                                   window=c["window"], n_sinks=c["sinks"], dtype=dt)
        size = kvec.kvec_prefill_workspace_size(cfg)
    else:
        cfg = kvec.PagedConfig(batch=c["batch"], n_kv_heads=c["kv"], n_q_heads=c["q"], head_dim=c["d"], page_size=c["page"], n_pages=s["k"].shape[0],
                               max_pages=s["table"].shape[1], dtype=dt)
        size = 0
        if c["op"] == "decode":
            size = kvec.kvec_paged_decode_workspace_size(cfg, c["T"], c["acc"])
        if c["op"] == "evict":
            size = kvec.kvec_paged_evict_workspace_size(cfg, c["T"], c["budget"])
    return kvec, cfg, torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


def _own(c, s):
    if "handle" not in s:
        s["handle"] = _handle(c, s)
    kvec, cfg, ws = s["handle"]
    if c["op"] == "append":
        q, k, v = s["new"]
        kvec.kvec_paged_append(cfg, q, k, v, s["positions"], s["slots"], s["q_out"], s["k"], s["v"], q_weight=s["weights"][0], k_weight=s["weights"][1],
                               eps=1e-6, inv_freq=s["inv_freq"], acc=s["acc"], pos=s["pos"])
    elif c["op"] == "decode":
        kvec.kvec_paged_decode(cfg, s["q"], s["k"], s["v"], s["table"], s["lens"], s["out"], ws, max_len=c["T"], window=c["window"], n_sinks=c["sinks"],
                               lse=s["lse"], acc=s["acc"] if c["acc"] else None)
    elif c["op"] == "evict":
        kvec.kvec_paged_evict(cfg, c["budget"], s["k"], s["v"], s["table"], s["lens"], s["lens"], s["meta"][0], s["meta"][1].view(torch.int32),
                              s["lens_out"], ws, window=c["window"], n_sinks=c["sinks"], kept=s["kept"], max_len=c["T"])
    else:
        kvec.kvec_prefill_attention(cfg, s["q"], s["k"], s["v"], s["out"], ws, lse=s["lse"], q_lens=s["q_lens"], kv_lens=s["kv_lens"])


_PLAIN = dict(append=_plain_append, decode=_plain_decode, evict=_plain_evict, prefill=_plain_prefill)


def run(s):
    c = s["case"]
    # every pass starts from the weights that the cache held before it
    if c["op"] == "decode" and c["acc"]:
        s["acc"].copy_(s["acc0"])
    if c["op"] == "evict":
        s["meta"].copy_(s["meta0"])
    if own:
        _own(c, s)
    else:
        _PLAIN[c["op"]](c, s)
    if c["op"] == "append":
        return dict(q=s["q_out"], k=s["k"], v=s["v"], acc=s["acc"], pos=s["pos"])
    if c["op"] == "decode":
        return dict(out=s["out"], lse=s["lse"], **(dict(acc=s["acc"]) if c["acc"] else {}))
    if c["op"] == "evict":
        return dict(k=s["k"], v=s["v"], acc=s["meta"][0], pos=s["meta"][1].view(torch.int32), kept=s["kept"], lens=s["lens_out"])
    return dict(out=s["out"], lse=s["lse"])


def _pairs(keys, rows, window, sinks):
    """(row, key) pairs that are visible when the rows are the last of the keys."""
    n = 0
    for p in range(keys - rows, keys):
        n += p + 1 if not window else min(p + 1, window) + max(0, min(sinks, p + 1 - window))
    return n


def work(case):
    """Inputs read once, outputs written once; the products of the visible pairs."""
    c, es = case, 2 if case["dtype"] == "bf16" else 4
    b, H, HQ, d = c["batch"], c["kv"], c["q"], c["d"]
    lens = _lens(c)
    if c["op"] == "append":
        return dict(bytes=c["T"] * (2 * (HQ + 2 * H) * d * es + 8 * H + 12), flops=4 * c["T"] * (HQ + H) * d)
    if c["op"] == "decode":
        seen = sum(_pairs(n, 1, c["window"], c["sinks"]) for n in lens)
        return dict(bytes=seen * H * (2 * d * es + (8 if c["acc"] else 0)) + b * HQ * (d * (es + 4) + 4), flops=4 * HQ * d * seen)
    if c["op"] == "evict":
        # a slot's weight and position; of the kept slots, as many move as were behind the budget
        B, moved = c["budget"], sum(min(n - c["budget"], c["budget"]) * c["budget"] / n for n in lens if n > c["budget"])
        return dict(bytes=int(sum(8 * n * H for n in lens) + moved * H * (4 * d * es + 16) + 4 * b * H * B), flops=0)
    pairs = sum(_pairs(n, min(n, c["rows"]), c["window"], c["sinks"]) for n in lens)
    rows = sum(min(n, c["rows"]) for n in lens)
    seen = sum(min(n, min(n, c["rows"]) + c["window"] + c["sinks"]) if c["window"] else n for n in lens)
    return dict(bytes=rows * HQ * (2 * d * es + 4) + 2 * seen * H * d * es, flops=4 * HQ * d * pairs)


# --- the definitions in 64 bits, one head (append: one tensor) at a time ---


def _softmax64(q, k, v, hidden):
    """q [rows][d], k and v [keys][d], all float64: out, lse, weights."""
    x = (q @ k.T) * q.shape[-1] ** -0.5
    x[hidden] = -math.inf
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[:, None])
    return p @ v, lse, p


def _exact_append(c, s):
    def value(x, w, i):  # one head, all tokens
        x = x[:, i].double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.double()
        out, n = x.clone(), c["rot"] // 2
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"])
        z = torch.complex(x[:, :n], x[:, n:2 * n]) * turn
        out[:, :n], out[:, n:2 * n] = z.real, z.imag
        return out

    q, k, _ = s["new"]
    out = dict(q=torch.stack([value(q, s["weights"][0], i) for i in range(c["q"])], 1), k=s["k"].double(), v=None, acc=None, pos=None)
    for i in range(c["kv"]):
        out["k"][s["slots"] // c["page"], i, s["slots"] % c["page"]] = value(k, s["weights"][1], i)
    return out


def _exact_decode(c, s):
    G = c["q"] // c["kv"]
    out = dict(out=torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), lse=torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda"))
    if c["acc"]:
        out["acc"] = s["acc0"].double()
    for i, n in enumerate(_lens(c)):
        slot = torch.arange(n, device="cuda")
        page, row = s["table"][i].long()[slot // c["page"]], slot % c["page"]
        hidden = (slot < n - c["window"]) & (slot >= c["sinks"]) if c["window"] else slot < 0
        for h in range(c["kv"]):
            own_heads = slice(h * G, h * G + G)
            o, l, p = _softmax64(s["q"][i, own_heads].double(), s["k"][page, h, row].double(), s["v"][page, h, row].double(), hidden.expand(G, n))
            out["out"][i, own_heads], out["lse"][i, own_heads] = o, l
            if c["acc"]:
                out["acc"][page, h, row] += p.mean(0)
    return out


def _exact_prefill(c, s):
    G, R = c["q"] // c["kv"], c["rows"]
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for i, n in enumerate(_lens(c)):
        m = min(n, R)
        p, t = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")
        seen = t <= p
        if c["window"]:
            seen &= (p - t < c["window"]) | (t < c["sinks"])
        for j in range(c["q"]):
            out[i, j, :m], lse[i, j, :m], _ = _softmax64(s["q"][i, j, :m].double(), s["k"][i, j // G, :n].double(), s["v"][i, j // G, :n].double(), ~seen)
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["op"] == "evict":
        return None  # picks and copied rows: no computed numbers
    return dict(append=_exact_append, decode=_exact_decode, prefill=_exact_prefill)[case["op"]](case, prepare(case, seed))

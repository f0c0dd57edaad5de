"""kvec_prefill_attention on the GPU against its definition in float64."""
import math

import numpy as np
import pytest

import serve_testlib as ref

pytestmark = pytest.mark.gpu


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _tensors(b, H, G, d, nq, nk, dt, seed, layout="bhtd"):
    """q, k, v; layout bthd: heads inside a token's row, as a projection leaves them."""
    import torch
    g = torch.Generator().manual_seed(seed)

    def one(h, n, scale):
        x = (torch.randn((b, h, n, d) if layout == "bhtd" else (b, n, h, d), generator=g) * scale).to(_dt(dt)).cuda()
        return x if layout == "bhtd" else x.transpose(1, 2)
    return one(H * G, nq, 1.5), one(H, nk, 1.5), one(H, nk, 1.0)


def _run(kv, q, k, v, window=0, sinks=0, q_lens=None, kv_lens=None, with_lse=True, stream=None):
    import torch
    b, HQ, nq, d = q.shape
    cfg = kv.AttentionConfig(b, k.shape[1], HQ, d, nq, k.shape[2], window, sinks, kv.KVEC_BF16 if q.dtype == torch.bfloat16 else kv.KVEC_F32)
    n = kv.kvec_prefill_workspace_size(cfg)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
    out = torch.full((b, HQ, nq, d), 77.0, dtype=q.dtype, device="cuda")
    lse = torch.full((b, HQ, nq), 77.0, device="cuda") if with_lse else None
    lens = [None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_lens, kv_lens)]
    kv.kvec_prefill_attention(cfg, q, k, v, out, ws, lse=lse, q_lens=lens[0], kv_lens=lens[1], stream=stream)
    return out, lse


def _check(q, k, v, out, lse, window=0, sinks=0, q_lens=None, kv_lens=None, rows=None):
    b, HQ, nq, d = q.shape
    G = HQ // k.shape[1]
    qn, kn, vn, on, ln = ref.f64(q), ref.f64(k), ref.f64(v), ref.f64(out), ref.f64(lse)
    bf16 = q.element_size() == 2
    u = ref.U_BF16 if bf16 else ref.U24
    for i in range(b):
        m = nq if q_lens is None else max(0, min(q_lens[i], nq))
        n = k.shape[2] if kv_lens is None else max(0, min(kv_lens[i], k.shape[2]))
        assert np.all(on[i, :, m:] == 77.0) and np.all(ln[i, :, m:] == 77.0)
        for r in range(m) if rows is None else [r for r in rows if r < m]:
            seen = ref.visible(n, n, n - m + r, window, sinks)
            for j in range(HQ):
                o, l, w, dx = ref.attend(qn[i, j, r], kn[i, j // G, :n], vn[i, j // G, :n], seen)
                # the probabilities rounded to bf16 (they are summed unrounded), then the output
                off = (2 * dx + ref.EXP + (u if bf16 else 0)) * (w @ np.abs(vn[i, j // G, :n])) + u * np.abs(o) * (1 + u) + 1e-30
                assert np.all(np.abs(on[i, j, r] - o) <= off), (i, j, r, np.max(np.abs(on[i, j, r] - o) / off))
                assert ln[i, j, r] == l or abs(ln[i, j, r] - l) <= dx + ref.EXP * (1 + abs(l)), (i, j, r, ln[i, j, r], l)


CASES = [  # b, H, G, d, q rows, keys, dtype, window, sinks, q_lens, kv_lens, layout
    (1, 1, 1, 128, 1, 1, "bf16", 0, 0, None, None, "bhtd"),
    (2, 2, 4, 128, 33, 33, "bf16", 0, 0, None, None, "bhtd"),
    (1, 4, 7, 128, 65, 65, "bf16", 0, 0, None, None, "bthd"),
    (1, 1, 16, 64, 130, 130, "bf16", 0, 0, None, None, "bhtd"),
    (2, 3, 1, 64, 200, 200, "bf16", 0, 0, None, None, "bthd"),
    (1, 2, 5, 128, 17, 300, "bf16", 0, 0, None, None, "bhtd"),
    (1, 2, 2, 64, 150, 150, "f32", 0, 0, None, None, "bhtd"),
    (2, 2, 3, 128, 40, 77, "f32", 0, 0, None, None, "bthd"),
    (1, 1, 16, 128, 9, 9, "f32", 0, 0, None, None, "bhtd"),
    # windows: one key, inside a tile, over tiles, with sinks that end inside a tile or reach the window
    (1, 2, 2, 64, 140, 140, "bf16", 1, 0, None, None, "bhtd"),
    (1, 2, 4, 128, 200, 260, "bf16", 37, 4, None, None, "bhtd"),
    (2, 1, 3, 64, 150, 300, "bf16", 100, 70, None, None, "bthd"),
    (1, 2, 1, 128, 100, 400, "bf16", 64, 350, None, None, "bhtd"),
    (1, 1, 2, 64, 90, 200, "f32", 33, 65, None, None, "bhtd"),
    (1, 1, 2, 64, 20, 50, "bf16", 50, 3, None, None, "bhtd"),
    # ragged: empty sequences, more rows than keys (rows that see nothing), lengths out of range
    (5, 2, 2, 64, 70, 90, "bf16", 0, 0, [70, 0, 33, 1, 100], [90, 40, 33, 0, 900], "bhtd"),
    (3, 1, 4, 128, 50, 64, "bf16", 20, 5, [50, 12, -4], [10, 64, 8], "bthd"),
    (3, 1, 2, 64, 40, 64, "f32", 9, 5, [40, 12, 3], [10, 64, 64], "bhtd"),
    # few rows, many keys: split
    (1, 2, 4, 128, 3, 2100, "bf16", 0, 0, None, None, "bhtd"),
    (2, 1, 7, 64, 1, 3000, "bf16", 0, 0, None, [2999, 130], "bthd"),
    (1, 1, 2, 128, 5, 1200, "f32", 0, 0, None, None, "bhtd"),
    (1, 1, 2, 64, 4, 4000, "bf16", 1500, 9, None, None, "bhtd"),
    (2, 1, 2, 64, 4, 2000, "bf16", 0, 0, [4, 2], [1, 2000], "bhtd"),
    # many sequences, many heads
    (300, 2, 1, 64, 3, 9, "bf16", 0, 0, None, None, "bhtd"),
    (1, 160, 1, 128, 20, 33, "bf16", 5, 2, None, None, "bthd"),
    (1, 96, 2, 64, 20, 33, "f32", 0, 0, None, None, "bhtd"),
]


@pytest.mark.parametrize("b,H,G,d,nq,nk,dt,window,sinks,q_lens,kv_lens,layout", CASES)
def test_prefill(gpu_lib, b, H, G, d, nq, nk, dt, window, sinks, q_lens, kv_lens, layout):
    q, k, v = _tensors(b, H, G, d, nq, nk, dt, seed=nq + nk + G, layout=layout)
    if kv_lens is not None:  # what lies behind a sequence's keys is not read
        for i, n in enumerate(kv_lens):
            k[i, :, max(0, n):] = math.nan
            v[i, :, max(0, n):] = math.inf
    out, lse = _run(gpu_lib, q, k, v, window, sinks, q_lens, kv_lens)
    _check(q, k, v, out, lse, window, sinks, q_lens, kv_lens)
    o2, _ = _run(gpu_lib, q, k, v, window, sinks, q_lens, kv_lens, with_lse=False)
    assert o2.equal(out)


LONG = [  # b, H, G, d, q rows, keys, dtype, window, sinks, q_lens, kv_lens
    (1, 2, 4, 128, 1300, 2500, "bf16", 0, 0, None, None),
    (1, 2, 4, 128, 1300, 2500, "bf16", 500, 20, None, None),
    (1, 2, 4, 128, 1300, 2500, "f32", 0, 0, None, None),
    # more row tiles than compute units
    (1, 8, 4, 128, 2100, 2100, "bf16", 0, 0, None, None),
    (2, 8, 2, 64, 4200, 4300, "bf16", 0, 0, [4200, 4111], [4300, 4000]),
    (3, 4, 7, 128, 1999, 2400, "bf16", 700, 100, [1999, 50, 1500], [2400, 2400, 1200]),
    (1, 8, 16, 64, 1100, 1100, "bf16", 300, 0, None, None),
    (1, 5, 5, 128, 2300, 2300, "bf16", 0, 0, None, None),
    # ... split over the keys
    (1, 8, 4, 128, 100, 5000, "bf16", 0, 0, None, None),
    (1, 8, 4, 64, 200, 9000, "bf16", 4000, 65, None, None),
    (1, 2, 4, 128, 600, 3000, "bf16", 0, 0, None, None),
    (2, 2, 4, 128, 1000, 2100, "bf16", 2000, 3, [1000, 997], [2100, 2040]),
    (1, 8, 4, 128, 500, 7001, "bf16", 0, 0, None, None),
    (1, 1, 8, 128, 2000, 30001, "bf16", 0, 0, None, None),
    (1, 4, 7, 128, 500, 8003, "bf16", 0, 0, None, None),
    # work-groups of four waves, alone or with the keys divided over several times as many
    (2, 4, 7, 128, 900, 900, "bf16", 100, 0, None, [900, 450]),
    (1, 8, 4, 128, 900, 2900, "bf16", 700, 10, None, None),
    (4, 8, 2, 64, 300, 1300, "bf16", 0, 0, [300, 1, 0, 299], [1300, 1290, 700, 0]),
    (2, 1, 8, 128, 300, 1501, "bf16", 0, 0, [300, 171], [1501, 1500]),
    (1, 3, 8, 64, 900, 900, "bf16", 0, 0, None, None),
    (1, 8, 4, 64, 200, 300, "bf16", 0, 0, None, None),
    (1, 4, 2, 64, 1500, 1500, "f32", 200, 0, None, None),
    (2, 4, 4, 128, 300, 300, "f32", 0, 0, None, [300, 211]),
    (2, 8, 4, 128, 260, 400, "f32", 0, 0, [260, 33], [399, 400]),
    (1, 1, 16, 64, 300, 900, "f32", 0, 0, None, None),
    (1, 1, 2, 64, 4, 4000, "f32", 0, 0, None, None),
    (1, 8, 2, 64, 300, 6000, "bf16", 0, 0, None, None),
]


@pytest.mark.parametrize("b,H,G,d,nq,nk,dt,window,sinks,q_lens,kv_lens", LONG)
def test_prefill_long(gpu_lib, b, H, G, d, nq, nk, dt, window, sinks, q_lens, kv_lens):
    """Many tiles and work-groups, some rows checked: the first and last of tiles."""
    q, k, v = _tensors(b, H, G, d, nq, nk, dt, seed=5)
    out, lse = _run(gpu_lib, q, k, v, window, sinks, q_lens, kv_lens)
    rows = sorted({r for r in (0, 1, 15, 16, 49, 63, 64, 99, 127, 255, 640, 1023, nq // 2, nq - 2, nq - 1) if r < nq})
    _check(q, k, v, out, lse, window, sinks, q_lens, kv_lens, rows=rows)


def test_prefill_extreme_logits(gpu_lib):
    """Logits of thousands that grow along the keys, fall along them, and are all equal."""
    import torch
    for n, H, every in ((300, 1, 7), (2100, 16, 211)):  # few and many row tiles
        for kind in ("grow", "fall", "equal", "one"):
            q, k, v = _tensors(1, H, 2, 64, n, n, "bf16", seed=6)
            ramp = torch.arange(n, device="cuda")[:, None].float()
            u = torch.ones(64, device="cuda")
            k.copy_((u * (ramp / 4 if kind == "grow" else -ramp / 4 if kind == "fall" else 0 * ramp + 1)).to(k.dtype))
            if kind == "one":  # a single key far above the others, behind many
                k[:, :, n // 2] *= 50
            q.copy_(q.abs())
            out, lse = _run(gpu_lib, q, k, v)
            _check(q[:, :2], k[:, :1], v[:, :1], out[:, :2], lse[:, :2], rows=list(range(0, n, every)))


def test_prefill_strides_of_outputs_and_shared_keys(gpu_lib):
    """out and lse inside larger tensors; one sequence's keys for the whole batch (stride 0)."""
    import torch
    kv = gpu_lib
    q, k, v = _tensors(2, 2, 2, 64, 70, 70, "bf16", seed=8)
    k, v = (x[:1].expand(2, -1, -1, -1) for x in (k, v))
    big, big_lse = torch.full((2, 75, 4, 64), 77.0, dtype=q.dtype, device="cuda"), torch.full((2, 6, 90), 77.0, device="cuda")
    out, lse = big[:, 2:72].transpose(1, 2), big_lse[:, 1:5, 3:73]
    cfg = kv.AttentionConfig(2, 2, 4, 64, 70, 70)
    kv.kvec_prefill_attention(cfg, q, k, v, out, lse=lse)
    _check(q, k, v, out, lse)
    assert torch.all(big[:, :2] == 77) and torch.all(big[:, 72:] == 77)
    assert torch.all(big_lse[:, 0] == 77) and torch.all(big_lse[:, 5] == 77) and torch.all(big_lse[:, :, :3] == 77) and torch.all(big_lse[:, :, 73:] == 77)


def test_prefill_far_offsets(gpu_lib):
    """Sequences 2^31 elements and more apart, and keys that span almost 2 GiB."""
    import torch
    kv, gap = gpu_lib, (1 << 31) + 4096
    q, k, v = _tensors(2, 1, 2, 64, 300, 300, "bf16", seed=12)
    out, lse = _run(kv, q, k, v)
    buf = torch.empty(gap + 300 * 64 * 2, dtype=torch.bfloat16, device="cuda")
    for x in (q, k, v):
        y = buf.as_strided(x.shape, (gap, x.stride(1), 64, 1))
        y.copy_(x)
        o2 = torch.empty_like(out)
        kv.kvec_prefill_attention(kv.AttentionConfig(2, 1, 2, 64, 300, 300), *(y if x is t else t for t in (q, k, v)), o2)
        assert o2.equal(out)
    y = buf.as_strided(out.shape, (gap, out.stride(1), 64, 1))
    y.fill_(0)
    kv.kvec_prefill_attention(kv.AttentionConfig(2, 1, 2, 64, 300, 300), q, k, v, y)
    assert torch.equal(y, out)
    row = ((1 << 30) - 1) // 300 // 8 * 8  # 300 rows of this stride: just below 2 GiB
    wide = buf.as_strided((1, 1, 300, 64), (0, 0, row, 1))
    wide.copy_(k[:1])
    o2 = torch.empty_like(out[:1])
    kv.kvec_prefill_attention(kv.AttentionConfig(1, 1, 2, 64, 300, 300), q[:1], wide, v[:1], o2)
    assert o2.equal(out[:1])


def test_prefill_graph_and_stream(gpu_lib):
    """Two captured calls that share a workspace, replayed with eager work between."""
    import torch
    kv = gpu_lib
    q, k, v = _tensors(1, 2, 4, 128, 4, 1500, "bf16", seed=9)
    cfg = kv.AttentionConfig(1, 2, 8, 128, 4, 1500)
    n = kv.kvec_prefill_workspace_size(cfg)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]
    args = [(q, k, v), (q.flip(2).contiguous(), k.flip(2).contiguous(), v)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    wants = [_run(kv, *a, stream=side)[0] for a in args]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for a, o in zip(args, outs):
            kv.kvec_prefill_attention(cfg, *a, o, ws)
    for _ in range(4):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.randn(300, 300, device="cuda").sum().item()
        for o, w in zip(outs, wants):
            assert o.equal(w)


def test_prompt_to_eviction_to_decode(gpu_lib):
    """A prompt's attention gives the normalisers that the eviction step takes; its kept
    rows become a paged cache that tokens are decoded over."""
    import torch
    kv, H, G, d, T, W, B = gpu_lib, 4, 2, 64, 700, 32, 128
    q, k, v = _tensors(1, H, G, d, T, T, "bf16", seed=10)
    out, lse = _run(kv, q, k, v)
    cfg = kv.Config(batch=1, n_layers=1, n_kv_heads=H, n_q_heads=H * G, head_dim=d, seq_len=T, window=16, window_ext=W, budget=B)
    ws = torch.empty(kv.kvec_workspace_size(cfg), dtype=torch.uint8, device="cuda")

    def evicted(call):
        idx = torch.empty((1, H, B), dtype=torch.int32, device="cuda")
        ko, vo = (torch.empty((1, H, B, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        bits = torch.zeros((1, 1, cfg.words), dtype=torch.int64, device="cuda")
        call(bits, idx, ko, vo)
        return idx, ko, vo
    q_win = q[:, :, T - W:]
    own = evicted(lambda bits, idx, ko, vo: kv.kvec_evict_layer(cfg, 0, q_win, k, v, bits, idx, ko, vo, ws))
    given = evicted(lambda bits, idx, ko, vo: kv.kvec_evict_layer_lse(cfg, 0, q_win, lse[:, :, T - W:], k, v, bits, idx, ko, vo, ws))
    same = (own[0][0].sort(-1).values == given[0][0].sort(-1).values).float().mean().item()
    assert same >= 0.99, same
    # the kept rows, with room for more tokens, as a cache of one page per sequence
    idx, ko, vo = given
    page = B + 16
    pc = kv.PagedConfig(1, H, H * G, d, page, 1, 1)
    kp, vp = (torch.full((1, H, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kp[:, :, :B], vp[:, :, :B] = ko, vo
    acc, pos = torch.zeros((1, H, page), device="cuda"), torch.full((1, H, page), -1, dtype=torch.int32, device="cuda")
    pos[:, :, :B] = idx
    table, lens = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([B], dtype=torch.int32, device="cuda")
    qd = torch.randn((1, H * G, d), device="cuda").bfloat16()
    got = torch.empty((1, H * G, d), device="cuda")
    kv.kvec_paged_decode(pc, qd, kp, vp, table, lens, got, torch.empty(kv.kvec_paged_decode_workspace_size(pc, None, True), dtype=torch.uint8, device="cuda"),
                         acc=acc)
    want = torch.empty_like(got)
    kv.kvec_decode_attention(cfg, qd, ko, vo, want, torch.empty(kv.kvec_decode_workspace_size(cfg, B), dtype=torch.uint8, device="cuda"))
    vmax = vo.float().abs().max().item()
    # both are within 1e-4 of the definition (the bar of kvec_decode_attention's own tests)
    assert (got - want).abs().max().item() <= 2e-4 * vmax
    assert abs(acc.sum().item() - H) < 1e-3  # every head's weights sum to one

"""Queries and keys that are no numbers, in the serving calls: a row whose logits hold a
NaN gets NaN, zeros and -inf are for rows that see nothing, and the rows beside it keep
their values."""
import math

import pytest

from test_gpu_paged import Cache, _decode, _dt
from test_gpu_prefill import _check, _run, _tensors

pytestmark = pytest.mark.gpu

PROMPTS = [  # b, H, G, d, q rows, keys, dtype, window, sinks: every kernel, in one piece and split
    (1, 2, 4, 128, 33, 33, "bf16", 0, 0),
    (1, 2, 4, 128, 4, 2100, "bf16", 0, 0),
    (1, 8, 4, 128, 700, 700, "bf16", 0, 0),
    (1, 8, 4, 128, 1100, 1100, "bf16", 300, 4),
    (1, 8, 4, 128, 2600, 2600, "bf16", 0, 0),
    (1, 1, 8, 128, 2000, 9001, "bf16", 0, 0),
    (1, 2, 2, 64, 150, 150, "bf16", 0, 0),
    (1, 8, 4, 64, 900, 900, "bf16", 0, 0),
    (2, 1, 7, 64, 3, 3000, "bf16", 0, 0),
    (1, 2, 2, 64, 150, 150, "f32", 0, 0),
    (2, 4, 4, 128, 300, 300, "f32", 0, 0),
    (1, 1, 2, 64, 4, 4000, "f32", 0, 0),
    (1, 1, 2, 128, 5, 1200, "f32", 200, 3),
]


@pytest.mark.parametrize("b,H,G,d,nq,nk,dt,window,sinks", PROMPTS)
def test_prompt_with_a_nan_query(gpu_lib, b, H, G, d, nq, nk, dt, window, sinks):
    import torch
    q, k, v = _tensors(b, H, G, d, nq, nk, dt, seed=nq + d)
    bad = sorted({0, nq // 2, nq - 1})
    q[:, :, bad, 5] = math.nan
    out, lse = _run(gpu_lib, q, k, v, window, sinks)
    assert torch.isnan(out[:, :, bad]).all() and torch.isnan(lse[:, :, bad]).all()
    near = {r + s for r in bad for s in (-2, -1, 1, 2, 17)}  # rows of the same tiles
    _check(q, k, v, out, lse, window, sinks, rows=sorted(r for r in near if 0 <= r < nq and r not in bad))


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_prompt_rows_that_see_nothing_stay_empty(gpu_lib, dt, d):
    """More rows than keys: a NaN query of a row before the first key is never used."""
    import torch
    q, k, v = _tensors(2, 2, 3, d, 50, 64, dt, seed=3)
    q[:, :, :20] = math.nan
    out, lse = _run(gpu_lib, q, k, v, q_lens=[50, 50], kv_lens=[30, 0])
    assert torch.all(out[0, :, :20] == 0) and torch.all(lse[0, :, :20] == -math.inf)
    assert torch.all(out[1] == 0) and torch.all(lse[1] == -math.inf)
    q[:, :, :20] = 0
    _check(q, k, v, out, lse, q_lens=[50, 50], kv_lens=[30, 0])


DECODES = [  # lens, H, G, d, dtype, window, sinks: in one launch and in two
    ([100, 40, 0], 2, 4, 128, "bf16", 0, 0),
    ([100, 77], 1, 16, 64, "f32", 20, 3),
    ([900, 40, 0, 2000], 2, 4, 128, "bf16", 0, 0),
    ([9000, 100], 1, 5, 64, "bf16", 700, 30),
    ([1500, 3], 2, 1, 128, "f32", 0, 0),
]


@pytest.mark.parametrize("lens,H,G,d,dt,window,sinks", DECODES)
def test_decode_with_a_nan_query(gpu_lib, lens, H, G, d, dt, window, sinks):
    """One query head of one KV head: NaN in its output and, through the mean over the
    heads, in the weights of that KV head's visible slots; all else keeps its bits."""
    import torch
    c = Cache(gpu_lib, lens, H, G, d, 16, dt, seed=d + G).cuda()
    q = c.rand(len(lens), H * G, d).to(_dt(dt)).cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks)
    want_acc = c.acc.clone()
    j = H * G - 1
    q[:, j, 7] = math.nan
    for acc in (False, True):
        c.acc.copy_(acc0)
        got, got_lse = _decode(c, q, window, sinks, acc=acc)
        for i, n in enumerate(lens):
            if n == 0:
                assert torch.all(got[i] == 0) and torch.all(got_lse[i] == -math.inf)
                continue
            assert torch.isnan(got[i, j]).all() and torch.isnan(got_lse[i, j])
            assert got[i, :j].equal(out[i, :j]) and got_lse[i, :j].equal(lse[i, :j])
    for i, n in enumerate(lens):
        page, row = c.slots(i, n)
        for s in range(n):
            seen = not window or s >= n - window or s < sinks
            want_acc[page[s], H - 1, row[s]] = math.nan if seen else acc0[page[s], H - 1, row[s]]
    assert torch.equal(c.acc.nan_to_num(-1), want_acc.nan_to_num(-1))


@pytest.mark.parametrize("n", [90, 1500])
def test_decode_of_logits_that_are_all_minus_infinity(gpu_lib, n):
    """No weight on any slot: zeros, -inf, and accumulated weights as they were."""
    import torch
    c = Cache(gpu_lib, [n], 1, 2, 64, 16, "f32", seed=2).cuda()
    page, row = c.slots(0, n)
    c.k[page, :, row] = -math.inf
    q = c.rand(1, 2, 64).abs().add_(0.1).cuda()
    acc0 = c.acc.clone()
    out, lse = _decode(c, q)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)
    assert torch.equal(c.acc.nan_to_num(-1), acc0.nan_to_num(-1))


UNSEEN = [  # b, H, G, d, rows, keys, dtype, window, sinks, keys that are no numbers
    (1, 2, 4, 128, 33, 33, "bf16", 0, 0, [20]),
    (1, 2, 4, 128, 8, 2100, "bf16", 0, 0, [2095, 2096]),
    (1, 2, 2, 128, 20, 2100, "bf16", 300, 7, [3, 9, 1795, 2085]),
    (1, 8, 4, 128, 700, 700, "bf16", 0, 0, [1, 65, 130, 300, 699]),
    (1, 8, 4, 128, 1100, 1100, "bf16", 300, 4, [0, 5, 63, 64, 500, 1000]),
    (1, 8, 4, 128, 2600, 2600, "bf16", 0, 0, [2000, 2559, 2560]),
    (1, 1, 8, 128, 2000, 9001, "bf16", 0, 0, [7500, 9000]),
    (1, 1, 2, 128, 2500, 2500, "bf16", 0, 0, [64, 2300]),
    (1, 8, 4, 128, 500, 500, "bf16", 0, 0, [31, 33, 400]),
    (1, 8, 2, 64, 1500, 1500, "bf16", 0, 0, [0, 700, 1400]),
    (1, 8, 2, 64, 1500, 1500, "bf16", 500, 2, [0, 1, 700, 1400]),
    (1, 2, 2, 64, 150, 150, "bf16", 0, 0, [0, 40, 149]),
    (1, 8, 4, 64, 900, 900, "bf16", 200, 40, [10, 41, 300, 640, 895]),
    (1, 16, 2, 64, 4100, 4100, "bf16", 0, 0, [1000, 4000]),
    (2, 1, 7, 64, 3, 3000, "bf16", 0, 0, [2998, 2999]),
    (1, 2, 2, 64, 150, 150, "f32", 0, 0, [0, 40, 149]),
    (1, 4, 2, 64, 1500, 1500, "f32", 200, 5, [2, 7, 700, 1490]),
    (2, 4, 4, 128, 300, 300, "f32", 0, 0, [31, 32, 200]),
    (1, 1, 2, 64, 4, 4000, "f32", 0, 0, [3997, 3998]),
    (1, 1, 2, 128, 5, 1200, "f32", 200, 3, [2, 4, 996, 999, 1197]),
]


@pytest.mark.parametrize("b,H,G,d,nq,nk,dt,window,sinks,keys", UNSEEN)
def test_keys_that_a_row_does_not_see_may_hold_anything(gpu_lib, b, H, G, d, nq, nk, dt, window, sinks, keys):
    """Rows that see one of these keys are no numbers where its value is none; all others
    are what they are without it."""
    import numpy as np
    import torch

    import serve_testlib as ref
    q, k, v = _tensors(b, H, G, d, nq, nk, dt, seed=nq + nk)
    want, want_lse = _run(gpu_lib, q, k, v, window, sinks)
    sees = np.stack([ref.visible(nk, nk, nk - nq + r, window, sinks)[keys].any() for r in range(nq)])
    clean, hit = (np.nonzero(x)[0].tolist() for x in (~sees, sees))
    for value in (math.nan, math.inf, -math.inf):
        w = v.clone()
        w[:, :, keys, d // 2:] = value
        out, lse = _run(gpu_lib, q, k, w, window, sinks)
        assert out[:, :, clean].equal(want[:, :, clean]) and lse.equal(want_lse)
        assert out[..., :d // 2].equal(want[..., :d // 2])
        assert not torch.isfinite(out[:, :, hit, d // 2:]).any()
        if value > 0:  # one sign: the value itself, where its weight is not rounded to 0
            assert (torch.isnan(out[:, :, hit, d // 2:]) | (out[:, :, hit, d // 2:] == value)).all()
    k2 = k.clone()
    k2[:, :, keys] = math.nan
    out, lse = _run(gpu_lib, q, k2, w, window, sinks)
    assert torch.isnan(out[:, :, hit]).all() and torch.isnan(lse[:, :, hit]).all()
    some = sorted({clean[i] for i in (0, len(clean) // 3, len(clean) // 2, -2, -1)} if len(clean) > 1 else clean)
    _check(q, k, v, out, lse, window, sinks, rows=some)

"""Attention behind a long shared prefix on the GPU, against its float64 definition: the kernels of
its weights that only long prefixes take, and splits whose page entries are looked up more than
once."""
import numpy as np
import pytest

from device_testlib import check_attention
from test_gpu_shared import Shared, _decode, _dt

pytestmark = pytest.mark.gpu


def _run(kv, prefix, lens, H, G, d, page, dt, window=0, sinks=0, missing=(), gone=(), rows_first=False):
    """missing: slots of the prefix whose pages are none; gone: such slots of the first sequence."""
    c = Shared(kv, prefix, lens, H, G, d, page, dt, seed=prefix + H, rows_first=rows_first).cuda()
    for i, s in enumerate(missing):
        c.pages[s // page] = [-1, c.cfg.n_pages, 2**31 - 1][i % 3]
    for s in gone:
        c.table[0, s // page] = -1
    b = len(lens)
    q = c.rand(b, H * G, d).mul_(2).to(_dt(dt)).cuda()
    q[[i for i, n in enumerate(lens) if n < 0]] = float("nan")
    acc0 = c.acc.clone()
    out, lse = _decode(c, q, window, sinks, max_prefix=prefix)
    first = c._rows(c.pages, prefix)
    rows = [None if n < 0 else [np.concatenate(x) for x in zip(first, c._rows(c.table[i], n))] for i, n in enumerate(lens)]
    check_attention(c.k.double(), c.v.double(), q, out, lse, rows, G, window, sinks, c.acc, acc0, columns=b * G)
    # without the weights: the same bits
    o2, l2 = _decode(c, q, window, sinks, acc=False, max_prefix=prefix)
    assert o2.equal(out) and l2.equal(lse)


WEIGHTS = [  # prefix, lens, H, G, window, sinks, missing: 128 slots a work-group from 256 of them over all heads on
    (1100, [3, 0, -1, 20], 32, 2, 0, 0, ()),
    (1100, [3, 0, -1, 20], 32, 2, 700, 5, (1090,)),
    (1001, [i % 23 for i in range(24)], 33, 4, 0, 0, (130, 900)),       # 96 columns
    (1001, [i % 23 for i in range(24)], 33, 4, 400, 300, ()),
    (8001, [5, 9], 5, 7, 0, 0, (4000,)),                                # few heads, a long prefix
    (8001, [5, 900], 5, 7, 3000, 17, (7777,)),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix,lens,H,G,window,sinks,missing", WEIGHTS)
def test_weights(gpu_lib, prefix, lens, H, G, window, sinks, missing, d):
    assert (prefix + 127) // 128 * H >= 256
    _run(gpu_lib, prefix, lens, H, G, d, 16, "bf16", window, sinks, missing)


SPLITS = [  # prefix, sequences, H, G, d, dtype, window, sinks: splits of more slots than one lookup of pages is for
    (4300, 3, 128, 1, 64, "bf16", 0, 0),      # 2150, 2048 a lookup
    (4500, 3, 128, 1, 64, "bf16", 4400, 5),
    (4400, 70, 64, 1, 128, "bf16", 0, 0),     # 1100, 1024 a lookup
    (4700, 35, 64, 2, 64, "bf16", 4500, 30),
    (4400, 5, 64, 1, 64, "f32", 0, 0),        # 1100, 1024
    (4700, 3, 64, 1, 128, "f32", 4500, 30),
]


@pytest.mark.parametrize("prefix,b,H,G,d,dt,window,sinks", SPLITS)
def test_splits_beyond_a_lookup(gpu_lib, prefix, b, H, G, d, dt, window, sinks):
    """Pages that are none lie in and behind what the first lookup of a split is for."""
    _run(gpu_lib, prefix, [i % 5 for i in range(b)], H, G, d, 16, dt, window, sinks, missing=(600, 1090, 2120, prefix - 20), rows_first=True)


def test_the_longest_rounds_of_weights(gpu_lib):
    """float32: more than 2^18 slots, so that a work-group of the weights takes more than one round."""
    _run(gpu_lib, 2**18 + 300, [4, 0], 1, 2, 64, 1024, "f32", missing=(100000,))


@pytest.mark.parametrize("dt,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_own_slots_beyond_a_lookup(gpu_lib, dt, d):
    """One sequence of 5000 own slots among 127 short ones of 8 heads: it is not split, and a wave
    has more than the 64 groups of one lookup."""
    _run(gpu_lib, 70, [5000] + [i % 3 for i in range(127)], 8, 1, d, 16, dt, gone=(700, 4100, 4990))

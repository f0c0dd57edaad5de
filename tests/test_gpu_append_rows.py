"""kvec_paged_append with two tokens a work-group: every query, key and value row."""
import numpy as np
import pytest

import serve_testlib as ref
from test_gpu_paged import Cache, _dt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,H,G,d,page,dt,rot,norm", [
    # an odd number of tokens leaves the last work-group one, an even one two
    (1539, 2, 1, 128, 256, "f32", 128, False), (1538, 2, 2, 64, 16, "bf16", 32, True), (1537, 1, 3, 128, 48, "bf16", 128, True)])
def test_every_row(gpu_lib, n, H, G, d, page, dt, rot, norm):
    import torch
    c = Cache(gpu_lib, [n], H, G, d, page, dt, seed=n).cuda()
    q, k, v = (c.rand(n, h, d).mul_(2).to(_dt(dt)).cuda() for h in (H * G, H, H))
    wq, wk = ((1 + 0.2 * c.rand(d)).to(_dt(dt)).cuda() if norm else None for _ in range(2))
    fr = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    positions = torch.randint(0, 100000, (n,), generator=c.gen, dtype=torch.int32).cuda()
    p, r = c.slots(0, n)
    q_out = torch.full_like(q, float("nan"))
    gpu_lib.kvec_paged_append(c.cfg, q, k, v, positions, torch.from_numpy(p.astype(np.int64) * page + r).cuda(), q_out, c.k, c.v, q_weight=wq,
                              k_weight=wk, eps=1e-5, inv_freq=fr, acc=c.acc, pos=c.pos)
    at, fn, u = positions.tolist(), ref.f64(fr), ref.half_step(_dt(dt))
    for x, w, got in ((q, wq, ref.f64(q_out)), (k, wk, ref.f64(c.k)[p, :, r])):
        x, w = ref.f64(x), None if w is None else ref.f64(w)
        for t in range(n):
            for j in range(x.shape[1]):
                y, off = ref.rotated(x[t, j], w, 1e-5, at[t], fn)
                assert np.all(np.abs(got[t, j] - y) <= off * (1 + u) + u * np.abs(y)), (t, j)
    assert np.array_equal(ref.f64(c.v)[p, :, r], ref.f64(v))
    assert np.all(ref.f64(c.acc)[p, :, r] == 0) and np.array_equal(ref.f64(c.pos)[p, :, r], np.repeat(ref.f64(positions)[:, None], H, 1))

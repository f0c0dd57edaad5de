"""The float64 definition of one token's attention, on the device: for caches whose sizes the
definitions in serve_testlib would take too long over.  The bounds are the same."""
import math

from serve_testlib import EXP, U24


def check_attention(k, v, q, out, lse, rows, G, window=0, sinks=0, acc=None, acc0=None, columns=1, more=0, terms=2.0 ** -24):
    """Pools k, v [pages][H][row][d] as float64 (anything in slots that no sequence sees), q
    [b][H G][d]; rows: of every sequence the (page, row) of its slots as numpy arrays, page -1
    where there is none, or None for a row that is no sequence.  more: roundings of a logit beyond
    those of a dot product; columns: sequences times G that add to one slot's weight."""
    import torch
    H, d = k.shape[1], k.shape[-1]
    want_acc, slack = (None, None) if acc is None else (acc0.double().clone(), torch.zeros_like(acc0, dtype=torch.float64))
    for i, where in enumerate(rows):
        o, l = out[i].double().view(H, G, d), lse[i].double().view(H, G)
        if where is not None:
            page, row = (torch.from_numpy(x).long().cuda() for x in where)
            n = len(page)
            slot = torch.arange(n, device="cuda")
            seen = page >= 0
            if window:
                seen &= (slot >= n - window) | (slot < sinks)
        if where is None or not seen.any():
            assert torch.all(o == 0) and torch.all(l == -math.inf), i
            continue
        page, row = page[seen], row[seen]
        kk, vv = (x[page, :, row].transpose(0, 1).contiguous() for x in (k, v))  # [H][n][d]
        qq, kt = q[i].double().view(H, G, d), kk.transpose(1, 2).contiguous()
        x = torch.bmm(qq, kt) / math.sqrt(d)
        dx = (d + 2 + more) * U24 * torch.bmm(qq.abs(), kt.abs_()).amax(-1) / math.sqrt(d)
        want_l = torch.logsumexp(x, -1)
        w = torch.exp(x - want_l[..., None])
        tol = (2 * dx + EXP + terms) * vv.abs().amax((1, 2)).clamp(min=1e-30)[:, None]
        off = (o - torch.bmm(w, vv)).abs().amax(-1)
        assert torch.all(off <= tol), (i, (off / tol).max())
        assert torch.all((l - want_l).abs() <= dx + EXP * (1 + want_l.abs())), i
        if acc is not None:
            want_acc[page, :, row] += w.sum(1).T / G
            slack[page, :, row] += (w * (2 * dx + EXP + (columns + 2) * U24)[..., None]).sum(1).T / G
    if acc is not None:
        a = acc.double()
        ok = ~want_acc.isnan()
        assert torch.equal(a.isnan(), ~ok)
        off = (a - want_acc).abs()
        assert torch.all((off <= slack + want_acc.abs() * 2 * U24)[ok]), off[ok].max()

"""Host-only checks of the largest batches and lengths that the attention behind a shared
prefix takes."""
import ctypes

import pytest

from paper_2606_29563_amd import kvec
from test_serve_abi import FAKE, UNS, WS, _i64, _status

LONG = 1 << 20


def _cfg(batch, H, G=1):
    return kvec.PagedConfig(batch, H, H * G, 64, 16, 1 << 20, LONG // 16)


@pytest.mark.parametrize("batch,H,G,most", [(32, 1024, 1, (1 << 19) - 1024), (32768, 1, 16, (1 << 19) - 1024), (16, 1024, 3, LONG - 1024),
                                            (16, 1023, 16, LONG)])
def test_joins_of_weights_stay_below_2_32_threads(batch, H, G, most):
    """The join has 256 threads for every 1024 own slots of a (sequence, KV head).  Shapes where
    these would be 2^32 are refused by both calls, before anything is launched; without weights
    the same shapes pass."""
    c = _cfg(batch, H, G)
    order = dict(cfg=c.ref, q=FAKE, qs=_i64(H * G * 64, 64), kp=FAKE, vp=FAKE, ps=_i64(H * 16 * 64, 16 * 64, 64), pages=FAKE, n_pages=4, plen=FAKE,
                 max_prefix=64, table=FAKE, lens=FAKE, max_len=most, window=0, sinks=0, out=FAKE, lse=None, acc=FAKE, ws=FAKE, n=16, st=None)
    call = kvec.load().kvec_paged_decode_shared
    assert kvec.kvec_paged_decode_shared_workspace_size(c, 64, most, True) > 0
    assert _status(call, order, {}) == WS
    if most < LONG:
        with pytest.raises(kvec.KvecError) as e:
            kvec.kvec_paged_decode_shared_workspace_size(c, 64, most + 1, True)
        assert e.value.status == UNS
        assert _status(call, order, dict(max_len=most + 1, n=1 << 60)) == UNS
        assert kvec.kvec_paged_decode_shared_workspace_size(c, 64, most + 1, False) > 0
        assert _status(call, order, dict(max_len=most + 1, acc=None)) == WS

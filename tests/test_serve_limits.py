"""Host-only checks of the largest shapes and strides that the serving calls take."""
import ctypes

import pytest

from paper_2606_29563_amd import kvec

INV, UNS, OK = kvec.KVEC_ERR_INVALID, kvec.KVEC_ERR_UNSUPPORTED, kvec.KVEC_OK


def _heads(batch, H):
    """The three size calls of one new token per sequence."""
    c = kvec.PagedConfig(batch=batch, n_kv_heads=H, n_q_heads=H, head_dim=64, page_size=16, n_pages=1, max_pages=1)
    return [lambda: kvec.kvec_prefill_workspace_size(kvec.AttentionConfig(batch, H, H, 64, 1, 16)),
            lambda: kvec.kvec_paged_decode_workspace_size(c, 16, True), lambda: kvec.kvec_paged_evict_workspace_size(c, 16, 8)]


def test_launches_stay_below_2_32_threads():
    """The widest launch has 1024 threads for every KV head of every sequence: fewer than
    2^22 of them are taken."""
    for call in _heads(4096, 1024):
        with pytest.raises(kvec.KvecError) as e:
            call()
        assert e.value.status == UNS
    for call in _heads(4095, 1024):
        call()


def test_a_prompts_launch_stays_below_2_32_threads():
    """4.1 million heads of 129 rows over many keys: three work-groups of 512 threads each."""
    many = kvec.AttentionConfig(batch=4064, n_kv_heads=1024, n_q_heads=1024, head_dim=64, q_len=129, kv_len=8192)
    with pytest.raises(kvec.KvecError) as e:
        kvec.kvec_prefill_workspace_size(many)
    assert e.value.status == UNS
    fewer = kvec.AttentionConfig(batch=2032, n_kv_heads=1024, n_q_heads=1024, head_dim=64, q_len=129, kv_len=8192)
    kvec.kvec_prefill_workspace_size(fewer)


FAKE = ctypes.c_void_p(1 << 20)  # aligned, never dereferenced


def _i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def test_strides_whose_offsets_pass_64_bits_are_refused():
    """Extent and stride of a dimension together reach 2^60 bytes: no tensor is that large,
    and an offset computed from it would wrap.  A dimension of one element may have any."""
    lib = kvec.load()
    far = (1 << 40) - 8
    paged = kvec.PagedConfig(2, 8, 32, 128, 64, 1 << 30, 16)
    token, pool = _i64(48 * 128, 128), _i64(8 * 64 * 128, 64 * 128, 128)
    append = dict(cfg=paged.ref, n=1 << 24, q=FAKE, qs=token, k=FAKE, ks=token, v=FAKE, vs=token, wq=None, wk=None, eps=1e-6, pos_in=FAKE, fr=FAKE,
                  rot=128, slots=FAKE, out=FAKE, os=token, kp=FAKE, vp=FAKE, ps=pool, acc=None, pos=None, st=None)
    for over in (dict(qs=_i64(far, 128)), dict(ks=_i64(far, 128)), dict(vs=_i64(far, 128)), dict(os=_i64(far, 128)), dict(ps=_i64(far, 64 * 128, 128))):
        assert lib.kvec_paged_append(*{**append, **over}.values()) == INV, over
    size = 1 << 40  # of a workspace
    decode = dict(cfg=paged.ref, q=FAKE, qs=token, kp=FAKE, vp=FAKE, ps=_i64(far, 64 * 128, 128), table=FAKE, lens=FAKE, max_len=1000, window=0,
                  sinks=0, out=FAKE, lse=None, acc=None, ws=FAKE, n=size, st=None)
    assert lib.kvec_paged_decode(*decode.values()) == INV
    evict = dict(cfg=paged.ref, budget=512, window=32, sinks=4, kp=FAKE, vp=FAKE, ps=_i64(far, 64 * 128, 128), table=FAKE, lens=FAKE, seen=FAKE,
                 max_len=1000, acc=FAKE, pos=FAKE, kept=None, lens_out=FAKE, ws=FAKE, n=size, st=None)
    assert lib.kvec_paged_evict(*evict.values()) == INV
    attn = kvec.AttentionConfig(2, 8, 32, 128, 1 << 20, 64)
    q, k = _i64(32 * 64 * 128, 64 * 128, 128), _i64(8 * 64 * 128, 64 * 128, 128)
    prompt = dict(cfg=attn.ref, q=FAKE, qs=q, k=FAKE, ks=k, v=FAKE, vs=k, ql=None, kl=None, out=FAKE, os=q, lse=FAKE, ls=_i64(32 << 20, 1 << 20),
                  ws=FAKE, n=size, st=None)
    for over in (dict(qs=_i64(8, 128, far)), dict(os=_i64(8, 128, far)), dict(ls=_i64(1 << 62, 1)), dict(ls=_i64(1, 1 << 60))):
        assert lib.kvec_prefill_attention(*{**prompt, **over}.values()) == INV, over
    # one element: its stride is never used; refused here for the workspace, behind the check of the strides
    few = kvec.AttentionConfig(1, 1, 4, 128, 1, 8192)
    one = {**prompt, "cfg": few.ref, "qs": _i64(far, 128, far), "os": _i64(far, 128, far), "ls": _i64(1 << 62, 1), "ks": _i64(far, far, 128),
           "vs": _i64(far, far, 128), "n": 0}
    assert lib.kvec_prefill_attention(*one.values()) == kvec.KVEC_ERR_WORKSPACE

"""Host-only checks of the serving entry points: every refusal comes back before the
device is touched (there is none here)."""
import ctypes

import pytest

from paper_2606_29563_amd import kvec

FAKE = ctypes.c_void_p(1 << 20)  # aligned, never dereferenced
OFF2, OFF4 = ctypes.c_void_p((1 << 20) + 2), ctypes.c_void_p((1 << 20) + 4)
INV, UNS, WS = kvec.KVEC_ERR_INVALID, kvec.KVEC_ERR_UNSUPPORTED, kvec.KVEC_ERR_WORKSPACE


def _i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _paged(**kw):
    return kvec.PagedConfig(**{**dict(batch=2, n_kv_heads=8, n_q_heads=32, head_dim=128, page_size=64, n_pages=40, max_pages=16), **kw})


def _attn(**kw):
    return kvec.AttentionConfig(**{**dict(batch=2, n_kv_heads=8, n_q_heads=32, head_dim=128, q_len=64, kv_len=8192), **kw})


HEADS = [(dict(batch=0), INV), (dict(n_kv_heads=0), INV), (dict(n_q_heads=33), INV), (dict(head_dim=0), INV), (dict(dtype=2), INV),
         (dict(batch=65536), UNS), (dict(n_kv_heads=2, n_q_heads=34), UNS), (dict(n_kv_heads=2048, n_q_heads=2048), UNS),
         (dict(head_dim=96), UNS), (dict(batch=4097, n_kv_heads=1024, n_q_heads=1024), UNS)]


@pytest.mark.parametrize("over,code", HEADS + [
    (dict(q_len=0), INV), (dict(kv_len=0), INV), (dict(window=-1), INV), (dict(n_sinks=-1), INV),
    (dict(q_len=(1 << 20) + 1), UNS), (dict(kv_len=(1 << 20) + 1), UNS), (dict(batch=64, n_q_heads=128, q_len=1 << 16), UNS)])
def test_attention_config(over, code):
    with pytest.raises(kvec.KvecError) as e:
        kvec.kvec_prefill_workspace_size(_attn(**over))
    assert e.value.status == code


@pytest.mark.parametrize("over,code", HEADS + [
    (dict(page_size=0), INV), (dict(n_pages=0), INV), (dict(max_pages=0), INV), (dict(page_size=24), UNS),
    (dict(max_pages=1 << 15), UNS)])
def test_paged_config(over, code):
    for call in (lambda c: kvec.kvec_paged_decode_workspace_size(c, 64), lambda c: kvec.kvec_paged_evict_workspace_size(c, 64, 32)):
        with pytest.raises(kvec.KvecError) as e:
            call(_paged(**over))
        assert e.value.status == code


def test_null_arguments_of_the_size_calls():
    lib, out = kvec.load(), ctypes.c_size_t(0)
    a, c = _attn().c(), _paged().c()
    assert lib.kvec_prefill_workspace_size(None, ctypes.byref(out)) == INV
    assert lib.kvec_prefill_workspace_size(ctypes.byref(a), None) == INV
    assert lib.kvec_paged_decode_workspace_size(None, 64, 0, ctypes.byref(out)) == INV
    assert lib.kvec_paged_decode_workspace_size(ctypes.byref(c), 64, 0, None) == INV
    assert lib.kvec_paged_evict_workspace_size(ctypes.byref(c), 64, 32, None) == INV
    for n in (0, -1, 64 * 16 + 1):
        assert lib.kvec_paged_decode_workspace_size(ctypes.byref(c), n, 0, ctypes.byref(out)) == INV
        assert lib.kvec_paged_evict_workspace_size(ctypes.byref(c), n, 32, ctypes.byref(out)) == INV
    assert lib.kvec_paged_evict_workspace_size(ctypes.byref(c), 64, 0, ctypes.byref(out)) == INV
    assert lib.kvec_paged_evict_workspace_size(ctypes.byref(c), 64, (1 << 20) + 1, ctypes.byref(out)) == UNS


def _status(lib_call, order, over):
    args = {**order, **over}
    return lib_call(*args.values())


def test_prefill_refusals():
    lib, c = kvec.load(), _attn().c()
    q, k = _i64(32 * 64 * 128, 64 * 128, 128), _i64(8 * 8192 * 128, 8192 * 128, 128)
    order = dict(cfg=ctypes.byref(c), q=FAKE, qs=q, k=FAKE, ks=k, v=FAKE, vs=k, ql=None, kl=None, out=FAKE, os=q, lse=None, ls=None, ws=FAKE,
                 n=1 << 40, st=None)
    far = _i64(0, 0, 1 << 18)
    for over, code in [(dict(cfg=None), INV), (dict(q=None), INV), (dict(k=OFF2), INV), (dict(v=None), INV), (dict(out=OFF4), INV),
                       (dict(qs=None), INV), (dict(ks=_i64(8, 8, 127)), INV), (dict(vs=_i64(-8, 8, 128)), INV), (dict(os=None), INV),
                       (dict(qs=_i64(1 << 40, 8, 128)), INV), (dict(ql=OFF2), INV), (dict(kl=OFF2), INV), (dict(lse=FAKE), INV),
                       (dict(lse=OFF2, ls=_i64(1, 1)), INV), (dict(lse=FAKE, ls=_i64(-1, 1)), INV), (dict(ks=far), UNS), (dict(vs=far), UNS)]:
        assert _status(lib.kvec_prefill_attention, order, over) == code, over
    # few rows over many keys are split: partial states in a workspace
    assert kvec.kvec_prefill_workspace_size(_attn(q_len=2)) > 0
    few = _attn(q_len=2).c()
    for over, code in [(dict(n=16), WS), (dict(ws=OFF4), INV), (dict(ws=None), INV)]:
        assert _status(lib.kvec_prefill_attention, {**order, "cfg": ctypes.byref(few)}, over) == code, over
    # ... a long prompt is not
    assert kvec.kvec_prefill_workspace_size(_attn(q_len=8192)) == 0


def test_append_refusals():
    lib, c = kvec.load(), _paged().c()
    t, p = _i64(48 * 128, 128), _i64(8 * 64 * 128, 64 * 128, 128)
    order = dict(cfg=ctypes.byref(c), n=5, q=FAKE, qs=t, k=FAKE, ks=t, v=FAKE, vs=t, wq=None, wk=None, eps=1e-6, pos_in=FAKE, fr=FAKE, rot=128,
                 slots=FAKE, out=FAKE, os=t, kp=FAKE, vp=FAKE, ps=p, acc=None, pos=None, st=None)
    for over, code in [(dict(cfg=None), INV), (dict(n=-1), INV), (dict(n=(1 << 24) + 1), UNS), (dict(q=None), INV), (dict(k=OFF2), INV),
                       (dict(v=None), INV), (dict(out=None), INV), (dict(qs=None), INV), (dict(ks=_i64(48 * 128, 4)), INV),
                       (dict(vs=_i64(-8, 8)), INV), (dict(os=None), INV), (dict(wq=OFF4), INV), (dict(wk=OFF4), INV),
                       (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(eps=float("inf")), INV), (dict(pos_in=None), INV),
                       (dict(fr=None), INV), (dict(rot=-16), INV), (dict(rot=144), INV), (dict(rot=40), UNS), (dict(slots=None), INV),
                       (dict(slots=OFF4), INV), (dict(kp=None), INV), (dict(vp=OFF4), INV), (dict(ps=None), INV),
                       (dict(ps=_i64(8 * 64 * 128, 64 * 128, 1 << 25)), UNS), (dict(acc=OFF2), INV), (dict(pos=OFF2), INV)]:
        assert _status(lib.kvec_paged_append, order, over) == code, over
    # no tokens: nothing to do, the token tensors need no address
    assert _status(lib.kvec_paged_append, order, dict(n=0, q=None, k=None, v=None, out=None, pos_in=None, slots=None)) == kvec.KVEC_OK


def test_decode_refusals():
    lib, c = kvec.load(), _paged().c()
    order = dict(cfg=ctypes.byref(c), q=FAKE, qs=_i64(32 * 128, 128), kp=FAKE, vp=FAKE, ps=_i64(8 * 64 * 128, 64 * 128, 128), table=FAKE,
                 lens=FAKE, max_len=1000, window=0, sinks=0, out=FAKE, lse=None, acc=None, ws=FAKE, n=1 << 40, st=None)
    for over, code in [(dict(cfg=None), INV), (dict(q=None), INV), (dict(q=OFF4), INV), (dict(qs=None), INV), (dict(qs=_i64(3, 128)), INV),
                       (dict(kp=None), INV), (dict(vp=OFF4), INV), (dict(ps=None), INV), (dict(table=None), INV), (dict(table=OFF2), INV),
                       (dict(lens=None), INV), (dict(max_len=0), INV), (dict(max_len=1025), INV), (dict(window=-1), INV),
                       (dict(sinks=-1), INV), (dict(out=None), INV), (dict(out=OFF2), INV), (dict(lse=OFF2), INV), (dict(acc=OFF2), INV),
                       (dict(ws=None), INV), (dict(ws=OFF4), INV), (dict(n=16), WS)]:
        assert _status(lib.kvec_paged_decode, order, over) == code, over
    # the accumulated weights need their logits in the workspace
    plain, acc = (kvec.kvec_paged_decode_workspace_size(_paged(), 1000, w) for w in (False, True))
    assert 0 < plain < acc
    assert _status(lib.kvec_paged_decode, order, dict(acc=FAKE, n=plain)) == WS


def test_evict_refusals():
    lib, c = kvec.load(), _paged().c()
    order = dict(cfg=ctypes.byref(c), budget=512, window=32, sinks=4, kp=FAKE, vp=FAKE, ps=_i64(8 * 64 * 128, 64 * 128, 128), table=FAKE,
                 lens=FAKE, seen=FAKE, max_len=1000, acc=FAKE, pos=FAKE, kept=None, lens_out=FAKE, ws=FAKE, n=1 << 40, st=None)
    for over, code in [(dict(cfg=None), INV), (dict(budget=0), INV), (dict(budget=(1 << 20) + 1), UNS), (dict(window=-1), INV),
                       (dict(sinks=-1), INV), (dict(window=509), INV), (dict(window=2**31 - 1, sinks=2**31 - 1), INV), (dict(kp=None), INV),
                       (dict(vp=OFF4), INV), (dict(ps=None), INV), (dict(table=None), INV), (dict(lens=OFF2), INV), (dict(seen=None), INV),
                       (dict(max_len=0), INV), (dict(max_len=1025), INV), (dict(acc=None), INV), (dict(pos=None), INV),
                       (dict(kept=OFF2), INV), (dict(lens_out=None), INV), (dict(ws=None), INV), (dict(n=16), WS)]:
        assert _status(lib.kvec_paged_evict, order, over) == code, over


def test_binding_checks_tensors():
    """Wrong shapes, types and devices are refused before a pointer leaves Python."""
    import torch
    c = _paged(batch=1, n_pages=2, max_pages=2)
    q, pool = torch.zeros(1, 32, 128, dtype=torch.bfloat16), torch.zeros(2, 8, 64, 128, dtype=torch.bfloat16)
    table, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    out, ws = torch.zeros(1, 32, 128), torch.zeros(1 << 20, dtype=torch.uint8)
    good = dict(q=q, k_pool=pool, v_pool=pool, page_table=table, lens=lens, out=out, ws=ws)
    for bad in (dict(q=q[:, :31]), dict(q=q.float()), dict(k_pool=pool[:1]), dict(v_pool=pool.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(page_table=table.long()), dict(page_table=table[:, :1]), dict(lens=lens.long()), dict(out=out.bfloat16()),
                dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), {}):  # the last: nothing is on a GPU
        with pytest.raises(AssertionError):
            kvec.kvec_paged_decode(c, **{**good, **bad})


@pytest.mark.parametrize("cfg", [_paged(), _attn(window=7)])
def test_configurations_copy(cfg):
    import copy
    import dataclasses
    import pickle
    for other in (copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg)), dataclasses.replace(cfg)):
        assert other == cfg and bytes(other.c()) == bytes(cfg.c())
    assert dataclasses.replace(cfg, batch=7).c().batch == 7
    with pytest.raises(dataclasses.FrozenInstanceError):
        cfg.batch = 3

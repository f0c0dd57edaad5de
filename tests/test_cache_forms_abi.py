"""Host-only checks of the paged cache's further forms, in eight bits and behind a shared
prefix: every refusal comes back before the device is touched (there is none here), and
names its argument."""
import copy
import ctypes
import dataclasses
import pickle

import pytest
import torch

from paper_2606_29563_amd import kvec
from test_serve_abi import FAKE, HEADS, INV, OFF2, OFF4, UNS, WS, _i64, _paged, _status

OK = kvec.KVEC_OK


def _q8(**kw):
    return kvec.PagedQ8Config(**{**dict(batch=2, n_kv_heads=8, n_q_heads=32, head_dim=128, page_size=64, n_pages=40, max_pages=16), **kw})


@pytest.mark.parametrize("over,code", HEADS + [
    (dict(page_size=0), INV), (dict(n_pages=0), INV), (dict(max_pages=0), INV), (dict(page_size=24), UNS),
    (dict(max_pages=1 << 15), UNS), (dict(format=2), INV), (dict(format=-1), INV)])
def test_q8_config(over, code):
    for call in (lambda c: kvec.kvec_paged_decode_q8_workspace_size(c, 64), lambda c: kvec.kvec_paged_evict_q8_workspace_size(c, 64, 32)):
        with pytest.raises(kvec.KvecError) as e:
            call(_q8(**over))
        assert e.value.status == code


@pytest.mark.parametrize("over,code", HEADS + [
    (dict(page_size=24), UNS), (dict(batch=32768), UNS), (dict(batch=8192, n_q_heads=128), UNS), (dict(batch=1024, n_kv_heads=1024, n_q_heads=1024), UNS)])
def test_shared_config(over, code):
    with pytest.raises(kvec.KvecError) as e:
        kvec.kvec_paged_decode_shared_workspace_size(_paged(**over), 500, 64)
    assert e.value.status == code
    # just below the largest number of columns
    kvec.kvec_paged_decode_shared_workspace_size(_paged(batch=32767), 500, 64)


def test_arguments_of_the_size_calls():
    lib, out = kvec.load(), ctypes.c_size_t(0)
    c, p = _q8().c(), _paged().c()
    ref = ctypes.byref
    assert lib.kvec_paged_decode_q8_workspace_size(None, 64, 0, ref(out)) == INV
    assert lib.kvec_paged_decode_q8_workspace_size(ref(c), 64, 0, None) == INV
    assert lib.kvec_paged_evict_q8_workspace_size(None, 64, 32, ref(out)) == INV
    assert lib.kvec_paged_evict_q8_workspace_size(ref(c), 64, 32, None) == INV
    assert lib.kvec_paged_decode_shared_workspace_size(None, 64, 64, 0, ref(out)) == INV
    assert lib.kvec_paged_decode_shared_workspace_size(ref(p), 64, 64, 0, None) == INV
    for n in (0, -1, 64 * 16 + 1):
        assert lib.kvec_paged_decode_q8_workspace_size(ref(c), n, 0, ref(out)) == INV
        assert lib.kvec_paged_evict_q8_workspace_size(ref(c), n, 32, ref(out)) == INV
        assert lib.kvec_paged_decode_shared_workspace_size(ref(p), 64, n, 0, ref(out)) == INV
    assert lib.kvec_paged_evict_q8_workspace_size(ref(c), 64, 0, ref(out)) == INV
    assert lib.kvec_paged_evict_q8_workspace_size(ref(c), 64, (1 << 20) + 1, ref(out)) == UNS
    assert lib.kvec_paged_decode_shared_workspace_size(ref(p), 0, 64, 0, ref(out)) == INV
    assert lib.kvec_paged_decode_shared_workspace_size(ref(p), (1 << 20) + 1, 64, 0, ref(out)) == UNS
    assert lib.kvec_paged_decode_shared_workspace_size(ref(p), 1 << 20, 64, 1, ref(out)) == OK


POOL = _i64(8 * 64 * 128, 64 * 128, 128)
POOLS = [(dict(kp=None), INV), (dict(vp=OFF4), INV), (dict(ps=None), INV), (dict(ps=_i64(8 * 64 * 128, 64 * 128, 132)), INV),
         (dict(ps=_i64(-128, 64 * 128, 128)), INV)]
SCALES = [(dict(ks=None), INV), (dict(vs=None), INV), (dict(ks=OFF2), INV), (dict(vs=OFF2), INV), (dict(ps=_i64(8 * 64 * 128, 64 * 128, 1 << 26)), UNS)]


def test_append_refusals():
    lib, c = kvec.load(), _q8().c()
    t = _i64(48 * 128, 128)
    order = dict(cfg=ctypes.byref(c), n=5, q=FAKE, qs=t, k=FAKE, kt=t, v=FAKE, vt=t, wq=None, wk=None, eps=1e-6, pos_in=FAKE, fr=FAKE, rot=128,
                 slots=FAKE, out=FAKE, os=t, kp=FAKE, vp=FAKE, ps=POOL, ks=FAKE, vs=FAKE, acc=None, pos=None, st=None)
    for over, code in POOLS + SCALES + [
            (dict(cfg=None), INV), (dict(n=-1), INV), (dict(n=(1 << 24) + 1), UNS), (dict(q=None), INV), (dict(k=OFF2), INV), (dict(v=None), INV),
            (dict(out=None), INV), (dict(qs=None), INV), (dict(kt=_i64(48 * 128, 4)), INV), (dict(vt=_i64(-8, 8)), INV), (dict(os=None), INV),
            (dict(wq=OFF4), INV), (dict(wk=OFF4), INV), (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(pos_in=None), INV),
            (dict(fr=None), INV), (dict(rot=-16), INV), (dict(rot=144), INV), (dict(rot=40), UNS), (dict(slots=None), INV), (dict(slots=OFF4), INV),
            (dict(acc=OFF2), INV), (dict(pos=OFF2), INV)]:
        assert _status(lib.kvec_paged_append_q8, order, over) == code, over
    assert _status(lib.kvec_paged_append_q8, order, dict(n=0, q=None, k=None, v=None, out=None, pos_in=None, slots=None)) == OK


def test_read_refusals():
    lib, c = kvec.load(), _q8().c()
    o = _i64(8 * 1000 * 128, 1000 * 128, 128)
    order = dict(cfg=ctypes.byref(c), kp=FAKE, vp=FAKE, ps=POOL, ks=FAKE, vs=FAKE, table=FAKE, lens=FAKE, max_len=1000, k=FAKE, kt=o, v=FAKE, vt=o, st=None)
    for over, code in POOLS + SCALES + [
            (dict(cfg=None), INV), (dict(table=None), INV), (dict(table=OFF2), INV), (dict(lens=None), INV), (dict(max_len=0), INV),
            (dict(max_len=1025), INV), (dict(k=None), INV), (dict(v=OFF4), INV), (dict(kt=None), INV), (dict(vt=_i64(8, 8, 4)), INV),
            (dict(kt=_i64(8, -8, 128)), INV), (dict(vt=_i64(8, 8, 1 << 50)), INV)]:
        assert _status(lib.kvec_paged_read_q8, order, over) == code, over


def test_decode_refusals():
    lib, c = kvec.load(), _q8().c()
    order = dict(cfg=ctypes.byref(c), q=FAKE, qs=_i64(32 * 128, 128), kp=FAKE, vp=FAKE, ps=POOL, ks=FAKE, vs=FAKE, table=FAKE, lens=FAKE, max_len=1000,
                 window=0, sinks=0, out=FAKE, lse=None, acc=None, ws=FAKE, n=1 << 40, st=None)
    for over, code in POOLS + SCALES + [
            (dict(cfg=None), INV), (dict(q=None), INV), (dict(q=OFF4), INV), (dict(qs=None), INV), (dict(qs=_i64(3, 128)), INV), (dict(table=None), INV),
            (dict(lens=None), INV), (dict(max_len=0), INV), (dict(max_len=1025), INV), (dict(window=-1), INV), (dict(sinks=-1), INV),
            (dict(out=None), INV), (dict(out=OFF2), INV), (dict(lse=OFF2), INV), (dict(acc=OFF2), INV), (dict(ws=None), INV), (dict(ws=OFF4), INV),
            (dict(n=16), WS)]:
        assert _status(lib.kvec_paged_decode_q8, order, over) == code, over
    plain, acc = (kvec.kvec_paged_decode_q8_workspace_size(_q8(), 1000, w) for w in (False, True))
    assert 0 < plain < acc
    assert _status(lib.kvec_paged_decode_q8, order, dict(acc=FAKE, n=plain)) == WS


def test_evict_refusals():
    lib, c = kvec.load(), _q8().c()
    order = dict(cfg=ctypes.byref(c), budget=512, window=32, sinks=4, kp=FAKE, vp=FAKE, ps=POOL, ks=FAKE, vs=FAKE, table=FAKE, lens=FAKE, seen=FAKE,
                 max_len=1000, acc=FAKE, pos=FAKE, kept=None, lens_out=FAKE, ws=FAKE, n=1 << 40, st=None)
    for over, code in POOLS + SCALES + [
            (dict(cfg=None), INV), (dict(budget=0), INV), (dict(budget=(1 << 20) + 1), UNS), (dict(window=-1), INV), (dict(sinks=-1), INV),
            (dict(window=509), INV), (dict(table=None), INV), (dict(lens=OFF2), INV), (dict(seen=None), INV), (dict(max_len=0), INV),
            (dict(max_len=1025), INV), (dict(acc=None), INV), (dict(pos=None), INV), (dict(kept=OFF2), INV), (dict(lens_out=None), INV),
            (dict(ws=None), INV), (dict(n=16), WS)]:
        assert _status(lib.kvec_paged_evict_q8, order, over) == code, over


def test_shared_refusals():
    lib, c = kvec.load(), _paged().c()
    order = dict(cfg=ctypes.byref(c), q=FAKE, qs=_i64(32 * 128, 128), kp=FAKE, vp=FAKE, ps=POOL, pages=FAKE, n_pages=20, plen=FAKE, max_prefix=1200,
                 table=FAKE, lens=FAKE, max_len=1000, window=0, sinks=0, out=FAKE, lse=None, acc=None, ws=FAKE, n=1 << 40, st=None)
    for over, code in POOLS + [
            (dict(cfg=None), INV), (dict(q=None), INV), (dict(q=OFF4), INV), (dict(qs=None), INV), (dict(qs=_i64(3, 128)), INV), (dict(pages=None), INV),
            (dict(pages=OFF2), INV), (dict(n_pages=0), INV), (dict(n_pages=-1), INV), (dict(plen=None), INV), (dict(plen=OFF2), INV),
            (dict(max_prefix=0), INV), (dict(max_prefix=1281), INV), (dict(n_pages=(1 << 14) + 1), UNS), (dict(table=None), INV), (dict(lens=None), INV),
            (dict(max_len=0), INV), (dict(max_len=1025), INV), (dict(window=-1), INV), (dict(sinks=-1), INV), (dict(out=None), INV),
            (dict(out=OFF2), INV), (dict(lse=OFF2), INV), (dict(acc=OFF2), INV), (dict(ws=None), INV), (dict(ws=OFF4), INV), (dict(n=16), WS)]:
        assert _status(lib.kvec_paged_decode_shared, order, over) == code, over
    plain, acc = (kvec.kvec_paged_decode_shared_workspace_size(_paged(), 1200, 1000, w) for w in (False, True))
    assert 0 < plain < acc
    assert _status(lib.kvec_paged_decode_shared, order, dict(acc=FAKE, n=plain)) == WS


@pytest.mark.parametrize("fmt", [kvec.KVEC_Q8_INT8, kvec.KVEC_Q8_E4M3])
def test_configurations_copy(fmt):
    cfg = _q8(format=fmt)
    for other in (copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg)), dataclasses.replace(cfg)):
        assert other == cfg and bytes(other.c()) == bytes(cfg.c())
    assert dataclasses.replace(cfg, batch=7).c().paged.batch == 7 and cfg.c().format == fmt
    with pytest.raises(dataclasses.FrozenInstanceError):
        cfg.batch = 3


# --- which argument a refusal of the binding is about ---

B, H, HQ, D, PAGE = 2, 2, 8, 64, 16
PLAIN, EIGHT = kvec.PagedConfig(B, H, HQ, D, PAGE, 6, 3), kvec.PagedQ8Config(B, H, HQ, D, PAGE, 6, 3, format=kvec.KVEC_Q8_E4M3)
I32, F32 = torch.int32, torch.float32


def _z(*shape, t=torch.bfloat16):
    return torch.zeros(shape, dtype=t)


CODES = dict(k_pool=_z(6, H, PAGE, D, t=torch.float8_e4m3fn), v_pool=_z(6, H, PAGE, D, t=torch.float8_e4m3fn), k_scale=_z(6, H, PAGE, t=F32),
             v_scale=_z(6, H, PAGE, t=F32))
SEQ = dict(page_table=_z(B, 3, t=I32), lens=_z(B, t=I32))
META = dict(acc=_z(6, H, PAGE, t=F32), pos=_z(6, H, PAGE, t=I32))
CALLS = {
    "append_q8": (lambda **k: kvec.kvec_paged_append_q8(EIGHT, **k),
                  dict(q=_z(3, HQ, D), k=_z(3, H, D), v=_z(3, H, D), positions=_z(3, t=I32), slots=_z(3, t=torch.int64), q_out=_z(3, HQ, D), **CODES,
                       q_weight=_z(D), k_weight=_z(D), inv_freq=_z(D // 2, t=torch.float64), **META),
                  {"q_weight", "k_weight", "inv_freq", "acc", "pos"}),
    "read_q8": (lambda **k: kvec.kvec_paged_read_q8(EIGHT, **k), dict(**CODES, **SEQ, k_out=_z(B, H, 40, D), v_out=_z(B, H, 40, D)), set()),
    "decode_q8": (lambda **k: kvec.kvec_paged_decode_q8(EIGHT, ws=None, **k),
                  dict(q=_z(B, HQ, D), **CODES, **SEQ, out=_z(B, HQ, D, t=F32), lse=_z(B, HQ, t=F32), acc=META["acc"]), {"lse", "acc"}),
    "evict_q8": (lambda **k: kvec.kvec_paged_evict_q8(EIGHT, 4, ws=None, **k),
                 dict(**CODES, **SEQ, n_seen=_z(B, t=I32), **META, lens_out=_z(B, t=I32), kept=_z(B, H, 4, t=I32)), {"kept"}),
    "decode_shared": (lambda **k: kvec.kvec_paged_decode_shared(PLAIN, ws=None, **k),
                      dict(q=_z(B, HQ, D), k_pool=_z(6, H, PAGE, D), v_pool=_z(6, H, PAGE, D), prefix_pages=_z(2, t=I32), prefix_len=_z(1, t=I32), **SEQ,
                           out=_z(B, HQ, D, t=F32), lse=_z(B, HQ, t=F32), acc=META["acc"]), {"lse", "acc"}),
}
FIRST = {"append_q8": "k_pool", "read_q8": "k_pool", "decode_q8": "q", "evict_q8": "k_pool", "decode_shared": "q"}


@pytest.mark.parametrize("call,arg", [(c, a) for c, (_, args, _) in CALLS.items() for a in args])
def test_misfits_are_named(call, arg):
    f, args, optional = CALLS[call]
    t = args[arg]
    bad = {"type": t.to(torch.float16), "contiguous": torch.cat([t.view(torch.uint8)] * 2, -1)[..., ::2].view(t.dtype) if t.element_size() == 1
           else torch.cat([t, t], -1)[..., ::2]}
    if arg not in ("inv_freq", "prefix_pages"):  # their lengths are sizes of their own
        bad["shape"] = t[..., :-1].contiguous()
    if t.shape[-1] == 1:  # one element is contiguous whatever its stride
        del bad["contiguous"]
    for kind, x in bad.items():
        want = {"type": str(t.dtype), "contiguous": "contiguous", "shape": r"\("}[kind]
        with pytest.raises(AssertionError, match=f"^kvec_\\w+: {arg} must be {want}"):
            f(**{**args, arg: x})
    first = FIRST[call]
    if arg in optional:  # without it only the device is wrong
        with pytest.raises(AssertionError, match=f": {first} must be on the GPU"):
            f(**{**args, arg: None})
    elif arg != first:
        with pytest.raises(AssertionError, match=f": {arg} must be given"):
            f(**{**args, arg: None})


@pytest.mark.parametrize("call", CALLS)
def test_a_configuration_of_another_kind_is_refused(call):
    kind = PLAIN if call == "decode_shared" else EIGHT
    f, args, _ = CALLS[call]
    more = {} if call in ("append_q8", "read_q8") else dict(ws=None)
    for other in (EIGHT if kind is PLAIN else PLAIN, kind.c(), None):
        with pytest.raises(AssertionError, match=f"^kvec_paged_{call}: cfg must be"):
            getattr(kvec, f"kvec_paged_{call}")(other, *([4] if call == "evict_q8" else []), **args, **more)


def test_codes_of_the_other_format_are_refused():
    f, args, _ = CALLS["decode_q8"]
    with pytest.raises(AssertionError, match="k_pool must be torch.float8_e4m3fn, not torch.int8"):
        f(**{**args, "k_pool": args["k_pool"].view(torch.int8), "v_pool": args["v_pool"].view(torch.int8)})

"""The serving calls' compiled marshalling module, with tensors on the GPU."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu


def _calls(kv):
    """(name, call, its arguments) of the four serving calls."""
    import torch
    b, H, HQ, d, page = 2, 2, 8, 64, 16
    cfg, attn = kv.PagedConfig(b, H, HQ, d, page, 6, 3), kv.AttentionConfig(b, H, HQ, d, 7, 40)
    i32, f32 = torch.int32, torch.float32
    zeros = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    pools = dict(k_pool=zeros(6, H, page, d), v_pool=zeros(6, H, page, d))
    seq = dict(page_table=torch.arange(6, dtype=i32, device="cuda").view(b, 3), lens=zeros(b, t=i32) + 5)
    meta = dict(acc=zeros(6, H, page, t=f32), pos=zeros(6, H, page, t=i32))
    ws = zeros(1 << 20, t=torch.uint8)
    return [
        ("append", lambda **k: kv.kvec_paged_append(cfg, **k),
         dict(q=zeros(3, HQ, d), k=zeros(3, H, d), v=zeros(3, H, d), positions=zeros(3, t=i32), slots=torch.arange(3, device="cuda"),
              q_out=zeros(3, HQ, d), **pools, q_weight=zeros(d), k_weight=zeros(d), inv_freq=zeros(d // 2, t=torch.float64), **meta)),
        ("decode", lambda **k: kv.kvec_paged_decode(cfg, **k),
         dict(q=zeros(b, HQ, d), **pools, **seq, out=zeros(b, HQ, d, t=f32), ws=ws, lse=zeros(b, HQ, t=f32), acc=meta["acc"])),
        ("evict", lambda **k: kv.kvec_paged_evict(cfg, 4, **k),
         dict(**pools, **seq, n_seen=zeros(b, t=i32), **meta, lens_out=zeros(b, t=i32), ws=ws, kept=zeros(b, H, 4, t=i32))),
        ("prompt", lambda **k: kv.kvec_prefill_attention(attn, **k),
         dict(q=zeros(b, HQ, 7, d), k=zeros(b, H, 40, d), v=zeros(b, H, 40, d), out=zeros(b, HQ, 7, d), ws=ws, lse=zeros(b, HQ, 7, t=f32),
              q_lens=zeros(b, t=i32), kv_lens=zeros(b, t=i32))),
    ]


def test_other_threads_run_during_a_call(gpu_lib):
    """The interpreter's lock is free while the C interface launches.  Its entry points
    are replaced by PyGILState_Check, which says whether the calling thread holds the
    lock: 1 would come back as an error."""
    kv = gpu_lib
    bind = kv._bound()
    held = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    entries = [ctypes.cast(getattr(kv.load(), n), ctypes.c_void_p).value
               for n in ("kvec_prefill_attention", "kvec_paged_append", "kvec_paged_decode", "kvec_paged_evict")]
    calls = _calls(kv)
    try:
        bind.bind(*[held] * 4)
        for _, call, args in calls:
            call(**args)
    finally:
        bind.bind(*entries)


def test_every_misfit_is_named(gpu_lib):
    """Each tensor argument in turn with a wrong type, a wrong shape or on the CPU: the
    error is about that argument."""
    import torch
    for _, call, args in _calls(gpu_lib):
        call(**args)
        for name, t in args.items():
            if name == "ws":
                with pytest.raises(AssertionError, match="workspace"):
                    call(**{**args, name: t.cpu()})
                continue
            for bad in (t.to(torch.float16), t[..., :-1].contiguous(), t.cpu()):
                if name == "inv_freq" and bad.dtype == t.dtype and bad.is_cuda:
                    continue  # any length is a shape of its own
                with pytest.raises(AssertionError, match=f": {name} must be"):
                    call(**{**args, name: bad})
        for name in ("acc", "pos", "n_seen", "lens", "page_table", "out", "slots"):
            if name in args and not (name in ("acc", "pos") and "n_seen" not in args):  # (elsewhere acc and pos are optional)
                with pytest.raises(AssertionError, match=f": {name} must be"):
                    call(**{**args, name: None})
        if "v_pool" in args:
            other = args["v_pool"].transpose(1, 2).contiguous().transpose(1, 2)
            with pytest.raises(AssertionError, match="same strides"):
                call(**{**args, "v_pool": other})
    torch.cuda.synchronize()


def test_two_threads_at_once(gpu_lib):
    """Calls of two threads, each with a stream and a workspace of its own: the same bits as
    one after the other."""
    import threading

    import torch
    kv = gpu_lib
    g = torch.Generator(device="cuda").manual_seed(3)
    cfg = kv.PagedConfig(2, 2, 8, 64, 16, 300, 140)
    pools = [torch.randn((300, 2, 16, 64), generator=g, device="cuda").bfloat16() for _ in range(2)]
    table = torch.randperm(300, generator=g, device="cuda")[:280].int().view(2, 140).contiguous()
    lens = torch.tensor([2200, 900], dtype=torch.int32, device="cuda")
    qs = [torch.randn((2, 8, 64), generator=g, device="cuda").bfloat16() for _ in range(2)]
    size = kv.kvec_paged_decode_workspace_size(cfg)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    wants = []
    for q, w in zip(qs, ws):
        wants.append(torch.empty((2, 8, 64), device="cuda"))
        kv.kvec_paged_decode(cfg, q, *pools, table, lens, wants[-1], w)
    torch.cuda.synchronize()
    outs = [[torch.empty((2, 8, 64), device="cuda") for _ in range(200)] for _ in range(2)]
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            for o in outs[i]:
                kv.kvec_paged_decode(cfg, qs[i], *pools, table, lens, o, ws[i], stream=stream)
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    assert all(o.equal(w) for i, w in enumerate(wants) for o in outs[i])

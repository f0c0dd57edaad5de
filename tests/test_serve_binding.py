"""Which argument of a serving call a refusal of the binding is about: its type, shape and
strides are looked at before the device is, so this needs no GPU."""
import pytest
import torch

from paper_2606_29563_amd import kvec

B, H, HQ, D, PAGE = 2, 2, 8, 64, 16
PAGED, ATTN = kvec.PagedConfig(B, H, HQ, D, PAGE, 6, 3), kvec.AttentionConfig(B, H, HQ, D, 7, 40)
I32, F32 = torch.int32, torch.float32


def _z(*shape, t=torch.bfloat16):
    return torch.zeros(shape, dtype=t)


POOLS = dict(k_pool=_z(6, H, PAGE, D), v_pool=_z(6, H, PAGE, D))
SEQ = dict(page_table=_z(B, 3, t=I32), lens=_z(B, t=I32))
META = dict(acc=_z(6, H, PAGE, t=F32), pos=_z(6, H, PAGE, t=I32))
CALLS = {
    "append": (lambda **k: kvec.kvec_paged_append(PAGED, **k),
               dict(q=_z(3, HQ, D), k=_z(3, H, D), v=_z(3, H, D), positions=_z(3, t=I32), slots=_z(3, t=torch.int64), q_out=_z(3, HQ, D), **POOLS,
                    q_weight=_z(D), k_weight=_z(D), inv_freq=_z(D // 2, t=torch.float64), **META),
               {"q_weight", "k_weight", "inv_freq", "acc", "pos"}),
    "decode": (lambda **k: kvec.kvec_paged_decode(PAGED, ws=None, **k),
               dict(q=_z(B, HQ, D), **POOLS, **SEQ, out=_z(B, HQ, D, t=F32), lse=_z(B, HQ, t=F32), acc=META["acc"]), {"lse", "acc"}),
    "evict": (lambda **k: kvec.kvec_paged_evict(PAGED, 4, ws=None, **k),
              dict(**POOLS, **SEQ, n_seen=_z(B, t=I32), **META, lens_out=_z(B, t=I32), kept=_z(B, H, 4, t=I32)), {"kept"}),
    "prompt": (lambda **k: kvec.kvec_prefill_attention(ATTN, **k),
               dict(q=_z(B, HQ, 7, D), k=_z(B, H, 40, D), v=_z(B, H, 40, D), out=_z(B, HQ, 7, D), lse=_z(B, HQ, 7, t=F32), q_lens=_z(B, t=I32),
                    kv_lens=_z(B, t=I32)), {"lse", "q_lens", "kv_lens"}),
}


@pytest.mark.parametrize("call,arg", [(c, a) for c, (_, args, _) in CALLS.items() for a in args])
def test_misfits_are_named(call, arg):
    f, args, optional = CALLS[call]
    t = args[arg]
    bad = {"type": t.to(torch.float16), "contiguous": torch.cat([t, t], -1)[..., ::2]}
    if arg != "inv_freq":  # its length is a size of its own
        bad["shape"] = t[..., :-1].contiguous()
    for kind, x in bad.items():
        want = {"type": str(t.dtype), "contiguous": "contiguous", "shape": r"\("}[kind]
        with pytest.raises(AssertionError, match=f"^kvec_\\w+: {arg} must be {want}"):
            f(**{**args, arg: x})
    first = "k_pool" if call in ("append", "evict") else "q"
    if arg in optional:  # without it only the device is wrong
        with pytest.raises(AssertionError, match=f": {first} must be on the GPU"):
            f(**{**args, arg: None})
    elif arg != first:
        with pytest.raises(AssertionError, match=f": {arg} must be given"):
            f(**{**args, arg: None})


@pytest.mark.parametrize("call", CALLS)
def test_a_configuration_of_another_kind_is_refused(call):
    """The compiled module reads the configuration by its address: the kind is checked first."""
    kinds = dict(kvec_paged_append=PAGED, kvec_paged_decode=PAGED, kvec_paged_evict=PAGED, kvec_prefill_attention=ATTN)
    name = "kvec_prefill_attention" if call == "prompt" else f"kvec_paged_{call}"
    _, args, _ = CALLS[call]
    more = {} if call in ("append", "prompt") else dict(ws=None, max_len=40)
    for other in (ATTN if kinds[name] is PAGED else PAGED, kinds[name].c(), None):
        with pytest.raises(AssertionError, match=f"^{name}: cfg must be"):
            getattr(kvec, name)(other, *([4] if call == "evict" else []), **args, **more)

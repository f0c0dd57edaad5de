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

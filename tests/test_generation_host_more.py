"""More of what the text-generation calls refuse and ask for, before anything touches a GPU."""
import ctypes as C

import pytest

import paper_2409_06941_amd as fr


def test_a_cache_in_host_memory_is_refused_by_itself():
    torch = pytest.importorskip("torch")
    x, slot = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    q, n, pages = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 1, dtype=torch.int32)
    for device in ("cpu", "meta"):
        k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device=device)
        cache = fr.KvPages(k, k.clone())
        for call in (lambda: fr.fr_kv_append(cache, x, x, slot), lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, 0.1, max_own_len=8)):
            with pytest.raises(ValueError, match="cache k: not on a GPU"):
                call()


def _need(n_tokens, n_seqs, max_q, prefix_len, max_own_len, n_q_heads=32, n_kv_heads=8, head_dim=128):
    """What fr_attend_shared_workspace_bytes answers: its code and the bytes."""
    d, need = fr.fr_attend_desc(), C.c_uint64(12345)
    d.cache = fr.fr_kv_pages(None, None, 10, 0, 0, 0, n_kv_heads, head_dim, 16, fr.FR_DTYPE_BF16)
    d.n_tokens, d.n_seqs, d.n_q_heads, d.max_q, d.prefix_len, d.max_own_len = n_tokens, n_seqs, n_q_heads, max_q, prefix_len, max_own_len
    return fr.lib().fr_attend_shared_workspace_bytes(C.byref(d), C.byref(need)), need.value


def test_sizes_that_no_launch_takes_are_refused_when_the_workspace_is_asked_for():
    assert _need(66047, 512, 65536, 0, 65536, n_q_heads=64)[0] == fr.FR_OK
    assert _need(1 << 20, 1 << 20, 1 << 20, 0, 100)[0] == fr.FR_ERR_ARG
    assert _need(1 << 20, 1 << 20, 1, 0, 100)[0] == fr.FR_OK

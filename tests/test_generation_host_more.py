"""More of what the text-generation calls refuse and ask for, before anything touches a GPU."""
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

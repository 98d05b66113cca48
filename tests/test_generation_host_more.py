"""More of what the text-generation calls refuse and ask for, before anything touches a GPU."""
import ctypes as C
import os
import random

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


def test_the_workspace_of_a_larger_call_is_enough_for_a_smaller_one():
    # batches that shrink, prompts that get shorter, prefixes and caches in between
    sizes = [(n, n, 1, P, L) for n in (256, 128, 64, 32, 8, 4, 1) for P in (0, 300, 8192) for L in (100, 4000, 60000)]
    sizes += [(n * t, n, t, P, max(t, L)) for n in (64, 16, 3, 1) for t in (700, 300, 40, 5) for P in (0, 512, 8192) for L in (0, 700, 5000)]
    rng = random.Random(0)
    for _ in range(4000):
        n, t = round(2 ** rng.uniform(0, 10)), round(2 ** rng.uniform(0, 12))
        sizes.append((rng.randint(1, n * t), n, t, rng.choice([0, round(2 ** rng.uniform(0, 16))]), rng.choice([0, round(2 ** rng.uniform(0, 16))])))
    for heads, kv, dim in ((32, 8, 128), (8, 8, 64), (40, 1, 64), (15, 5, 128)):
        answers = [_need(*s, n_q_heads=heads, n_kv_heads=kv, head_dim=dim) for s in sizes]
        assert all(code == fr.FR_OK for code, _ in answers)
        small = sizes[:1200]
        for s, (_, need) in zip(small, answers):
            for _ in range(4):
                less = tuple(rng.randint(0 if i > 2 else 1, x) if rng.random() < 0.6 and x else x for i, x in enumerate(s))
                assert _need(*less, n_q_heads=heads, n_kv_heads=kv, head_dim=dim)[1] <= need, (s, less)
    # and the two that a server met: a batch that shrinks, questions that get shorter
    assert _need(32, 32, 1, 0, 4000)[1] <= _need(256, 256, 1, 0, 4000)[1]
    assert _need(16 * 300, 16, 300, 8192, 700)[1] <= _need(16 * 700, 16, 700, 8192, 700)[1]
    # a decoding step asks for some MB, not for what the largest possible cut would take
    assert _need(64, 64, 1, 16384, 1500)[1] < 64 << 20


def test_a_module_built_from_another_header_is_not_loaded(monkeypatch, tmp_path):
    pytest.importorskip("torch")
    fr.binding._torch_calls()
    other = type("fr_sample_desc", (C.Structure,), {"_fields_": list(reversed(fr.fr_sample_desc._fields_))})
    assert C.sizeof(other) == C.sizeof(fr.fr_sample_desc)
    monkeypatch.setattr(fr.binding, "_calls", None)
    monkeypatch.setattr(fr.binding, "fr_sample_desc", other)
    with pytest.raises(RuntimeError, match="another include/freeride.h"):
        fr.binding._torch_calls()
    # and an old one is built anew where only what is stale is built
    build = fr.binding._build
    module = tmp_path / "module.so"
    monkeypatch.setattr(build, "TORCH_CALLS", str(module))
    assert build.torch_calls_is_stale()
    module.write_bytes(b"")
    assert not build.torch_calls_is_stale() and build.build_torch_calls(force=False) == str(module)
    os.utime(module, (1, 1))
    assert build.torch_calls_is_stale()

"""What the text-generation calls refuse, and what they ask for, before anything touches a GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2409_06941_amd as fr
from oracle import generation as oracle

STRUCTS = ["fr_kv_pages", "fr_kv_append_desc", "fr_attend_desc", "fr_sample_desc"]
A = 1 << 20                                            # an address that is never read: the calls below refuse first


def test_struct_sizes_match_the_header_layout(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "freeride.h"\nint main(void) {\n' +
                   "".join('  printf("%s %%zu\\n", sizeof(%s));\n' % (n, n) for n in STRUCTS) + "  return 0;\n}\n")
    exe = tmp_path / "sizes"
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-std=c11", "-I", include, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    sizes = dict((line.split()[0], int(line.split()[1])) for line in out.splitlines())
    for n in STRUCTS:
        assert C.sizeof(getattr(fr.binding, n)) == sizes[n], n


def _pages(**change):
    c = fr.fr_kv_pages(A, A, 10, 8 * 16 * 128, 16 * 128, 128, 8, 128, 16, fr.FR_DTYPE_BF16)
    for k, x in change.items():
        setattr(c, k, x)
    return c


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=A + 8), dict(n_pages=0), dict(n_pages=1 << 31), dict(page_stride=-8),
             dict(page_stride=4), dict(head_stride=1), dict(slot_stride=127), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96),
             dict(head_dim=0), dict(page_size=0), dict(page_size=24), dict(page_size=8192), dict(dtype=fr.FR_DTYPE_F32), dict(dtype=7)]


def _append(**change):
    d = fr.fr_kv_append_desc()
    d.cache = _pages()
    d.k, d.v, d.q, d.q_out, d.slot, d.position, d.rotary = A, A, A, A, A, A, A
    d.k_stride = d.v_stride = 1024
    d.q_stride = d.q_out_stride = 4096
    d.n_positions, d.rotary_dim, d.n_tokens, d.n_q_heads = 100, 128, 4, 32
    for k, x in change.items():
        setattr(d, k, x)
    return fr.lib().fr_kv_append(C.byref(d), None)


@pytest.mark.parametrize("change", [dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(slot=None), dict(position=None), dict(rotary=None),
                                    dict(k=A + 2), dict(v=A + 8), dict(q=A + 4), dict(q_out=A + 8), dict(rotary=A + 4), dict(k_stride=1016), dict(k_stride=1028),
                                    dict(v_stride=-1024), dict(q_stride=8), dict(q_out_stride=4088), dict(q_stride=8192), dict(n_positions=0),
                                    dict(rotary_dim=130), dict(rotary_dim=24), dict(rotary_dim=-16), dict(style=2), dict(n_tokens=-1), dict(n_q_heads=-1),
                                    dict(n_q_heads=1025)] + [dict(cache=_pages(**p)) for p in BAD_PAGES])
def test_append_refuses(change):
    assert _append(**change) == fr.FR_ERR_ARG


def test_append_of_nothing_is_no_launch():
    assert _append(n_tokens=0) == fr.FR_OK and _append(n_tokens=0, k=None, slot=None) == fr.FR_OK
    assert fr.lib().fr_kv_append(None, None) == fr.FR_ERR_ARG


def _attend(**change):
    d = fr.fr_attend_desc()
    d.cache = _pages()
    d.q, d.out, d.q_begin, d.prefix_pages, d.pages, d.own_len, d.workspace = A, 2 * A, A, A, A, A, A
    d.q_stride = d.out_stride = 4096
    d.pages_stride, d.n_tokens, d.n_seqs, d.n_q_heads, d.max_q = 8, 4, 4, 32, 1
    d.prefix_len, d.max_own_len, d.scale, d.workspace_bytes = 1000, 128, 0.1, 1 << 40
    for k, x in change.items():
        setattr(d, k, x)
    return fr.lib().fr_attend_shared(C.byref(d), None)


@pytest.mark.parametrize("change", [dict(q=None), dict(out=None), dict(out=A), dict(q=A + 2), dict(out=A + 8), dict(prefix_pages=None), dict(pages=None),
                                    dict(own_len=None), dict(q_stride=4088), dict(out_stride=4097), dict(q_stride=-4096), dict(pages_stride=7),
                                    dict(n_tokens=-1), dict(n_seqs=-1), dict(n_q_heads=0), dict(n_q_heads=12), dict(n_q_heads=2048), dict(max_q=0),
                                    dict(prefix_len=-1), dict(max_own_len=-1), dict(prefix_len=0x7fffffff), dict(scale=0.0), dict(scale=-1.0),
                                    dict(scale=float("nan")), dict(scale=float("inf")), dict(q_begin=None, n_seqs=3)] + [dict(cache=_pages(**p)) for p in BAD_PAGES])
def test_attend_refuses(change):
    assert _attend(**change) == fr.FR_ERR_ARG


def test_attend_of_nothing_is_no_launch_and_workspaces_are_asked_for():
    assert _attend(n_tokens=0) == fr.FR_OK and _attend(n_seqs=0, q=None) == fr.FR_OK
    d, need = fr.fr_attend_desc(), C.c_uint64()
    d.cache = _pages(k=None, v=None)
    d.n_tokens, d.n_seqs, d.n_q_heads, d.max_q, d.prefix_len, d.max_own_len = 64, 64, 32, 1, 16384, 1500
    f = fr.lib().fr_attend_shared_workspace_bytes
    assert f(C.byref(d), C.byref(need)) == fr.FR_OK
    if need.value:
        assert _attend(n_tokens=64, n_seqs=64, prefix_len=16384, max_own_len=1500, pages_stride=100, workspace_bytes=need.value - 1) == fr.FR_ERR_ARG
        assert _attend(n_tokens=64, n_seqs=64, prefix_len=16384, max_own_len=1500, pages_stride=100, workspace=None) == fr.FR_ERR_ARG
        assert _attend(n_tokens=64, n_seqs=64, prefix_len=16384, max_own_len=1500, pages_stride=100, workspace=A + 16) == fr.FR_ERR_ARG
    assert f(None, C.byref(need)) == fr.FR_ERR_ARG and f(C.byref(d), None) == fr.FR_ERR_ARG
    d.n_q_heads = 33
    assert f(C.byref(d), C.byref(need)) == fr.FR_ERR_ARG


def _sample(**change):
    d = fr.fr_sample_desc()
    d.logits, d.uniform, d.token, d.workspace = A, A, A, A
    d.row_stride, d.n_rows, d.n_vocab, d.dtype, d.workspace_bytes = 1000, 3, 1000, fr.FR_DTYPE_F32, 1 << 40
    for k, x in change.items():
        setattr(d, k, x)
    return fr.lib().fr_sample(C.byref(d), None)


@pytest.mark.parametrize("change", [dict(logits=None), dict(uniform=None), dict(token=None), dict(logits=A + 2), dict(logits=A + 1, dtype=fr.FR_DTYPE_F16),
                                    dict(row_stride=999), dict(row_stride=-1000), dict(n_rows=-1), dict(n_vocab=0), dict(n_vocab=(1 << 19) + 1), dict(dtype=3),
                                    dict(dtype=-1)])
def test_sample_refuses(change):
    assert _sample(**change) == fr.FR_ERR_ARG


def test_sample_of_nothing_is_no_launch_and_workspaces_are_asked_for():
    assert _sample(n_rows=0) == fr.FR_OK and _sample(n_rows=0, logits=None) == fr.FR_OK
    assert fr.lib().fr_sample(None, None) == fr.FR_ERR_ARG
    d, need = fr.fr_sample_desc(), C.c_uint64()
    d.n_rows, d.n_vocab, d.dtype = 3, 1000, fr.FR_DTYPE_F32
    f = fr.lib().fr_sample_workspace_bytes
    assert f(C.byref(d), C.byref(need)) == fr.FR_OK
    if need.value:
        assert _sample(workspace_bytes=need.value - 1) == fr.FR_ERR_ARG and _sample(workspace=None) == fr.FR_ERR_ARG and _sample(workspace=A + 16) == fr.FR_ERR_ARG
    assert f(None, C.byref(need)) == fr.FR_ERR_ARG and f(C.byref(d), None) == fr.FR_ERR_ARG


def test_the_binding_refuses_tensors_the_library_cannot_read():
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fr.KvPages(k, torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        fr.KvPages(k.transpose(2, 3), k.transpose(2, 3))
    cache, x, slot = fr.KvPages(k, k.clone()), torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(TypeError):
        fr.fr_kv_append(cache, x.half(), x, slot)
    with pytest.raises(TypeError):
        fr.fr_kv_append(cache, x, x, slot.int())
    with pytest.raises(ValueError):
        fr.fr_kv_append(cache, x[:2], x, slot)
    with pytest.raises(ValueError):
        fr.fr_kv_append(cache, torch.zeros(3, 4, 64, dtype=torch.bfloat16)[:, ::2], x, slot)
    q, n = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        fr.fr_attend_shared(cache, q, q.clone(), torch.zeros(3, 1, dtype=torch.int32), n, 0.1, max_own_len=9)
    with pytest.raises(ValueError):
        fr.fr_attend_shared(cache, q, q.clone(), None, None, 0.1, prefix_len=9, prefix_pages=n[:1])
    with pytest.raises(TypeError):
        fr.fr_attend_shared(cache, q, q.clone(), torch.zeros(3, 1, dtype=torch.int64), n, 0.1, max_own_len=8)
    with pytest.raises(TypeError):
        fr.fr_sample(torch.zeros(3, 10), torch.zeros(3, dtype=torch.float64), n)
    with pytest.raises(ValueError):
        fr.fr_sample(torch.zeros(10, 3).t(), torch.zeros(3), n)
    with pytest.raises(TypeError):
        fr.fr_sample(torch.zeros(3, 10, dtype=torch.int32), torch.zeros(3), n)


def test_calls_refuse_host_memory_other_objects_and_numbers_out_of_range():
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    cache, x, slot = fr.KvPages(k, k.clone()), torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    q, n = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    pages, logits, u = torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, 10), torch.zeros(3)
    for call in (lambda: fr.fr_kv_append(cache, x, x, slot), lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, 0.1, max_own_len=8),
                 lambda: fr.fr_sample(logits, u, n)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
    for call in (lambda: fr.fr_kv_append(cache, None, x, slot), lambda: fr.fr_kv_append(cache, x, x, 0), lambda: fr.fr_sample(logits, u, [0, 0, 0]),
                 lambda: fr.fr_attend_shared(cache, 1, q, pages, n, 0.1), lambda: fr.fr_kv_append(cache, x, x, slot, q=q),
                 lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, "1")):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, 0.1, prefix_len=1 << 31),
                 lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, 0.1, max_q=-(1 << 40)),
                 lambda: fr.fr_kv_append(cache, x, x, slot, style=1 << 33), lambda: fr.fr_kv_append(cache, x, x, slot, q=q, q_out=q[:, :3]),
                 lambda: fr.fr_kv_append(cache, x, x, slot, rotary=torch.zeros(64)),
                 lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, 0.1, q_begin=torch.zeros(0, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()


def test_oracle_against_closed_forms():
    # a rotation keeps lengths and turns by the sum of two angles; pairs and halves are the same up to the order
    rng = np.random.default_rng(0)
    x, a, b = rng.standard_normal((3, 8)), rng.uniform(0, 6, 3), rng.uniform(0, 6, 3)
    once = oracle.rotate(oracle.rotate(x, np.cos(a), np.sin(a), 6, False), np.cos(b), np.sin(b), 6, False)
    assert np.allclose(once, oracle.rotate(x, np.cos(a + b), np.sin(a + b), 6, False))
    assert np.allclose((once ** 2).sum(1), (x ** 2).sum(1)) and np.array_equal(once[:, 6:], x[:, 6:])
    mixed = np.empty_like(x)
    mixed[:, 0:6:2], mixed[:, 1:6:2], mixed[:, 6:] = x[:, :3], x[:, 3:6], x[:, 6:]
    y = oracle.rotate(mixed, np.cos(a), np.sin(a), 6, True)
    assert np.allclose(np.concatenate([y[:, 0:6:2], y[:, 1:6:2], y[:, 6:]], 1), oracle.rotate(x, np.cos(a), np.sin(a), 6, False))
    # equal scores average the values; one dominant score picks its value
    v = rng.standard_normal((5, 4))
    o, lse, _, _ = oracle.attend_row(np.zeros(4), rng.standard_normal((5, 4)), v, 1.0)
    assert np.allclose(o, v.mean(0)) and np.isclose(lse, np.log(5))
    assert oracle.attend_row(np.zeros(4), np.zeros((0, 4)), np.zeros((0, 4)), 1.0)[1] == -np.inf
    assert [oracle.visible(7, 5, 3, i) for i in range(3)] == [10, 11, 12] and oracle.visible(7, 1, 3, 0) == 7
    # shares 1/2, 1/4, 1/8, 1/8
    x = np.log([2.0, 8.0, 4.0, 2.0])
    assert [oracle.sample(x, u) for u in (0.0, 0.12, 0.13, 0.62, 0.63, 0.87, 0.88, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert list(oracle.kept(x, 1.0, top_k=3)[0]) == [0, 1, 2] and list(oracle.kept(x, 1.0, top_p=0.5)[0]) == [1]
    assert list(oracle.kept(x, 1.0, top_p=0.51)[0]) == [1, 2] and list(oracle.kept(x, 1.0, min_p=0.3)[0]) == [1, 2]

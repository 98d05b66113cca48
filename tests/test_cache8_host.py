"""What the calls of a cache held in 8 bits refuse, and what they ask for, before anything touches a GPU; the oracle's codes."""
import ctypes as C
import os
import random
import subprocess

import numpy as np
import pytest

import paper_2409_06941_amd as fr
from oracle import cache8

STRUCTS = ["fr_kv8_pages", "fr_kv8_append_desc", "fr_attend_kv8_desc", "fr_kv_copy_desc"]
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


def _pages8(**change):
    c = fr.fr_kv8_pages(A, A, A, A, 10, 8 * 16 * 128, 16 * 128, 128, 8, 1, 1, 8, 128, 16, 16, fr.FR_DTYPE_BF16, 0)
    for k, x in change.items():
        setattr(c, k, x)
    return c


BAD_PAGES = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=A + 8), dict(v=A + 1), dict(n_pages=0), dict(n_pages=1 << 31),
             dict(page_stride=-16), dict(page_stride=8), dict(head_stride=1), dict(slot_stride=120), dict(slot_stride=1 << 31), dict(scale_page_stride=-1),
             dict(scale_head_stride=1 << 31), dict(scale_block_stride=-1), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96), dict(head_dim=0),
             dict(page_size=0), dict(page_size=24), dict(page_size=8192), dict(block=0), dict(block=32), dict(block=3), dict(page_size=256, block=256),
             dict(dtype=fr.FR_DTYPE_F32), dict(dtype=7)]


def _append(**change):
    d = fr.fr_kv8_append_desc()
    d.cache = _pages8()
    d.k, d.v, d.q, d.q_out, d.slot, d.position, d.rotary = A, A, A, A, A, A, A
    d.k_stride = d.v_stride = 1024
    d.q_stride = d.q_out_stride = 4096
    d.n_positions, d.rotary_dim, d.n_tokens, d.n_q_heads = 100, 128, 4, 32
    for k, x in change.items():
        setattr(d, k, x)
    return fr.lib().fr_kv8_append(C.byref(d), None)


@pytest.mark.parametrize("change", [dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(slot=None), dict(position=None), dict(rotary=None),
                                    dict(k=A + 2), dict(v=A + 8), dict(q=A + 4), dict(q_out=A + 8), dict(rotary=A + 4), dict(k_stride=1016), dict(k_stride=1028),
                                    dict(v_stride=-1024), dict(n_tokens=1, k_stride=-8), dict(q_stride=8), dict(q_out_stride=4088), dict(q_stride=8192),
                                    dict(n_positions=0), dict(rotary_dim=130), dict(rotary_dim=24), dict(rotary_dim=-16), dict(style=2), dict(n_tokens=-1),
                                    dict(n_q_heads=-1), dict(n_q_heads=1025)] + [dict(cache=_pages8(**p)) for p in BAD_PAGES])
def test_append_refuses(change):
    assert _append(**change) == fr.FR_ERR_ARG


def test_append_of_nothing_is_no_launch():
    assert _append(n_tokens=0) == fr.FR_OK and _append(n_tokens=0, k=None, slot=None) == fr.FR_OK
    assert fr.lib().fr_kv8_append(None, None) == fr.FR_ERR_ARG


def _attend_desc(**change):
    d = fr.fr_attend_kv8_desc()
    d.cache = _pages8()
    d.q, d.out, d.q_begin, d.pages, d.lens, d.workspace = A, 2 * A, A, A, A, A
    d.q_stride = d.out_stride = 4096
    d.pages_stride, d.n_tokens, d.n_seqs, d.n_q_heads, d.max_q = 80, 4, 4, 32, 1
    d.max_len, d.scale, d.workspace_bytes = 1280, 0.1, 1 << 40
    for k, x in change.items():
        setattr(d, k, x)
    return d


def _attend(**change):
    return fr.lib().fr_attend_kv8(C.byref(_attend_desc(**change)), None)


@pytest.mark.parametrize("change", [dict(q=None), dict(out=None), dict(out=A), dict(q=A + 2), dict(out=A + 8), dict(pages=None), dict(lens=None),
                                    dict(q_stride=4088), dict(out_stride=4097), dict(q_stride=-4096), dict(pages_stride=79), dict(pages_stride=-1),
                                    dict(n_tokens=-1), dict(n_seqs=-1), dict(n_q_heads=0), dict(n_q_heads=12), dict(n_q_heads=2048), dict(max_q=0),
                                    dict(max_len=-1), dict(max_len=0x7fffffff), dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0),
                                    dict(scale=float("nan")), dict(scale=float("inf")), dict(q_begin=None, n_seqs=3)] + [dict(cache=_pages8(**p)) for p in BAD_PAGES])
def test_attend_refuses(change):
    assert _attend(**change) == fr.FR_ERR_ARG


def _need(n_tokens, n_seqs, max_q, max_len, window=0, sinks=0, n_q_heads=32, n_kv_heads=8, head_dim=128):
    d, need = _attend_desc(n_tokens=n_tokens, n_seqs=n_seqs, max_q=max_q, max_len=max_len, window=window, sinks=sinks, n_q_heads=n_q_heads), C.c_uint64(12345)
    d.cache = _pages8(k=None, v=None, k_scale=None, v_scale=None, n_kv_heads=n_kv_heads, head_dim=head_dim)
    return fr.lib().fr_attend_kv8_workspace_bytes(C.byref(d), C.byref(need)), need.value


def test_attend_of_nothing_is_no_launch_and_workspaces_are_asked_for():
    assert _attend(n_tokens=0) == fr.FR_OK and _attend(n_seqs=0, q=None) == fr.FR_OK
    code, need = _need(64, 64, 1, 16384)
    assert code == fr.FR_OK
    more = dict(n_tokens=64, n_seqs=64, max_len=16384, pages_stride=1024)
    if need:
        assert _attend(workspace_bytes=need - 1, **more) == fr.FR_ERR_ARG
        assert _attend(workspace=None, **more) == fr.FR_ERR_ARG
        assert _attend(workspace=A + 16, **more) == fr.FR_ERR_ARG
    f, out = fr.lib().fr_attend_kv8_workspace_bytes, C.c_uint64()
    assert f(None, C.byref(out)) == fr.FR_ERR_ARG and f(C.byref(_attend_desc()), None) == fr.FR_ERR_ARG
    assert _need(64, 64, 1, 1000, n_q_heads=33)[0] == fr.FR_ERR_ARG


def test_the_workspace_of_a_larger_call_is_enough_for_a_smaller_one():
    sizes = [(n, n, 1, L) for n in (256, 128, 64, 32, 8, 4, 1) for L in (0, 100, 4000, 60000)]
    sizes += [(n * t, n, t, max(t, L)) for n in (64, 16, 3, 1) for t in (700, 300, 40, 5) for L in (0, 700, 5000)]
    rng = random.Random(0)
    for _ in range(3000):
        n, t = round(2 ** rng.uniform(0, 10)), round(2 ** rng.uniform(0, 12))
        sizes.append((rng.randint(1, n * t), n, t, rng.choice([0, round(2 ** rng.uniform(0, 17))])))
    for heads, kv, dim in ((32, 8, 128), (8, 8, 64), (40, 1, 64), (15, 5, 128)):
        for s in sizes[:1200]:
            code, need = _need(*s, n_q_heads=heads, n_kv_heads=kv, head_dim=dim)
            assert code == fr.FR_OK
            for _ in range(3):
                less = tuple(rng.randint(0 if i > 2 else 1, x) if rng.random() < 0.6 and x else x for i, x in enumerate(s))
                window, sinks = rng.choice([(0, 0), (1, 0), (100, 4), (4096, 4), (0x7fffffff, 0x7fffffff)])
                assert _need(*less, window, sinks, n_q_heads=heads, n_kv_heads=kv, head_dim=dim)[1] <= need, (s, less, window)
    assert _need(64, 64, 1, 16384)[1] < 64 << 20


def _copy(**change):
    wide = fr.fr_kv_pages(A, A, 10, 8 * 16 * 128, 16 * 128, 128, 8, 128, 16, fr.FR_DTYPE_BF16)
    for k, x in change.pop("wide", {}).items():
        setattr(wide, k, x)
    narrow = _pages8(**change.pop("narrow", {}))
    d = fr.fr_kv_copy_desc(C.pointer(wide), C.pointer(narrow), 1, 1, A, A, A, 4, 0)
    for k, x in change.items():
        setattr(d, k, x)
    return fr.lib().fr_kv_copy_pages(C.byref(d), None)


@pytest.mark.parametrize("change", [dict(source=None), dict(target=None), dict(n_caches=-1), dict(n_caches8=-1), dict(n_caches=4097), dict(caches=None),
                                    dict(caches8=None), dict(n_pairs=-1), dict(n_pairs=(1 << 16) + 1), dict(wide=dict(n_pages=11)), dict(narrow=dict(n_pages=9)),
                                    dict(wide=dict(k=None)), dict(wide=dict(head_dim=96))] + [dict(narrow=p) for p in BAD_PAGES])
def test_copy_refuses(change):
    assert _copy(**change) == fr.FR_ERR_ARG


def test_copy_of_nothing_is_no_launch():
    assert _copy(n_pairs=0, source=None, target=None) == fr.FR_OK
    assert _copy(n_caches=0, n_caches8=0, caches=None, caches8=None) == fr.FR_OK
    assert fr.lib().fr_kv_copy_pages(None, None) == fr.FR_ERR_ARG


def test_tensors_that_do_not_fit_are_refused():
    torch = pytest.importorskip("torch")
    codes, scale = torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 4, dtype=torch.uint8)
    make = lambda k=codes, v=codes, ks=scale, vs=scale, dtype=torch.bfloat16: fr.Kv8Pages(k, v, ks, vs, dtype)
    assert make().desc.block == 4 and make(k=codes.view(torch.float8_e4m3fn), v=codes.view(torch.float8_e4m3fn)).desc.k == codes.data_ptr()
    for bad in (dict(k=codes[:3]), dict(k=codes.float(), v=codes.float()), dict(k=codes.view(torch.int8), v=codes.view(torch.int8)), dict(ks=scale[:3], vs=scale[:3]),
                dict(ks=scale.int(), vs=scale.int()), dict(ks=scale[:, :, :3], vs=scale[:, :, :3]), dict(ks=scale.transpose(0, 0)[:, :, ::2]), dict(dtype=torch.float32),
                dict(k=codes.transpose(2, 3), v=codes.transpose(2, 3)), dict(ks=scale[:, :, :0], vs=scale[:, :, :0])):
        with pytest.raises((ValueError, TypeError)):
            make(**bad)
    x, slot = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    q, n, pages = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 1, dtype=torch.int32)
    cache, wide = make(), fr.KvPages(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16))
    for call in (lambda: fr.fr_kv8_append(cache, x, x, slot), lambda: fr.fr_attend_kv8(cache, q, q.clone(), pages, n, 0.1, max_len=8),
                 lambda: fr.fr_kv_copy_pages([cache, wide], n, n)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
    for call in (lambda: fr.fr_kv8_append(cache, x.half(), x, slot), lambda: fr.fr_kv8_append(cache, x, x, slot.int()), lambda: fr.fr_kv8_append(wide, x, x, slot),
                 lambda: fr.fr_attend_kv8(cache, q.half(), q.half(), pages, n, 0.1, max_len=8), lambda: fr.fr_attend_kv8(wide, q, q, pages, n, 0.1, max_len=8),
                 lambda: fr.fr_kv_copy_pages([cache, codes], n, n), lambda: fr.fr_kv_copy_pages(cache, n.long(), n), lambda: fr.fr_kv_copy_pages(cache, n, None)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: fr.fr_kv8_append(cache, x, x[:2], slot), lambda: fr.fr_attend_kv8(cache, q, q.clone(), pages, n, 0.1, max_len=17),
                 lambda: fr.fr_attend_kv8(cache, q, q.clone(), pages, n[:2], 0.1, max_len=8), lambda: fr.fr_attend_kv8(cache, q, q.clone(), pages, n, 0.1, max_len=1 << 40),
                 lambda: fr.fr_kv_copy_pages(cache, n, n[:2]), lambda: fr.fr_kv_copy_pages(cache, n, n, copied=n[:1])):
        with pytest.raises(ValueError):
            call()


def test_codes_of_the_oracle_are_those_of_the_type():
    torch = pytest.importorskip("torch")
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(want, cache8.VALUES, equal_nan=True)
    rng = np.random.default_rng(0)
    x = (rng.normal(0, 1, 20000) * 2.0 ** rng.uniform(-12, 8, 20000)).astype(np.float32)
    x = np.concatenate([x[np.abs(x) <= 448], cache8._MIDDLE.astype(np.float32), -cache8._MIDDLE.astype(np.float32)])
    assert np.array_equal(torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), cache8.encode(x))
    for dt, (lo, hi) in cache8.RANGE.items():
        for s in range(lo, hi):
            top = np.array([448 * 2.0 ** (s - 127)])
            assert cache8.need(top, dt) == s and cache8.need(np.nextafter(top, np.inf), dt) == s + 1

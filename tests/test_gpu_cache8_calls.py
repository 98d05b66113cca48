"""Calls of the operators of a cache held in 8 bits that go another way than their sizes alone would say."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2409_06941_amd as fr              # noqa: E402
from test_gpu_cache8 import DT, I32, _append_case, _attend_case, _copy_case          # noqa: E402


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hk,longest", [(16, 2, 300), (8, 8, 20), (8, 1, 5000)])
def test_one_token_a_sequence_whatever_max_q(dt, Hq, Hk, longest):
    # without q_begin every sequence has one token: a larger max_q, that of a program's other calls, changes neither result nor kernel
    print("attend max_q", dt, Hq, Hk, longest, flush=True)
    g = torch.Generator(device="cuda").manual_seed(longest)
    n, D, page = 9, 64, 16
    width = -(-longest // page)
    codes = [torch.randint(0, 120, (n * width, Hk, page, D), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scale = [torch.full((n * width, Hk, 1), 118, device="cuda", dtype=torch.uint8) for _ in range(2)]
    cache = fr.Kv8Pages(*codes, *scale, DT[dt])
    q = torch.randn((n, Hq, D), generator=g, device="cuda").to(DT[dt])
    table = torch.randperm(n * width, generator=g, device="cuda").to(I32).view(n, width)
    lens = torch.randint(1, longest, (n,), generator=g, device="cuda").to(I32)
    lens[0], lens[1] = longest, 0
    results = []
    for max_q in (1, 8, 64, 1 << 20):
        out, lse = torch.full_like(q, 9.0), torch.full((n, Hq), 9.0, device="cuda")
        ws = torch.full((max(1, fr.fr_attend_kv8_workspace_bytes(cache, q, n, max_len=longest)),), 255, dtype=torch.uint8, device="cuda")
        fr.fr_attend_kv8(cache, q, out, table, lens, 0.125, max_len=longest, max_q=max_q, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        results.append((out, lse))
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


def test_copy_without_caches_touches_nothing():
    source, copied = torch.arange(3, dtype=I32, device="cuda"), torch.full((3,), 7, dtype=I32, device="cuda")
    fr.fr_kv_copy_pages([], source, source + 3, copied=copied)
    torch.cuda.synchronize()
    assert copied.tolist() == [7, 7, 7]


@pytest.mark.parametrize("dt,Hq,Hk,D", [("bf16", 8, 1, 64), ("f16", 12, 2, 128)])
@pytest.mark.parametrize("seqs,window", [(64, 0), (65, 0), (130, 50)])
def test_attend_many_rows_of_many_sequences(dt, Hq, Hk, D, seqs, window):
    # 128 rows a workgroup; up to 64 sequences go by falling lengths, more of them in their own order
    print("attend many rows", dt, Hq, Hk, D, seqs, window, flush=True)
    rng = np.random.default_rng(seqs)
    new = [int(x) for x in rng.integers(0, 10, seqs)]
    lens = [int(x) for x in rng.integers(0, 150, seqs)]
    new[3], new[-1], lens[-1] = 40, 9, 333
    _attend_case(dt, Hq, Hk, D, 16, 8, lens, new, seqs, window, 3 if window else 0)


@pytest.mark.parametrize("T", [767, 1023, 1024, 2047, 4095, 4096, 8192])
@pytest.mark.parametrize("block", [1, 16])
def test_append_tokens_of_a_workgroup(T, block):
    # how many tokens' keys and values a workgroup has goes by their number: runs that begin and end at its border and elsewhere, padding
    print("append", T, block, flush=True)
    rng = np.random.default_rng(T)
    slot, at = [], 0
    while len(slot) < T:
        n = int(rng.integers(1, 40))
        begin = at * 16 + int(rng.integers(0, 16))
        slot += [begin + i for i in range(n)] if n < 30 else [-1] * (n - 29)
        at += 4
    _append_case("bf16", T, 2, 1, 64, 16, block, 64, 0, T, slot=slot[:T], pages=at)


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("Hq,Hk,new", [(8, 1, 4), (11, 1, 3), (16, 2, 5), (10, 2, 9), (24, 3, 6), (7, 1, 7)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_attend_about_as_many_rows_as_are_few(dt, D, Hq, Hk, new, window, sinks):
    # 32 to 49 rows of a sequence and key head: two, three tiles of 16, and the first that go by 128
    print("attend rows", dt, D, Hq, Hk, new, window, flush=True)
    lens = [0, 1, new, 31, 33, 130, 700, 257]
    _attend_case(dt, Hq, Hk, D, 16, 8, lens, [min(n, new) for n in lens], Hq + new, window, sinks, rows=400)
    _attend_case(dt, Hq, Hk, D, 16, 1, [90, 40], [new, new - 1], Hq + new, window, sinks, nan_at=[(0, 89, 3, True), (0, 30, 8, True), (1, 37, 0, False)])


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f16", 64)])
def test_attend_three_tiles_of_rows_dealt_out_evenly(dt, D):
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 17000, 5)]
    lens[0], lens[3] = 17000, 4
    _attend_case(dt, 56, 8, D, 16, 8, lens, [6, 5, 0, 4, 6], 9, rows=150)


@pytest.mark.parametrize("longest", [1, 250, 288, 300, 511, 512, 513, 600, 1000])
@pytest.mark.parametrize("kind", ["equal", "any"])
def test_attend_short_sequences_with_room_for_long_ones(longest, kind):
    # tiles are dealt out evenly among workers, by whole sequences where all of them are short
    print("attend short", longest, kind, flush=True)
    rng = np.random.default_rng(longest)
    lens = [longest] * 16 if kind == "equal" else [int(x) for x in rng.integers(0, longest + 1, 15)] + [longest]
    _attend_case("bf16", 16, 8, 64, 16, 8, lens, [1] * 16, longest, max_len=40000)
    _attend_case("f16", 6, 2, 128, 16, 8, lens, [1] * 16, longest, max_len=140000)


@pytest.mark.parametrize("n", [511, 512, 1023, 1024, 1537])
def test_copy_caches_of_a_workgroup(n):
    rng = np.random.default_rng(n)
    source, target = np.full(n, -1), rng.integers(0, 23, n)
    for i, (a, b) in zip((0, n // 3, n // 2, n - 1), ((1, 2), (1, 7), (4, 5), (6, 2))):
        source[i], target[i] = a, b
    _copy_case([(8, 3, 8, 64, 4, "slots")] * 5 + [(16, 2, 4, 128, 1, "heads")], source.tolist(), target.tolist(), n)

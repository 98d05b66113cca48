"""GPU parity of the text-generation operators against the fp64 oracle: fr_kv_append, fr_attend_shared, fr_sample."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2409_06941_amd as fr              # noqa: E402
from oracle import generation as oracle        # noqa: E402

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # half an ulp of 8 and of 11 significant bits
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -25}        # half the smallest subnormal


def _f64(x):
    return x.detach().double().cpu().numpy()


# ---------------------------------------------------------------- append

def _append_case(T, Hq, Hk, D, page, pages, R, style, dt, seed, pad=(), strided=False, in_place=False, layout="heads"):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g).to(DT[dt])
    if layout == "heads":
        ck, cv = rnd(pages, Hk, page, D).cuda(), rnd(pages, Hk, page, D).cuda()
    elif layout == "slots":                            # [page][slot][head][i]: the heads of a slot side by side
        ck, cv = (rnd(pages, page, Hk, D).cuda().transpose(1, 2) for _ in range(2))
    else:                                              # K and V of a page in one array
        both = rnd(pages, 2, Hk, page, D).cuda()
        ck, cv = both[:, 0], both[:, 1]
    if strided:                                        # views of one projection's rows, with something behind them
        row = rnd(T, Hq + 2 * Hk + 1, D).cuda()
        q, k, v = row[:, :Hq], row[:, Hq:Hq + Hk], row[:, Hq + Hk:Hq + 2 * Hk]
    else:
        q, k, v = rnd(T, Hq, D).cuda(), rnd(T, Hk, D).cuda(), rnd(T, Hk, D).cuda()
    slot = torch.randperm(pages * page, generator=g)[:T].to(torch.int64)
    for i, x in pad:
        slot[i] = x
    positions = 777
    position = torch.randint(0, positions, (T,), generator=g).to(torch.int32)
    angle = torch.rand((positions, max(R // 2, 1)), generator=g) * 6.3
    table = torch.cat([angle.cos(), angle.sin()], 1)[:, :R].contiguous() if R else None
    q0, k0, v0, ck0, cv0 = (_f64(x) for x in (q, k, v, ck, cv))
    q_out = q if in_place else torch.full((T, Hq, D), 7.0, dtype=DT[dt], device="cuda")
    cache = fr.KvPages(ck, cv)
    fr.fr_kv_append(cache, k, v, slot.cuda(), q=q if Hq else None, q_out=q_out if Hq else None,
                    position=position.cuda() if R else None, rotary=table.cuda() if R else None, style=style,
                    stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    got_k, got_v, got_q = _f64(ck), _f64(cv), _f64(q_out)
    want_k, want_v, bound_k = ck0.copy(), cv0.copy(), np.zeros_like(ck0)
    pairs = style == fr.FR_ROTARY_PAIRS

    def both(x, t):
        if not R:
            return x, np.zeros_like(x)
        c, s = _f64(table[position[t]])[:R // 2], _f64(table[position[t]])[R // 2:]
        y = oracle.rotate(x, c, s, R, pairs)
        # two products and a sum of 32 bits, then the type's rounding
        e = 3 * 2.0 ** -24 * oracle.rotate(np.abs(x), np.abs(c), -np.abs(s), R, pairs)
        e = np.maximum(np.abs(e), 3 * 2.0 ** -24 * np.abs(oracle.rotate(np.abs(x), np.abs(c), np.abs(s), R, pairs)))
        e[:, R:] = 0
        near = e + UNIT[dt] * (np.abs(y) + e) + TINY[dt]
        near[:, R:] = 0
        return y, near
    for t in range(T):
        if 0 <= slot[t] < pages * page:
            p, o = int(slot[t]) // page, int(slot[t]) % page
            want_k[p, :, o], bound_k[p, :, o] = both(k0[t], t)
            want_v[p, :, o] = v0[t]
        if Hq:
            y, near = both(q0[t], t)
            assert np.all(np.abs(got_q[t] - y) <= near), t
    assert np.all(np.abs(got_k - want_k) <= bound_k)       # (0 where nothing was stored and where nothing was turned)
    assert np.array_equal(got_v, want_v)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,Hq,Hk,D,page,R,style", [
    (1, 4, 1, 64, 16, 64, 0), (1, 1, 1, 128, 1, 128, 1), (2, 8, 8, 128, 8, 64, 0), (37, 15, 5, 64, 8, 32, 1),
    (65, 3, 3, 64, 32, 48, 0), (129, 32, 8, 128, 16, 128, 0), (130, 7, 1, 128, 64, 16, 1), (9, 0, 2, 64, 4, 64, 0),
    (5, 4, 2, 128, 2, 0, 0), (300, 20, 5, 64, 32, 32, 1)])
def test_append(dt, T, Hq, Hk, D, page, R, style):
    print("append", dt, T, Hq, Hk, D, page, R, style, flush=True)
    _append_case(T, Hq, Hk, D, page, -(-(T + 5) // page) + 1, R, style, dt, seed=T + Hq)


@pytest.mark.parametrize("layout", ["heads", "slots", "joined"])
@pytest.mark.parametrize("strided,in_place", [(True, False), (True, True), (False, True)])
def test_append_layouts_strides_and_in_place(layout, strided, in_place):
    print("append", layout, strided, in_place, flush=True)
    _append_case(19, 6, 2, 128, 16, 4, 128, 0, "bf16", 5, strided=strided, in_place=in_place, layout=layout)
    _append_case(19, 6, 2, 64, 16, 4, 32, 1, "f16", 6, strided=strided, in_place=in_place, layout=layout)


def test_append_leaves_padding_out():
    far = 1 << 40
    _append_case(40, 4, 2, 64, 8, 9, 64, 0, "bf16", 8, pad=[(0, -1), (3, -far), (17, 72), (39, far), (20, (1 << 63) - 1)])


def test_append_positions_outside_the_table_and_empty_calls():
    D, T = 64, 4
    k = torch.randn(T, 1, D, device="cuda").to(torch.bfloat16)
    ck = torch.zeros(2, 1, 4, D, dtype=torch.bfloat16, device="cuda")
    cv = torch.zeros_like(ck)
    table = torch.randn(3, D, device="cuda")
    cache, slot = fr.KvPages(ck, cv), torch.arange(T, device="cuda")
    fr.fr_kv_append(cache, k, k, slot, position=torch.tensor([-5, 0, 2, 1 << 30], dtype=torch.int32, device="cuda"), rotary=table)
    a = ck.clone()
    fr.fr_kv_append(cache, k, k, slot, position=torch.tensor([0, 0, 2, 2], dtype=torch.int32, device="cuda"), rotary=table)
    torch.cuda.synchronize()
    assert torch.equal(a, ck) and bool((a[0] != 0).any())
    fr.fr_kv_append(cache, k[:0], k[:0], slot[:0], position=slot[:0].int(), rotary=table)
    torch.cuda.synchronize()
    assert torch.equal(a, ck)


# ---------------------------------------------------------------- attend

def _attend_case(dt, Hq, Hk, D, page, P, own, new, seed, layout="heads", q_begin=True, strided=False, spoil=0.0, scale=None,
                 std=1.0, stream=None, extra=3):
    """own, new: own keys and new tokens of every sequence.  spoil: what stands in slots behind a length."""
    g = torch.Generator().manual_seed(seed)
    n = len(own)
    width = max(1, -(-max(own + [0]) // page)) + 1
    counts = [-(-x // page) for x in own]
    P_pages = -(-P // page)
    pages = P_pages + sum(counts) + extra
    shape = (pages, Hk, page, D)
    fill = lambda: torch.randn(shape, generator=g)
    k, v = fill(), fill()
    order = torch.randperm(pages, generator=g).to(torch.int32)
    prefix_pages = order[:P_pages].clone()
    table = torch.full((n, width), 1 << 30, dtype=torch.int32)         # ids behind a sequence's pages lead nowhere
    at = P_pages
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    used = torch.zeros((pages, page), dtype=torch.bool)
    for j in range(P):
        used[prefix_pages[j // page], j % page] = True
    for b in range(n):
        for j in range(own[b]):
            used[table[b, j // page], j % page] = True
    k[~used[:, None, :].expand(-1, Hk, -1)] = spoil
    v[~used[:, None, :].expand(-1, Hk, -1)] = spoil
    k, v = k.to(DT[dt]).cuda(), v.to(DT[dt]).cuda()
    if layout == "slots":
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    elif layout == "joined":
        both = torch.stack([k, v], 1).contiguous()
        k, v = both[:, 0], both[:, 1]
    begin = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(begin[-1])
    q = (torch.randn((T, Hq + (2 if strided else 0), D), generator=g) * std).to(DT[dt]).cuda()[:, :Hq]
    out = torch.full((T, Hq + (1 if strided else 0), D), 9.0, dtype=DT[dt], device="cuda")[:, :Hq]
    lse = torch.full((T, Hq), 9.0, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    cache = fr.KvPages(k, v)
    lim = dict(prefix_len=P, max_own_len=max(own + [0]), max_q=max(max(new), 1) if q_begin else 1)
    need = fr.fr_attend_shared_workspace_bytes(cache, q, n, **lim)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")      # (NaNs, in whatever type it is read)
    torch.cuda.synchronize()
    fr.fr_attend_shared(cache, q, out, table.cuda() if max(own + [0]) else None, torch.tensor(own, dtype=torch.int32, device="cuda"),
                        scale, prefix_pages=prefix_pages.cuda() if P else None,
                        q_begin=torch.from_numpy(begin).cuda() if q_begin else None, lse=lse, workspace=ws,
                        stream=stream or torch.cuda.current_stream(), **lim)
    torch.cuda.synchronize()
    _check_attend(dt, q, k, v, prefix_pages, table, P, own, begin, scale, out, lse)
    return out, lse


def _check_attend(dt, q, k, v, prefix_pages, table, P, own, begin, scale, out, lse, rows=None):
    Hq, D, Hk, page = q.shape[1], q.shape[2], k.shape[1], k.shape[2]
    q64, k64, v64, o64, l64 = (_f64(x) for x in (q, k, v, out, lse))
    u = UNIT[dt]
    for b in range(len(own)):
        t = int(begin[b + 1] - begin[b])
        ids = np.concatenate([np.repeat(prefix_pages.numpy(), page)[:P], np.repeat(table[b].numpy(), page)[:own[b]]]).astype(np.int64)
        slots = np.concatenate([np.arange(P) % page, np.arange(own[b]) % page]).astype(np.int64)
        for h in range(Hq):
            kk, vv = k64[ids, h // (Hq // Hk), slots], v64[ids, h // (Hq // Hk), slots]
            for i in range(t):
                n = oracle.visible(P, own[b], t, i)
                row = int(begin[b]) + i
                o, l, a, x = oracle.attend_row(q64[row, h], kk[:n], vv[:n], scale)
                if n == 0:
                    assert not o64[row, h].any() and l64[row, h] == -math.inf
                    continue
                if not np.isfinite(o).all() or not np.isfinite(l):
                    assert np.array_equal(np.isfinite(o64[row, h]), np.isfinite(o)), (b, i, h)
                    continue
                # scores: sums of D products of 32 bits; each weight off by that, by a few ulps of exp, and by the type's
                # rounding; sums of n of them; the result's rounding.  Weights of 16 bits end at half the smallest subnormal.
                d = (D + 4) * 2.0 ** -24 * x + 2.0 ** -20
                near = (u + 2 * d + n * 2.0 ** -23) * a + u * np.abs(o) * 1.01 + TINY[dt] + (n * 2.0 ** -25 * np.abs(vv[:n]).max() if dt == "f16" else 0.0)
                assert np.all(np.abs(o64[row, h] - o) <= near), (b, i, h, np.abs(o64[row, h] - o).max(), near.max())
                assert abs(l64[row, h] - l) <= d + n * 2.0 ** -23 + 2.0 ** -20 * (1 + abs(l)), (b, i, h)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hk,D,page,P,own,new", [
    (1, 1, 64, 1, 0, [1], [1]),                                    # one key of one sequence
    (4, 2, 128, 16, 0, [0, 1, 15, 16, 17], [1, 1, 1, 1, 1]),       # a sequence that sees nothing; pages that end
    (8, 2, 64, 16, 37, [1, 30, 16], [1, 1, 1]),
    (8, 8, 128, 8, 64, [0, 0], [1, 1]),                            # the prefix alone
    (15, 5, 64, 8, 131, [3, 0, 77, 129], [3, 0, 2, 7]),
    (12, 1, 128, 32, 200, [65, 64, 63, 1], [1, 1, 1, 1]),
    (3, 3, 128, 64, 1, [2, 300], [2, 5]),
    (32, 2, 64, 4, 63, [5] * 9, [2] * 9),
    (40, 1, 128, 16, 257, [33, 2], [3, 2]),                        # forty heads to a key
    (6, 2, 128, 16, 0, [130, 70], [130, 70]),                      # prompts alone
    (4, 2, 64, 16, 100, [150, 9, 260], [70, 9, 33]),
    (16, 4, 128, 16, 600, [140, 33], [140, 33]),
    (2, 1, 64, 16, 0, [2, 5], [4, 5]),                             # more tokens than own keys: the first see nothing
    (2, 1, 128, 16, 3, [2, 0], [4, 3])])
def test_attend(dt, Hq, Hk, D, page, P, own, new):
    print("attend", dt, Hq, Hk, D, page, P, own, new, flush=True)
    _attend_case(dt, Hq, Hk, D, page, P, own, new, seed=Hq + P)


@pytest.mark.parametrize("P,own,new", [(2100, [900, 5, 0], [1, 1, 1]), (1025, [4097, 1, 640], [1, 1, 1]), (3000, [50] * 40, [1] * 40),
                                       (5001, [700, 20], [5, 7]), (0, [5000, 4095, 4096], [1, 1, 1]), (700, [600, 300], [300, 300])])
def test_attend_longer(P, own, new):
    print("attend longer", P, own, new, flush=True)
    _attend_case("bf16", 8, 2, 128, 16, P, own, new, seed=P + 1)
    _attend_case("f16", 8, 2, 64, 16, P, own, new, seed=P + 2)


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("P,new", [(0, 1), (150, 1), (700, 1), (150, 3)])
def test_attend_many_short_sequences(dt, D, P, new):
    # enough of them for a wavefront each: lengths from none to several parts, one and several tokens
    print("attend many", dt, D, P, new, flush=True)
    rng = np.random.default_rng(P + new)
    own = [int(x) for x in rng.integers(0, 40, 66)] + [0, 1, 31, 32, 33, 255, 256, 257, 600]
    t = [min(x, int(rng.integers(1, new + 1))) if new > 1 else 1 for x in own]
    _attend_case(dt, 16, 8, D, 16, P, own, t, seed=P + D)


@pytest.mark.parametrize("layout", ["slots", "joined"])
def test_attend_layouts_and_strides(layout):
    print("attend", layout, flush=True)
    _attend_case("bf16", 8, 2, 128, 16, 150, [40, 3, 90], [1, 1, 1], 3, layout=layout, strided=True, q_begin=False)
    _attend_case("f16", 8, 2, 64, 16, 150, [40, 3, 190], [20, 3, 100], 4, layout=layout, strided=True)


@pytest.mark.parametrize("spoil", [math.nan, math.inf, -math.inf, 60000.0])
def test_attend_never_uses_slots_behind_a_length(spoil):
    print("attend spoiled", spoil, flush=True)
    for dt in ("bf16", "f16"):
        _attend_case(dt, 8, 2, 128, 32, 70, [1, 33, 45], [1, 1, 1], 11, spoil=spoil)
        _attend_case(dt, 8, 2, 64, 32, 70, [150, 33, 45], [100, 3, 45], 12, spoil=spoil)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D,G,t", [(128, 2, 5), (64, 4, 40), (128, 4, 90)])
def test_attend_keys_that_a_token_may_not_see_do_not_touch_it(bad, D, G, t):
    # the last tokens' keys and values are not finite: tokens before them must come out as if they were not there
    print("attend hidden", bad, D, G, t, flush=True)
    page, P, L, Hk = 16, 50, t + 20, 2
    g = torch.Generator().manual_seed(t)
    pages = -(-P // page) + -(-L // page)
    k, v = (torch.randn((pages, Hk, page, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    prefix_pages, table = torch.arange(4, dtype=torch.int32), torch.arange(4, pages, dtype=torch.int32)[None, :].contiguous()
    for j, which in ((L - 1, v), (L - 2, k), (L - 3, v)):
        which[4 + j // page, :, j % page, 3:60] = bad
    q = torch.randn((t, Hk * G, D), generator=g).to(torch.bfloat16).cuda()
    out, lse = torch.zeros_like(q), torch.zeros(t, Hk * G, device="cuda")
    lim = dict(prefix_len=P, max_own_len=L, max_q=t)
    cache = fr.KvPages(k, v)
    ws = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(cache, q, 1, **lim)), dtype=torch.uint8, device="cuda")
    fr.fr_attend_shared(cache, q, out, table.cuda(), torch.tensor([L], dtype=torch.int32, device="cuda"), D ** -0.5,
                        prefix_pages=prefix_pages.cuda(), q_begin=torch.tensor([0, t], dtype=torch.int32, device="cuda"), lse=lse,
                        workspace=ws, stream=torch.cuda.current_stream(), **lim)
    torch.cuda.synchronize()
    # tokens t - 3 and later see at least one of the three keys; the others none
    clean = t - 3
    assert bool(torch.isfinite(out[:clean].float()).all()) and bool(torch.isfinite(lse[:clean]).all())
    k2, v2 = torch.nan_to_num(k.float(), 0, 0, 0).to(k.dtype), torch.nan_to_num(v.float(), 0, 0, 0).to(v.dtype)
    begin = np.array([0, clean], dtype=np.int32)
    _check_attend("bf16", q[:clean], k2, v2, prefix_pages, table, P, [L - 3], begin, D ** -0.5, out[:clean], lse[:clean])
    assert not bool(torch.isfinite(out[t - 3].float()).all())      # a value that is seen and not finite shows


def test_attend_large_scores_and_scales():
    _attend_case("bf16", 4, 2, 128, 16, 100, [50, 60], [1, 1], 21, std=30.0)
    _attend_case("f16", 4, 2, 64, 16, 100, [50, 60], [2, 9], 22, std=20.0)
    _attend_case("bf16", 4, 2, 64, 16, 100, [50, 60], [1, 1], 23, scale=1e-3)
    _attend_case("bf16", 4, 2, 64, 16, 0, [350, 60], [1, 1], 24, scale=3.0, std=4.0)


def test_attend_numbers_from_the_device_are_bounded():
    # lengths beyond max_own_len, q_begin beyond n_tokens, page ids outside: results of the bounded numbers, no access outside
    D, page = 64, 16
    k = torch.randn(4, 1, page, D, device="cuda").to(torch.bfloat16)
    v = torch.randn(4, 1, page, D, device="cuda").to(torch.bfloat16)
    cache, q = fr.KvPages(k, v), torch.randn(3, 2, D, device="cuda").to(torch.bfloat16)

    def call(own, begin, table, P=0, prefix=None):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(q)
        lim = dict(prefix_len=P, max_own_len=32, max_q=1)
        ws = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(cache, q, 3, **lim)), dtype=torch.uint8, device="cuda")
        fr.fr_attend_shared(cache, q, out, i32(table), i32(own), 0.125, q_begin=i32(begin), prefix_pages=i32(prefix) if P else None,
                            workspace=ws, stream=torch.cuda.current_stream(), **lim)
        torch.cuda.synchronize()
        return out
    same = [[0, 1], [1, 2], [3, 0]]
    assert torch.equal(call([1000, -7, 5], [0, 1, 2, 3], same), call([32, 0, 5], [0, 1, 2, 3], same))
    assert torch.equal(call([9, 9, 5], [-4, 1, 2, 900], same), call([9, 9, 5], [0, 1, 2, 3], same))
    assert torch.equal(call([20, 20, 20], [0, 1, 2, 3], [[-1, 1], [1, 99], [1 << 30, 0]]), call([20, 20, 20], [0, 1, 2, 3], [[0, 1], [1, 3], [3, 0]]))
    assert torch.equal(call([20, 20, 20], [0, 1, 2, 3], same, 20, [77, -3]), call([20, 20, 20], [0, 1, 2, 3], same, 20, [3, 0]))


def test_attend_in_a_long_cache_beyond_32_bits():
    # pages whose bytes lie beyond 2^32 from the start
    D, page, Hk = 128, 64, 8
    pages = 36000
    k = torch.zeros((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() * 2 > 1 << 32
    used = [0, pages - 1, pages // 2, pages - 2]
    g = torch.Generator().manual_seed(1)
    q = torch.randn((2, 16, D), generator=g).to(torch.bfloat16).cuda()
    knew, vnew = (torch.randn((4 * page, Hk, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    slot = torch.cat([torch.arange(page) + p * page for p in used]).to(torch.int64).cuda()
    cache = fr.KvPages(k, v)
    fr.fr_kv_append(cache, knew, vnew, slot, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(k[used], knew.view(4, page, Hk, D).transpose(1, 2)) and torch.equal(v[used], vnew.view(4, page, Hk, D).transpose(1, 2))
    assert int((k != 0).sum()) == int((knew != 0).sum())
    own = [100, 30]
    table = torch.tensor([[pages - 1, 0], [pages - 2, 0]], dtype=torch.int32)
    prefix_pages = torch.tensor([pages // 2, 0], dtype=torch.int32)
    out, lse = torch.zeros_like(q), torch.zeros(2, 16, device="cuda")
    lim = dict(prefix_len=70, max_own_len=100, max_q=1)
    ws = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(cache, q, 2, **lim)), dtype=torch.uint8, device="cuda")
    fr.fr_attend_shared(cache, q, out, table.cuda(), torch.tensor(own, dtype=torch.int32, device="cuda"), D ** -0.5,
                        prefix_pages=prefix_pages.cuda(), lse=lse, workspace=ws, stream=torch.cuda.current_stream(), **lim)
    torch.cuda.synchronize()
    place = {p: i for i, p in enumerate(used)}
    small = lambda x: torch.tensor([[place.get(int(y), 0) for y in r] for r in x], dtype=torch.int32)
    _check_attend("bf16", q, k[used], v[used], small(prefix_pages[None])[0], small(table), 70, own, np.array([0, 1, 2]), D ** -0.5, out, lse)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hk,D,page,P,own,new", [
    (4, 1, 128, 16, 8200, [50, 61], [41, 40]),                     # two questions about a long document
    (4, 1, 64, 16, 2100, [70, 66, 0, 33, 1, 64, 50, 90], [64, 40, 0, 33, 1, 64, 50, 64]),
    (3, 1, 128, 8, 300, [60] * 12, [50] * 12),                     # many about a short one
    (8, 2, 64, 32, 3000, [200], [170]),                            # a prompt that goes on
    (4, 2, 128, 16, 0, [1999, 10, 500], [100, 10, 0]),
    (2, 2, 64, 16, 4000, [0, 0, 0], [45, 60, 1]),                  # nothing but the document
    # and where the document is gone through once for all of them
    (8, 2, 128, 16, 8200, [50, 61], [41, 40]),
    (8, 2, 64, 16, 2048, [70, 66, 60, 33, 1, 64, 50, 90], [40, 40, 37, 33, 1, 40, 40, 40]),
    (8, 8, 64, 16, 4000, [0, 0, 0], [45, 60, 1]),
])
def test_attend_questions_about_a_document(dt, Hq, Hk, D, page, P, own, new):
    print("attend questions", dt, Hq, Hk, D, page, P, own, new, flush=True)
    _attend_case(dt, Hq, Hk, D, page, P, own, new, seed=P + len(own), spoil=math.nan)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hk,D,page,P,n,most,tokens", [
    # few rows, a long prefix
    (8, 8, 128, 16, 6000, 3, 77, 1),
    (12, 6, 64, 8, 9000, 3, 77, 4),
    (3, 3, 128, 16, 9000, 3, 0, 1),
    # more, the prefix' rows in tiles of 128
    (16, 8, 64, 16, 1500, 40, 200, 1),
    (15, 5, 64, 8, 5001, 9, 300, 3),
    (8, 8, 128, 16, 3000, 40, 9, 1),
    (16, 8, 128, 32, 700, 64, 100, 1),
    (8, 2, 64, 16, 1200, 70, 300, 2),
    # many short ones by themselves, behind a few shared keys, and not quite as many
    (8, 8, 64, 16, 0, 130, 200, 1),
    (16, 16, 128, 16, 0, 70, 256, 2),
    (8, 8, 128, 64, 40, 130, 150, 1),
    (8, 8, 128, 16, 0, 60, 700, 1),
])
def test_attend_ways_to_cut_few_rows(dt, Hq, Hk, D, page, P, n, most, tokens):
    print("attend ways", dt, Hq, Hk, D, page, P, n, most, tokens, flush=True)
    rng = np.random.default_rng(P + n)
    own = [int(x) for x in rng.integers(0, most + 1, n)]
    own[0], own[-1] = most, min(1, most)
    new = [min(max(1, x) if tokens == 1 else x, tokens) for x in own]
    _attend_case(dt, Hq, Hk, D, page, P, own, new, seed=n, spoil=math.nan)


def test_attend_on_another_stream_masked_and_captured():
    print("attend streams", flush=True)
    side = torch.cuda.Stream()
    a, _ = _attend_case("bf16", 8, 2, 128, 16, 900, [300, 40, 7], [1, 1, 1], 31)
    b, _ = _attend_case("bf16", 8, 2, 128, 16, 900, [300, 40, 7], [1, 1, 1], 31, stream=side)
    assert torch.equal(a, b)
    ctx = fr.Context(device_id=0, cu_count=16)
    _attend_case("bf16", 8, 2, 128, 16, 900, [300, 40, 7], [1, 1, 1], 31, stream=ctx.fr_side_stream())
    ctx.fr_destroy()


# ---------------------------------------------------------------- sample

def _sample(logits, uniform, **settings):
    n = logits.shape[0]
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((max(1, fr.fr_sample_workspace_bytes(logits)),), 255, dtype=torch.uint8, device="cuda")
    kinds = dict(temperature=torch.float32, top_k=torch.int32, top_p=torch.float32, min_p=torch.float32)
    s = {k: torch.tensor(x, dtype=kinds[k], device="cuda") for k, x in settings.items()}
    fr.fr_sample(logits, torch.tensor(uniform, dtype=torch.float32, device="cuda"), token, workspace=ws,
                 stream=torch.cuda.current_stream(), **s)
    torch.cuda.synchronize()
    return token.cpu().numpy()


def _middle(rng, index, w):
    """A random number in the middle of an entry's share, and the entry: shares of 2^-14 and more, so that roundings of
    2^-24 a weight cannot move the choice."""
    run = np.cumsum(w[index])
    share = w[index] / run[-1]
    big = np.flatnonzero(share >= 2.0 ** -14)
    j = int(rng.choice(big)) if len(big) else None
    return (None, None) if j is None else (float((run[j] - w[index][j] / 2) / run[-1]), int(index[j]))


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4099, 32768, 100003, 131072])
def test_sample(dt, V):
    print("sample", dt, V, flush=True)
    rng = np.random.default_rng(V)
    n = 24
    x = 10.0 - 1.7 * np.log1p(np.stack([rng.permutation(V) for _ in range(n)])) + 0.5 * rng.standard_normal((n, V))
    x[rng.random((n, V)) < 0.01] = -np.inf
    x[rng.random((n, V)) < 0.01] = np.nan
    x[np.arange(n), rng.integers(0, V, n)] = 10.0                      # (never a row without a logit)
    logits = torch.from_numpy(x).to(DT[dt]).cuda()
    x = _f64(logits)
    T, K, P, M, U, want = [], [], [], [], [], []
    for r in range(n):
        t = float(np.float32(rng.uniform(0.5, 1.5)))
        k = int(rng.integers(1, min(V, 300) + 1)) if r % 2 else 0
        m = float(np.float32(rng.uniform(0.005, 0.1))) if r % 3 == 1 else 0.0
        p = 1.0
        if r % 4 >= 2:
            # a limit in the middle of an entry's share: the entry is the last one kept
            w, y = oracle.weights(x[r], t)
            order = np.argsort(-y, kind="stable")[: k or V]
            run = np.cumsum(w[order])
            big = np.flatnonzero(w[order] / run[-1] >= 2.0 ** -12)
            j = int(rng.choice(big))
            p = float(np.float32((run[j] - w[order][j] / 2) / run[-1]))
        if m and not np.all(np.abs(oracle.weights(x[r], t)[0] - m) > 1e-5 * m):
            m = 0.0
        index, w = oracle.kept(x[r], t, k, p, m)
        u, token = _middle(rng, index, w)
        T.append(t), K.append(k), P.append(p), M.append(m), U.append(u if u is not None else 0.0), want.append(token)
    got = _sample(logits, U, temperature=T, top_k=K, top_p=P, min_p=M)
    for r in range(n):
        assert want[r] is None or got[r] == want[r], (r, T[r], K[r], P[r], M[r], U[r])


def test_sample_share_of_every_entry():
    # equally spaced random numbers meet an entry as often as its share says
    x = np.array([0.0, 1.0, -2.0, 3.0, -np.inf, 0.5])
    n = 4096
    logits = torch.tensor(np.repeat(x[None], n, 0), dtype=torch.float32, device="cuda")
    got = _sample(logits, (np.arange(n) + 0.5) / n)
    share = np.exp(x - x.max()) / np.exp(x - x.max()).sum()
    assert np.all(np.abs(np.bincount(got, minlength=6) - n * share) <= 1.0 + 1e-3)
    assert np.all(np.diff(got) >= 0)


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
def test_sample_ties_masks_and_empty_rows(dt):
    print("sample ties", dt, flush=True)
    V, low = 5000, float(torch.finfo(DT[dt]).min)
    rows = {
        "equal": np.full(V, 1.25), "lowest": np.full(V, low), "nothing": np.full(V, -np.inf), "nan": np.full(V, np.nan),
        "zeros": np.where(np.arange(V) % 2, 0.0, -0.0), "infinite": np.where(np.arange(V) % 1000 == 7, np.inf, 1.0),
        "one": np.where(np.arange(V) == 4321, 2.0, -np.inf), "half": np.where(np.arange(V) < 100, low, 3.0),
    }
    x = torch.from_numpy(np.stack(list(rows.values()))).to(DT[dt]).cuda()
    n = len(rows)
    name = {k: i for i, k in enumerate(rows)}
    got = _sample(x, [0.5] * n, temperature=[0.0] * n)
    assert list(got) == [0, 0, -1, -1, 0, 7, 4321, 100]                 # the largest logit, the lowest index
    got = _sample(x, [0.50005] * n)
    assert list(got) == [2500, 2500, -1, -1, 2500, 2007, 4321, 100 + int(0.50005 * 4900)]
    got = _sample(x, [0.9999] * n, top_k=[10] * n)                      # ten of equals: the lowest indices
    assert list(got) == [9, 9, -1, -1, 9, 4007, 4321, 109]
    got = _sample(x, [0.9999] * n, top_p=[0.1001] * n)                  # 501 of 5000, one of five, 491 of 4900
    assert list(got) == [500, 500, -1, -1, 500, 7, 4321, 590]
    got = _sample(x, [0.9999] * n, top_k=[100] * n, top_p=[0.4951] * n)
    assert list(got) == [49, 49, -1, -1, 49, 2007, 4321, 149]
    got = _sample(x, [0.9999] * n, min_p=[5.0] * n, top_k=[3] * n)      # (above 1 counts as 1)
    assert list(got) == [2, 2, -1, -1, 2, 2007, 4321, 102]
    got = _sample(x, [1.0, 2.0, 0.0, 0.0, math.nan, -3.0, math.inf, 0.0])
    assert list(got) == [4999, 4999, -1, -1, 0, 7, 4321, 100]
    got = _sample(x, [0.0] * n, top_p=[0.0] * n)                        # one entry at least
    assert list(got) == [0, 0, -1, -1, 0, 7, 4321, 100]


def test_sample_extreme_temperatures_and_ranges():
    x = np.concatenate([[3e38, -3e38, 0.0], np.linspace(-50, 50, 997)])
    logits = torch.tensor(np.stack([x] * 4), dtype=torch.float32, device="cuda")
    assert list(_sample(logits, [0.9] * 4, temperature=[1e-30, 1e-42, 1.0, math.nan])) == [0, 0, 0, 0]
    flat = torch.tensor([[1.0, 2.0, 3.0, -math.inf]] * 4, device="cuda")
    assert list(_sample(flat, [0.1, 0.5, 0.9, 0.999], temperature=[math.inf] * 4)) == [0, 1, 2, 2]
    assert list(_sample(flat, [0.1, 0.9, 0.1, 0.9], temperature=[math.inf] * 4, top_k=[2, 2, 1, 1])) == [1, 2, 2, 2]


def test_sample_strides_offsets_and_a_flat_row():
    V = 131072
    g = torch.Generator().manual_seed(5)
    for dt in ("bf16", "f32"):
        wide = (torch.rand((5, V + 37), generator=g) * 0.25).to(DT[dt]).cuda()
        for off in (0, 1, 3, 8):
            view = wide[:, off:off + V]
            x = _f64(view)
            for k, p in ((0, 1.0), (70000, 1.0), (0, 0.75), (60000, 0.5)):
                index = [oracle.kept(x[r], 1.0, k, p)[0] for r in range(5)]
                got = _sample(view, [0.0, 0.25, 0.5, 0.75, 1.0], temperature=[1.0] * 5, top_k=[k] * 5, top_p=[p] * 5)
                for r in range(5):                      # flat: the place is known to some entries
                    run = np.cumsum(oracle.weights(x[r], 1.0)[0][index[r]])
                    at = min(np.searchsorted(run, [0.0, 0.25, 0.5, 0.75, 1.0][r] * run[-1], side="right"), len(run) - 1)
                    j = np.searchsorted(index[r], got[r])
                    assert abs(int(j) - int(at)) <= 4 and abs(int(got[r]) - int(index[r][at])) <= 64


def _both_ways(logits, uniform, k, p, m, T):
    """The same rows, once as they are and once with a limit on the count that only leaves out an entry without mass: a limit beyond
    1024 of a large vocabulary sends a row through every step of the long way."""
    n, V = logits.shape
    a = _sample(logits, uniform, temperature=T, top_k=k, top_p=p, min_p=m)
    b = _sample(logits, uniform, temperature=T, top_k=[x if x else V - 1 for x in k], top_p=p, min_p=m)
    assert np.array_equal(a, b), [(r, k[r], p[r], m[r], T[r], a[r], b[r]) for r in np.flatnonzero(a != b)][:5]
    return a


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [6000, 50021, 131072, 300001])
def test_sample_by_every_way_gives_the_same(dt, V):
    print("sample ways", dt, V, flush=True)
    rng = np.random.default_rng(V + 1)
    n = 40
    fall = rng.uniform(0.0, 3.0, (n, 1))                               # from flat rows to steep ones
    x = 12.0 - fall * np.log1p(np.stack([rng.permutation(V) for _ in range(n)])) + 0.3 * rng.standard_normal((n, V))
    x[rng.random((n, V)) < 0.002] = np.nan
    x[5] = np.round(x[5])                                              # many equal ones
    x[6] = np.sort(x[6])                                               # the largest side by side
    x[7, : V // 2] = -60.0
    x[:, V // 3] = -np.inf
    logits = torch.from_numpy(x).to(DT[dt]).cuda()
    for rounds in range(3):
        p = [float(np.float32(y)) for y in rng.choice([1.0, 0.3, 0.7, 0.9, 0.95, 0.99, 0.9999], n)]
        m = [float(np.float32(y)) for y in rng.choice([0.0, 0.0, 0.02, 0.3], n)]
        T = [float(np.float32(y)) for y in rng.choice([1.0, 0.3, 0.7, 1.5, 20.0], n)]
        u = list(rng.random(n))
        got = _both_ways(logits, u, [0] * n, p, m, T)
        assert got.min() >= 0 and not np.any(np.isnan(x[np.arange(n), got]))
        # and where the kept entries end exactly at an entry, as nearly as 32 bits of p can say
        q = []
        for r in range(n):
            w, y = oracle.weights(_f64(logits[r]), T[r])
            run = np.cumsum(np.sort(w)[::-1])
            q.append(float(np.float32(run[min(int(rng.integers(0, 400)), V - 1)] / run[-1])))
        _both_ways(logits, [0.999999] * n, [0] * n, q, [0.0] * n, T)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_sample_counts_beyond_a_thousand_and_equal_entries_at_the_end(dt):
    print("sample counts", dt, flush=True)
    rng = np.random.default_rng(9)
    V, n = 70001, 12
    x = 8.0 - 1.1 * np.log1p(np.stack([rng.permutation(V) for _ in range(n)]))
    x[:, 100:30000] = 2.0                                              # a third of the entries are equal
    logits = torch.from_numpy(x).to(DT[dt]).cuda()
    x = _f64(logits)
    K = [1, 2, 50, 1000, 1024, 1025, 3000, 20000, 40000, 70000, 70001, 0]
    for u in (0.0, 0.9999999):
        got = _sample(logits, [u] * n, temperature=[50.0] * n, top_k=K)
        for r in range(n):                              # nearly equal weights: the first and the last of the kept indices
            index, _ = oracle.kept(x[r], 50.0, K[r])
            assert got[r] == (index[0] if u == 0.0 else index[-1]), (r, K[r])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5000, 70003, 131072])
def test_sample_flat_rows_of_every_width(dt, V):
    # From rows of nearly equal entries, of which thousands are a cut's last ones, to rows over a wide range.  A 32-bit weight is off by
    # less than 2^-20 of itself here ((x - top) by 2^-24 of at most 16, its product by as much, exp by 2^-23), so the place of a number
    # is off by less than 2^-20 of the mass, and by four entries at the end where a limit falls between them.
    print("sample widths", dt, V, flush=True)
    rng = np.random.default_rng(V)
    width = np.array([0.0, 0.001, 0.015, 0.03, 0.1, 0.3, 1.0, 3.0, 8.0, 16.0])
    n = len(width)
    logits = torch.from_numpy(rng.random((n, V)) * width[:, None] - 3.0).to(DT[dt]).cuda()
    x = _f64(logits)
    u = [0.1, 0.3, 0.5, 0.7, 0.99] * 2
    for k, p, m in ((0, 0.9, 0.0), (0, 0.3, 0.0), (V // 2, 1.0, 0.0), (V // 3, 0.8, 0.0), (2000, 1.0, 0.0), (2000, 0.5, 0.0), (0, 0.95, 0.25), (0, 1.0, 0.3),
                    (V - 1, 0.999, 0.0)):
        p, m = float(np.float32(p)), float(np.float32(m))
        got = _sample(logits, u, temperature=[1.0] * n, top_k=[k] * n, top_p=[p] * n, min_p=[m] * n)
        for r in range(n):
            w = oracle.weights(x[r], 1.0)[0]
            index = oracle.kept(x[r], 1.0, k, p, m)[0]
            run, last = np.cumsum(w[index]), w[index].min()
            slack, at = 2.0 ** -20 * run[-1] + 4 * last, float(np.float32(u[r])) * run[-1]
            j = int(np.searchsorted(index, got[r]))
            before = run[j - 1] if j else 0.0
            assert before - slack <= at <= before + w[got[r]] + slack, (r, k, p, m, before, at, run[-1])
            assert w[got[r]] >= last * (1 - 2.0 ** -19), (r, k, p, m)


# ---------------------------------------------------------------- graphs

def test_a_captured_step_replays():
    D, Hk, Hq, page, n, V = 128, 2, 8, 16, 5, 4099
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    ck, cv = rnd(24, Hk, page, D), rnd(24, Hk, page, D)
    cache = fr.KvPages(ck, cv)
    q, k, v, logits = rnd(n, Hq, D), rnd(n, Hk, D), rnd(n, Hk, D), rnd(n, V)
    table = torch.arange(4, 24, dtype=torch.int32).view(n, 4).cuda()
    prefix, own = torch.arange(4, dtype=torch.int32).cuda(), torch.tensor([3, 17, 0, 33, 60], dtype=torch.int32).cuda()
    rotary, position = torch.randn(200, D, generator=g).cuda(), (own + 60).int()
    lim = dict(prefix_len=60, max_own_len=64)
    ws = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(cache, q, n, **lim)), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(max(1, fr.fr_sample_workspace_bytes(logits)), dtype=torch.uint8, device="cuda")
    qr, out, token, uniform = torch.empty_like(q), torch.empty_like(q), torch.empty(n, dtype=torch.int32, device="cuda"), torch.rand(n, generator=g).cuda()
    slot, length = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")

    def step():
        s = torch.cuda.current_stream()
        fr.fr_kv_append(cache, k, v, slot, q=q, q_out=qr, position=position, rotary=rotary, stream=s)
        fr.fr_attend_shared(cache, qr, out, table, length, D ** -0.5, prefix_pages=prefix, workspace=ws, stream=s, **lim)
        fr.fr_sample(logits, uniform, token, workspace=ws2, stream=s)

    def inputs(i):
        length.copy_(own + 1 + i)
        place = (own + i).long()
        slot.copy_(table.long().gather(1, (place // page)[:, None])[:, 0] * page + place % page)
        uniform.copy_(torch.rand(n, generator=torch.Generator().manual_seed(i)).cuda())
        k.copy_(torch.randn((n, Hk, D), generator=torch.Generator().manual_seed(i)).cuda())
    inputs(0)
    warm = torch.cuda.Stream()
    with torch.cuda.stream(warm):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        inputs(i)
        torch.cuda.synchronize()
        out.zero_(), token.zero_()
        graph.replay()
        torch.cuda.synchronize()
        a, b = out.clone(), token.clone()
        out.zero_(), token.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, token) and bool(out.any())

"""GPU parity of the operators of a cache held in 8 bits against the fp64 oracle: fr_kv8_append, fr_attend_kv8, fr_kv_copy_pages."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2409_06941_amd as fr              # noqa: E402
from oracle import cache8, generation          # noqa: E402

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # half an ulp of 8 and of 11 significant bits
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -25}        # half the smallest subnormal
I32 = torch.int32


def _f64(x):
    return x.detach().double().cpu().numpy()


def _codes_like(a, b):
    """Codes that are the same number, any NaN counting as NaN."""
    return np.array_equal(np.where(a & 127 == 127, 127, a), np.where(b & 127 == 127, 127, b))


def _views(arrays, layout):
    """[pages, heads, slots, dim] (or [pages, heads, blocks]) tensors on the GPU, lying as `layout` says."""
    x = [torch.from_numpy(a).cuda() for a in arrays]
    if layout == "slots":                              # the heads of a slot side by side
        return [y.transpose(1, 2).contiguous().transpose(1, 2) for y in x]
    if layout == "joined":                             # K and V of a page in one array
        both = torch.stack(x, 1).contiguous()
        return [both[:, 0], both[:, 1]]
    return x


# ---------------------------------------------------------------- append

def _append_case(dt, T, Hq, Hk, D, page, block, R, style, seed, slot=None, pages=None, std=1.0, layout="heads", spread=0.0, bad=(), strided=False, in_place=False,
                 k=None, v=None):
    """slot: where tokens go (default: runs of pages).  spread: how far the tokens' magnitudes lie apart (powers of two, standard deviation)."""
    rng = np.random.default_rng(seed)
    if pages is None:
        pages = -(-T // page) + 3
    if slot is None:
        order = rng.permutation(pages)
        slot = np.array([order[t // page] * page + t % page for t in range(T)])
    slot = np.asarray(slot, dtype=np.int64)
    lo, hi = cache8.RANGE[dt]
    ck, cv = (rng.integers(0, 256, (pages, Hk, page, D)).astype(np.uint8) for _ in range(2))
    sk, sv = (rng.integers(lo + 1, hi + 3, (pages, Hk, page // block)).astype(np.uint8) if seed % 2 else
              rng.integers(115, 125, (pages, Hk, page // block)).astype(np.uint8) for _ in range(2))
    size = std * 2.0 ** np.round(rng.normal(0, spread, (T, 1, 1)))
    make = lambda h: torch.from_numpy(rng.normal(0, 1, (T, h, D)) * size).to(DT[dt])
    k = make(Hk) if k is None else k
    v = make(Hk) if v is None else v
    for t, h, i, x in bad:
        k[t, h, i] = x
        v[t, h, (i + 1) % D] = x
    q = make(Hq)
    if strided:                                        # views of one projection's rows, with something behind them
        row = torch.cat([q, k, v, q], 1).cuda()
        qg, kg, vg = row[:, :Hq], row[:, Hq:Hq + Hk], row[:, Hq + Hk:Hq + 2 * Hk]
    else:
        qg, kg, vg = q.cuda(), k.cuda(), v.cuda()
    positions = 777
    position = torch.from_numpy(rng.integers(0, positions, T)).to(I32)
    angle = rng.random((positions, max(R // 2, 1))) * 6.3
    table = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)[:, :R]).float().contiguous() if R else None
    gk, gv = _views([ck, cv], layout)
    gsk, gsv = _views([sk, sv], "joined" if layout == "joined" else "heads")
    q_out = qg if in_place else torch.full((T, Hq, D), 7.0, dtype=DT[dt], device="cuda")
    fr.fr_kv8_append(fr.Kv8Pages(gk, gv, gsk, gsv, DT[dt]), kg, vg, torch.from_numpy(slot).cuda(), q=qg if Hq else None, q_out=q_out if Hq else None,
                     position=position.cuda() if R else None, rotary=table.cuda() if R else None, style=style, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    cos = _f64(table[position.long()])[:, :R // 2] if R else None
    sin = _f64(table[position.long()])[:, R // 2:] if R else None
    pairs = style == fr.FR_ROTARY_PAIRS
    cache8.append(ck, cv, sk, sv, _f64(k), _f64(v), slot, block, dt, cos, sin, R, pairs)
    # scales and codes are those of the exact numbers: the same bits
    assert np.array_equal(gsk.cpu().numpy(), sk) and np.array_equal(gsv.cpu().numpy(), sv)
    assert _codes_like(gk.cpu().numpy(), ck) and _codes_like(gv.cpu().numpy(), cv)
    got, q0 = _f64(q_out), _f64(q)
    for t in range(T if Hq else 0):
        if not R:
            assert np.array_equal(got[t], q0[t])
            continue
        y = generation.rotate(q0[t], cos[t], sin[t], R, pairs)
        # two products and a sum of 32 bits, then the type's rounding
        e = 3 * 2.0 ** -24 * np.abs(generation.rotate(np.abs(q0[t]), np.abs(cos[t]), -np.abs(sin[t]), R, pairs))
        e = np.maximum(e, 3 * 2.0 ** -24 * np.abs(generation.rotate(np.abs(q0[t]), np.abs(cos[t]), np.abs(sin[t]), R, pairs)))
        near = e + UNIT[dt] * (np.abs(y) + e) + TINY[dt]
        near[:, R:] = 0
        e[:, R:] = 0
        assert np.all(np.abs(got[t] - y) <= near), t


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,Hq,Hk,D,page,block,R,style", [
    (1, 4, 1, 64, 16, 16, 64, 0), (1, 1, 1, 128, 1, 1, 128, 1), (2, 8, 8, 128, 8, 4, 64, 0), (37, 15, 5, 64, 8, 1, 32, 1),
    (65, 3, 3, 64, 32, 32, 48, 0), (129, 32, 8, 128, 16, 16, 128, 0), (130, 7, 1, 128, 64, 64, 16, 1), (9, 0, 2, 64, 4, 2, 64, 0),
    (5, 4, 2, 128, 2, 2, 0, 0), (300, 20, 5, 64, 256, 128, 32, 1), (301, 4, 2, 128, 128, 128, 128, 0), (70, 2, 9, 64, 32, 8, 64, 0)])
def test_append(dt, T, Hq, Hk, D, page, block, R, style):
    print("append", dt, T, Hq, Hk, D, page, block, R, style, flush=True)
    _append_case(dt, T, Hq, Hk, D, page, block, R, style, seed=T + Hq)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("block", [1, 4, 16, 64])
@pytest.mark.parametrize("seed", [2, 3])
def test_append_runs_that_begin_and_end_anywhere(dt, block, seed):
    # sequences go on in the middle of a block: a token each, a few, over several blocks; scales that grow and that do not
    print("append runs", dt, block, seed, flush=True)
    rng = np.random.default_rng(seed)
    page, D = 64, 128 if block > 4 else 64
    runs = [1, 1, 1, 2, 3, 15, 16, 17, 40, 64, 65, 100, 1, 5]
    order, slot, at = rng.permutation(4 * len(runs)), [], 0
    for n in runs:
        begin = int(rng.integers(0, page))
        slot += [int(order[at + (begin + i) // page]) * page + (begin + i) % page for i in range(n)]
        at += 4
    _append_case(dt, len(slot), 4, 2, D, page, block, D, 0, seed, slot=slot, pages=4 * len(runs), spread=3.0)
    _append_case(dt, len(slot), 0, 3, D, page, block, D // 2, 1, seed + 10, slot=slot, pages=4 * len(runs), std=2.0 ** -6)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_append_the_ends_of_the_range(dt):
    # from the type's smallest numbers to its largest, zeros, and numbers next to a change of the scale
    print("append ends", dt, flush=True)
    info = torch.finfo(DT[dt])
    D, values = 64, []
    top = 1.75 * 2.0 ** np.arange(-20, 16) if dt == "f16" else 1.75 * 2.0 ** np.arange(-100, 120, 7)
    for x in [0.0, info.smallest_normal, info.max, info.tiny * info.eps, *top]:
        x = min(float(x), info.max)
        values += [x, float(torch.nextafter(torch.tensor(x, dtype=torch.float32), torch.tensor(0.0))), x * 1.01]
    k = torch.zeros(len(values), 1, D, dtype=torch.float64)
    k[:, 0, 5] = torch.tensor(values, dtype=torch.float64).clamp(max=info.max)
    k[:, 0, 6] = -k[:, 0, 5] / 3
    k[:, 0, 7:] = k[:, 0, 5:6] * torch.logspace(0, -7, D - 7, base=10.0, dtype=torch.float64)
    k = k.to(DT[dt])
    for block in (1, 4):
        _append_case(dt, len(values), 1, 1, D, 16, block, 0, 0, 4, k=k.clone(), v=-k.clone())
    _append_case(dt, len(values), 1, 1, D, 16, 1, 64, 0, 5, k=k.clone(), v=k.clone())


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_append_every_number_near_a_border_between_codes(dt):
    # all numbers of the type between 2^-10 and 1: ties to even among them, and all codes
    print("append borders", dt, flush=True)
    lo, hi = (int(torch.tensor(x, dtype=DT[dt]).view(torch.int16)) for x in (2.0 ** -11, 1.0))
    bits = torch.arange(lo, hi + 1, dtype=torch.int16)
    D = 64
    n = -(-len(bits) // (D - 1))
    x = torch.zeros(n * (D - 1), dtype=DT[dt])
    x[: len(bits)] = bits.view(DT[dt])
    k = torch.cat([torch.full((n, 1), 448 / 512.0, dtype=DT[dt]), x.view(n, D - 1)], 1)[:, None, :].contiguous()
    _append_case(dt, n, 0, 1, D, 16, 1, 0, 0, 6, k=k, v=-k)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_append_what_is_not_finite(dt):
    inf, nan = math.inf, math.nan
    bad = [(0, 0, 0, inf), (3, 1, 5, -inf), (4, 0, 63, nan), (17, 1, 62, nan), (18, 1, 1, inf)]
    _append_case(dt, 30, 2, 2, 64, 16, 8, 64, 0, 7, bad=bad)
    _append_case(dt, 30, 2, 2, 64, 16, 1, 32, 1, 8, bad=bad)
    k = torch.full((3, 1, 64), nan, dtype=DT[dt])      # nothing finite in a block: the least scale
    _append_case(dt, 3, 1, 1, 64, 16, 16, 0, 0, 9, k=k, v=torch.full_like(k, inf))


@pytest.mark.parametrize("layout", ["heads", "slots", "joined"])
@pytest.mark.parametrize("strided,in_place", [(True, False), (True, True), (False, True)])
def test_append_layouts_strides_and_in_place(layout, strided, in_place):
    print("append", layout, strided, in_place, flush=True)
    _append_case("bf16", 19, 6, 2, 128, 16, 8, 128, 0, 5, layout=layout, strided=strided, in_place=in_place)
    _append_case("f16", 19, 6, 2, 64, 16, 2, 32, 1, 6, layout=layout, strided=strided, in_place=in_place)


def test_append_leaves_padding_out():
    far = 1 << 40
    slot = np.arange(40)
    for i, x in [(0, -1), (3, -far), (17, 72), (39, far), (20, (1 << 63) - 1), (21, -(1 << 63))]:
        slot[i] = x
    _append_case("bf16", 40, 4, 2, 64, 8, 1, 64, 0, 8, slot=slot, pages=9)
    _append_case("bf16", 8, 4, 2, 64, 8, 8, 64, 0, 8, slot=[-1, -1, 8, 9, 10, -1, 71, 72], pages=9)
    _append_case("bf16", 2, 4, 2, 64, 8, 8, 64, 0, 8, slot=[-5, 1 << 50], pages=9)


def test_append_positions_outside_the_table_and_empty_calls():
    D, T = 64, 4
    k = torch.randn(T, 1, D, device="cuda").to(torch.bfloat16)
    codes = lambda: torch.zeros(2, 1, 4, D, dtype=torch.uint8, device="cuda")
    ck, cv, sk, sv = codes(), codes(), torch.zeros(2, 1, 1, dtype=torch.uint8, device="cuda"), torch.zeros(2, 1, 1, dtype=torch.uint8, device="cuda")
    table = torch.randn(3, D, device="cuda")
    cache, slot = fr.Kv8Pages(ck, cv, sk, sv, torch.bfloat16), torch.arange(T, device="cuda")
    fr.fr_kv8_append(cache, k, k, slot, position=torch.tensor([-5, 0, 2, 1 << 30], dtype=I32, device="cuda"), rotary=table)
    a = ck.clone()
    fr.fr_kv8_append(cache, k, k, slot, position=torch.tensor([0, 0, 2, 2], dtype=I32, device="cuda"), rotary=table)
    torch.cuda.synchronize()
    assert torch.equal(a, ck) and bool((a[0] != 0).any())
    fr.fr_kv8_append(cache, k[:0], k[:0], slot[:0], position=slot[:0].int(), rotary=table)
    torch.cuda.synchronize()
    assert torch.equal(a, ck)


# ---------------------------------------------------------------- attend

def _attend_case(dt, Hq, Hk, D, page, block, lens, new, seed, window=0, sinks=0, layout="heads", q_begin=True, strided=False, scale=None, std=1.0, stream=None,
                 extra=3, scales=(117, 122), nan_at=(), max_len=None, rows=None):
    """lens, new: keys and new tokens of every sequence.  Slots behind a length, and pages that no token sees, hold NaN codes and any scale.
    nan_at: (sequence, key, first element, is it V) whose codes are NaN."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    counts = [-(-x // page) for x in lens]
    pages = sum(counts) + extra
    width = max(1, -(-(max(lens + [0]) if max_len is None else max_len) // page)) + 1
    order = rng.permutation(pages)
    table = np.full((n, width), 1 << 30, dtype=np.int32)               # ids of pages that are not seen lead nowhere
    used = np.zeros((pages, page), dtype=bool)
    draws = cache8.encode(rng.normal(0, 100, 1 << 16))
    ck, cv = (draws[rng.integers(0, 1 << 16, (pages, Hk, page, D), dtype=np.uint16)] for _ in range(2))
    sk, sv = (rng.integers(scales[0], scales[1] + 1, (pages, Hk, page // block)).astype(np.uint8) for _ in range(2))
    at = 0
    place = []
    for b, c in enumerate(counts):
        ids = order[at:at + c]
        at += c
        first = max(0, lens[b] - new[b] + 1 - window) if window else 0
        j = np.arange(lens[b])
        j = j[(j >= first) | (j < sinks)] if window else j
        table[b, np.unique(j // page)] = ids[np.unique(j // page)]
        used[ids[j // page], j % page] = True
        place.append(ids)
    for codes in (ck, cv):
        codes[np.broadcast_to(~used[:, None, :], (pages, Hk, page))] = 0x7f
    any_scale = ~used.reshape(pages, page // block, block).any(2)
    for s in (sk, sv):
        s[np.broadcast_to(any_scale[:, None, :], s.shape)] = 255
    for b, j, e, value in nan_at:
        (cv if value else ck)[place[b][j // page], :, j % page, e:e + 5] = 0xff
    gk, gv = _views([ck, cv], layout)
    gsk, gsv = _views([sk, sv], layout)
    begin = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(begin[-1])
    q = torch.from_numpy(rng.normal(0, std, (T, Hq + (2 if strided else 0), D))).to(DT[dt]).cuda()[:, :Hq]
    out = torch.full((T, Hq + (1 if strided else 0), D), 9.0, dtype=DT[dt], device="cuda")[:, :Hq]
    lse = torch.full((T, Hq), 9.0, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    cache = fr.Kv8Pages(gk, gv, gsk, gsv, DT[dt])
    lim = dict(max_len=max(lens + [0]) if max_len is None else max_len, max_q=max(max(new), 1) if q_begin else 1, window=window, sinks=sinks)
    need = fr.fr_attend_kv8_workspace_bytes(cache, q, n, **lim)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")      # (NaNs, in whatever type it is read)
    torch.cuda.synchronize()
    fr.fr_attend_kv8(cache, q, out, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=I32, device="cuda"), scale,
                     q_begin=torch.from_numpy(begin).cuda() if q_begin else None, lse=lse, workspace=ws, stream=stream or torch.cuda.current_stream(), **lim)
    torch.cuda.synchronize()
    _check_attend(dt, q, Numbers(ck, sk, block, dt), Numbers(cv, sv, block, dt), place, page, lens, begin, window, sinks, scale, out, lse, rows)
    return out, lse


class Numbers:
    """What codes and scales stand for, made where they are asked for: [pages, a head, slots]."""

    def __init__(self, codes, scale, block, dt):
        self.codes, self.scale, self.block, self.dt, self.shape = codes, scale, block, dt, codes.shape

    def __getitem__(self, at):
        p, h, o = at
        return cache8.VALUES[self.codes[p, h, o]] * cache8.scale_of(self.scale[p, h, o // self.block], self.dt)[:, None]


def _check_attend(dt, q, K, V, place, page, lens, begin, window, sinks, scale, out, lse, rows=None):
    """rows: check only about so many rows, spread over all."""
    Hq, Hk = q.shape[1], K.shape[1]
    q64, o64, l64, u = _f64(q), _f64(out), _f64(lse), UNIT[dt]
    every = 1 if rows is None else max(1, q64.shape[0] * Hq // rows)
    count = 0
    for b in range(len(lens)):
        t = int(begin[b + 1] - begin[b])
        j = np.arange(lens[b])
        for h in range(Hq):
            kk = vv = None
            for i in range(t):
                count += 1
                if every > 1 and count % every and i not in (0, t - 1):
                    continue
                if kk is None:
                    kk, vv = K[place[b][j // page], h // (Hq // Hk), j % page], V[place[b][j // page], h // (Hq // Hk), j % page]
                see, row = cache8.seen(lens[b], t, i, window, sinks), int(begin[b]) + i
                o, l, a, x = generation.attend_row(q64[row, h], kk[see], vv[see], scale)
                n = len(see)
                if n == 0:
                    assert not o64[row, h].any() and l64[row, h] == -math.inf, (b, i, h)
                    continue
                if not np.isfinite(o).all() or not np.isfinite(l):
                    assert np.array_equal(np.isnan(o64[row, h]), np.isnan(o)) and np.isnan(l64[row, h]) == np.isnan(l), (b, i, h)
                    o, a = o[~np.isnan(o)], a[~np.isnan(o)]
                    if np.isnan(l) or not o.size:
                        continue
                # scores: sums of D products of 32 bits; each weight off by that, by a few ulps of exp, and by the type's rounding; sums of n of
                # them; the result's rounding.  Weights of fp16 end at 2^-32 of the largest.  (What the codes stand for is exact.)
                d = (q64.shape[2] + 4) * 2.0 ** -24 * x + 2.0 ** -20
                got = o64[row, h][~np.isnan(o64[row, h])]
                big = np.nanmax(np.abs(vv[see]))
                near = (u + 2 * d + n * 2.0 ** -23) * a + u * np.abs(o) * 1.01 + TINY[dt] + (n * 2.0 ** -32 * big if dt == "f16" else 0.0)
                assert np.all(np.abs(got - o) <= near), (b, i, h, np.abs(got - o).max(), near.max())
                assert abs(l64[row, h] - l) <= d + n * 2.0 ** -23 + 2.0 ** -20 * (1 + abs(l)), (b, i, h)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hk,D,page,block,lens,new", [
    (1, 1, 64, 1, 1, [1], [1]),                                    # one key of one sequence
    (4, 2, 128, 16, 16, [0, 1, 15, 16, 17], [1, 1, 1, 1, 1]),      # a sequence that sees nothing; pages that end
    (8, 2, 64, 16, 4, [1, 30, 16], [1, 1, 1]),
    (8, 8, 128, 8, 2, [31, 32, 33, 63, 64, 65], [1] * 6),
    (15, 5, 64, 8, 1, [3, 0, 77, 129], [3, 0, 2, 7]),
    (12, 1, 128, 32, 32, [65, 64, 63, 1], [1, 1, 1, 1]),
    (3, 3, 128, 64, 8, [2, 300], [2, 5]),
    (32, 2, 64, 4, 4, [5] * 9, [2] * 9),
    (40, 1, 128, 16, 1, [33, 2], [3, 2]),                          # forty heads to a key
    (6, 2, 128, 16, 8, [130, 70], [130, 70]),                      # prompts alone
    (4, 2, 64, 16, 16, [150, 9, 260], [70, 9, 33]),
    (16, 4, 128, 256, 128, [740, 33], [140, 33]),
    (2, 1, 64, 16, 2, [2, 5], [4, 5]),                             # more tokens than keys: the first see nothing
    (2, 1, 128, 16, 16, [2, 0], [4, 3])])
def test_attend(dt, Hq, Hk, D, page, block, lens, new):
    print("attend", dt, Hq, Hk, D, page, block, lens, new, flush=True)
    _attend_case(dt, Hq, Hk, D, page, block, lens, new, seed=Hq + page)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (31, 0), (32, 32), (33, 33), (64, 4), (65, 63), (100, 64), (100, 65), (128, 130),
                                          (1000, 0), (1 << 30, 5), (2, 1 << 30), (0, 9)])
def test_attend_windows(dt, window, sinks):
    print("attend window", dt, window, sinks, flush=True)
    lens = [0, 1, 2, 40, 64, 65, 100, 127, 128, 129, 200, 333, 700]
    _attend_case(dt, 6, 2, 128, 16, 4, lens, [1] * len(lens), window + 1, window, sinks)
    _attend_case(dt, 4, 1, 64, 8, 1, lens, [min(n, 5) for n in lens], window + 2, window, sinks)
    _attend_case(dt, 4, 2, 128, 32, 16, [40, 129, 333], [40, 100, 90], window + 3, window, sinks)
    _attend_case(dt, 2, 2, 64, 16, 8, [260, 64], [260, 30], window + 4, window, sinks)


@pytest.mark.parametrize("lens,new,window,sinks", [([2900, 5, 0], [1, 1, 1], 0, 0), ([4097, 1, 640], [1, 1, 1], 2000, 3), ([50] * 40, [1] * 40, 0, 0),
                                                   ([5700, 20], [5, 7], 3000, 70), ([5000, 4095, 4096], [1, 1, 1], 0, 0), ([1600, 300], [300, 300], 0, 0),
                                                   ([1600, 700], [300, 700], 256, 10)])
def test_attend_longer(lens, new, window, sinks):
    print("attend longer", lens, new, window, sinks, flush=True)
    _attend_case("bf16", 8, 2, 128, 16, 16, lens, new, 11, window, sinks, rows=300)
    _attend_case("f16", 8, 2, 64, 16, 1, lens, new, 12, window, sinks, rows=300)


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("window,new", [(0, 1), (150, 1), (20, 3)])
def test_attend_many_short_sequences(dt, D, window, new):
    print("attend many", dt, D, window, new, flush=True)
    rng = np.random.default_rng(window + new)
    lens = [int(x) for x in rng.integers(0, 40, 66)] + [0, 1, 31, 32, 33, 255, 256, 257, 600]
    t = [min(x, int(rng.integers(1, new + 1))) if new > 1 else 1 for x in lens]
    _attend_case(dt, 16, 8, D, 16, 8, lens, t, window + D, window, 2)


def _ragged(kind, seqs, most, rng):
    if kind == "any":
        return [int(x) for x in rng.integers(0, most, seqs - 3)] + [0, 1, most]
    if kind == "equal":
        return [most - int(x) for x in rng.integers(0, 40, seqs)]
    if kind == "one":
        return [0, 3] * (seqs // 2 - 1) + [most, 17]
    return [32 * int(x) for x in rng.integers(0, most // 32, seqs - 1)] + [most]          # whole tiles: items that end where a worker's share does


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("kind,seqs,most,Hq,Hk,new,window", [
    ("any", 16, 8400, 8, 8, 1, 0), ("equal", 16, 8300, 8, 8, 1, 0), ("whole", 16, 8320, 16, 8, 1, 0), ("one", 10, 17000, 20, 5, 1, 0), ("any", 8, 17000, 16, 4, 6, 0),
    ("any", 16, 20000, 8, 8, 1, 9000), ("any", 70, 2100, 12, 4, 7, 0)])
def test_attend_lengths_that_are_dealt_out_evenly(dt, D, kind, seqs, most, Hq, Hk, new, window):
    # many keys in sequences that differ: workers go through several items, and items through several workers
    print("attend dealt", dt, D, kind, seqs, most, Hq, Hk, new, window, flush=True)
    rng = np.random.default_rng(seqs + most)
    lens = _ragged(kind, seqs, most, rng)
    t = [min(n, int(rng.integers(0, new + 1))) if new > 1 else 1 for n in lens]
    _attend_case(dt, Hq, Hk, D, 16, 8, lens, t, most, window, 5 if window else 0, rows=160)


def test_attend_lengths_dealt_out_among_few_units():
    ctx = fr.Context(device_id=0, cu_count=16)
    rng = np.random.default_rng(1)
    for kind, seqs, most, Hq, Hk, new in (("any", 4, 8300, 4, 2, 1), ("any", 3, 17000, 16, 2, 3), ("whole", 4, 8320, 2, 2, 1), ("one", 8, 8300, 3, 1, 1), ("equal", 4, 9000, 2, 2, 1)):
        lens = _ragged(kind, seqs, most, rng)
        t = [min(n, int(rng.integers(0, new + 1))) if new > 1 else 1 for n in lens]
        _attend_case("bf16", Hq, Hk, 64, 16, 16, lens, t, most, stream=ctx.fr_side_stream(), rows=100)
        _attend_case("f16", Hq, Hk, 128, 32, 1, lens, t, most, 8250, 40, stream=ctx.fr_side_stream(), rows=100, nan_at=[(len(lens) - 1, lens[-1] - 1, 3, True)])
    for kind, seqs, most, Hq, Hk, new in (("any", 11, 700, 8, 4, 1), ("any", 40, 300, 6, 3, 5), ("one", 30, 2000, 2, 2, 1)):
        lens = _ragged(kind, seqs, most, rng)
        t = [min(n, int(rng.integers(0, new + 1))) if new > 1 else 1 for n in lens]
        _attend_case("bf16", Hq, Hk, 64, 16, 16, lens, t, most, stream=ctx.fr_side_stream(), rows=400)
        _attend_case("f16", Hq, Hk, 128, 32, 1, lens, t, most, 250, 40, stream=ctx.fr_side_stream(), rows=400)
        _attend_case("bf16", Hq, Hk, 128, 16, 16, lens, t, most, stream=ctx.fr_side_stream(), rows=400, nan_at=[(len(lens) - 1, 2, 3, True)])
    ctx.fr_destroy()


@pytest.mark.parametrize("layout", ["slots", "joined"])
def test_attend_layouts_and_strides(layout):
    print("attend", layout, flush=True)
    _attend_case("bf16", 8, 2, 128, 16, 4, [40, 3, 90], [1, 1, 1], 3, layout=layout, strided=True, q_begin=False)
    _attend_case("f16", 8, 2, 64, 16, 1, [40, 3, 190], [20, 3, 100], 4, 50, 3, layout=layout, strided=True)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D,G,t,window", [(128, 2, 5, 0), (64, 4, 40, 0), (128, 4, 90, 0), (64, 2, 90, 30), (128, 1, 3, 16)])
def test_attend_nan_shows_to_those_that_see_it_alone(dt, D, G, t, window):
    # the last tokens' keys and values, one in the middle and a first one are NaN: tokens that do not see them come out as if they were not there
    print("attend nan", dt, D, G, t, window, flush=True)
    L = t + 20
    nan_at = [(0, L - 1, 3, True), (0, L - 2, 3, False), (0, L - 3, 60, True)]
    _attend_case(dt, 2 * G, 2, D, 16, 8, [L, 30], [t, 1], t, window, 2, nan_at=nan_at)
    if window:
        _attend_case(dt, 2 * G, 2, D, 16, 1, [L, 30], [t, 1], t, window, 2, nan_at=[(0, 22, 3, True), (0, 23, 0, True), (0, L - t // 2, 9, False)])
        _attend_case(dt, 2 * G, 2, D, 16, 1, [L, 30], [t, 1], t, window, 2, nan_at=[(0, 1, 3, True), (1, 0, 0, False)])


@pytest.mark.parametrize("dt,scales", [("bf16", (0, 30)), ("bf16", (225, 255)), ("bf16", (100, 140)), ("f16", (0, 115)), ("f16", (130, 255)), ("f16", (112, 134))])
def test_attend_scales_from_end_to_end(dt, scales):
    # queries as large or small as keep the scores of order one
    print("attend scales", dt, scales, flush=True)
    top = cache8.scale_of(scales[1], dt) * 448
    scale = float(min(1e30, max(1e-30, 1.0 / top / 12)))
    for lens, new in (([40, 3, 190], [1, 1, 1]), ([190, 77], [100, 77])):
        _attend_case(dt, 4, 2, 128, 16, 1, lens, new, 5, scales=scales, scale=scale, std=0.5)
        _attend_case(dt, 4, 2, 64, 16, 16, lens, new, 6, 50, 3, scales=scales, scale=scale, std=0.5)


def test_attend_large_scores_and_scales():
    _attend_case("bf16", 4, 2, 128, 16, 4, [150, 60], [1, 1], 21, std=30.0)
    _attend_case("f16", 4, 2, 64, 16, 4, [150, 60], [2, 9], 22, std=20.0)
    _attend_case("bf16", 4, 2, 64, 16, 16, [150, 60], [1, 1], 23, scale=1e-3)
    _attend_case("bf16", 4, 2, 64, 16, 16, [350, 60], [1, 1], 24, scale=3.0, std=4.0)
    _attend_case("f16", 4, 2, 128, 16, 16, [350, 160], [200, 160], 25, scale=1.0, std=4.0)


def test_attend_numbers_from_the_device_are_bounded():
    # lengths beyond max_len, q_begin beyond n_tokens, page ids outside: results of the bounded numbers, no access outside
    D, page = 64, 16
    codes = [torch.randint(0, 126, (4, 1, page, D), device="cuda", dtype=torch.uint8) for _ in range(2)]
    scale = [torch.full((4, 1, 2), 118, device="cuda", dtype=torch.uint8) for _ in range(2)]
    cache, q = fr.Kv8Pages(*codes, *scale, torch.bfloat16), torch.randn(3, 2, D, device="cuda").to(torch.bfloat16)

    def call(lens, begin, table, **more):
        i32 = lambda x: torch.tensor(x, dtype=I32, device="cuda")
        out = torch.zeros_like(q)
        lim = dict(max_len=32, max_q=1, **more)
        ws = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(cache, q, 3, **lim)), dtype=torch.uint8, device="cuda")
        fr.fr_attend_kv8(cache, q, out, i32(table), i32(lens), 0.125, q_begin=i32(begin), workspace=ws, stream=torch.cuda.current_stream(), **lim)
        torch.cuda.synchronize()
        return out
    same = [[0, 1], [1, 2], [3, 0]]
    assert torch.equal(call([1000, -7, 5], [0, 1, 2, 3], same), call([32, 0, 5], [0, 1, 2, 3], same))
    assert torch.equal(call([9, 9, 5], [-4, 1, 2, 900], same), call([9, 9, 5], [0, 1, 2, 3], same))
    assert torch.equal(call([20, 20, 20], [0, 1, 2, 3], [[-1, 1], [1, 99], [1 << 30, 0]]), call([20, 20, 20], [0, 1, 2, 3], [[0, 1], [1, 3], [3, 0]]))
    # a window and sinks far beyond every length
    big = 0x7fffffff
    assert torch.equal(call([20, 9, 32], [0, 1, 2, 3], same, window=big, sinks=big), call([20, 9, 32], [0, 1, 2, 3], same))
    assert torch.equal(call([20, 9, 32], [0, 1, 2, 3], same, window=3, sinks=big), call([20, 9, 32], [0, 1, 2, 3], same))


@pytest.mark.parametrize("t,n", [(1, 5), (40, 5), (200, 2)])
def test_attend_rows_that_are_in_no_sequence_or_beyond_max_q_stay(t, n):
    D, page, H = 64, 16, 4
    codes = [torch.randint(0, 126, (40, 2, page, D), device="cuda", dtype=torch.uint8) for _ in range(2)]
    scale = [torch.full((40, 2, 4), 118, device="cuda", dtype=torch.uint8) for _ in range(2)]
    cache = fr.Kv8Pages(*codes, *scale, torch.bfloat16)
    T = n * (t + 3) + 7
    q = torch.randn(T, H, D, device="cuda").to(torch.bfloat16)
    begin = [5 + b * (t + 3) for b in range(n + 1)]     # five tokens before the first sequence, two behind the last; three of each beyond max_q
    table = torch.arange(n * 16, device="cuda", dtype=I32).view(n, 16) % 40
    lens = torch.tensor([min(256, t + 3 + 11 * b) for b in range(n)], dtype=I32, device="cuda")
    out, lse = torch.full_like(q, 5.0), torch.full((T, H), 5.0, device="cuda")
    for max_len in (256,):
        lim = dict(max_len=max_len, max_q=t)
        ws = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(cache, q, n, **lim)), dtype=torch.uint8, device="cuda")
        fr.fr_attend_kv8(cache, q, out, table, lens, 0.125, q_begin=torch.tensor(begin, dtype=I32, device="cuda"), lse=lse, workspace=ws, **lim)
    torch.cuda.synchronize()
    computed = torch.zeros(T, dtype=torch.bool)
    for b in range(n):
        computed[begin[b]: begin[b] + t] = True
    stay = ~computed.cuda()
    assert bool((out[stay] == 5).all()) and bool((lse[stay] == 5).all())
    assert not bool((lse[~stay] == 5).any())


def test_attend_in_a_long_cache_beyond_32_bits():
    # pages whose codes lie beyond 2^32 from the start
    D, page, Hk, block = 128, 64, 8, 16
    pages = 70000
    ck = torch.zeros((pages, Hk, page, D), dtype=torch.uint8, device="cuda")
    cv = torch.zeros_like(ck)
    sk, sv = (torch.zeros((pages, Hk, page // block), dtype=torch.uint8, device="cuda") for _ in range(2))
    assert ck.numel() > 1 << 32
    used = np.array([0, pages - 1, pages // 2, pages - 2])
    rng = np.random.default_rng(1)
    q = torch.from_numpy(rng.normal(0, 1, (2, 16, D))).to(torch.bfloat16).cuda()
    k, v = (torch.from_numpy(rng.normal(0, 1, (4 * page, Hk, D))).to(torch.bfloat16).cuda() for _ in range(2))
    slot = torch.from_numpy((used[:, None] * page + np.arange(page)[None, :]).reshape(-1).astype(np.int64)).cuda()
    cache = fr.Kv8Pages(ck, cv, sk, sv, torch.bfloat16)
    fr.fr_kv8_append(cache, k, v, slot)
    lens, table = [4 * page, 3 * page - 5], np.array([used, used[::-1]], dtype=np.int32)
    out, lse = torch.zeros_like(q), torch.zeros(2, 16, device="cuda")
    lim = dict(max_len=4 * page)
    ws = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(cache, q, 2, **lim)), dtype=torch.uint8, device="cuda")
    fr.fr_attend_kv8(cache, q, out, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=I32, device="cuda"), D ** -0.5, lse=lse, workspace=ws, **lim)
    # and a copy from the far end to the start
    extra = torch.tensor([pages - 3], dtype=I32, device="cuda")
    fr.fr_kv_copy_pages(cache, torch.tensor([pages - 1], dtype=I32, device="cuda"), extra)
    torch.cuda.synchronize()
    ids = torch.from_numpy(used).cuda()
    small = [x[ids].cpu().numpy() for x in (ck, cv, sk, sv)]
    want = [np.zeros_like(x) for x in small]
    cache8.append(*want, _f64(k), _f64(v), np.arange(4 * page), block, "bf16")
    for x, y in zip(small, want):
        assert np.array_equal(x, y)
    K, V = cache8.numbers(small[0], small[2], block, "bf16"), cache8.numbers(small[1], small[3], block, "bf16")
    place = [np.array([0, 1, 2, 3]), np.array([3, 2, 1, 0])]
    _check_attend("bf16", q, K, V, place, page, lens, np.array([0, 1, 2]), 0, 0, D ** -0.5, out, lse)
    assert torch.equal(ck[pages - 3], ck[pages - 1]) and torch.equal(sv[pages - 3], sv[pages - 1])
    assert int(ck.view(pages, -1)[1:pages // 2].max()) == 0


# ---------------------------------------------------------------- copy

def _copy_case(caches, source, target, seed, want_copied=True):
    """caches: (8 or 16, heads, page, dim, block, layout) of as many pages."""
    pages, rng = 23, np.random.default_rng(seed)
    tensors, handles = [], []
    for bits, H, page, D, block, layout in caches:
        if bits == 16:
            x = _views([rng.integers(-9999, 9999, (pages, H, page, D)).astype(np.int16) for _ in range(2)], layout)
            x = [y.view(torch.float16) for y in x]
            handles.append(fr.KvPages(*x))
            tensors.append([y.view(torch.int16) for y in x])
        else:
            x = _views([rng.integers(0, 256, (pages, H, page, D)).astype(np.uint8) for _ in range(2)], layout)
            x += _views([rng.integers(0, 256, (pages, H, page // block)).astype(np.uint8) for _ in range(2)], layout)
            handles.append(fr.Kv8Pages(*x, torch.float16))
            tensors.append(x)
    before = [[y.cpu().numpy().copy() for y in x] for x in tensors]
    copied = torch.full((len(source),), 7, dtype=I32, device="cuda") if want_copied else None
    fr.fr_kv_copy_pages(handles, torch.tensor(source, dtype=I32, device="cuda"), torch.tensor(target, dtype=I32, device="cuda"), copied=copied)
    torch.cuda.synchronize()
    do = cache8.copies(source, target, pages)
    if want_copied:
        assert copied.cpu().tolist() == [int(x) for x in do]
    for x, y in zip(tensors, before):
        for a, b in zip(x, y):
            c = b.copy()
            for i, d in enumerate(do):
                if d:
                    c[target[i]] = b[source[i]]
            assert np.array_equal(a.cpu().numpy(), c)


ONE = [(8, 2, 16, 64, 8, "heads")]


@pytest.mark.parametrize("caches", [ONE, [(16, 3, 8, 128, 1, "slots")], [(8, 5, 4, 64, 1, "slots"), (8, 5, 4, 64, 1, "slots")], [(8, 1, 1, 128, 1, "joined")],
                                    [(8, 8, 16, 128, 16, "heads")] * 70, [(16, 2, 16, 64, 1, "joined"), (8, 2, 16, 64, 4, "joined"), (16, 2, 16, 64, 1, "joined"), (8, 3, 8, 128, 2, "heads")]])
def test_copy(caches):
    print("copy", len(caches), caches[0], flush=True)
    _copy_case(caches, [3, 3, 9, 0], [5, 22, 1, 12], 1)
    _copy_case(caches, [22], [0], 2, want_copied=False)


def test_copy_pairs_that_are_left_out():
    big = 0x7fffffff
    _copy_case(ONE, [1, -1, 23, 3, big, 5, 6], [2, 4, 5, 23, 6, -big, 6], 3)             # padding, pages outside, a page with itself
    _copy_case(ONE, [1, 2, 3, 4], [7, 8, 7, 7], 4)                                       # one target of several pairs: the last
    _copy_case(ONE, [1, 2, 3], [2, 3, 4], 5)                                             # a chain: what is written is not read
    _copy_case(ONE, [1, 2], [2, 1], 6)                                                   # a swap
    _copy_case(ONE, [1, 2, 2], [2, 9, 2], 7)                                             # a target that is padding's source
    _copy_case(ONE, [1, 1, 1], [9, 9, 9], 8)
    _copy_case(ONE, [], [], 9)


def test_copy_many_pairs():
    rng = np.random.default_rng(5)
    source = rng.integers(-2, 25, 1500)
    _copy_case(ONE + [(8, 2, 16, 64, 8, "slots")], source.tolist(), rng.integers(-2, 25, 1500).tolist(), 10)
    # so many that a workgroup has several caches: padding but for a few
    for n in (2100, 5000):
        source, target = np.full(n, -1), np.full(n, 3)
        source[[5, n // 2, n - 1]], target[[5, n // 2, n - 1]] = [1, 2, 2], [7, 8, 9]
        _copy_case([(8, 2, 16, 64, 8, "heads")] * 7 + [(16, 1, 4, 64, 1, "heads")] * 3, source.tolist(), target.tolist(), n)


def test_attend_of_nothing_at_all_gives_zeros():
    cache = fr.Kv8Pages(*(torch.zeros(1, 1, 1, 64, dtype=torch.uint8, device="cuda") for _ in range(2)), *(torch.zeros(1, 1, 1, dtype=torch.uint8, device="cuda") for _ in range(2)),
                        torch.float16)
    for t in (1, 40):
        q = torch.ones(3 * t, 2, 64, dtype=torch.float16, device="cuda")
        out, lse = torch.full_like(q, 3.0), torch.zeros(3 * t, 2, device="cuda")
        fr.fr_attend_kv8(cache, q, out, None, None, 0.125, max_len=0, max_q=t, q_begin=torch.arange(0, 3 * t + 1, t, dtype=I32, device="cuda"), lse=lse)
        torch.cuda.synchronize()
        assert not bool(out.any()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("Hq,t", [(1024, 1), (300, 2)])
def test_attend_hundreds_of_heads_to_a_key_head(Hq, t):
    # rows of one token are many: tiles of 128 rows that all see the same keys
    _attend_case("bf16", Hq, 1, 64, 16, 4, [100, 0, 70], [t, 0, t], Hq, 30, 3, rows=300)
    _attend_case("f16", Hq, 1, 128, 16, 16, [300], [t], Hq + 1, rows=300)


# ---------------------------------------------------------------- together

def test_a_prompt_that_forks_and_goes_on():
    # a prompt in two pieces, three sequences that go on from it in pages of their own, a window; every code and every row against the oracle
    dt, Hq, Hk, D, page, block, pages = "bf16", 8, 2, 128, 16, 8, 30
    rng = np.random.default_rng(3)
    oracle = [np.zeros((pages, Hk, page, D), np.uint8), np.zeros((pages, Hk, page, D), np.uint8)] + [np.zeros((pages, Hk, page // block), np.uint8) for _ in range(2)]
    gpu = [torch.from_numpy(x.copy()).cuda() for x in oracle]
    cache = fr.Kv8Pages(*gpu, DT[dt])
    order = rng.permutation(pages)
    tables = np.tile(order[:4], (3, 1)).astype(np.int32)                 # the prompt's pages stand in all tables ...
    tables = np.concatenate([tables, order[4:4 + 9].reshape(3, 3).astype(np.int32)], 1)
    angle = rng.random((200, 32)) * 6.3
    table = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float()

    def run(new, lens, tables, window, sinks):
        """new tokens of every sequence, the last of its lens keys: appended and attended to"""
        T = sum(new)
        q, k, v = (torch.from_numpy(rng.normal(0, 1, (T, h, D)) * 2.0 ** rng.integers(-3, 4, (T, 1, 1))).to(DT[dt]) for h in (Hq, Hk, Hk))
        where = np.concatenate([np.arange(n - t, n) for n, t in zip(lens, new)])
        seq = np.repeat(np.arange(len(new)), new)
        slot = (tables[seq, where // page] * page + where % page).astype(np.int64)
        begin = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        qg, out, lse = q.cuda(), torch.full((T, Hq, D), 9.0, dtype=DT[dt], device="cuda"), torch.zeros(T, Hq, device="cuda")
        fr.fr_kv8_append(cache, k.cuda(), v.cuda(), torch.from_numpy(slot).cuda(), q=qg, q_out=qg, position=torch.from_numpy(where.astype(np.int32)).cuda(), rotary=table.cuda())
        lim = dict(max_len=max(lens), max_q=max(new), window=window, sinks=sinks)
        ws = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(cache, qg, len(new), **lim)), dtype=torch.uint8, device="cuda")
        fr.fr_attend_kv8(cache, qg, out, torch.from_numpy(np.ascontiguousarray(tables)).cuda(), torch.tensor(lens, dtype=I32, device="cuda"), D ** -0.5,
                         q_begin=torch.from_numpy(begin).cuda(), lse=lse, workspace=ws, **lim)
        torch.cuda.synchronize()
        cache8.append(*oracle, _f64(k), _f64(v), slot, block, dt, _f64(table)[where, :32], _f64(table)[where, 32:], 64, False)
        for a, b in zip(gpu, oracle):
            assert np.array_equal(a.cpu().numpy(), b)
        K, V = cache8.numbers(oracle[0], oracle[2], block, dt), cache8.numbers(oracle[1], oracle[3], block, dt)
        _check_attend(dt, qg, K, V, [t for t in tables], page, lens, begin, window, sinks, D ** -0.5, out, lse)

    run([33], [33], tables[:1], 0, 0)
    run([26], [59], tables[:1], 20, 2)                                   # (59 tokens: the fourth page is not full)
    source, target = np.full(2, order[3]), tables[1:, 4]
    copied = torch.zeros(2, dtype=I32, device="cuda")
    fr.fr_kv_copy_pages([cache], torch.from_numpy(source.astype(np.int32)).cuda(), torch.from_numpy(np.ascontiguousarray(target)).cuda(), copied=copied)
    for x in oracle:
        x[target] = x[source]
    assert copied.tolist() == [1, 1]
    tables[1:, 3] = target                                               # ... but for the last one, of which the others have copies
    tables[:, 4:6] = np.stack([tables[0, 4:6], tables[1, 5:7], tables[2, 5:7]])
    lens = [59, 59, 59]
    for new in ([1, 1, 1], [1, 1, 1], [5, 1, 7], [1, 0, 1], [20, 3, 11]):
        lens = [n + t for n, t in zip(lens, new)]
        run(new, lens, tables, 24, 3)
        if new[0] == 5:
            run([0, 1, 0], [lens[0], lens[1] + 1, lens[2]], tables, 0, 0)
            lens[1] += 1


def _step(dt=torch.bfloat16, seqs=6, Hq=8, Hk=2, D=64, page=16, block=16, longest=900, window=0, seed=0):
    """A step that reads from the device where it stands: append, then attend; and what it works on."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = longest // page
    codes = [torch.randint(0, 120, (seqs * n, Hk, page, D), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scale = [torch.full((seqs * n, Hk, page // block), 118, device="cuda", dtype=torch.uint8) for _ in range(2)]
    s = dict(cache=fr.Kv8Pages(*codes, *scale, dt), tensors=codes + scale, pages=torch.randperm(seqs * n, generator=g, device="cuda").to(I32).view(seqs, n),
             at=torch.arange(seqs, device="cuda") * 131 % (longest - 40), row=torch.randn((seqs, Hq + 2 * Hk, D), generator=g, device="cuda").to(dt),
             out=torch.zeros((seqs, Hq, D), dtype=dt, device="cuda"), lse=torch.zeros(seqs, Hq, device="cuda"), rows=torch.arange(seqs, device="cuda"))
    lim = dict(max_len=n * page, window=window, sinks=2 if window else 0)
    s["workspace"] = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(s["cache"], s["out"], seqs, **lim)), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        q, k, v = s["row"].split([Hq, Hk, Hk], 1)
        slot = s["pages"][s["rows"], s["at"] // page].long() * page + s["at"] % page
        fr.fr_kv8_append(s["cache"], k, v, slot, stream=stream)
        s["at"].add_(1)
        fr.fr_attend_kv8(s["cache"], q.contiguous(), s["out"], s["pages"], s["at"].int(), D ** -0.5, lse=s["lse"], workspace=s["workspace"], stream=stream, **lim)
        s["row"].copy_(s["row"].roll(1, 0) * 1.01)
    return s, step


def test_captured_steps_replay_beside_one_another():
    # two graphs that share a workspace, replayed in turn with eager work and other calls between: the bits of eager steps
    make = lambda: [_step(seed=1), _step(seed=2, window=100)]
    want, steps = [], make()
    steps[1][0]["workspace"] = steps[0][0]["workspace"] = max((s["workspace"] for s, _ in steps), key=lambda w: w.numel())
    for _ in range(8):
        for s, step in steps:
            step()
            want.append((s["out"].clone(), s["lse"].clone(), [x.clone() for x in s["tensors"]]))
    steps = make()
    steps[1][0]["workspace"] = steps[0][0]["workspace"] = max((s["workspace"] for s, _ in steps), key=lambda w: w.numel())
    graphs = []
    for s, step in steps:
        keep = {k: s[k].clone() for k in ("at", "row")}
        tensors = [x.clone() for x in s["tensors"]]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for k, x in keep.items():
            s[k].copy_(x)
        for a, b in zip(s["tensors"], tensors):
            a.copy_(b)
        graphs.append(graph)
    other = _step(seed=9)[1]
    for i in range(8):
        for j, (s, _) in enumerate(steps):
            graphs[j].replay()
            if i % 3 == 1:
                other()
            if i % 2:
                torch.cuda.synchronize()
            out, lse, tensors = want[2 * i + j]
            assert torch.equal(s["out"], out) and torch.equal(s["lse"], lse), (i, j)
            assert all(torch.equal(a, b) for a, b in zip(s["tensors"], tensors)), (i, j)


def test_calls_on_streams_of_their_own_side_by_side():
    alone = []
    for seed in (4, 5):
        s, step = _step(seed=seed, seqs=40, longest=1600)
        for _ in range(6):
            step()
        torch.cuda.synchronize()
        alone.append((s["out"].clone(), s["tensors"][0].clone()))
    pairs, streams = [_step(seed=seed, seqs=40, longest=1600) for seed in (4, 5)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(6):
        for (s, step), stream in zip(pairs, streams):
            with torch.cuda.stream(stream):
                step()                                 # (without a stream: torch's current one)
    torch.cuda.synchronize()
    for (s, _), (out, codes) in zip(pairs, alone):
        assert torch.equal(s["out"], out) and torch.equal(s["tensors"][0], codes)


def test_a_masked_stream_gives_the_same_result():
    # fewer units: keys are cut in other parts, results are those of the definition all the same
    ctx = fr.Context(device_id=0, cu_count=16)
    for lens, new in (([2000, 1, 300], [1, 1, 1]), ([400, 90], [200, 90])):
        _attend_case("bf16", 8, 2, 128, 16, 16, lens, new, 31, stream=ctx.fr_side_stream(), rows=200)
        _attend_case("f16", 8, 2, 64, 16, 4, lens, new, 32, 128, 2, stream=ctx.fr_side_stream(), rows=200)
    ctx.fr_destroy()


@pytest.mark.parametrize("window,sinks,prompt", [(0, 0, 500), (64, 4, 512), (300, 1, 250)])
def test_the_example_in_8_bits(window, sinks, prompt):
    from examples import generate_in_bubbles as example
    make = lambda: example.Decoder(prompt=prompt, new=20, seed=6, cache_bits=8, window=window, sinks=sinks)
    model = make()
    model.prefill()
    for _ in range(20):
        model.step()
    torch.cuda.synchronize()
    want = model.tokens.clone()
    assert int(want.min()) >= 0 and len(set(want[:, 0].tolist())) > 1 and bool(torch.isfinite(model.logits.float()).all())
    model = make()
    model.prefill()
    model.capture()
    got, step_ns = example.standalone(model)
    assert torch.equal(got, want)
    again, progress, bubble_ns = example.harvest(model, step_ns, epochs=10)
    assert progress.steps == 20 and bubble_ns > 0 and torch.equal(again, want)

"""The ends of what fr_attend_kv8 takes, the scale's among them, against the fp64 oracle or exact results."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2409_06941_amd as fr                 # noqa: E402
import test_gpu_cache8 as cases                   # noqa: E402
from oracle import cache8, generation             # noqa: E402
from test_gpu_cache8 import DT, I32, _attend_case          # noqa: E402

SHAPES = [([40, 3, 190], [1, 1, 1]), ([190, 77], [100, 77])]           # few rows; many


@pytest.mark.parametrize("dt,std,scale", [
    ("bf16", 0.0, 2.0 ** 120), ("f16", 0.0, 2.0 ** 120),               # queries of zeros: the mean of the values, whatever the scale
    ("bf16", 0.0, 2.0 ** -149), ("f16", 0.0, 2.0 ** -149),
    ("bf16", 1.0, 2.0 ** -149), ("f16", 1.0, 2.0 ** -149), ("f16", 1.0, 2.0 ** -126)])
def test_attend_largest_and_smallest_scale(dt, std, scale):
    print("attend scale", dt, std, scale, flush=True)
    for lens, new in SHAPES:
        _attend_case(dt, 4, 2, 128, 16, 1, lens, new, 5, scale=scale, std=std)
        _attend_case(dt, 4, 2, 64, 16, 16, lens, new, 6, 50, 3, scale=scale, std=std)


# Codes are some 2^6.6 times their block's power, so that scores of 128 elements are of order one where
# scale x std x 2^(byte - 120.4) is about 2^-3.5.  (fp16 has no such numbers.)
@pytest.mark.parametrize("std,scale,byte", [
    (2.0 ** 30, 2.0 ** 20, 67), (2.0 ** -12, 2.0 ** 119, 10), (2.0 ** 100, 2.0 ** 7, 10),              # large scales
    (2.0 ** -50, 2.0 ** -79, 246), (1.0, 2.0 ** -129, 246), (2.0 ** 10, 2.0 ** -139, 246), (2.0 ** 60, 2.0 ** -30, 87),
    (2.0 ** -20, 2.0 ** -64, 201), (2.0 ** -20, 2.0 ** -109, 246)])
def test_attend_queries_and_keys_far_apart(std, scale, byte):
    print("attend far apart", std, scale, byte, flush=True)
    for lens, new in SHAPES:
        _attend_case("bf16", 4, 2, 128, 16, 1, lens, new, 7, scales=(byte, byte), scale=scale, std=std)
        _attend_case("bf16", 4, 2, 64, 16, 16, lens, new, 8, 50, 3, scales=(byte, byte), scale=scale, std=std)


@pytest.mark.parametrize("dt,q,scale,byte", [
    ("bf16", 2.0 ** 80, 2.0 ** 60, 10), ("bf16", 2.0 ** 127, 1.0, 10), ("bf16", 2.0 ** 127, 2.0 ** -64, 70), ("bf16", 2.0 ** 127, 2.0 ** -64, 160),
    ("bf16", 2.0 ** -62, 2.0 ** -60, 246), ("bf16", 2.0 ** 7, 2.0 ** 120, 10), ("f16", 2.0 ** 15, 2.0 ** 80, 134), ("f16", 2.0 ** -14, 2.0 ** 120, 112),
    ("f16", 2.0 ** 15, 2.0 ** -24, 134), ("bf16", 2.0 ** -20, 2.0 ** 120, 10)])          # (the last: products among the subnormal numbers of 32 bits)
@pytest.mark.parametrize("t", [1, 70])
def test_attend_scores_in_range_whatever_makes_them(dt, q, scale, byte, t):
    # One element of q and k that is not 0: scores are powers of two times 1, 2, 4, .. 128, exactly, whose largest is all that counts but where they
    # are small: then they are 0 to the last bit that 32 bits show.
    print("attend in range", dt, q, scale, byte, t, flush=True)
    n, D, page = 80, 64, 16
    ck = torch.zeros(n // page, 1, page, D, dtype=torch.uint8, device="cuda")
    exponent = torch.arange(n, device="cuda") * 5 % 8
    ck[:, 0, :, 9] = (56 + 8 * exponent).to(torch.uint8).view(-1, page)            # (0x38 is 1)
    cv = torch.randint(0, 120, (n // page, 1, page, D), device="cuda", dtype=torch.uint8)
    s = [torch.full((n // page, 1, 1), x, device="cuda", dtype=torch.uint8) for x in (byte, 120)]
    cache = fr.Kv8Pages(ck, cv, *s, DT[dt])
    x = torch.zeros(t, 1, D, dtype=DT[dt], device="cuda")
    x[:, :, 9] = q
    out, lse = torch.full_like(x, 9.0), torch.full((t, 1), 9.0, device="cuda")
    lim = dict(max_len=n, max_q=t)
    ws = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(cache, x, 1, **lim)), dtype=torch.uint8, device="cuda")
    fr.fr_attend_kv8(cache, x, out, torch.arange(n // page, dtype=I32, device="cuda").view(1, -1), torch.tensor([n], dtype=I32, device="cuda"), scale,
                     q_begin=torch.tensor([0, t], dtype=I32, device="cuda"), lse=lse, workspace=ws, **lim)
    torch.cuda.synchronize()
    v = cv.view(torch.float8_e4m3fn).double().view(n, D) * 2.0 ** (120 - 127)
    for i in range(t):
        seen = n - t + 1 + i
        score = scale * q * 2.0 ** (byte - 127) * 2.0 ** exponent[:seen].double()
        assert score.max() < 2.0 ** 127
        w = torch.softmax(score, 0)
        want = w @ v[:seen]
        # weights and result rounded to the type; scores are exact, their product with log2 e and the exponential off by a few units
        unit = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11
        assert bool(((out[i, 0].double() - want).abs() <= (2 * unit + 2.0 ** -16) * (w @ v[:seen].abs()) + 2.0 ** -20).all()), i
        assert abs(float(lse[i, 0]) - float(torch.logsumexp(score, 0))) <= 2.0 ** -20 * (1 + abs(float(torch.logsumexp(score, 0)))), i


class _Uncut(cases.Numbers):
    """What codes and scale bytes would stand for if one end of the range did not cut the bytes."""

    def __init__(self, end, *of):
        super().__init__(*of)
        self.end = end

    def __getitem__(self, at):
        p, h, o = at
        lo, hi = cache8.RANGE[self.dt]
        byte = np.clip(self.scale[p, h, o // self.block].astype(np.int64), -1000 if self.end == "lo" else lo, 1000 if self.end == "hi" else hi)
        return cache8.VALUES[self.codes[p, h, o]] * (2.0 ** (byte - 127))[:, None]


# Most blocks' bytes lie beyond the cut, the others next to it; scores are of order one.
@pytest.mark.parametrize("dt,end,scales,std,scale", [
    ("bf16", "lo", (0, 11), 2.0 ** -12, 2.0 ** 119), ("bf16", "hi", (245, 255), 2.0 ** -20, 2.0 ** -109),
    ("f16", "lo", (100, 113), 1.0, 2.0 ** 5), ("f16", "hi", (133, 145), 2.0 ** -8, 2.0 ** -9)])
def test_attend_scale_bytes_are_cut(monkeypatch, dt, end, scales, std, scale):
    print("attend cut", dt, end, flush=True)
    spread, row, plain = [], generation.attend_row, cases.Numbers

    def noting(q, k, v, scale):
        if len(k):
            spread.append(float(scale * np.abs(k @ q).max()))
        return row(q, k, v, scale)
    monkeypatch.setattr(generation, "attend_row", noting)

    def call(lens, new):
        _attend_case(dt, 4, 2, 128, 16, 1, lens, new, 15, scales=scales, scale=scale, std=std)
        _attend_case(dt, 4, 2, 64, 16, 16, lens, new, 16, 50, 3, scales=scales, scale=scale, std=std)
    for lens, new in SHAPES:
        call(lens, new)
    # (the bound of the comparison grows with 2^-17 of the largest score: nothing beside the type's rounding)
    assert 1 < max(spread) < 16
    # and the comparison sees a cut that is missing, of K's bytes alone and of V's alone
    for wrong in (0, 1):
        for lens, new in SHAPES:
            made = []

            def numbers(*of):
                made.append(len(made))
                return _Uncut(end, *of) if made[-1] % 2 == wrong else plain(*of)
            monkeypatch.setattr(cases, "Numbers", numbers)
            with np.errstate(all="ignore"), pytest.raises(AssertionError):
                call(lens, new)
            monkeypatch.setattr(cases, "Numbers", plain)


@pytest.mark.parametrize("t", [1, 40])
@pytest.mark.parametrize("Hq,n", [(1, 20), (4, 2048)])
def test_attend_largest_and_smallest_values(t, Hq, n):
    # bfloat16: 2^11 values of the largest magnitude, all of one sign; and values of some 2^-126 .. 2^-118
    print("attend values", t, Hq, n, flush=True)
    D, page = 64, 16
    pages = -(-n // page)
    g = torch.Generator(device="cuda").manual_seed(n + t)
    codes = lambda lo, hi: torch.randint(lo, hi, (pages, 1, page, D), generator=g, device="cuda", dtype=torch.uint8)
    byte = lambda x: torch.full((pages, 1, 1), x, device="cuda", dtype=torch.uint8)
    q = torch.randn((t, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    i32 = lambda x: torch.tensor(x, dtype=I32, device="cuda")

    def call(ck, cv, v_byte):
        cache, out = fr.Kv8Pages(ck, cv, byte(119), byte(v_byte), torch.bfloat16), torch.full_like(q, 9.0)
        lim = dict(max_len=n, max_q=t)
        ws = torch.empty(max(1, fr.fr_attend_kv8_workspace_bytes(cache, q, 1, **lim)), dtype=torch.uint8, device="cuda")
        fr.fr_attend_kv8(cache, q, out, torch.arange(pages, dtype=I32, device="cuda").view(1, -1), i32([n]), D ** -0.5, q_begin=i32([0, t]), workspace=ws, **lim)
        torch.cuda.synchronize()
        return out.double().cpu().numpy()
    ck = codes(0, 256) & 0xbf                          # (below 2: scores of some units)
    top = call(ck, torch.full_like(ck, 0x7e), 250)
    # equal values: off by the weights' rounding and the result's
    assert not top[: max(0, t - n)].any()              # (they see nothing)
    top = top[max(0, t - n):]
    assert np.all(np.abs(top / (448 * 2.0 ** 119) - 1) <= 2 * 2.0 ** -8 + 2.0 ** -16)
    cv = codes(0, 17)
    got = call(ck, cv, 3)
    K = cache8.VALUES[ck.cpu().numpy()].transpose(0, 2, 1, 3).reshape(-1, D) * 2.0 ** (119 - 127)
    V = cache8.VALUES[cv.cpu().numpy()].transpose(0, 2, 1, 3).reshape(-1, D) * 2.0 ** -117
    q = q.double().cpu().numpy()
    for i in range(t):
        for h in range(Hq):
            seen = n - t + 1 + i
            o, _, a, x = generation.attend_row(q[i, h], K[:seen], V[:seen], D ** -0.5)
            if seen > 0:
                # the bound of ordinary values; and sums of weights 2^-20 times theirs, the largest one 1 at least, whose steps are 2^-149: half a
                # step for every eight keys or fewer that are added at once, for every time that the maximum rises, and for every part that is joined
                near = (2.0 ** -8 + 2 * ((D + 4) * 2.0 ** -24 * x + 2.0 ** -20) + n * 2.0 ** -23) * a + 2.0 ** -8 * np.abs(o) + 2.0 ** -134 + (n / 8 + 64) * 2.0 ** -130
                assert np.all(np.abs(got[i, h] - o) <= near), (i, h)

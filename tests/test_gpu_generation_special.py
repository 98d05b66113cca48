"""Values that are not finite, small weights, tokens outside of a call, large calls and shared workspaces of the text-generation operators."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2409_06941_amd as fr              # noqa: E402
from oracle import generation as oracle        # noqa: E402

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # half an ulp of 8 and of 11 significant bits
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -25}        # half the smallest subnormal


def _f64(x):
    return x.detach().double().cpu().numpy()


class _Batch:
    """A cache with sequences of own[b] keys and new[b] tokens behind P shared keys; pages in any order."""

    def __init__(self, dt, Hq, Hk, D, page, P, own, new, seed):
        g = torch.Generator().manual_seed(seed)
        self.dt, self.Hq, self.Hk, self.D, self.page, self.P, self.own, self.new = dt, Hq, Hk, D, page, P, own, new
        prefix_pages, counts = -(-P // page), [-(-x // page) for x in own]
        pages = prefix_pages + sum(counts) + 2
        self.k, self.v = (torch.randn((pages, Hk, page, D), generator=g).to(DT[dt]) for _ in range(2))
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.prefix_pages = order[:prefix_pages].contiguous()
        self.table = torch.zeros((len(own), max(1, max(counts))), dtype=torch.int32)
        at = prefix_pages
        for b, c in enumerate(counts):
            self.table[b, :c] = order[at:at + c]
            at += c
        self.begin = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.q = torch.randn((int(self.begin[-1]), Hq, D), generator=g).to(DT[dt])
        self.scale = D ** -0.5

    def place(self, b, j):
        """Page and slot of key j that sequence b sees (counted through the prefix)."""
        own = j - self.P
        return (int(self.prefix_pages[j // self.page]), j % self.page) if own < 0 else (int(self.table[b, own // self.page]), own % self.page)

    def prepare(self):
        self.gk, self.gv, self.gq = self.k.cuda(), self.v.cuda(), self.q.cuda()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        self.cache = fr.KvPages(self.gk, self.gv)
        self.out = torch.full_like(self.gq, 9.0)
        self.lse = torch.full(self.q.shape[:2], 9.0, device="cuda")
        self.limits = dict(prefix_len=self.P, max_own_len=max(self.own), max_q=max(max(self.new), 1))
        need = fr.fr_attend_shared_workspace_bytes(self.cache, self.gq, len(self.own), **self.limits)
        self.workspace = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")
        self.args = (self.table.cuda() if max(self.own) else None, i32(self.own))
        self.more = dict(prefix_pages=self.prefix_pages.cuda() if self.P else None, q_begin=i32(self.begin))
        return self

    def call(self):
        fr.fr_attend_shared(self.cache, self.gq, self.out, *self.args, self.scale, lse=self.lse, workspace=self.workspace,
                            stream=torch.cuda.current_stream(), **self.more, **self.limits)

    def check(self):
        """Every row against the oracle: the same infinities, NaN where it has NaN, near it elsewhere."""
        self.prepare()
        self.call()
        torch.cuda.synchronize()
        q, k, v, out, lse = (_f64(x) for x in (self.q, self.k, self.v, self.out, self.lse))
        u, G = UNIT[self.dt], self.Hq // self.Hk
        for b in range(len(self.own)):
            places = np.array([self.place(b, j) for j in range(self.P + self.own[b])], dtype=np.int64).reshape(-1, 2)
            for h in range(self.Hq):
                kk, vv = k[places[:, 0], h // G, places[:, 1]], v[places[:, 0], h // G, places[:, 1]]
                for i in range(self.new[b]):
                    n, row = oracle.visible(self.P, self.own[b], self.new[b], i), int(self.begin[b]) + i
                    with np.errstate(invalid="ignore"):
                        o, l, _, x = oracle.attend_row(q[row, h], kk[:n], vv[:n], self.scale)
                        at = (b, i, h, n)
                        assert np.array_equal(np.isnan(out[row, h]), np.isnan(o)), at
                        inf = np.isinf(o)
                        assert np.array_equal(np.isinf(out[row, h]), inf) and np.array_equal(out[row, h][inf], o[inf]), at
                        there = np.isfinite(o)
                        if n == 0:
                            assert not out[row, h].any() and lse[row, h] == -math.inf, at
                            continue
                        # scores: sums of D products of 32 bits; a weight is off by that, by a few ulps of exp and by the type's rounding;
                        # sums of n of them; the result's rounding.  Weights of 16 bits end at half the smallest subnormal.
                        finite = np.where(np.isfinite(vv[:n]), vv[:n], 0.0)
                        e = np.exp(self.scale * (kk[:n] @ q[row, h]) - l)
                        d = (self.D + 4) * 2.0 ** -24 * x + 2.0 ** -20
                        near = (u + 2 * d + n * 2.0 ** -23) * (e @ np.abs(finite)) + u * np.abs(np.where(there, o, 0.0)) * 1.01 + TINY[self.dt]
                        near = near + (n * 2.0 ** -25 * np.abs(finite).max() if self.dt == "f16" else 0.0)
                    assert np.all(np.abs(out[row, h] - o)[there] <= near[there]), at
                    assert abs(lse[row, h] - l) <= d + n * 2.0 ** -23 + 2.0 ** -20 * (1 + abs(l)), at


# the kinds of work that a call is made of: few rows and many, by themselves and behind a prefix, in one part and in several
KINDS = [
    (8, 2, 128, 16, 0, [50, 1, 33], [1, 1, 1]),
    (4, 2, 64, 16, 0, [5001, 70], [1, 1]),
    (8, 8, 64, 16, 0, [int(x) for x in 1 + np.arange(130) * 7 % 199], [1] * 130),
    (8, 2, 128, 16, 37, [50, 0, 33], [1, 1, 1]),
    (8, 8, 128, 16, 6001, [77, 3, 0], [1, 1, 1]),
    (16, 8, 64, 16, 1501, [int(x) for x in 1 + np.arange(40) * 13 % 197], [1] * 40),
    (16, 8, 128, 32, 701, [int(x) for x in 1 + np.arange(64) * 7 % 99], [1] * 64),
    (8, 8, 128, 16, 3001, [0] * 40, [1] * 40),
    (8, 2, 64, 16, 37, [40, 9, 0], [5, 9, 0]),
    (6, 2, 128, 16, 0, [130, 70], [130, 70]),
    (4, 2, 64, 16, 100, [150, 9, 260], [70, 9, 33]),
    (4, 1, 128, 16, 8203, [50, 61], [41, 40]),
]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_infinite_values_that_are_seen_stay_what_they_are(dt, kind):
    Hq, Hk, D, page, P, own, new = KINDS[kind]
    print("attend infinite", dt, *KINDS[kind][:5], len(own), flush=True)
    c = _Batch(dt, Hq, Hk, D, page, P, own, new, seed=kind)
    ends = [(b, P + n - 1) for b, n in enumerate(own) if n] + ([(0, P - 1)] if P else [])
    for b, j in ends:                                  # the last key of a sequence, and of the prefix
        page_, slot = c.place(b, j)
        c.v[page_, :, slot, 3], c.v[page_, :, slot, 5], c.v[page_, :, slot, 40] = math.inf, -math.inf, math.nan
    first = [(b, 0) for b in range(1)] if P else [(b, 0) for b, n in enumerate(own) if n > 2]
    for b, j in first:                                 # the first key: the same sign, and another one
        page_, slot = c.place(b, j)
        c.v[page_, :, slot, 3], c.v[page_, :, slot, 5], c.v[page_, :, slot, 21] = math.inf, math.inf, -math.inf
    c.check()


@pytest.mark.parametrize("D,G,P,t", [(128, 2, 50, 5), (64, 4, 50, 40), (128, 4, 0, 90), (128, 1, 300, 200), (64, 8, 4000, 3)])
def test_values_that_only_later_tokens_see(D, G, P, t):
    print("attend later", D, G, P, t, flush=True)
    c = _Batch("bf16", 2 * G, 2, D, 16, P, [t + 20, 7], [t, 1], seed=t)
    for back, e, x in ((1, 3, math.inf), (2, 4, math.nan), (3, 3, -math.inf), (t // 2, 9, math.inf), (t, 10, -math.inf), (t + 5, 11, math.inf)):
        page, slot = c.place(0, P + t + 20 - back)
        c.v[page, :, slot, e] = x
    c.check()


@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_scores_of_infinity(kind):
    # keys whose score is -infinity have no weight; a row that sees no others gets zeros and -infinity; +infinity makes NaN
    Hq, Hk, D, page, P, own, new = KINDS[kind]
    print("attend scores", *KINDS[kind][:5], len(own), flush=True)
    c = _Batch("bf16", Hq, Hk, D, page, P, own, new, seed=kind)
    c.q[:, :, 0] = 1.0
    for b in range(len(own)):
        for j in range(own[b]):                        # all own keys
            at, slot = c.place(b, P + j)
            c.k[at, :, slot, 0] = -math.inf
    if P:
        c.prepare()                                    # (every token sees the prefix, and that alone counts)
        c.call()
        torch.cuda.synchronize()
        out, lse = _f64(c.out), _f64(c.lse)
        k, v, q = _f64(c.k), _f64(c.v), _f64(c.q)
        places = np.array([c.place(0, j) for j in range(P)])
        for row in range(0, q.shape[0], max(1, q.shape[0] // 50)):
            for h in range(0, Hq, 3):
                o, l, a, x = oracle.attend_row(q[row, h], k[places[:, 0], h // (Hq // Hk), places[:, 1]], v[places[:, 0], h // (Hq // Hk), places[:, 1]], c.scale)
                d = (D + 4) * 2.0 ** -24 * x + 2.0 ** -20
                near = (UNIT["bf16"] + 2 * d + P * 2.0 ** -23) * a + UNIT["bf16"] * np.abs(o) * 1.01 + TINY["bf16"]
                assert np.all(np.abs(out[row, h] - o) <= near) and abs(lse[row, h] - l) <= d + P * 2.0 ** -23 + 2.0 ** -20 * (1 + abs(l)), (row, h)
    else:
        c.prepare()
        c.call()
        torch.cuda.synchronize()
        assert not c.out.any() and bool((c.lse == -math.inf).all())
    if own[0]:
        at, slot = c.place(0, 0)
        c.k[at, :, slot, 0] = math.inf
        c.prepare()
        c.call()
        torch.cuda.synchronize()
        first = c.out[: new[0]] if not P else c.out
        assert bool(torch.isnan(first.float()).all())


def test_small_weights_of_many_keys_add_up():
    # one key far ahead of the others, whose weights of 2^-26 are too small for 16 bits by themselves but not together
    n, D = 2000, 64
    for dt in ("f16", "bf16"):
        for Hk, new in ((8, [40] * 32), (1, [1]), (8, [1] * 200)):
            print("attend small weights", dt, Hk, len(new), flush=True)
            c = _Batch(dt, Hk, Hk, D, 16, 0, [n] * len(new), new, seed=1)
            c.k.zero_()
            c.v.fill_(256.0)
            for b in range(len(new)):
                page, slot = c.place(b, 0)
                c.k[page, :, slot, 0], c.v[page, :, slot] = 8.0, 0.0
            c.q.zero_()
            c.q[:, :, 0] = 1.0
            c.scale = float(np.float32(26 * math.log(2.0) / 8.0))
            c.prepare()
            c.call()
            torch.cuda.synchronize()
            w = math.exp(-8.0 * c.scale)
            for i in (0, new[0] // 2, new[0] - 1):
                seen = n - new[0] + i
                want = 256.0 * seen * w / (1 + seen * w)
                # 2^-7 of a weight (2^-26 but for the rounding of the scale), the sums of n weights in 32 bits, half an ulp of the result
                assert np.all(np.abs(_f64(c.out)[i::new[0]] - want) <= want * (2.0 ** -7 + n * 2.0 ** -24 + UNIT[dt])), (dt, Hk, len(new), i)


def test_a_value_that_is_not_finite_does_not_make_a_call_long():
    # 4 questions about a document that they go through themselves, with one bad value in the document, and one in the questions
    def us(spoil):
        c = _Batch("bf16", 16, 4, 128, 16, 4096, [300, 280, 310, 290], [300, 280, 310, 290], seed=2)
        for b, j in spoil:
            page, slot = c.place(b, j)
            c.v[page, :, slot, 17] = math.nan
        c.prepare()
        c.call()
        torch.cuda.synchronize()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(10):
            c.call()
        end.record()
        torch.cuda.synchronize()
        return begin.elapsed_time(end) * 100
    clean, document, question = us([]), us([(0, 5)]), us([(1, 4096 + 100)])
    print("clean %.0f us, a bad value in the document %.0f, in a question %.0f" % (clean, document, question), flush=True)
    # (keys that not all rows of a tile see are gone through again, at a third of the pace)
    assert document <= 1.5 * clean + 20 and question <= 4 * clean + 100


@pytest.mark.parametrize("Hk,G,n,most,P", [(8, 1, 16, 2, 250), (8, 8, 64, 4, 128), (8, 1, 100, 3, 250), (8, 4, 100, 40, 250), (2, 1, 3, 4, 20), (2, 4, 5, 4, 9000)])
def test_tokens_outside_of_the_sequences_are_not_computed(Hk, G, n, most, P):
    # tokens before and behind the sequences, a sequence without any, some with more than max_q; no keys but the prefix
    print("attend outside", Hk, G, n, most, P, flush=True)
    counts = [1 + b * 5 % (most + 3) for b in range(n)]
    counts[n // 2] = 0
    begin = np.concatenate([[2], 2 + np.cumsum(counts)]).astype(np.int32)
    c = _Batch("bf16", Hk * G, Hk, 128, 16, P, [0] * n, [int(begin[-1]) + 3] + [0] * (n - 1), seed=P)
    c.prepare()
    c.limits["max_q"] = most
    c.more["q_begin"] = torch.from_numpy(begin).cuda()
    c.workspace = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(c.cache, c.gq, n, **c.limits)), dtype=torch.uint8, device="cuda")
    c.call()
    torch.cuda.synchronize()
    there = np.zeros(c.q.shape[0], dtype=bool)
    for b in range(n):
        there[begin[b]:begin[b] + min(counts[b], most)] = True
    out, lse = _f64(c.out), _f64(c.lse)
    assert np.all(out[~there] == 9.0) and np.all(lse[~there] == 9.0)
    assert np.all(lse[there] != 9.0) and np.all(np.abs(out[there]) < 5.0)


def test_one_workspace_for_the_largest_call_and_smaller_ones():
    print("attend one workspace", flush=True)
    sizes = [([4000] * 64, [1] * 64, 0), ([4000] * 8, [1] * 8, 0), ([300] * 16, [70] * 16, 2048), ([300] * 16, [40] * 16, 2048), ([9] * 3, [2] * 3, 2000)]
    shape = dict(dt="bf16", Hq=8, Hk=2, D=128, page=16)
    most = torch.empty((16 * 70, 8, 128), dtype=torch.bfloat16, device="cuda")
    for i, (own, new, P) in enumerate(sizes):
        c = _Batch(own=own, new=new, P=P, seed=i, **shape)
        c.prepare()
        c.call()
        torch.cuda.synchronize()
        want = c.out.clone()
        need = fr.fr_attend_shared_workspace_bytes(c.cache, most, 64, prefix_len=2048, max_own_len=4000, max_q=70)
        c.workspace = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        c.out.zero_()
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want), i


def test_append_of_more_tokens_than_a_grid_has_threads_for():
    print("append many", flush=True)
    T, D = (1 << 24) + 5, 64
    k = torch.empty((T, 1, D), dtype=torch.int16, device="cuda").random_(-30000, 30000).view(torch.bfloat16)
    ck, cv = (torch.zeros((-(-T // 16), 1, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slot = torch.arange(T - 1, -1, -1, device="cuda")
    fr.fr_kv_append(fr.KvPages(ck, cv), k, k, slot, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for x in (ck, cv):
        assert torch.equal(x.view(-1, D)[:T].view(torch.int16), k.view(T, D).view(torch.int16).flip(0))


def test_sample_of_more_rows_than_a_grid_has_threads_for():
    print("sample many", flush=True)
    n = (1 << 22) + 3
    r = torch.arange(n, device="cuda")
    logits = torch.zeros((n, 2), device="cuda")
    logits[:, 1] = torch.where(r % 11 == 0, -2.0, 0.0)                 # (the second entry has a weight of 0.135 or 1)
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    f32 = lambda x: x.to(torch.float32)
    fr.fr_sample(logits, f32(torch.where(r % 7 == 0, 0.25, 0.95)), token, temperature=f32(r % 5 != 0), top_k=(r % 5 == 1).int(),
                 top_p=f32(torch.where(r % 5 == 2, 0.25, 1.0)), min_p=f32(torch.where(r % 5 == 3, 0.5, 0.0)), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    first = (r % 7 == 0) | (r % 5 <= 2) | ((r % 5 == 3) & (r % 11 == 0))
    assert torch.equal(token, (~first).int())


def test_one_long_prompt_beside_many_single_tokens():
    # sizes at which sequences times the longest prompt are more workgroups than one dimension of a grid takes
    print("attend ragged", flush=True)
    n, most, Hq, Hk, D, page = 1024, 4177, 512, 64, 64, 16
    new = [1] * n
    new[500] = most
    own = [int(x) for x in 1 + np.arange(n) * 37 % 60]
    own[500] = most
    c = _Batch("bf16", Hq, Hk, D, page, 0, own, new, seed=3)
    c.prepare()
    c.call()
    torch.cuda.synchronize()
    k, v = _f64(c.k), _f64(c.v)
    rng = np.random.default_rng(0)
    for b in [0, 1, 499, 501, n - 1] + [500] * 12:
        i, h = int(rng.integers(0, new[b])), int(rng.integers(0, Hq))
        places = np.array([c.place(b, j) for j in range(own[b])])
        count = oracle.visible(0, own[b], new[b], i)
        kk, vv = k[places[:count, 0], h // (Hq // Hk), places[:count, 1]], v[places[:count, 0], h // (Hq // Hk), places[:count, 1]]
        row = int(c.begin[b]) + i
        o, l, a, x = oracle.attend_row(_f64(c.q[row, h]), kk, vv, c.scale)
        d = (D + 4) * 2.0 ** -24 * x + 2.0 ** -20
        near = (UNIT["bf16"] + 2 * d + count * 2.0 ** -23) * a + UNIT["bf16"] * np.abs(o) * 1.01 + TINY["bf16"]
        assert np.all(np.abs(_f64(c.out[row, h]) - o) <= near), (b, i, h)
        assert abs(float(c.lse[row, h]) - l) <= d + count * 2.0 ** -23 + 2.0 ** -20 * (1 + abs(l)), (b, i, h)
    assert bool((c.lse != 9.0).all())


def test_a_cache_that_is_not_on_the_gpu_is_refused():
    print("host cache", flush=True)
    host = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    there = host.cuda()
    x, slot = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.arange(3, device="cuda")
    q, n, pages = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda"), torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    for k, v, name in ((host, host, "cache k"), (host, there, "cache k"), (there, host, "cache v"), (host.to("meta"), there, "cache k")):
        cache = fr.KvPages(k, v)
        for call in (lambda: fr.fr_kv_append(cache, x, x, slot), lambda: fr.fr_attend_shared(cache, q, q.clone(), pages, n, 0.1, max_own_len=8)):
            with pytest.raises(ValueError, match=name + ": not on a GPU"):
                call()


def test_calls_without_a_stream_work_on_the_current_one():
    print("current stream", flush=True)
    D, n = 64, 40
    side = torch.cuda.Stream()
    ck, cv = (torch.zeros(4, 1, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = fr.KvPages(ck, cv)
    k = torch.zeros(n, 1, D, dtype=torch.bfloat16, device="cuda")
    slot, pages = torch.arange(n, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")[None]
    q, out = torch.zeros(1, 2, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, D, dtype=torch.bfloat16, device="cuda")
    own = torch.tensor([n], dtype=torch.int32, device="cuda")
    ws = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(cache, q, 1, 0, n)), dtype=torch.uint8, device="cuda")
    logits, token = torch.zeros(1, 100, device="cuda"), torch.full((1,), -7, dtype=torch.int32, device="cuda")
    uniform = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                 # what follows is still to come when the calls are made
        k.fill_(3.0)
        logits[0, 77] = 50.0
        fr.fr_kv_append(cache, k, k, slot)
        fr.fr_attend_shared(cache, q, out, pages, own, 0.1, max_own_len=n, workspace=ws)
        fr.fr_sample(logits, uniform, token)
        a, b = out.clone(), token.clone()
    side.synchronize()
    assert bool((a == 3.0).all()) and int(b) == 77


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_sample_shares_of_nothing_and_next_to_nothing(dt):
    # top_p of 0, below 0 and too small for any share but the first entry's: the largest logit, the lowest index of equals
    print("sample nothing", dt, flush=True)
    V = 70001
    p = [0.0, -0.0, -1.0, -math.inf, 1e-12, 1e-30, 1e-45, -1e-45]
    g = torch.Generator().manual_seed(1)
    logits = torch.randn((2 * len(p), V), generator=g).to(torch.bfloat16 if dt == "bf16" else torch.float32).cuda()
    logits[:, 500:600] = 9.0
    logits[len(p):, 600:60000] = 9.0                   # (many equal ones)
    token = torch.full((2 * len(p),), -7, dtype=torch.int32, device="cuda")
    fr.fr_sample(logits, torch.full((2 * len(p),), 0.99, device="cuda"), token, top_p=torch.tensor(p * 2, dtype=torch.float32, device="cuda"))
    torch.cuda.synchronize()
    assert token.tolist() == [500] * (2 * len(p))


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [4095, 4096, 4097])
def test_sample_vocabularies_about_what_there_is_room_for(dt, V):
    # 4096 entries have room, and up to 1740 of more are taken in one go; rows without and with equal entries
    print("sample room", dt, V, flush=True)
    rng = np.random.default_rng(V)
    n = 24
    x = 10.0 - 1.7 * np.log1p(np.stack([rng.permutation(V) for _ in range(n)])) + 0.5 * rng.standard_normal((n, V))
    x[n // 2:] = np.round(x[n // 2:])
    x[n - 1] = 3.0
    types = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    logits = torch.from_numpy(x).to(types[dt]).cuda()
    x = _f64(logits)
    for top_k, top_p in ((0, 1.0), (0, 0.95), (0, 0.5), (1739, 1.0), (1740, 1.0), (1741, 1.0), (1740, 0.9), (1741, 0.9), (V - 1, 1.0), (V - 1, 0.9), (V, 0.9)):
        T, K, P, U, want = [], [], [], [], []
        for r in range(n):
            t = float(np.float32(rng.uniform(0.5, 1.5)))
            w, y = oracle.weights(x[r], t)
            order = np.argsort(-y, kind="stable")[: top_k or V]
            run = np.cumsum(w[order])
            p = 1.0
            if top_p < 1:                              # the middle of an entry's share, so that roundings of 32 bits do not decide
                j = int(np.searchsorted(run, top_p * run[-1]))
                p = float(np.float32((run[j] - w[order][j] / 2) / run[-1]))
            index, w = oracle.kept(x[r], t, top_k, p, 0.0)
            run = np.cumsum(w[index])
            big = np.flatnonzero(w[index] / run[-1] >= 2.0 ** -14)
            j = int(rng.choice(big))
            T.append(t), K.append(top_k), P.append(p), U.append(float((run[j] - w[index][j] / 2) / run[-1])), want.append(int(index[j]))
        token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        f = lambda y, kind=torch.float32: torch.tensor(y, dtype=kind, device="cuda")
        fr.fr_sample(logits, f(U), token, temperature=f(T), top_k=f(K, torch.int32), top_p=f(P))
        got = token.tolist()
        assert got == want, (top_k, top_p, [r for r in range(n) if got[r] != want[r]])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_sample_counts_about_the_last_that_is_taken_in_one_go(dt):
    # 1740 is the last; what is above the line that so many values of threads are above has room, or nearly
    print("sample counts", dt, flush=True)
    rng = np.random.default_rng(3)
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    for V in (4097, 5000, 20011, 131072):
        K = [1023, 1024, 1025, 1738, 1739, 1740, 1741, 1742]
        for spread in (0.01, 1.0, 30.0):
            x = rng.standard_normal((len(K), V)) * spread
            x[3] = np.sort(x[3])                       # the largest side by side, in few threads' shares
            x[4] = np.sort(x[4])[::-1]
            x[5, : V // 2] = x[5].max()
            logits = torch.from_numpy(x).to(types[dt]).cuda()
            y = _f64(logits)
            for u in (0.0, 0.9999999):
                token = torch.full((len(K),), -7, dtype=torch.int32, device="cuda")
                f = lambda z, kind=torch.float32: torch.tensor(z, dtype=kind, device="cuda")
                fr.fr_sample(logits, f([u] * len(K)), token, temperature=f([1e4] * len(K)), top_k=f(K, torch.int32))
                got = token.tolist()
                for r, k in enumerate(K):              # weights nearly equal: the first and the last of the kept indices
                    index = np.sort(np.argsort(-y[r], kind="stable")[:k])
                    assert got[r] == (index[0] if u == 0.0 else index[-1]), (V, spread, k, u)


@pytest.mark.parametrize("P,own,T", [(0, 5000, 6000), (3000, 900, 4000)])
def test_few_tokens_of_many_are_in_a_sequence(P, own, T):
    # parts of all tokens' results would take more than the call has room for: it is made in one
    print("attend few of many", P, own, T, flush=True)
    c = _Batch("bf16", 8, 2, 128, 16, P, [own, own // 2, 3], [T, 0, 0], seed=P)
    c.prepare()
    begin = np.array([T // 2, T // 2 + 1, T // 2 + 2, T // 2 + 3], dtype=np.int32)
    c.limits["max_q"] = 1
    c.more["q_begin"] = torch.from_numpy(begin).cuda()
    c.workspace = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(c.cache, c.gq, 3, **c.limits)), dtype=torch.uint8, device="cuda")
    c.call()
    torch.cuda.synchronize()
    out, lse = c.out.clone(), c.lse.clone()
    there = slice(T // 2, T // 2 + 3)
    few = _Batch("bf16", 8, 2, 128, 16, P, [own, own // 2, 3], [1, 1, 1], seed=P)
    few.k, few.v, few.prefix_pages, few.table, few.q = c.k, c.v, c.prefix_pages, c.table, c.q[there].contiguous()
    few.check()
    assert bool(((out[there].float() - few.out.float()).abs() <= 2.0 ** -7 * few.out.float().abs() + 2.0 ** -8).all())
    assert bool(((lse[there] - few.lse).abs() <= 1e-4).all())
    out[there], lse[there] = 9.0, 9.0
    assert bool((out == 9.0).all()) and bool((lse == 9.0).all())

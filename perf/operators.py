"""Timed work of text generation as a side task: the cache of keys and values, the attention that reads it, the choice of a token.

A case is a dict of plain values; `kind` says which operator it is:
  append   fr_kv_append: queries and keys rotated by their positions, keys and values stored into pages of a cache
  attend   fr_attend_shared: attention of a batch whose sequences share a prefix, each with keys of its own behind it
  sample   fr_sample: one token a row from logits, with temperature, top-k, top-p, min-p and a given random number
The plain forms are elementary torch operations in float32 (integers of 64 bits for the masses of a sampler, whose sums then do
not depend on their order). Which lengths a batch has follows from the case alone, so that its work does too; the values follow
from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
ROTARY_BASE = 10000.0
MASS_ONE = float(1 << 43)          # a sampler's mass of weight 1: sums over 2^19 tokens stay below 2^63


def listed():
    return [
        # one decoding step of 64 sequences: one token each, anywhere in the cache; latency counts
        dict(name="append_step", kind="append", dtype="bf16", tokens=64, q_heads=32, kv_heads=8, head_dim=128, page=16,
             slots=8192, rotary_dim=128, style="halves", padding=0),
        # prompts of several sequences in one go, padded to a common count; half of every head rotated, neighbouring pairs
        dict(name="append_ragged", kind="append", dtype="f16", tokens=4099, q_heads=20, kv_heads=5, head_dim=64, page=32,
             slots=10016, rotary_dim=32, style="pairs", padding=61),
        # a batch of long prompts: four of the larger stage's sequences of 4096 tokens
        dict(name="append_prompts", kind="append", dtype="bf16", tokens=16384, q_heads=64, kv_heads=8, head_dim=128, page=64,
             slots=20480, rotary_dim=128, style="halves", padding=0),
        # a few sequences behind a short instruction: the smallest call
        dict(name="attend_few", kind="attend", dtype="bf16", seqs=4, q_heads=8, kv_heads=2, head_dim=64, page=16, prefix=37,
             own_lo=1, own_hi=30, new_lo=1, new_hi=1, lens=1),
        # decoding step, 64 sequences of up to 1500 tokens behind one prompt of 16384
        dict(name="attend_step", kind="attend", dtype="bf16", seqs=64, q_heads=32, kv_heads=8, head_dim=128, page=16,
             prefix=16384, own_lo=1, own_hi=1500, new_lo=1, new_hi=1, lens=2),
        # decoding step of a wide batch with more heads to a key: many rows share what is read of the prefix
        dict(name="attend_wide", kind="attend", dtype="f16", seqs=256, q_heads=64, kv_heads=8, head_dim=128, page=64,
             prefix=4096, own_lo=1, own_hi=512, new_lo=1, new_hi=1, lens=3),
        # several guessed tokens a sequence are checked at once; odd sizes, an empty sequence, three heads to a key
        dict(name="attend_guesses", kind="attend", dtype="f16", seqs=33, q_heads=15, kv_heads=5, head_dim=64, page=8,
             prefix=5001, own_lo=0, own_hi=777, new_lo=0, new_hi=7, lens=4),
        # decoding without a shared prompt from long caches
        dict(name="attend_long", kind="attend", dtype="bf16", seqs=8, q_heads=32, kv_heads=8, head_dim=128, page=128,
             prefix=0, own_lo=20000, own_hi=65536, new_lo=1, new_hi=1, lens=5),
        # questions of up to 700 tokens about one shared document: matrix products bind
        dict(name="attend_questions", kind="attend", dtype="bf16", seqs=16, q_heads=32, kv_heads=8, head_dim=128, page=16,
             prefix=8192, own_lo=300, own_hi=700, new_lo=300, new_hi=700, lens=6),
        # one sequence's next token
        dict(name="sample_one", kind="sample", dtype="f32", rows=1, vocab=32768, flat=0),
        # a batch with settings of its own for every row, an odd vocabulary
        dict(name="sample_mixed", kind="sample", dtype="bf16", rows=64, vocab=100003, flat=0),
        # a wide batch over a large vocabulary
        dict(name="sample_wide", kind="sample", dtype="f32", rows=256, vocab=131072, flat=1),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["append", "attend", "sample"], [3, 6, 3])[0]
    if kind == "append":
        head_dim, kv_heads = rng.choice([64, 128]), rng.choice([1, 2, 5, 8])
        tokens, page = _log_uniform(rng, 1, 16384), rng.choice([8, 16, 32, 64, 128])
        slots = -(-int(tokens * rng.uniform(1.2, 2.0) + 64) // page) * page
        return dict(kind=kind, dtype=rng.choice(["bf16", "f16"]), tokens=tokens, q_heads=kv_heads * rng.choice([1, 3, 4, 8]),
                    kv_heads=kv_heads, head_dim=head_dim, page=page, slots=slots, rotary_dim=rng.choice([head_dim, head_dim // 2]),
                    style=rng.choice(["halves", "pairs"]), padding=rng.choice([0, tokens // 50]))
    if kind == "attend":
        head_dim, kv_heads = rng.choice([64, 128]), rng.choice([1, 2, 5, 8])
        case = dict(kind=kind, dtype=rng.choice(["bf16", "f16"]), q_heads=kv_heads * rng.choice([1, 3, 4, 8]), kv_heads=kv_heads,
                    head_dim=head_dim, page=rng.choice([8, 16, 32, 64, 128]), lens=rng.randrange(1 << 20))
        form = rng.choice(["step", "step", "guesses", "questions", "long"])
        if form == "step":
            case.update(seqs=_log_uniform(rng, 1, 256), prefix=_log_uniform(rng, 16, 16384), own_lo=1,
                        own_hi=_log_uniform(rng, 2, 1500), new_lo=1, new_hi=1)
        elif form == "guesses":
            case.update(seqs=_log_uniform(rng, 2, 64), prefix=_log_uniform(rng, 16, 8192), own_lo=0,
                        own_hi=_log_uniform(rng, 8, 1000), new_lo=0, new_hi=rng.randrange(2, 9))
        elif form == "questions":
            hi = _log_uniform(rng, 16, 700)
            case.update(seqs=_log_uniform(rng, 1, 16), prefix=_log_uniform(rng, 64, 8192), own_lo=max(1, hi // 3), own_hi=hi,
                        new_lo=max(1, hi // 3), new_hi=hi)
        else:
            hi = _log_uniform(rng, 1000, 40000)
            case.update(seqs=_log_uniform(rng, 1, 8), prefix=0, own_lo=hi // 3, own_hi=hi, new_lo=1, new_hi=1)
        return case
    return dict(kind=kind, dtype=rng.choice(["bf16", "f16", "f32"]), rows=_log_uniform(rng, 1, 256),
                vocab=_log_uniform(rng, 1000, 131072), flat=rng.randrange(2))


def lengths(case):
    """Own keys and new tokens of every sequence; a sequence has no more new tokens than keys of its own."""
    rng = random.Random(case["lens"])
    own_len = [rng.randint(case["own_lo"], case["own_hi"]) for _ in range(case["seqs"])]
    own_len[rng.randrange(len(own_len))] = case["own_hi"]
    new = [min(n, rng.randint(case["new_lo"], case["new_hi"])) for n in own_len]
    return own_len, new


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, dtype, gen, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(dtype)


def _rotary_table(positions, rotary_dim):
    """[positions, rotary_dim] float32: cosines, then sines, of position * base^(-2 i / rotary_dim)."""
    inv = ROTARY_BASE ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64, device="cuda") / rotary_dim)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * inv[None, :]
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().contiguous()


# ---------------------------------------------------------------- append

def _append_inputs(case, seed):
    gen, dt = _generator(seed), DTYPES[case["dtype"]]
    T, D, page = case["tokens"], case["head_dim"], case["page"]
    pages = case["slots"] // page
    s = {}
    # one row of a fused projection: queries, keys and values of a token side by side
    heads = case["q_heads"] + 2 * case["kv_heads"]
    qkv = _normal((T, heads, D), dt, gen)
    s["q"], s["k"], s["v"] = qkv.split([case["q_heads"], case["kv_heads"], case["kv_heads"]], dim=1)
    s["cache_k"] = _normal((pages, case["kv_heads"], page, D), dt, gen)
    s["cache_v"] = _normal((pages, case["kv_heads"], page, D), dt, gen)
    s["table"] = _rotary_table(max(4096, 2 * case["slots"]), case["rotary_dim"])
    s["position"] = torch.randint(0, s["table"].shape[0], (T,), generator=gen, device="cuda", dtype=torch.int32)
    # runs of 8 slots anywhere in the cache
    order = torch.randperm(case["slots"] // 8, generator=gen, device="cuda")[: (T + 7) // 8]
    slot = (order[:, None] * 8 + torch.arange(8, device="cuda")[None, :]).reshape(-1)[:T].to(torch.int64).contiguous()
    if case["padding"]:
        slot[T - case["padding"]:] = -1
    s["slot"] = slot
    return s


def _rotate(x, cos, sin, rotary_dim, style):
    """x [tokens, heads, head_dim] float32; cos, sin [tokens, rotary_dim / 2]."""
    c, n = cos[:, None, :], sin[:, None, :]
    y = x.clone()
    if style == "halves":
        a, b = x[..., : rotary_dim // 2], x[..., rotary_dim // 2: rotary_dim]
        y[..., : rotary_dim // 2] = a * c - b * n
        y[..., rotary_dim // 2: rotary_dim] = b * c + a * n
    else:
        a, b = x[..., 0:rotary_dim:2], x[..., 1:rotary_dim:2]
        y[..., 0:rotary_dim:2] = a * c - b * n
        y[..., 1:rotary_dim:2] = b * c + a * n
    return y


def _append_plain(case, s):
    dt, half = DTYPES[case["dtype"]], case["rotary_dim"] // 2
    row = s["table"][s["position"].long()]
    cos, sin = row[:, :half], row[:, half:]
    q = _rotate(s["q"].float(), cos, sin, case["rotary_dim"], case["style"]).to(dt)
    k = _rotate(s["k"].float(), cos, sin, case["rotary_dim"], case["style"]).to(dt)
    stored = case["tokens"] - case["padding"]          # (padding stands at the end)
    page, offset = s["slot"][:stored] // case["page"], s["slot"][:stored] % case["page"]
    s["cache_k"][page, :, offset] = k[:stored]
    s["cache_v"][page, :, offset] = s["v"][:stored]
    return {"q": q, "k": s["cache_k"], "v": s["cache_v"]}


def _append_exact(case, seed):
    s = _append_inputs(case, seed)
    table = s["table"].double().cpu().numpy()[s["position"].cpu().numpy()]
    R, half = case["rotary_dim"], case["rotary_dim"] // 2
    turn = table[:, :half] + 1j * table[:, half:]      # a rotation is a product of complex numbers

    def rotated(x):
        x = x.double().cpu().numpy()
        z = x[..., :half] + 1j * x[..., half:R] if case["style"] == "halves" else x[..., 0:R:2] + 1j * x[..., 1:R:2]
        z = z * turn[:, None, :]
        y = x.copy()
        if case["style"] == "halves":
            y[..., :half], y[..., half:R] = z.real, z.imag
        else:
            y[..., 0:R:2], y[..., 1:R:2] = z.real, z.imag
        return y

    slot = s["slot"].cpu().numpy()
    k, v = rotated(s["k"]), s["v"].double().cpu().numpy()
    cache_k, cache_v = s["cache_k"].double().cpu().numpy(), s["cache_v"].double().cpu().numpy()
    put = slot >= 0
    cache_k[slot[put] // case["page"], :, slot[put] % case["page"]] = k[put]
    cache_v[slot[put] // case["page"], :, slot[put] % case["page"]] = v[put]
    return {"q": rotated(s["q"]), "k": cache_k, "v": cache_v}


# ---------------------------------------------------------------- attend

def _attend_inputs(case, seed):
    gen, dt = _generator(seed), DTYPES[case["dtype"]]
    D, page, Hk = case["head_dim"], case["page"], case["kv_heads"]
    own_len, new = lengths(case)
    prefix_pages, width = -(-case["prefix"] // page), max(1, -(-max(own_len) // page))
    counts = [-(-n // page) for n in own_len]
    pages = prefix_pages + sum(counts) + 3
    s = {"cache_k": _normal((pages, Hk, page, D), dt, gen), "cache_v": _normal((pages, Hk, page, D), dt, gen)}
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)      # pages lie anywhere
    s["prefix_pages"] = order[:prefix_pages].contiguous()
    table = torch.zeros((case["seqs"], width), dtype=torch.int32, device="cuda")
    at = prefix_pages
    for b, n in enumerate(counts):
        table[b, :n] = order[at: at + n]
        at += n
    s["pages"] = table
    s["own_len"] = torch.tensor(own_len, dtype=torch.int32, device="cuda")
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    s["q_begin"] = torch.tensor(begin, dtype=torch.int32, device="cuda")
    s["q"] = _normal((begin[-1], case["q_heads"], D), dt, gen, std=1.5)
    s["begin"], s["lens"] = begin, own_len
    return s


def _keys_of(cache, pages, length):
    """[kv_heads, length, head_dim] float32 of the first `length` slots of these pages."""
    x = cache[pages.long()]                             # [n, kv_heads, page, head_dim]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :length].float()


def _attend_plain(case, s):
    D, Hk, G = case["head_dim"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    P, page, dt = case["prefix"], case["page"], DTYPES[case["dtype"]]
    T = s["begin"][-1]
    q = (s["q"].float() * D ** -0.5).view(T, Hk, G, D).transpose(0, 1).contiguous()          # [kv_heads, T, G, D]
    out = torch.zeros((Hk, T, G, D), dtype=torch.float32, device="cuda")
    lse = torch.full((Hk, T, G), -math.inf, dtype=torch.float32, device="cuda")
    # the prefix once for all tokens
    pk, pv = _keys_of(s["cache_k"], s["prefix_pages"], P), _keys_of(s["cache_v"], s["prefix_pages"], P)
    for b in range(case["seqs"]):
        t0, t1, L = s["begin"][b], s["begin"][b + 1], s["lens"][b]
        t = t1 - t0
        if t == 0 or P + L == 0:
            continue
        pages = s["pages"][b, : -(-L // page)]
        k, v = torch.cat([pk, _keys_of(s["cache_k"], pages, L)], 1), torch.cat([pv, _keys_of(s["cache_v"], pages, L)], 1)
        x = torch.matmul(q[:, t0:t1].reshape(Hk, t * G, D), k.transpose(1, 2).contiguous()).view(Hk, t, G, P + L)
        if t > 1:
            limit = P + L - t + 1 + torch.arange(t, device="cuda")
            hidden = torch.arange(P + L, device="cuda")[None, :] >= limit[:, None]
            x = torch.where(hidden[None, :, None, :], torch.full_like(x, -math.inf), x)
        m = x.amax(-1, keepdim=True)
        e = torch.exp(x - m)
        total = e.sum(-1, keepdim=True)
        out[:, t0:t1] = torch.matmul(e.view(Hk, t * G, P + L), v).view(Hk, t, G, D) / total
        lse[:, t0:t1] = (m + torch.log(total))[..., 0]
    return {"out": out.transpose(0, 1).reshape(T, Hk * G, D).to(dt), "lse": lse.transpose(0, 1).reshape(T, Hk * G).contiguous()}


def _attend_exact(case, seed):
    s = _attend_inputs(case, seed)
    own_len, new = lengths(case)
    H, Hk, D, P, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["prefix"], case["page"]
    T = sum(new)
    out = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device="cuda")

    def slots(pages, n):                                # [n] indices into the cache as [pages * page] slots
        j = torch.arange(n, device="cuda")
        return pages.long()[j // page] * page + j % page

    shared = slots(s["prefix_pages"], P) if P else torch.zeros(0, dtype=torch.long, device="cuda")
    for h in range(Hk):
        K = s["cache_k"][:, h].reshape(-1, D)
        V = s["cache_v"][:, h].reshape(-1, D)
        at = 0
        for b in range(case["seqs"]):
            n, L = new[b], own_len[b]
            index = torch.cat([shared, slots(s["pages"][b], L)]) if L else shared
            if n and index.numel():
                k, v = K[index].double(), V[index].double()
                for g in range(H // Hk):
                    head = h * (H // Hk) + g
                    score = s["q"][at: at + n, head].double() @ k.T / math.sqrt(D)
                    seen = torch.ones((n, index.numel()), dtype=torch.bool, device="cuda").tril(index.numel() - n)
                    score = score.masked_fill(~seen, -math.inf)
                    lse[at: at + n, head] = torch.logsumexp(score, 1)
                    out[at: at + n, head] = torch.softmax(score, 1) @ v
            at += n
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- sample

def _sample_inputs(case, seed):
    gen, n, V = _generator(seed), case["rows"], case["vocab"]
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda")
    # logits of a language model: they fall with the logarithm of the rank, over vocabulary entries in any order
    rank = torch.argsort(rand(n, V), dim=1).float()
    fall = 1.6 + 0.8 * rand(n, 1)
    logits = 16.0 - fall * torch.log1p(rank) + 0.5 * torch.randn((n, V), generator=gen, device="cuda")
    banned = rand(n, V)
    logits[banned < 0.002] = -math.inf                  # words that are not allowed
    logits[(banned > 0.002) & (banned < 0.004)] = float(torch.finfo(DTYPES[case["dtype"]]).min)
    s = {"logits": logits.to(DTYPES[case["dtype"]])}
    s["uniform"] = rand(n)
    s["temperature"] = 0.6 + 0.6 * rand(n)
    off = torch.arange(n, device="cuda") % 8            # rows in turn: greedy, one rule alone, several together
    s["temperature"][off == 7] = 0.0
    s["top_k"] = torch.randint(1, 200, (n,), generator=gen, device="cuda", dtype=torch.int32)
    s["top_p"] = 0.7 + 0.28 * rand(n)
    s["min_p"] = 0.01 + 0.09 * rand(n)
    s["top_k"][(off == 2) | (off == 3) | (off == 6)] = 0
    s["top_p"][(off == 1) | (off == 3)] = 1.0
    s["min_p"][(off == 0) | (off == 1) | (off == 2)] = 0.0
    if case["flat"]:                                    # no limit on the count: rows cut by mass or weight alone
        s["top_k"].zero_()
        s["top_p"][off == 1] = 0.9
    return s


def _sample_plain(case, s):
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    n, V = x.shape
    top = x.amax(1, keepdim=True)
    greedy = ~(s["temperature"] > 0)
    per_t = 1.0 / torch.where(greedy, torch.ones_like(s["temperature"]), s["temperature"])
    w = torch.exp((x - top) * per_t[:, None])
    w = torch.where(x == top, torch.ones_like(w), w)
    w = torch.where(torch.isneginf(x), torch.zeros_like(w), w)
    mass = (w * MASS_ONE).to(torch.int64)
    value, order = torch.sort(x, dim=1, descending=True, stable=True)
    sorted_mass = torch.gather(mass, 1, order)
    place = torch.arange(V, device="cuda")[None, :]
    k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    sorted_mass = torch.where(place < k, sorted_mass, torch.zeros_like(sorted_mass))
    before = torch.cumsum(sorted_mass, 1) - sorted_mass
    total = sorted_mass.sum(1, keepdim=True)
    need = torch.ceil(s["top_p"].double()[:, None] * total.double()).to(torch.int64).clamp(min=1)
    keep = (place < k) & ((before < need) | ~(s["top_p"][:, None] < 1))
    keep = torch.zeros_like(keep).scatter(1, order, keep)
    keep &= w >= s["min_p"].clamp(max=1.0)[:, None]
    kept = torch.where(keep, mass, torch.zeros_like(mass))
    run = torch.cumsum(kept, 1)
    at = torch.floor(s["uniform"].double()[:, None] * run[:, -1:].double()).to(torch.int64)
    token = (run <= at).sum(1)
    token = torch.where(greedy, order[:, 0], token)
    return torch.where(torch.isneginf(top[:, 0]), torch.full_like(token, -1), token).to(torch.int32)


def _sample_exact(case, seed):
    s = {k: v.double().cpu().numpy() for k, v in _sample_inputs(case, seed).items()}
    out = np.empty(case["rows"], dtype=np.int32)
    for r in range(case["rows"]):
        x = s["logits"][r]
        order = np.argsort(-x, kind="stable")
        T = s["temperature"][r]
        if not np.isfinite(x[order[0]]):
            out[r] = -1
            continue
        if T <= 0:
            out[r] = order[0]
            continue
        w = np.exp((x - x[order[0]]) / T)
        if s["top_k"][r] > 0:
            order = order[: int(s["top_k"][r])]
        if s["top_p"][r] < 1:
            before = np.cumsum(w[order]) - w[order]
            order = order[before < s["top_p"][r] * w[order].sum()]
        order = np.sort(order[w[order] >= s["min_p"][r]])
        run = np.cumsum(w[order])
        out[r] = order[np.searchsorted(run, s["uniform"][r] * run[-1], side="right")]
    return out


# ---------------------------------------------------------------- what the tools call

def prepare(case, seed):
    s = {"append": _append_inputs, "attend": _attend_inputs, "sample": _sample_inputs}[case["kind"]](case, seed)
    if own:
        import paper_2409_06941_amd as fr
        if case["kind"] == "append":
            s["cache"] = fr.KvPages(s["cache_k"], s["cache_v"])
            s["q_out"] = torch.empty((case["tokens"], case["q_heads"], case["head_dim"]), dtype=s["q"].dtype, device="cuda")
        elif case["kind"] == "attend":
            s["cache"] = fr.KvPages(s["cache_k"], s["cache_v"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
            new = max(1, max(b - a for a, b in zip(s["begin"], s["begin"][1:])))
            s["limits"] = dict(prefix_len=case["prefix"], max_own_len=max(s["lens"]), max_q=new)
            need = fr.fr_attend_shared_workspace_bytes(s["cache"], s["q"], case["seqs"], **s["limits"])
            s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        else:
            s["token"] = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
            need = fr.fr_sample_workspace_bytes(s["logits"])
            s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    s["case"] = case
    return s


def run(state):
    case, s = state["case"], state
    if not own:
        return {"append": _append_plain, "attend": _attend_plain, "sample": _sample_plain}[case["kind"]](case, s)
    import paper_2409_06941_amd as fr
    stream = torch.cuda.current_stream()
    if case["kind"] == "append":
        style = fr.FR_ROTARY_HALVES if case["style"] == "halves" else fr.FR_ROTARY_PAIRS
        fr.fr_kv_append(s["cache"], s["k"], s["v"], s["slot"], q=s["q"], q_out=s["q_out"], position=s["position"],
                        rotary=s["table"], style=style, stream=stream)
        return {"q": s["q_out"], "k": s["cache_k"], "v": s["cache_v"]}
    if case["kind"] == "attend":
        fr.fr_attend_shared(s["cache"], s["q"], s["out"], s["pages"], s["own_len"], scale=case["head_dim"] ** -0.5,
                            prefix_pages=s["prefix_pages"], q_begin=s["q_begin"], lse=s["lse"], workspace=s["workspace"],
                            stream=stream, **s["limits"])
        return {"out": s["out"], "lse": s["lse"]}
    fr.fr_sample(s["logits"], s["uniform"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                 min_p=s["min_p"], workspace=s["workspace"], stream=stream)
    return s["token"]


def work(case):
    e = BYTES[case["dtype"]]
    if case["kind"] == "append":
        T, D, stored = case["tokens"], case["head_dim"], case["tokens"] - case["padding"]
        row = (case["q_heads"] + 2 * case["kv_heads"]) * D * e
        moved = T * (row + 4 + 8 + case["rotary_dim"] * 4) + T * case["q_heads"] * D * e + stored * 2 * case["kv_heads"] * D * e
        return {"bytes": moved, "flops": 3 * T * (case["q_heads"] + case["kv_heads"]) * case["rotary_dim"]}
    if case["kind"] == "attend":
        own_len, new = lengths(case)
        D, T = case["head_dim"], sum(new)
        keys = case["prefix"] + sum(n for n, t in zip(own_len, new) if t)
        seen = sum(t * (case["prefix"] + n) - t * (t - 1) // 2 for n, t in zip(own_len, new))
        return {"bytes": 2 * keys * case["kv_heads"] * D * e + 2 * T * case["q_heads"] * D * e + T * case["q_heads"] * 4,
                "flops": 4 * D * case["q_heads"] * seen}
    return {"bytes": case["rows"] * (case["vocab"] * e + 24), "flops": 4 * case["rows"] * case["vocab"]}


def exact(case, seed):
    return {"append": lambda c, s: _append_exact(c, s), "attend": _attend_exact, "sample": _sample_exact}[case["kind"]](case, seed)

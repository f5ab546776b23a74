"""The operators of the 8-bit context cache as a user's program calls them:
attention over the cache (single tokens, the slots of an action expert, whole
prompts, windows with sinks, with or without the attention mass that each
token drew), storing tokens into it, and evicting its lightest tokens.

Definitions (B robots, Hkv KV heads of G = Hq / Hkv query heads each):

* A cache holds a robot's keys and values per KV head in e4m3 (4 exponent and 3
  mantissa bits) with one power of two for each block of 16 tokens, keys and
  values apart: the smallest 2^e, e >= -100, for which the block's largest
  magnitude is at most 448 * 2^e.  Values are rounded to nearest, ties to even.
  When a token arrives in a block that has some, e never falls; where it grows,
  the tokens already there are rounded again.
* Query i of the c that a robot has sits at position p = L - c + i of its L
  tokens; it sees every token (causal = False), the tokens up to p (causal), or
  of those the last `window` and the first `sinks`.  out = softmax(q k / sqrt(hd)) v
  over what it sees; a query that sees nothing, or does not exist, is zeros.
  mass[b, h, j] is the sum of token j's softmax weights over robot b's queries
  and the query heads of KV head h.
* Eviction keeps `keep` tokens of each robot and KV head, in their order: the
  first `sinks`, the last `recent` and the heaviest of the rest (ties: the
  earlier token), and rounds them into blocks of 16 anew.

Sizes are those of this repository's experts (the tiny one, the 18-layer one
with 8 query heads on one KV head of 256, the wider one with 16 on 4 of 64, the
ragged test expert with 6 on 2 of 40), its prefixes of 256 to 2048 tokens and
its batches of 1 to 64 robots, with longer caches for what accumulates over an
episode."""
import math

import torch

own = False

TINY = dict(hq=4, hkv=1, hd=64)
PI05 = dict(hq=8, hkv=1, hd=256)
WIDE = dict(hq=16, hkv=4, hd=64)
ODD = dict(hq=6, hkv=2, hd=40)
BLOCK, TOP, E_MIN = 16, 448.0, -100


def _attend(name, heads, dtype, batch, n, tokens, causal=True, window=0, sinks=0, ragged=False, mass=False):
    """n queries per robot over up to `tokens` cached tokens; ragged: robots of
    different lengths and query counts."""
    return dict(name=name, kind="attend", **heads, dtype=dtype, batch=batch, n=n, tokens=tokens, causal=causal,
                window=window, sinks=sinks, ragged=ragged, mass=mass)


def _store(name, heads, dtype, batch, n, start, ragged=False):
    """n new tokens per robot behind `start` tokens, and the blocks that they
    are in read back."""
    return dict(name=name, kind="store", **heads, dtype=dtype, batch=batch, n=n, start=start, ragged=ragged)


def _evict(name, heads, dtype, batch, tokens, keep, sinks, recent, ragged=False):
    """Caches of up to `tokens` tokens down to `keep`, read back."""
    return dict(name=name, kind="evict", **heads, dtype=dtype, batch=batch, tokens=tokens, keep=keep, sinks=sinks,
                recent=recent, ragged=ragged)


def listed():
    return [
        # one robot decodes a text token (a subtask, say) over its prefix: latency
        _attend("token_b1", PI05, "bf16", 1, 1, 816),
        # the robots of one GPU each decode a token, contexts of every length
        _attend("token_b64", PI05, "bf16", 64, 1, 2048, ragged=True),
        # a few robots whose caches hold a long episode, soon to be evicted from
        _attend("token_long", WIDE, "bf16", 4, 1, 131071, mass=True),
        # the 50 action slots of 16 robots read their prefixes
        _attend("slots_b16", PI05, "bf16", 16, 50, 816, causal=False),
        # whole prompts of 16 robots, every token sees every other
        _attend("prompt_b16", PI05, "bf16", 16, 816, 816, causal=False),
        # a long prompt under a sliding window whose first tokens stay visible
        _attend("prompt_window", WIDE, "bf16", 2, 8191, 8191, window=1024, sinks=4),
        # short prompts in fp32 at ragged sizes
        _attend("fp32_odd", ODD, "fp32", 3, 37, 301, ragged=True),
        # prompts whose tokens' attention mass is wanted for eviction
        _attend("mass_prompt_b4", PI05, "bf16", 4, 816, 816, causal=False, mass=True),
        # every robot of a fleet stores the token that it decoded
        _store("store_token_b64", PI05, "bf16", 64, 1, 816, ragged=True),
        # prompts of 16 robots go into the cache and out to the expert's context
        _store("store_prompt_b16", PI05, "bf16", 16, 816, 0),
        # the prefixes of 64 robots shrink before the expert reads them
        _evict("evict_b64", PI05, "bf16", 64, 816, 256, 4, 32),
        # one long episode shrinks to a fixed budget
        _evict("evict_long", WIDE, "fp32", 1, 65537, 4095, 4, 1024),
    ]


def _log(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() * 1.000001))


def draw(rng):
    most = [work(c) for c in listed()]
    flops, size = max(w["flops"] for w in most), max(w["bytes"] for w in most)
    while True:
        c = _draw(rng)
        pairs = c["batch"] * c["hq"] * c.get("n", 1) * c.get("tokens", 1)   # scores of the plain form
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= size and pairs <= 2 * 16 * 8191 * 8191:
            c.pop("name")
            return c


def _draw(rng):
    heads = rng.choice([TINY, PI05, WIDE, ODD, dict(hq=rng.choice([1, 3, 8]), hkv=1, hd=8 * rng.randint(4, 32)),
                        dict(hq=12, hkv=rng.choice([2, 4, 12]), hd=8 * rng.randint(4, 16))])
    kind = rng.choice(["token", "token", "slots", "prompt", "prompt", "store", "evict"])
    batch = _log(rng, 1, 64)
    ragged = rng.random() < 0.6
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "store":
        n = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
        return _store("", heads, dtype, batch, n, rng.choice([0, _log(rng, 1, 4096)]), ragged)
    if kind == "evict":
        tokens = _log(rng, 200, 65536)
        keep = _log(rng, 64, max(65, tokens))
        return _evict("", heads, dtype, batch, tokens, keep, rng.choice([0, 4, 16]), rng.choice([0, 1, 17, 40]), ragged)
    mass = rng.random() < 0.3
    if kind == "token":
        tokens, n = _log(rng, 64, 131072), 1 if rng.random() < 0.7 else rng.randint(2, 8)
    elif kind == "slots":
        tokens, n = _log(rng, 64, 4096), rng.randint(8, 60)
    else:
        tokens = _log(rng, 64, 8192)
        n = tokens if rng.random() < 0.5 else _log(rng, 60, max(61, tokens))
    causal = rng.random() < 0.6
    window = rng.choice([0, _log(rng, 16, 2048)]) if causal else 0
    return _attend("", heads, dtype, batch, min(n, tokens), tokens, causal, window, rng.choice([0, 4, 20]) if window else 0,
                   ragged, mass)


def _lengths(case):
    """Lengths and query (or token) counts of the robots."""
    most = case.get("tokens", 0) or case["start"]
    batch, n, ragged = case["batch"], case.get("n", 0), case["ragged"]
    lengths = [most - b * 7919 % (most // 2 + 1) if ragged and b else most for b in range(batch)]
    counts = [max(1, n - b * 131 % (n // 2 + 1)) if ragged and b else n for b in range(batch)]
    return lengths, [min(c, m) if case["kind"] == "attend" else c for c, m in zip(counts, lengths)]


def _blocks(n):
    return -(-n // BLOCK)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def work(case):
    hq, hkv, hd, batch = case["hq"], case["hkv"], case["hd"], case["batch"]
    size = 2 if case["dtype"] == "bf16" else 4
    lengths, counts = _lengths(case)
    per = hkv * (2 * hd + 2 / BLOCK)   # bytes of a cached token
    if case["kind"] == "store":
        new = sum(counts)
        back = batch * _back(case)   # what is read back
        return {"bytes": int(new * (2 * hkv * hd * size + per) + back * 2 * hkv * hd * size), "flops": 0}
    if case["kind"] == "evict":
        kept = sum(min(case["keep"], m) for m in lengths)
        return {"bytes": int(sum(lengths) * hkv * 4 + kept * (per + hkv * 8 + 2 * hkv * hd * size)), "flops": 0}
    pairs = tokens = 0
    for m, c in zip(lengths, counts):
        if not case["causal"]:
            pairs, tokens = pairs + m * c, tokens + m
        elif not case["window"]:
            pairs, tokens = pairs + sum(range(m - c + 1, m + 1)), tokens + m
        else:
            w, s = case["window"], case["sinks"]
            pairs += sum(min(p, w) + min(s, max(0, p - w)) for p in range(m - c + 1, m + 1))
            tokens += min(m, c - 1 + w + s)
    moved = 2 * sum(counts) * hq * hd * size + tokens * per + (batch * hkv * case["tokens"] * 4 if case["mass"] else 0)
    return {"bytes": int(moved), "flops": 4 * hd * hq * pairs}


def _back(case):
    """Tokens per robot that are read back from the first block stored into."""
    return case["n"] if not case["start"] else BLOCK * _blocks(case["n"] + BLOCK - 1)


# ---- inputs ---------------------------------------------------------------------


def _inputs(case, seed):
    """Keys and values have channels of different scales, padding is NaN."""
    dev, dt = "cuda", _dtype(case)
    g = torch.Generator(dev).manual_seed(seed)
    hq, hkv, hd, batch = case["hq"], case["hkv"], case["hd"], case["batch"]
    lengths, counts = _lengths(case)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    channels = torch.exp(0.5 * normal(hkv, hd))

    def kv(tokens):
        return (normal(batch, tokens, hkv, hd) * channels).to(dt), normal(batch, tokens, hkv, hd).to(dt)

    def padded(x, counts):
        there = torch.arange(x.shape[1], device=dev)[None] < ints(counts)[:, None]
        return torch.where(there[:, :, None, None], x, torch.full_like(x, math.nan))

    if case["kind"] == "store":
        starts = lengths if case["start"] else [0] * batch
        k, v = kv(case["n"])
        old_k, old_v = kv(BLOCK)
        return dict(k=padded(k, counts), v=padded(v, counts), old_k=old_k, old_v=old_v, starts=ints(starts),
                    counts=ints(counts), firsts=ints([s // BLOCK * BLOCK for s in starts]),
                    filled=ints([s % BLOCK for s in starts]), ends=ints([s + c for s, c in zip(starts, counts)]))
    k, v = kv(case["tokens"])
    out = dict(k=padded(k, lengths), v=padded(v, lengths), lengths=ints(lengths))
    if case["kind"] == "evict":
        out["mass"] = torch.rand((batch, hkv, case["tokens"]), generator=g, device=dev) ** 4
        return out
    q = (2.0 * normal(batch, case["n"], hq, hd)).to(dt)
    out.update(q=padded(q, counts), counts=ints(counts))
    return out


def prepare(case, seed):
    x = _inputs(case, seed)
    dev = x["k"].device
    state = dict(case=case, x=x)
    batch = case["batch"]
    if own:
        from paper_2609_34170_gb300 import ContextCache

        def cache(tokens):
            return ContextCache(layers=1, n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["hd"],
                                max_tokens=tokens, max_batch=batch, max_queries=case.get("n", 1), dtype=case["dtype"])

        zero = torch.zeros(batch, dtype=torch.int32, device=dev)
        if case["kind"] == "store":
            most = int(x["firsts"].max()) + BLOCK * _blocks(case["n"] + BLOCK)
            state["cache"] = cache(most)
            state["cache"].append(0, x["old_k"], x["old_v"], x["firsts"], counts=x["filled"])
        else:
            state["cache"] = cache(case["tokens"])
            state["cache"].append(0, x.pop("k"), x.pop("v"), zero, counts=x["lengths"])
            if case["kind"] == "evict":
                state["to"] = cache(case["keep"])
            else:
                state["out"] = torch.empty_like(x["q"])
                state["mass"] = (torch.empty((batch, case["hkv"], case["tokens"]), device=dev) if case["mass"] else None)
        torch.cuda.synchronize()
    elif case["kind"] == "store":
        state["old"] = _quantise(x["old_k"].float(), x["old_v"].float(), x["filled"])
    else:
        state["held"] = _quantise(x.pop("k").float(), x.pop("v").float(), x["lengths"])
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    case, x, cache = state["case"], state["x"], state["cache"]
    if case["kind"] == "store":
        cache.append(0, x["k"], x["v"], x["starts"], counts=x["counts"])
        return cache.read(0, case["batch"], _back(case), firsts=x["firsts"], lengths=x["ends"])
    if case["kind"] == "evict":
        lengths, index, mass = cache.evict(0, state["to"], 0, x["lengths"], x["mass"], case["keep"], sinks=case["sinks"],
                                           recent=case["recent"])
        k, v = state["to"].read(0, case["batch"], case["keep"], lengths=lengths)
        return lengths, index, mass, k, v
    out = cache.attend(0, x["q"], x["lengths"], counts=x["counts"], causal=case["causal"], window=case["window"],
                       sinks=case["sinks"], out=state["out"], mass=state["mass"])
    return out if state["mass"] is None else (out, state["mass"])


# ---- the plain form ---------------------------------------------------------------
# A cache here is (key codes, key exponents, value codes, value exponents): codes
# [B, Hkv, blocks, 16, hd] e4m3, exponents [B, Hkv, blocks] int8.


def _exponent(x, least=E_MIN):
    """The blocks' exponents e: max |x| <= 448 * 2^e; x [..., 16, hd]."""
    most = x.abs().amax((-1, -2))
    part, e = torch.frexp(most)
    return torch.clamp(torch.where(most > 0, e - 9 + (part > 0.875).int(), E_MIN), min=least)


def _codes(x, e):
    return torch.ldexp(x, -e[..., None, None]).to(torch.float8_e4m3fn)


def _fit(x):
    """[B, T, H, hd] -> [B, H, blocks, 16, hd], zeros behind."""
    more = _blocks(x.shape[1]) * BLOCK - x.shape[1]
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, more)).transpose(1, 2)
    return x.reshape(*x.shape[:2], -1, BLOCK, x.shape[-1])


def _quantise(k, v, counts):
    there = (torch.arange(k.shape[1], device=k.device)[None] < counts[:, None])[:, :, None, None]
    out = []
    for x in (k, v):
        x = _fit(torch.where(there, x, torch.zeros_like(x)))
        e = _exponent(x)
        out += [_codes(x, e), e.to(torch.int8)]
    return out


def _values(codes, e):
    """[B, H, T, hd] fp32"""
    return torch.ldexp(codes.float(), e.int()[..., None, None]).flatten(2, 3)


def _run_plain(state):
    case, x = state["case"], state["x"]
    return {"store": _plain_store, "evict": _plain_evict, "attend": _plain_attend}[case["kind"]](state, case, x)


def _plain_store(state, case, x):
    n, back, dt = case["n"], _back(case), _dtype(case)
    dev = x["k"].device
    place = torch.arange(BLOCK * _blocks(n + BLOCK), device=dev)[None]   # from the first block on
    at = place - x["filled"][:, None]                                     # index among the new tokens
    new = (at >= 0) & (at < x["counts"][:, None])
    out = []
    for name, codes, e_old in (("k", *state["old"][:2]), ("v", *state["old"][2:])):
        rows = torch.gather(x[name].float(), 1, at.clamp(0, n - 1)[:, :, None, None].expand(-1, -1, *x[name].shape[2:]))
        rows = _fit(torch.where(new[:, :, None, None], rows, torch.zeros_like(rows)))
        e = _exponent(rows)
        some = (x["filled"] > 0)[:, None]
        e[:, :, 0] = torch.where(some, torch.maximum(e[:, :, 0], e_old[:, :, 0].int()), e[:, :, 0])
        old = _values(codes, e_old)   # zeros where nothing is
        rows[:, :, 0] += old
        out.append(_values(_codes(rows, e), e)[:, :, :back].to(dt).contiguous())
    return tuple(out)


def _plain_evict(state, case, x):
    kc, ke, vc, ve = state["held"]
    keep, tokens = case["keep"], case["tokens"]
    place = torch.arange(tokens, device=kc.device)[None, None]
    m = x["lengths"][:, None, None]
    always = (place < case["sinks"]) | (place >= m - case["recent"])
    rank = torch.where(always, math.inf, x["mass"])
    rank = torch.where(place < m, rank, -math.inf)
    index = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :min(keep, tokens)]
    index = torch.where(torch.gather(rank, 2, index) > -math.inf, index, tokens).sort(-1).values
    index = torch.nn.functional.pad(index, (0, keep - index.shape[-1]), value=tokens)
    there = index < tokens
    lengths = x["lengths"].clamp(max=keep)
    safe = index.clamp(max=tokens - 1)
    mass = torch.where(there, torch.gather(x["mass"], 2, safe), 0.0)
    out = []
    for codes, e in ((kc, ke), (vc, ve)):
        rows = torch.gather(_values(codes, e), 2, safe[..., None].expand(-1, -1, -1, case["hd"]))
        rows = _fit(torch.where(there[..., None], rows, 0.0).transpose(1, 2))
        e2 = _exponent(rows)
        out.append(_values(_codes(rows, e2), e2)[:, :, :keep].to(_dtype(case)).contiguous())
    return lengths, torch.where(there, index, -1).int(), mass, *out


def _visible(case, lengths, counts, lo, hi):
    """[B, hi - lo, tokens]: what queries lo .. hi - 1 see."""
    dev = lengths.device
    i = torch.arange(lo, hi, device=dev)[None, :, None]
    j = torch.arange(case["tokens"], device=dev)[None, None]
    m, c = lengths[:, None, None], counts[:, None, None]
    see = (j < m) & (i < c)
    if case["causal"]:
        p = m - c + i
        see &= j <= p
        if case["window"]:
            see &= (j > p - case["window"]) | (j < case["sinks"])
    return see


def _plain_attend(state, case, x):
    batch, n, hq, hkv, hd, tokens = (case[k] for k in ("batch", "n", "hq", "hkv", "hd", "tokens"))
    k = _values(*state["held"][:2])[:, :, :tokens]
    v = _values(*state["held"][2:])[:, :, :tokens]
    q = x["q"].float().reshape(batch, n, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4) / math.sqrt(hd)
    out = torch.empty((batch, n, hkv, hq // hkv, hd), device=q.device)
    mass = torch.zeros((batch, hkv, tokens), device=q.device)
    step = max(1, (1 << 28) // (batch * hq * tokens))
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        see = _visible(case, x["lengths"], x["counts"], lo, hi)[:, None, None]
        s = torch.where(see, q[:, :, :, lo:hi] @ k[:, :, None].transpose(-1, -2), -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
        out[:, lo:hi] = (p @ v[:, :, None]).permute(0, 3, 1, 2, 4)
        if case["mass"]:
            mass += p.sum((2, 3))
    out = out.reshape(batch, n, hq, hd).to(_dtype(case))
    return (out, mass) if case["mass"] else out


# ---- the definition in 64 bits -------------------------------------------------------


def _held64(x):
    """What a block [..., 16, hd] holds, in 64 bits."""
    x = x.double()
    top = x.abs().flatten(-2).max(-1).values
    e = torch.full_like(top, float(E_MIN))
    some = top > 0
    e[some] = torch.ceil(torch.log2(top[some]) - math.log2(TOP))
    for step in (1.0, -1.0):   # the logarithm may be off by one
        e = torch.where(some & (top > TOP * torch.exp2(e)), e + step, e) if step > 0 else \
            torch.where(some & (top <= TOP * torch.exp2(e - 1)), e - 1, e)
    return _round64(x, e.clamp(min=E_MIN)), e.clamp(min=E_MIN)


def _round64(x, e):
    unit = torch.exp2(e)[..., None, None]
    y = x / unit
    size = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -40)))
    size = torch.where(y.abs() < torch.exp2(size), size - 1, torch.where(y.abs() >= torch.exp2(size + 1), size + 1, size))
    grid = torch.exp2(size.clamp(min=-6) - 3)
    return torch.round(y / grid) * grid * unit


def _split64(x, counts):
    """[B, T, H, hd] -> held values [B, H, T', hd], T' a multiple of 16."""
    x = x.double().transpose(1, 2).clone()
    for b, c in enumerate(counts):
        x[b, :, c:] = 0
    full = torch.zeros((*x.shape[:2], _blocks(x.shape[2]) * BLOCK, x.shape[3]), dtype=x.dtype, device=x.device)
    full[:, :, :x.shape[2]] = x
    return _held64(full.unflatten(2, (-1, BLOCK)))[0].flatten(2, 3)


def exact(case, seed):
    x = _inputs(case, seed)
    lengths, counts = _lengths(case)
    dt = torch.float64
    if case["kind"] == "store":
        back, out = _back(case), []
        for new, old in ((x["k"], x["old_k"]), (x["v"], x["old_v"])):
            res = torch.zeros((case["batch"], case["hkv"], back, case["hd"]), dtype=dt, device=new.device)
            for b in range(case["batch"]):
                fill, c = int(x["filled"][b]), counts[b]
                rows = torch.zeros((case["hkv"], BLOCK * _blocks(fill + c), case["hd"]), dtype=dt, device=new.device)
                rows[:, fill:fill + c] = new[b, :c].double().transpose(0, 1)
                held, e = _held64(rows.unflatten(1, (-1, BLOCK)))
                if fill:
                    first = torch.zeros((case["hkv"], BLOCK, case["hd"]), dtype=dt, device=new.device)
                    first[:, :fill] = old[b, :fill].double().transpose(0, 1)
                    first, e_old = _held64(first)
                    first[:, fill:] = rows[:, fill:BLOCK]
                    held[:, 0] = _round64(first, torch.maximum(e[:, 0], e_old))
                held = held.flatten(1, 2)[:, :back]
                res[b, :, :held.shape[1]] = held
            out.append(res)
        return tuple(out)
    k, v = (_split64(x[name], lengths) for name in ("k", "v"))
    if case["kind"] == "evict":
        return _exact_evict(case, x, k, v, lengths)
    batch, n, hq, hkv, hd, tokens = (case[name] for name in ("batch", "n", "hq", "hkv", "hd", "tokens"))
    group = hq // hkv
    out = torch.zeros((batch, n, hq, hd), dtype=dt, device=k.device)
    mass = torch.zeros((batch, hkv, tokens), dtype=dt, device=k.device)
    step = max(1, (1 << 26) // (group * tokens))
    for b in range(batch):
        m, c = lengths[b], counts[b]
        j = torch.arange(m, device=k.device)[None]
        for lo in range(0, c, step):
            hi = min(c, lo + step)
            p = m - c + torch.arange(lo, hi, device=k.device)[:, None]
            hide = torch.zeros((hi - lo, m), dtype=torch.bool, device=k.device)
            if case["causal"]:
                hide |= j > p
            if case["window"]:
                hide |= (j <= p - case["window"]) & (j >= case["sinks"])
            for h in range(hkv):
                q = x["q"][b, lo:hi, h * group:(h + 1) * group].double()
                s = torch.einsum("igd,jd->igj", q, k[b, h, :m]) / hd ** 0.5
                w = torch.softmax(s.masked_fill(hide[:, None], -math.inf), -1)
                out[b, lo:hi, h * group:(h + 1) * group] = torch.einsum("igj,jd->igd", w, v[b, h, :m])
                mass[b, h, :m] += w.sum((0, 1))
    return (out, mass) if case["mass"] else out


def _exact_evict(case, x, k, v, lengths):
    batch, hkv, keep = case["batch"], case["hkv"], case["keep"]
    dev = k.device
    index = torch.full((batch, hkv, keep), -1, dtype=torch.int32, device=dev)
    mass = torch.zeros((batch, hkv, keep), dtype=torch.float64, device=dev)
    rows = [torch.zeros((batch, hkv, _blocks(keep) * BLOCK, case["hd"]), dtype=torch.float64, device=dev) for _ in "kv"]
    for b in range(batch):
        m = lengths[b]
        for h in range(hkv):
            if m <= keep:
                chosen = torch.arange(m, device=dev)
            else:
                s, r = case["sinks"], case["recent"]
                rest = torch.sort(-x["mass"][b, h, s:m - r], stable=True).indices[:keep - s - r] + s
                chosen = torch.cat([torch.arange(s, device=dev), rest, torch.arange(m - r, m, device=dev)]).sort().values
            n = len(chosen)
            index[b, h, :n] = chosen.int()
            mass[b, h, :n] = x["mass"][b, h, chosen].double()
            rows[0][b, h, :n] = k[b, h, chosen]
            rows[1][b, h, :n] = v[b, h, chosen]
    held = [_held64(r.unflatten(2, (-1, BLOCK)))[0].flatten(2, 3)[:, :, :keep] for r in rows]
    return x["lengths"].clamp(max=keep), index, mass, *held

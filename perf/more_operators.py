"""The operators of a VLM's decode step beside the context cache as a user's
program calls them: rotary positions (on their own and on the way into the
cache), products of few rows with 4-bit weights, and drawing a token from
logits.

Definitions:

* Rotary positions.  Of a head's dims the first `dims` turn in pairs, (i, i +
  dims / 2) or interleaved (2i, 2i + 1): by the angle a = p f_i, p the token's
  position, (x, y) becomes amplitude * (x cos a - y sin a, x sin a + y cos a); the
  other dims stay.  f_i = base^(-2i / dims), divided by `factor`; with an original
  length, a frequency that makes t = length * f_i / 2 pi turns over it is divided
  in full for t <= low, not at all for t >= high, and in between is
  f_i (g + (1 - g) / factor), g = (t - low) / (high - low).
* Storing with rotation.  A token's query heads and its key are turned to its
  position; key and value go into the 8-bit cache (e4m3 values under one power
  of two for each block of 16 tokens, the smallest 2^e, e >= -100, for which the
  block's largest magnitude is at most 448 * 2^e).  Nothing but that rounding
  lies between the turned key and the cache.
* 4-bit weights.  Row n of a [N, K] matrix is w[n, k] = (c - z) s with a code c of
  0 .. 15 for each k and a zero point z of 0 .. 15 and a scale s for each group of
  `group` ks.  y = x w^T + bias; then stored, SiLU(y) stored, added to a residual
  stream, or GeGLU: rows come in blocks of 64 gate rows and the 64 matching up
  rows, gelu_tanh(gate) * up is stored.
* Drawing a token.  Of logits x and a temperature T, weight w_i = exp((x_i - max x) / T).
  Tokens are ordered by their logit, equal ones by their index.  What stays: the
  first top_k of them; of those the shortest run from the first on whose weights
  sum to at least top_p of their sum; of those the ones with w_i >= min_p.  The
  token drawn is the lowest index for which the weights of what stays, summed in
  the order of the index, exceed u times their sum; its log-probability is
  log(w_i / sum).  T = 0: the first token of the order, log-probability 0.  A
  logit of -inf is never drawn.

Sizes are those of this repository's experts (the 18-layer one with 8 query heads
on one KV head of 256, width 1024 and an MLP of 4096; the wider one with 16 heads
on 4 of 64; the ragged test expert with 6 on 2 of 40), its prefixes and batches of
1 to 64 robots, with generic larger matrices, vocabularies and lengths."""
import math

import torch

own = False

PI05 = dict(hq=8, hkv=1, hd=256)
WIDE = dict(hq=16, hkv=4, hd=64)
ODD = dict(hq=6, hkv=2, hd=40)
BLOCK, TOP, E_MIN = 16, 448.0, -100


def _turn(name, heads, dtype, batch, n, dims, first=0, interleaved=False, base=10000.0, factor=1.0, length=0, ragged=False):
    """Query and key heads of n tokens per robot, columns of a projection's rows,
    from position `first` on; ragged: robots of different positions and counts."""
    return dict(name=name, kind="turn", **heads, dtype=dtype, batch=batch, n=n, dims=dims, first=first,
                interleaved=interleaved, base=base, factor=factor, length=length, ragged=ragged)


def _store(name, heads, batch, n, start, dims, gap=0, interleaved=False, base=10000.0, factor=1.0, length=0, ragged=False):
    """n new tokens per robot into a cache behind `start` tokens, at positions `gap`
    further on (what an eviction took away), and the blocks that they are in read
    back."""
    return dict(name=name, kind="store", **heads, dtype="bf16", batch=batch, n=n, start=start, dims=dims, gap=gap,
                interleaved=interleaved, base=base, factor=factor, length=length, ragged=ragged)


def _product(name, m, n, k, group, epi="store", out="bf16", bias=False):
    """m rows of K = k values times N = n rows of 4-bit weights."""
    return dict(name=name, kind="product", m=m, n=n, k=k, group=group, epi=epi, out=out, bias=bias)


def _draw_token(name, dtype, batch, vocab, temperature, top_k=0, top_p=1.0, min_p=0.0, spread=3.0, mixed=False):
    """A token for each robot; mixed: every robot has settings of its own, every
    fourth takes the likeliest token and every third has most of its vocabulary
    masked."""
    return dict(name=name, kind="draw", dtype=dtype, batch=batch, vocab=vocab, temperature=temperature, top_k=top_k,
                top_p=top_p, min_p=min_p, spread=spread, mixed=mixed)


def listed():
    return [
        # prompts of 16 robots: Q and K columns of the projection before they are attended to
        _turn("turn_prompt_b16", PI05, "bf16", 16, 816, 256),
        # one long context in fp32, half of each head, frequencies stretched for eight times the length
        _turn("turn_long", WIDE, "fp32", 1, 65536, 32, interleaved=True, base=500000.0, factor=8.0, length=8192),
        # every robot of a fleet stores the token that it decoded, far behind an evicted prefix
        _store("store_token_b64", PI05, 64, 1, 816, 256, gap=100000, factor=4.0, ragged=True),
        # prompts of ragged length go into the cache
        _store("store_prompt_b16", WIDE, 16, 816, 0, 64, interleaved=True, ragged=True),
        # one robot's decode: the projection to queries, keys and values
        _product("qkv_b1", 1, 2560, 1024, 128),
        # four robots: gate and up projection with GeGLU
        _product("gate_up_b4", 4, 8192, 1024, 64, epi="geglu"),
        # sixteen robots: down projection into the residual stream
        _product("down_b16", 16, 1024, 4096, 32, epi="add", out="fp32"),
        # a few rows of sizes that fit no tile
        _product("odd", 3, 777, 1003, 32, epi="silu", out="fp32", bias=True),
        # a fleet's logits over a large vocabulary, the largest matrix
        _product("head_b64", 64, 65536, 8192, 128, out="fp32"),
        # one robot's next token under the usual three limits: latency
        _draw_token("draw_b1", "bf16", 1, 65536, 0.8, top_k=40, top_p=0.95, min_p=0.02),
        # a fleet over a large vocabulary, most of the mass stays
        _draw_token("draw_b64", "fp32", 64, 128001, 1.0, top_p=0.9),
        # robots with settings and masks of their own, flat logits with many ties
        _draw_token("draw_mixed_b24", "bf16", 24, 32003, 1.3, top_k=500, top_p=0.8, min_p=0.01, spread=0.5, mixed=True),
    ]


def _log(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() * 1.000001))


def draw(rng):
    most = [work(c) for c in listed()]
    flops, size = max(w["flops"] for w in most), max(w["bytes"] for w in most)
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= size and (c["kind"] in ("product", "draw") or w["bytes"] <= 300e6):
            c.pop("name")
            return c


def _draw(rng):
    kind = rng.choice(["turn", "store", "product", "product", "draw", "draw"])
    if kind == "product":
        epi = rng.choice(["store", "store", "silu", "add", "geglu"])
        n = 128 * _log(rng, 1, 256) if epi == "geglu" else _log(rng, 40, 65536)
        out = {"add": "fp32", "geglu": "bf16"}.get(epi) or rng.choice(["bf16", "fp32"])
        k = _log(rng, 40, 8192)
        return _product("", 1 if rng.random() < 0.25 else _log(rng, 1, 64), n, k if rng.random() < 0.3 else 8 * -(-k // 8),
                        rng.choice([32, 64, 128]), epi, out, rng.random() < 0.4)
    if kind == "draw":
        return _draw_token("", rng.choice(["bf16", "fp32"]), _log(rng, 1, 64), _log(rng, 200, 200000), 0.3 + 1.4 * rng.random(),
                           rng.choice([0, 0, _log(rng, 1, 2000)]), rng.choice([1.0, 0.3 + 0.69 * rng.random()]),
                           rng.choice([0.0, 0.1 * rng.random()]), rng.choice([0.2, 1.0, 3.0, 6.0]), rng.random() < 0.4)
    heads = rng.choice([PI05, WIDE, ODD, dict(hq=rng.choice([1, 3, 8]), hkv=1, hd=8 * rng.randint(2, 32)),
                        dict(hq=12, hkv=rng.choice([2, 4, 12]), hd=8 * rng.randint(4, 16))])
    dims = heads["hd"] if rng.random() < 0.6 else 2 * rng.randint(1, heads["hd"] // 2)
    n = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
    more = dict(interleaved=rng.random() < 0.5, base=rng.choice([1e4, 5e5]), factor=rng.choice([1.0, 4.0, 8.0]),
                length=rng.choice([0, 2048, 8192]), ragged=rng.random() < 0.5)
    batch = _log(rng, 1, 64)
    if kind == "turn":
        return _turn("", heads, rng.choice(["bf16", "fp32"]), batch, n, dims, rng.choice([0, _log(rng, 1, 1000000)]), **more)
    return _store("", heads, batch, n, rng.choice([0, _log(rng, 1, 4096)]), dims, rng.choice([0, _log(rng, 1, 100000)]), **more)


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _counts(case):
    """Where each robot's tokens begin (in the cache, or their position), and how many there are."""
    batch, n = case["batch"], case["n"]
    at = case["start"] if case["kind"] == "store" else case["first"]
    if not case["ragged"]:
        return [at] * batch, [n] * batch
    return ([at - b * 7919 % (at // 2 + 1) if b else at for b in range(batch)],
            [max(1, n - b * 131 % (n // 2 + 1)) if b else n for b in range(batch)])


def _blocks(n):
    return -(-n // BLOCK)


def _back(case):
    """Tokens per robot that are read back from the first block stored into."""
    return case["n"] if not case["start"] else BLOCK * _blocks(case["n"] + BLOCK - 1)


def work(case):
    kind = case["kind"]
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        groups = -(-k // case["group"])
        wide = 2 if case["out"] == "bf16" else 4
        outs = m * (n // 2 if case["epi"] == "geglu" else n) * wide * (2 if case["epi"] == "add" else 1)
        return {"bytes": int(n * k / 2 + n * groups * 2.5 + 2 * m * k + outs + (4 * n if case["bias"] else 0)), "flops": 2 * m * n * k}
    if kind == "draw":
        # a row's logits once; an exponential and a sum each (counted as eight operations)
        return {"bytes": case["batch"] * (case["vocab"] * _size(case) + 28), "flops": 8 * case["batch"] * case["vocab"]}
    hq, hkv, hd, size = case["hq"], case["hkv"], case["hd"], _size(case)
    new = sum(_counts(case)[1])
    flops = 6 * new * (hq + hkv) * case["dims"] // 2
    if kind == "turn":
        return {"bytes": 2 * new * (hq + hkv) * hd * size, "flops": flops}
    held = hkv * (2 * hd + 2 / BLOCK)
    return {"bytes": int(new * (2 * hq * hd * size + 2 * hkv * hd * size + held) + case["batch"] * _back(case) * 2 * hkv * hd * size),
            "flops": flops}


# ---- inputs ---------------------------------------------------------------------


def _inputs(case, seed):
    return {"turn": _token_inputs, "store": _token_inputs, "product": _product_inputs, "draw": _logit_inputs}[case["kind"]](case, seed)


def _token_inputs(case, seed):
    """Keys have channels of different scales."""
    dev, dt = "cuda", _dtype(case["dtype"])
    g = torch.Generator(dev).manual_seed(seed)
    hq, hkv, hd, batch, n = case["hq"], case["hkv"], case["hd"], case["batch"], case["n"]
    starts, counts = _counts(case)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    channels = torch.exp(0.5 * normal(hq + 2 * hkv, hd))
    qkv = (normal(batch, n, hq + 2 * hkv, hd) * channels).to(dt)
    x = dict(qkv=qkv, starts=ints(starts), counts=ints(counts))
    if case["kind"] == "store":
        x["positions"] = x["starts"][:, None] + torch.arange(n, dtype=torch.int32, device=dev)[None] + case["gap"]
        x["old_k"], x["old_v"] = ((normal(batch, BLOCK, hkv, hd) * channels[at:at + hkv]).to(dt) for at in (hq, hq + hkv))
        x["firsts"] = ints([s // BLOCK * BLOCK for s in starts])
        x["filled"] = ints([s % BLOCK for s in starts])
        x["ends"] = ints([s + c for s, c in zip(starts, counts)])
    return x


def _product_inputs(case, seed):
    """Codes as a round-to-nearest quantiser of bell-shaped weights leaves them;
    activations with channels of different scales."""
    dev = "cuda"
    g = torch.Generator(dev).manual_seed(seed)
    m, n, k = case["m"], case["n"], case["k"]
    groups = -(-k // case["group"])
    pairs = -(-k // 2)
    codes = torch.empty((n, pairs), dtype=torch.uint8, device=dev)
    for part in codes.split(8192):   # low nibble: even k
        c = (torch.randn((*part.shape, 2), generator=g, device=dev) * 2.6 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
        part.copy_(c[..., 0] | c[..., 1] << 4)
    scales = ((0.5 + torch.rand((n, groups), generator=g, device=dev)) / (2.6 * math.sqrt(k))).to(torch.bfloat16)
    zeros = torch.randint(6, 10, (n, groups), generator=g, device=dev, dtype=torch.uint8)
    x = torch.randn((m, k), generator=g, device=dev) * torch.exp(0.5 * torch.randn((k,), generator=g, device=dev))
    bias = 0.5 * torch.randn((n,), generator=g, device=dev) if case["bias"] else None
    out = torch.randn((m, n), generator=g, device=dev) if case["epi"] == "add" else None
    return dict(codes=codes, scales=scales, zeros=zeros, x=x.to(torch.bfloat16), bias=bias, residual=out)


def _logit_inputs(case, seed):
    dev = "cuda"
    g = torch.Generator(dev).manual_seed(seed)
    batch, vocab = case["batch"], case["vocab"]
    x = case["spread"] * torch.randn((batch, vocab), generator=g, device=dev)
    rows = torch.arange(batch, device=dev)
    full = dict(u=torch.rand((batch,), generator=g, device=dev))
    ones = torch.ones((batch,), device=dev)
    t, k, p, q = ones * case["temperature"], (ones * case["top_k"]).int(), ones * case["top_p"], ones * case["min_p"]
    if case["mixed"]:
        t = torch.where(rows % 4 == 3, 0.0, t * (0.6 + 0.4 * (rows % 3)))
        k = torch.where(rows % 5 == 1, 0, k + 7 * rows.int()).int()
        p = torch.where(rows % 7 == 2, 1.0, p * (0.9 + 0.02 * (rows % 6)))
        q = torch.where(rows % 2 == 0, 0.0, q)
        hide = torch.rand((batch, vocab), generator=g, device=dev) < 0.9
        x = torch.where(hide & (rows % 3 == 1)[:, None], -math.inf, x)
    full.update(logits=x.to(_dtype(case["dtype"])), temperature=t, top_k=k, top_p=p, min_p=q)
    return full


def _rotary_settings(case):
    return dict(base=case["base"], interleaved=case["interleaved"], factor=case["factor"], original_length=case["length"])


def prepare(case, seed):
    x = _inputs(case, seed)
    state = dict(case=case, x=x)
    kind = case["kind"]
    if kind == "product":
        cols = case["n"] // 2 if case["epi"] == "geglu" else case["n"]
        state["out"] = x.pop("residual") if case["epi"] == "add" else \
            torch.empty((case["m"], cols), dtype=_dtype(case["out"]), device=x["x"].device)
    elif kind == "turn":
        state["out"] = torch.zeros((case["batch"], case["n"], case["hq"] + case["hkv"], case["hd"]), dtype=x["qkv"].dtype,
                                   device=x["qkv"].device)
    elif kind == "store":
        state["q_out"] = torch.zeros_like(x["qkv"][:, :, :case["hq"]])
        if not own:
            state["old"] = _quantise(x["old_k"].float(), x["old_v"].float(), x["filled"])
    if own:
        _prepare_own(state, case, x)
        torch.cuda.synchronize()
    return state


def _prepare_own(state, case, x):
    from paper_2609_34170_gb300 import ContextCache, Rotary, Weights4
    kind = case["kind"]
    if kind == "product":
        state["w"] = Weights4(case["n"], case["k"], case["group"])
        state["w"].load(x.pop("codes"), x.pop("scales"), x.pop("zeros"))
    if kind in ("turn", "store"):
        state["rotary"] = Rotary(case["dims"], **_rotary_settings(case))
    if kind == "store":
        most = int(x["firsts"].max()) + BLOCK * _blocks(case["n"] + BLOCK)
        state["cache"] = ContextCache(layers=1, n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["hd"],
                                      max_tokens=most, max_batch=case["batch"], max_queries=1)
        state["cache"].append(0, x["old_k"], x["old_v"], x["firsts"], counts=x["filled"])


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    case, x = state["case"], state["x"]
    kind, hq, hkv = case["kind"], case.get("hq"), case.get("hkv")
    if kind == "product":
        return state["w"].product(x["x"], out=state["out"], epi=case["epi"], bias=x["bias"])
    if kind == "draw":
        from paper_2609_34170_gb300 import draw_tokens
        return draw_tokens(x["logits"], x["u"], temperature=x["temperature"], top_k=x["top_k"], top_p=x["top_p"], min_p=x["min_p"],
                           log_probs=True)
    if kind == "turn":
        return state["rotary"].apply(x["qkv"][:, :, :hq + hkv], starts=x["starts"], counts=x["counts"], out=state["out"])
    qkv, cache = x["qkv"], state["cache"]
    q = cache.append_rotary(0, state["rotary"], qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], x["starts"],
                            counts=x["counts"], positions=x["positions"], q_out=state["q_out"])
    return q, *cache.read(0, case["batch"], _back(case), firsts=x["firsts"], lengths=x["ends"])


# ---- the plain form ---------------------------------------------------------------


def _run_plain(state):
    case, x = state["case"], state["x"]
    return {"turn": _plain_turn, "store": _plain_store, "product": _plain_product, "draw": _plain_draw}[case["kind"]](state, case, x)


def _cos_sin(case, positions):
    """[B, n, 1, dims / 2] fp32: the angles in 64 bits."""
    i = torch.arange(case["dims"] // 2, device=positions.device, dtype=torch.float64)
    f = case["base"] ** (-2.0 * i / case["dims"])
    if case["length"]:
        turns = case["length"] * f / (2 * math.pi)
        g = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (g + (1.0 - g) / case["factor"])
    else:
        f = f / case["factor"]
    a = positions.double()[:, :, None, None] * f
    return torch.cos(a).float(), torch.sin(a).float()


def _turned(case, x, positions):
    """fp32 [B, n, H, hd]"""
    d = case["dims"]
    c, s = _cos_sin(case, positions)
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:d:2], y[..., 1:d:2]
        turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    else:
        a, b = y[..., :d // 2], y[..., d // 2:d]
        turned = torch.cat((a * c - b * s, a * s + b * c), -1)
    return torch.cat((turned, y[..., d:]), -1)


def _there(x, n):
    return (torch.arange(n, device=x["counts"].device)[None] < x["counts"][:, None])[:, :, None, None]


def _plain_turn(state, case, x):
    heads = x["qkv"][:, :, :case["hq"] + case["hkv"]]
    positions = x["starts"][:, None].long() + torch.arange(case["n"], device=heads.device)[None]
    y = _turned(case, heads, positions).to(heads.dtype)
    return torch.where(_there(x, case["n"]), y, state["out"])


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


def _quantise_one(x, counts):
    there = (torch.arange(x.shape[1], device=x.device)[None] < counts[:, None])[:, :, None, None]
    x = _fit(torch.where(there, x, torch.zeros_like(x)))
    e = _exponent(x)
    return _codes(x, e), e.to(torch.int8)


def _quantise(k, v, counts):
    return *_quantise_one(k, counts), *_quantise_one(v, counts)


def _values(codes, e):
    """[B, H, T, hd] fp32"""
    return torch.ldexp(codes.float(), e.int()[..., None, None]).flatten(2, 3)


def _stored(case, x, new, codes, e_old):
    """Values read back of new tokens [B, n, Hkv, hd] stored behind those held."""
    n, back = case["n"], _back(case)
    dev = new.device
    place = torch.arange(BLOCK * _blocks(n + BLOCK), device=dev)[None]   # from the first block on
    at = place - x["filled"][:, None]                                     # index among the new tokens
    fresh = (at >= 0) & (at < x["counts"][:, None])
    rows = torch.gather(new, 1, at.clamp(0, n - 1)[:, :, None, None].expand(-1, -1, *new.shape[2:]))
    rows = _fit(torch.where(fresh[:, :, None, None], rows, torch.zeros_like(rows)))
    e = _exponent(rows)
    some = (x["filled"] > 0)[:, None]
    e[:, :, 0] = torch.where(some, torch.maximum(e[:, :, 0], e_old[:, :, 0].int()), e[:, :, 0])
    rows[:, :, 0] += _values(codes, e_old)
    return _values(_codes(rows, e), e)[:, :, :back].to(_dtype(case["dtype"])).contiguous()


def _plain_store(state, case, x):
    hq, hkv = case["hq"], case["hkv"]
    qkv = x["qkv"]
    turned = _turned(case, qkv[:, :, :hq + hkv], x["positions"])
    q = torch.where(_there(x, case["n"]), turned[:, :, :hq].to(qkv.dtype), state["q_out"])
    return (q, _stored(case, x, turned[:, :, hq:], *state["old"][:2]), _stored(case, x, qkv[:, :, hq + hkv:].float(), *state["old"][2:]))


def _unpacked(case, x):
    """fp32 [N, K]"""
    n, k, group = case["n"], case["k"], case["group"]
    codes = torch.stack((x["codes"] & 15, x["codes"] >> 4), -1).flatten(1)[:, :k].float()
    at = torch.arange(k, device=codes.device) // group
    return (codes - x["zeros"].float()[:, at]) * x["scales"].float()[:, at]


def _gelu(g):
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def _plain_product(state, case, x):
    y = x["x"].float() @ _unpacked(case, x).t()
    if x["bias"] is not None:
        y = y + x["bias"]
    if case["epi"] == "add":
        return state["out"].add_(y)
    if case["epi"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    if case["epi"] == "geglu":
        y = y.unflatten(1, (-1, 2, 64))
        y = (_gelu(y[:, :, 0]) * y[:, :, 1]).flatten(1)
    return y.to(state["out"].dtype)


def _plain_draw(state, case, x):
    """Weights and sums in 64 bits: a token next to a limit, or next to u, is in or out by less than 32 hold."""
    logits = x["logits"].float()
    vocab = logits.shape[1]
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    t = x["temperature"].double()[:, None]
    greedy = t <= 0
    z = (order.values.double() - order.values[:, :1].double()) / torch.where(greedy, 1.0, t)
    w = torch.exp(z)
    rank = torch.arange(vocab, device=logits.device)[None]
    k = x["top_k"][:, None]
    w = torch.where((k > 0) & (rank >= k), 0.0, w)
    before = torch.nn.functional.pad(torch.cumsum(w, 1), (1, -1))
    p = x["top_p"].double()[:, None]
    stays = (p >= 1) | (before < p * w.sum(1, keepdim=True)) | (rank == 0)
    stays &= (w >= x["min_p"].double()[:, None].clamp(max=1.0)) & ~(greedy & (rank > 0))
    w = torch.zeros_like(w).scatter_(1, order.indices, torch.where(stays, w, 0.0))   # by index again
    cum = torch.cumsum(w, 1)
    total = cum[:, -1:]
    token = torch.argmax((cum > x["u"].double()[:, None] * total).int(), 1, keepdim=True)
    return token[:, 0].int(), torch.log(torch.gather(w, 1, token) / total)[:, 0].float()


# ---- the definition in 64 bits -------------------------------------------------------


def _frequencies64(case):
    out = []
    for i in range(case["dims"] // 2):
        f = math.exp(-2.0 * i / case["dims"] * math.log(case["base"]))
        if not case["length"]:
            out.append(f / case["factor"])
            continue
        turns = case["length"] * f / (2 * math.pi)
        if turns <= 1.0:
            out.append(f / case["factor"])
        elif turns >= 32.0:
            out.append(f)
        else:
            g = (turns - 1.0) / 31.0
            out.append(g * f + (1.0 - g) * f / case["factor"])
    return out


def _turned64(case, x, positions):
    """x [n, H, hd] of one robot at positions [n]"""
    f = torch.tensor(_frequencies64(case), dtype=torch.float64, device=x.device)
    turn = torch.exp(1j * positions.double()[:, None] * f)[:, None]
    d = case["dims"]
    y = x.double().clone()
    first, second = (slice(0, d, 2), slice(1, d, 2)) if case["interleaved"] else (slice(0, d // 2), slice(d // 2, d))
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _held64(x):
    """What a block [..., 16, hd] holds, in 64 bits."""
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


def _stored64(case, new, old, fill):
    """One robot's new tokens [c, Hkv, hd] behind `fill` old ones of their first block."""
    c = new.shape[0]
    rows = torch.zeros((case["hkv"], BLOCK * _blocks(fill + c), case["hd"]), dtype=torch.float64, device=new.device)
    rows[:, fill:fill + c] = new.transpose(0, 1)
    held, e = _held64(rows.unflatten(1, (-1, BLOCK)))
    if fill:
        first = torch.zeros((case["hkv"], BLOCK, case["hd"]), dtype=torch.float64, device=new.device)
        first[:, :fill] = old[:fill].double().transpose(0, 1)
        first, e_old = _held64(first)
        first[:, fill:] = rows[:, fill:BLOCK]
        held[:, 0] = _round64(first, torch.maximum(e[:, 0], e_old))
    return held.flatten(1, 2)[:, :_back(case)]


def _exact_tokens(case, x):
    hq, hkv, hd, batch, n = (case[key] for key in ("hq", "hkv", "hd", "batch", "n"))
    starts, counts = _counts(case)
    dev = x["qkv"].device
    store = case["kind"] == "store"
    out = torch.zeros((batch, n, hq if store else hq + hkv, hd), dtype=torch.float64, device=dev)
    back = [torch.zeros((batch, hkv, _back(case), hd), dtype=torch.float64, device=dev) for _ in "kv"] if store else []
    for b in range(batch):
        c = counts[b]
        positions = starts[b] + torch.arange(c, device=dev) + case.get("gap", 0)
        y = _turned64(case, x["qkv"][b, :c, :hq + hkv], positions)
        out[b, :c] = y[:, :out.shape[2]]
        if store:
            fill = starts[b] % BLOCK
            for to, new, old in ((back[0], y[:, hq:], x["old_k"]), (back[1], x["qkv"][b, :c, hq + hkv:].double(), x["old_v"])):
                held = _stored64(case, new, old[b], fill)
                to[b, :, :held.shape[1]] = held
    return (out, *back) if store else out


def _exact_product(case, x):
    n, k, group = case["n"], case["k"], case["group"]
    acts = x["x"].double()
    y = torch.empty((case["m"], n), dtype=torch.float64, device=acts.device)
    for lo in range(0, n, 8192):
        c = x["codes"][lo:lo + 8192]
        w = torch.empty((c.shape[0], 2 * c.shape[1]), dtype=torch.float64, device=c.device)
        w[:, 0::2], w[:, 1::2] = (c % 16).double(), (c // 16).double()
        w = w[:, :k].contiguous()
        for g in range(-(-k // group)):
            part = w[:, g * group:(g + 1) * group]
            part -= x["zeros"][lo:lo + 8192, g, None].double()
            part *= x["scales"][lo:lo + 8192, g, None].double()
        y[:, lo:lo + 8192] = torch.einsum("mk,nk->mn", acts, w)
    if x["bias"] is not None:
        y += x["bias"].double()
    if case["epi"] == "add":
        return x["residual"].double() + y
    if case["epi"] == "silu":
        return y * torch.sigmoid(y)
    if case["epi"] == "geglu":
        gate, up = (torch.cat([y[:, b + at:b + at + 64] for b in range(0, n, 128)], 1) for at in (0, 64))
        inner = math.sqrt(2.0 / math.pi) * (gate + 0.044715 * gate ** 3)
        return gate * torch.sigmoid(2.0 * inner) * up   # (1 + tanh x) / 2 = sigmoid(2 x)
    return y


def _exact_draw(case, x):
    tokens, logs = [], []
    for b in range(case["batch"]):
        row = x["logits"][b].double()
        t, k, p, q = (x[key][b].item() for key in ("temperature", "top_k", "top_p", "min_p"))
        top = row.max()
        if t <= 0:
            tokens.append(int((row == top).nonzero()[0]))
            logs.append(0.0)
            continue
        order = torch.argsort(-row, stable=True)
        if k > 0:
            order = order[:k]
        w = torch.exp((row[order] - top) / t)
        if p < 1:
            reached = (torch.cumsum(w, 0) >= p * w.sum()).nonzero()
            order = order[:int(reached[0]) + 1] if len(reached) else order
        left = order[torch.exp((row[order] - top) / t) >= min(q, 1.0)].sort().values
        w = torch.exp((row[left] - top) / t)
        cum = torch.cumsum(w, 0)
        at = int((cum <= x["u"][b].double() * cum[-1]).sum())
        tokens.append(int(left[at]))
        logs.append(float(torch.log(w[at] / cum[-1])))
    dev = x["logits"].device
    return torch.tensor(tokens, dtype=torch.int32, device=dev), torch.tensor(logs, dtype=torch.float64, device=dev)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "product":
        return _exact_product(case, x)
    if case["kind"] == "draw":
        return _exact_draw(case, x)
    return _exact_tokens(case, x)

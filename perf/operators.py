"""The operators around the decode step that long contexts need, through the public entry points.

Five kinds of call, over the two families of model shapes that the benchmark and the tests use
(Pythia-160M: 12 query heads of 64, one to four KV heads, rotary on 16 channels; Llama-2-7B: 32
query heads of 128, 8 KV heads, rotary on all channels):

  qkv     mlkv_qk_norm_rope: the projections' queries, keys and values of `b` sequences of `s` tokens,
          as rows of one fused projection, to what the cache's calls take: RMS norm of every query and
          key head with a learned gain, rotary position encoding, values moved along
  store   the prompt's keys and values into a cache of 4-bit codes (MLKVQ4Cache.load_prefix), and what
          the cache then holds (MLKVQ4Cache.read); the single-token form is MLKVQ4Cache.append
  q4      decode attention over that cache (MLKVQ4Cache.decode_attention), all positions visible or
          a sliding window and the first tokens (sinks)
  window  decode attention over the bf16 cache with a sliding window and sinks
          (MLKVCache.decode_attention_window)
  prompt  causal prefill with a sliding window and sinks (MLKVCache.prefill_window), an owner layer's:
          it stores the prompt's keys and values too

The 4-bit cache: each 32 consecutive channels of one position of one KV head share a scale, the
bf16 nearest to their largest magnitude / 7; a channel is held as the whole number in [-7, 7] nearest
to value / scale, halves away from zero.

A query at position t sees position u <= t if u < sinks or u > t - window (window 0: all u <= t).

Inputs are bf16 normals, the Llama keys of the attention cases at half the scale (a trained model's
logits are less spread than random ones); lengths are one for all sequences or uniform in [1, L].
"""
import math
import random

import torch

own = False   # set from outside: the library's kernels in place of the plain forms

MODELS = {"pythia": {"h": 12, "d": 64, "rot": 16, "sigma_k": 1.0},
          "llama": {"h": 32, "d": 128, "rot": 128, "sigma_k": 0.5}}
GROUP = 32      # channels that share a scale
EPS = 1e-6
N_POS = 32768   # rows of the rotary table


def _case(name, kind, model, g, b, L, ragged=False, window=0, sinks=0):
    return {"name": name, "kind": kind, "model": model, "g": g, "b": b, "L": L, "ragged": ragged,
            "window": window, "sinks": sinks}


def listed():
    return [
        # one decode step of a serving batch: a token a sequence, nothing but latency
        _case("qkv-llama-b32-step", "qkv", "llama", 8, 32, 1),
        # prompts of the large model, of an odd length
        _case("qkv-llama-b4-s4001", "qkv", "llama", 8, 4, 4001),
        # the new token of a serving batch
        _case("store-pythia-g1-b64-append", "append", "pythia", 1, 64, 2000),
        # prompts of the large model into the cache
        _case("store-llama-b8-s4096", "store", "llama", 8, 8, 4096),
        # one user, a short chat turn: nothing but latency
        _case("q4-pythia-g4-b1-L128", "q4", "pythia", 4, 1, 128),
        # continuous batching of the large model: every sequence at a length of its own
        _case("q4-llama-b64-ragged8192", "q4", "llama", 8, 64, 8192, True),
        # one very long document, one KV head for twelve query heads
        _case("q4-pythia-g1-b1-L131072", "q4", "pythia", 1, 1, 131072),
        # long conversations of which the last 4096 tokens and the first four stay visible
        _case("q4-llama-b32-L20000-w4096", "q4", "llama", 8, 32, 20000, False, 4096, 4),
        # the same on the bf16 cache, uneven lengths
        _case("window-llama-b32-ragged16384-w2048", "window", "llama", 8, 32, 16384, True, 2048, 16),
        # the small model, a short window
        _case("window-pythia-g1-b64-L6000-w511", "window", "pythia", 1, 64, 6000, False, 511, 4),
        # prompts longer than the window; uneven short ones of the small model
        _case("prompt-llama-b1-s8192-w1024", "prompt", "llama", 8, 1, 8192, False, 1024, 4),
        _case("prompt-pythia-g4-b32-ragged777-w200", "prompt", "pythia", 4, 32, 777, True, 200, 1),
    ]


def _cost(case):
    """What a drawn case is held to: operations for prompts, else bytes."""
    return work(case)["flops" if case["kind"] == "prompt" else "bytes"]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["qkv", "qkv", "append", "store", "q4", "q4", "q4", "window", "window", "prompt",
                       "prompt"])
    model = rng.choice(["pythia", "llama"])
    g = rng.choice([1, 3, 4, 12] if model == "pythia" else [2, 4, 8])
    b = _log(rng, 1, 128)
    c = _case("", kind, model, g, b, 1, kind in ("q4", "window", "prompt") and rng.random() < 0.5)
    del c["name"]
    if kind == "qkv":
        c["L"] = rng.choice([1, _log(rng, 1, 4096)])
    elif kind in ("append", "store"):
        c["L"] = _log(rng, 1, 8192)
    elif kind == "prompt":
        c["L"] = _log(rng, 16, 8192)
    else:
        c["L"] = _log(rng, 16, 131072 if kind == "q4" else 32768)
    if kind in ("window", "prompt") or (kind == "q4" and rng.random() < 0.5):
        c["window"] = _log(rng, 1, 4096)
        c["sinks"] = rng.choice([0, 1, 4, 16, rng.randint(0, 300)])
    # No more than the kind's largest listed one; and what the plain forms hold at a time stays small:
    # a prompt's scores, the bf16 rows of a cache's positions.
    most = max(_cost(x) for x in listed() if x["kind"] == kind)

    def too_large():
        if kind == "prompt" and c["b"] * MODELS[model]["h"] * c["L"] ** 2 > 2.2e9:
            return True
        return 4.0 * c["b"] * c["g"] * c["L"] * MODELS[model]["d"] > 6e9 or _cost(c) > most

    while too_large():
        if c["b"] > 1:
            c["b"] = max(1, c["b"] * 2 // 3)
        else:
            c["L"] = max(1, c["L"] * 2 // 3)
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------


def _lens(case):
    """The sequences' lengths: part of the case, not of its inputs."""
    if not case["ragged"]:
        return [case["L"]] * case["b"]
    r = random.Random("%(model)s %(b)d %(L)d" % case)
    return [r.randint(1, case["L"]) for _ in range(case["b"])]


def _normal(seed, what, shape, sigma=1.0):
    gen = torch.Generator(device="cuda").manual_seed((seed * 1000003 + what) % (1 << 62))
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)


def _owners(case):
    return [0, 0]   # an owner layer and one that reads its cache


def _kv(case, seed, n):
    s = MODELS[case["model"]]
    shape = (case["b"], case["g"], n, s["d"])
    return _normal(seed, 2, shape, s["sigma_k"]), _normal(seed, 3, shape)


def _qkv_inputs(case, seed):
    s = MODELS[case["model"]]
    h, d, g = s["h"], s["d"], case["g"]
    fused = _normal(seed, 4, (case["b"], case["L"], h + 2 * g, d))
    # trained gains spread around one
    gains = [(1.0 + 0.2 * _normal(seed, 5 + i, (d,)).float()).bfloat16() for i in range(2)]
    half = s["rot"] // 2
    angle = (torch.arange(N_POS, device="cuda", dtype=torch.float64)[:, None] *
             10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64)[None] / half))
    gen = torch.Generator(device="cuda").manual_seed(seed % (1 << 62))
    # a step's tokens stand anywhere; a prompt's follow one another
    start = torch.randint(0, N_POS - case["L"] + 1, (case["b"], 1), device="cuda", generator=gen)
    positions = (start + torch.arange(case["L"], device="cuda")[None]).int()
    return fused, gains, angle, positions


def prepare(case, seed):
    s = MODELS[case["model"]]
    h, d, g, b, L, kind = s["h"], s["d"], case["g"], case["b"], case["L"], case["kind"]
    state = {"case": case}
    if own:
        import paper_2406_09297_gb300 as mlkv
    if kind == "qkv":
        fused, gains, angle, positions = _qkv_inputs(case, seed)
        state.update(Q=fused[:, :, :h], K=fused[:, :, h:h + g], V=fused[:, :, h + g:], gains=gains,
                     cos=angle.cos().float(), sin=angle.sin().float(), positions=positions,
                     Q_out=torch.zeros((b, L, h, d), dtype=torch.bfloat16, device="cuda"),
                     K_out=torch.zeros((b, g, L, d), dtype=torch.bfloat16, device="cuda"),
                     V_out=torch.zeros((b, g, L, d), dtype=torch.bfloat16, device="cuda"))
        if own:
            state["call"] = mlkv.mlkv_qk_norm_rope
        return state
    lens = _lens(case)
    K, V = _kv(case, seed, 1 if kind == "append" else L)
    state["K"], state["V"] = K, V
    if kind in ("append", "store"):
        state["K_out"], state["V_out"] = torch.zeros_like(K), torch.zeros_like(V)
    else:
        rows = (b, L) if kind == "prompt" else (b,)
        state["Q"] = _normal(seed, 1, rows + (h, d))
        state["out"] = torch.zeros_like(state["Q"])
    # What a program keeps from call to call: with the library a cache (its memory is the library's
    # own), for the plain forms the same contents as tensors.
    if own:
        Cache = mlkv.MLKVQ4Cache if kind in ("append", "store", "q4") else mlkv.MLKVCache
        cache = Cache(2, h, d, _owners(case), g, b, L)
        state["cache"], state["lens"] = cache, mlkv.as_seq_lens(lens)
        if kind in ("q4", "window"):
            cache.load_prefix(0, K, V, L)
            torch.cuda.synchronize()   # the cache copies its prefix from tensors that end here
            del state["K"], state["V"]
        if kind == "prompt":
            state["stored"] = _stored(cache)
    else:
        state["lens"] = torch.tensor(lens, device="cuda")
        if kind == "q4":
            state["K"], state["V"] = _quantise(K), _quantise(V)
        if kind == "prompt":
            state["stored"] = [torch.zeros_like(K), torch.zeros_like(V)]
    return state


class _DeviceMemory:
    """A view of cache memory for torch; it keeps the cache alive as long as a tensor uses it."""

    def __init__(self, cache, ptr, shape, strides):
        self.cache = cache
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": shape, "typestr": "<i2",
                                         "strides": tuple(2 * x for x in strides), "version": 3}


def _stored(cache):
    """The owner's keys and values where they lie in the bf16 cache."""
    k, v, st = cache.kv_ptr(0)
    return [torch.as_tensor(_DeviceMemory(cache, ptr, (cache.b, cache.g, cache.max_seq, cache.d), st),
                            device="cuda").view(torch.bfloat16) for ptr in (k, v)]


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(state, case, case["kind"])


def _run_own(state, case, kind):
    if kind == "qkv":
        state["call"](state["Q"], state["K"], state["V"], *state["gains"], state["cos"],
                      state["sin"], state["positions"], state["Q_out"], state["K_out"],
                      state["V_out"], eps=EPS)
        return {k: state[k + "_out"] for k in "QKV"}
    cache = state["cache"]
    if kind in ("append", "store"):
        if kind == "append":
            cache.append(0, state["K"], state["V"], state["lens"])
            cache.read(0, state["K_out"], state["V_out"], case["L"] - 1, 1)
        else:
            cache.load_prefix(0, state["K"], state["V"], case["L"])
            cache.read(0, state["K_out"], state["V_out"], 0, case["L"])
        return {"K": state["K_out"], "V": state["V_out"]}
    if kind == "prompt":
        cache.prefill_window(0, state["Q"], state["K"], state["V"], state["out"], state["lens"],
                             case["window"], case["sinks"])
        return {"out": state["out"], "stored": state["stored"]}
    call = cache.decode_attention if kind == "q4" else cache.decode_attention_window
    call(1, state["Q"], state["out"], state["lens"], case["window"], case["sinks"])
    return state["out"]


def _run_plain(state, case, kind):
    if kind == "qkv":
        return {"Q": _norm_rope(state["Q"], state["gains"][0], state),
                "K": _norm_rope(state["K"], state["gains"][1], state).transpose(1, 2).contiguous(),
                "V": state["V"].transpose(1, 2).contiguous()}
    if kind in ("append", "store"):
        return {k: _values(*_quantise(state[k])).bfloat16() for k in "KV"}
    lens, Q = state["lens"], state["Q"]
    w, sinks = case["window"], case["sinks"]
    if kind == "prompt":
        K, V = state["K"].float(), state["V"].float()
        at = torch.arange(case["L"], device="cuda")
        t, u = at[:, None], at[None]
        visible = ((u <= t) & ((u < sinks) | (u > t - w)))[None, None, None]   # [1][1][1][s][s]
        b, s, h, d = Q.shape
        q = Q.float().view(b, s, K.shape[1], -1, d).permute(0, 2, 3, 1, 4)       # [b][g][G][s][d]
        out = _attend(q, K[:, :, None], V[:, :, None], visible).permute(0, 3, 1, 2, 4).reshape(Q.shape)
        # rows past a prompt's end are not written
        live = (at[None] < lens[:, None])[:, :, None, None]
        state["out"].copy_(torch.where(live, out.bfloat16(), state["out"]))
        for to, kv in zip(state["stored"], (state["K"], state["V"])):
            to.copy_(kv)
        return {"out": state["out"], "stored": state["stored"]}
    # decode: the visible positions, sinks first, gathered into rows of one width
    if w == 0:
        at = torch.arange(case["L"], device="cuda").expand(case["b"], -1)
    else:
        first = (lens[:, None] - w).clamp(min=0)
        n_sink = min(sinks, case["L"])
        at = torch.cat([torch.arange(n_sink, device="cuda").expand(case["b"], -1),
                        first + torch.arange(min(w, case["L"]), device="cuda")[None]], 1)
        # a sink that the window holds too counts once
        twice = (torch.arange(at.shape[1], device="cuda")[None] < n_sink) & (at >= first)
        at = torch.where(twice, case["L"], at)
    visible = at < lens[:, None]
    at = at.clamp(max=case["L"] - 1)
    if kind == "q4":
        K, V = (_values(*(_take(x, at, w) for x in state[k])) for k in "KV")
    else:
        K, V = _take(state["K"], at, w).float(), _take(state["V"], at, w).float()
    q = Q.float().view(Q.shape[0], K.shape[1], -1, Q.shape[2])
    return _attend(q, K, V, visible[:, None, None]).reshape(Q.shape).bfloat16()


def _take(x, at, w):
    """Positions at[b] of x [b][g][L][...]."""
    return x if w == 0 else x.gather(2, at[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3]))


def _attend(q, k, v, visible):
    """softmax(q k^T / sqrt(d)) v over the visible positions, in 32 bits; a row without any gives 0."""
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(q.shape[-1])
    s = s.masked_fill(~visible, -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    return torch.matmul(e, v) / e.sum(-1, keepdim=True)


def _quantise(x):
    """(codes in [-7, 7], scales) of the channels of x [...][d] in groups of 32."""
    y = x.float().unflatten(-1, (-1, GROUP))
    scale = (y.abs().amax(-1) / 7.0).bfloat16()
    ratio = y / scale.float().clamp(min=2.0 ** -126)[..., None]
    code = torch.sign(ratio) * torch.floor(ratio.abs() + 0.5)
    return code.clamp(-7, 7).to(torch.int8).flatten(-2), scale


def _values(code, scale):
    return (code.float().unflatten(-1, (-1, GROUP)) * scale.float()[..., None]).flatten(-2)


def _norm_rope(x, gain, state):
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.float()
    cos, sin = (state[k][state["positions"].long()][:, :, None] for k in ("cos", "sin"))
    half = cos.shape[-1]
    a, b, rest = y[..., :half], y[..., half:2 * half], y[..., 2 * half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1).bfloat16()


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------


def _seen(n, w, sinks):
    """Positions that a query at the end of n positions sees."""
    return n if w == 0 else min(n, min(w, n) + min(sinks, max(0, n - w)))


def _pairs(n, w, sinks):
    """The sum of _seen over the lengths 1 .. n (w > 0)."""
    near, far = min(n, w), max(0, n - w)
    ramp = min(far, sinks)
    return near * (near + 1) / 2 + far * w + ramp * (ramp + 1) / 2 + (far - ramp) * sinks


def work(case):
    s = MODELS[case["model"]]
    h, d, g, b, L, kind = s["h"], s["d"], case["g"], case["b"], case["L"], case["kind"]
    w, sinks = case["window"], case["sinks"]
    if kind == "qkv":
        # heads in and out, each token's position and its row of the table; per channel a square, a
        # sum, two products of the norm and three operations of the rotation
        return {"bytes": 4.0 * b * L * (h + 2 * g) * d + b * L * (4.0 + 4 * s["rot"]),
                "flops": 7.0 * b * L * (h + g) * d}
    if kind in ("append", "store"):
        # bf16 in, codes and scales stored and read again, bf16 out; per channel a magnitude, a
        # maximum, a product, a rounding and a product
        n = 2.0 * b * g * (1 if kind == "append" else L) * d
        return {"bytes": n * (2 + 2 * (0.5 + 2 / GROUP) + 2), "flops": 5.0 * n}
    lens = _lens(case)
    if kind == "prompt":
        # queries in, outputs out, the prompt's keys and values in and into the cache
        total = float(sum(lens))
        return {"bytes": 2.0 * 2 * total * h * d + 2.0 * 2 * (total + b * L) * g * d,
                "flops": 4.0 * h * d * sum(_pairs(n, w, sinks) for n in lens)}
    seen = float(sum(_seen(n, w, sinks) for n in lens))
    per = 2 * d * (0.5 + 2 / GROUP) if kind == "q4" else 4.0 * d
    return {"bytes": seen * g * per + 4.0 * b * h * d, "flops": 4.0 * h * d * seen}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits
# ------------------------------------------------------------------------------------------------


def _held(x):
    """What the 4-bit cache holds of x, from the definition: the scale the bf16 nearest to the exact
    quotient, the code the nearest whole number."""
    b, g, n, d = x.shape
    y = x.double().reshape(b, g, n, d // GROUP, GROUP)
    largest = y.abs().max(-1, keepdim=True).values
    scale = (largest / 7).to(torch.bfloat16).double()
    code = torch.where(scale > 0, y / torch.where(scale > 0, scale, torch.ones_like(scale)),
                       torch.zeros_like(y))
    code = torch.where(code < 0, -((-code + 0.5).floor()), (code + 0.5).floor())
    return (code * scale).reshape(b, g, n, d)


def exact(case, seed):
    s = MODELS[case["model"]]
    h, d, g, b, L, kind = s["h"], s["d"], case["g"], case["b"], case["L"], case["kind"]
    w, sinks = case["window"], case["sinks"]
    if kind == "qkv":
        fused, gains, angle, positions = _qkv_inputs(case, seed)
        turn = torch.polar(torch.ones_like(angle), angle)[positions.long()][:, :, None]
        out = {}
        for name, x, gain in (("Q", fused[:, :, :h], gains[0]), ("K", fused[:, :, h:h + g], gains[1])):
            y = x.double()
            y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
            half = s["rot"] // 2
            z = torch.complex(y[..., :half], y[..., half:s["rot"]]) * turn
            out[name] = torch.cat([z.real, z.imag, y[..., s["rot"]:]], -1)
        out["K"] = out["K"].permute(0, 2, 1, 3).contiguous()
        out["V"] = fused[:, :, h + g:].double().permute(0, 2, 1, 3).contiguous()
        return out
    if kind in ("append", "store"):
        K, V = _kv(case, seed, 1 if kind == "append" else L)
        return {"K": _held(K), "V": _held(V)}
    if kind == "prompt" and 4.0 * b * h * L * L * d > 1e13:
        return None   # the square of the lengths, in 64 bits
    K, V = _kv(case, seed, L)
    Q = _normal(seed, 1, ((b, L) if kind == "prompt" else (b,)) + (h, d))
    out = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    for i, n in enumerate(_lens(case)):
        if kind == "prompt":
            u = torch.arange(n, device="cuda")
            hidden = (u > u[:, None]) | ((u >= sinks) & (u <= u[:, None] - w))
            for j in range(h):
                k, v = K[i, j // (h // g), :n].double(), V[i, j // (h // g), :n].double()
                sc = (Q[i, :n, j].double() @ k.T / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                out[i, :n, j] = torch.softmax(sc, -1) @ v
            continue
        u = torch.arange(n, device="cuda")
        u = u if w == 0 else u[(u < sinks) | (u >= n - w)]
        k, v = K[i:i + 1, :, u], V[i:i + 1, :, u]
        k, v = (_held(k)[0], _held(v)[0]) if kind == "q4" else (k[0].double(), v[0].double())
        q = Q[i].double().view(g, h // g, d)
        sc = torch.einsum("gqd,gtd->gqt", q, k) / math.sqrt(d)
        out[i] = torch.einsum("gqt,gtd->gqd", torch.softmax(sc, -1), v).reshape(h, d)
    if kind == "prompt":
        return {"out": out, "stored": [K.double(), V.double()]}
    return out

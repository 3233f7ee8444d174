"""The operators that bound what a step reads of a long cache, and what a cache keeps, through the public
entry points.

Six kinds of call, over the two families of model shapes that the benchmark and the tests use
(Pythia-160M: 12 query heads of 64, one to twelve KV heads; Llama-2-7B: 32 query heads of 128, 2 to 8 KV
heads):

  prefix   decode attention of a batch whose sequences share long beginnings, each held once in a cache of
           its own (MLKVCache.decode_attention_prefix)
  prompt   causal prefill of prompts that go on behind such a beginning (MLKVCache.prefill_prefix), an owner
           layer's: it stores the prompts' keys and values too
  bounds   the least and the largest value of every key channel in each block of 64 positions, in 8 bits
           (MLKVCache.block_bounds), of whole prompts or of the newest block alone
  blocks   one step's attention over the blocks that those bounds promise the largest scores
           (MLKVCache.select_blocks, MLKVCache.decode_attention_blocks)
  weights  decode attention that also adds up the weight that each position got
           (MLKVCache.decode_attention_weights)
  evict    the positions of the largest such weights, and the newest ones, into a smaller cache, in order
           (MLKVCache.evict)

Bounds of a block: with amax the largest |k| of its positions and channels, scale = 2^e for the least whole
number e in [-60, 40] with amax <= 127 * 2^e; codes floor(min / scale) and ceil(max / scale) a channel.
Score of a block for a query head: the query in 8 bits, q8 = q / 2^f rounded (halves to even), f as e but
of the query head; sum over channels of max(q8 lo, q8 hi), times 2^f scale.  Whole numbers below 2^24
times a power of two: exact in fp32, in any order.  A KV head takes the largest score of its query heads,
and of equal scores the block of the lower index.

Inputs are bf16 normals.  The keys of the block cases have channels with offsets, as trained models' do; the
Llama keys are at half the scale (a trained model's logits are less spread than random ones).  The weights
that an eviction goes by are log-normal, since attention favours few positions.
"""
import math
import random

import torch

own = False   # set from outside: the library's kernels in place of the plain forms

MODELS = {"pythia": {"h": 12, "d": 64, "sigma_k": 1.0},
          "llama": {"h": 32, "d": 128, "sigma_k": 0.5}}
BLOCK = 64      # positions of a block
FIRST, LAST = 1, 2   # blocks at either end that are always selected


def _case(name, kind, model, g, b, L, ragged=False, P=0, n_prefix=0, n_select=0, keep=0):
    """L: positions of the sequences' own caches (prompts' lengths for "prompt"); P: of the n_prefix shared
    beginnings; n_select: blocks; keep: positions that stay, a quarter of them the newest."""
    return {"name": name, "kind": kind, "model": model, "g": g, "b": b, "L": L, "ragged": ragged, "P": P,
            "n_prefix": n_prefix, "n_select": n_select, "keep": keep}


def listed():
    return [
        # four users' first answer tokens behind a short common instruction: nothing but latency
        _case("prefix-pythia-g4-b4-P300-L20", "prefix", "pythia", 4, 4, 20, False, 300, 1),
        # five applications on one server, each with an instruction of its own, some users without any
        _case("prefix-llama-b48-5xP6001-ragged3000", "prefix", "llama", 8, 48, 3000, True, 6001, 5),
        # many questions about one long document
        _case("prefix-llama-b128-P32768-L1024", "prefix", "llama", 8, 128, 1024, False, 32768, 1),
        # uneven short questions behind a common instruction, small model
        _case("prompt-pythia-g4-b16-P1000-ragged200", "prompt", "pythia", 4, 16, 200, True, 1000, 1),
        # questions about a document
        _case("prompt-llama-b8-P8192-s500", "prompt", "llama", 8, 8, 500, False, 8192, 1),
        # the prompts' blocks, after prefill
        _case("bounds-llama-b8-ragged16000", "bounds", "llama", 8, 8, 16000, True),
        # one very long document, one KV head for twelve query heads
        _case("blocks-pythia-g1-b1-L131072-n64", "blocks", "pythia", 1, 1, 131072, n_select=64),
        # a serving batch of long conversations of uneven lengths
        _case("blocks-llama-b32-ragged32768-n64", "blocks", "llama", 8, 32, 32768, True, n_select=64),
        # short uneven sequences: latency
        _case("weights-pythia-g4-b8-ragged777", "weights", "pythia", 4, 8, 777, True),
        # a full cache of a serving batch
        _case("weights-llama-b32-L8192", "weights", "llama", 8, 32, 8192),
        # prompts of the small model cut down to a short cache
        _case("evict-pythia-g1-b16-L2000-k500", "evict", "pythia", 1, 16, 2000, keep=500),
        # long prompts of the large model, of which a quarter stays
        _case("evict-llama-b16-ragged16384-k4096", "evict", "llama", 8, 16, 16384, True, keep=4096),
    ]


def _cost(case):
    """What a drawn case is held to: operations for prompts, else bytes."""
    return work(case)["flops" if case["kind"] == "prompt" else "bytes"]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["prefix", "prefix", "prompt", "prompt", "bounds", "blocks", "blocks", "weights",
                       "weights", "evict", "evict"])
    model = rng.choice(["pythia", "llama"])
    c = _case("", kind, model, rng.choice([1, 3, 4, 12] if model == "pythia" else [2, 4, 8]),
              _log(rng, 1, 128), 1, rng.random() < 0.5)
    del c["name"]
    if kind in ("prefix", "prompt"):
        c["n_prefix"] = rng.choice([1, 1, rng.randint(2, 6)])
        c["P"] = _log(rng, 16, 32768 if kind == "prefix" else 8192)
        c["L"] = _log(rng, 1, 4096) if kind == "prefix" else _log(rng, 1, 1000)
    elif kind == "blocks":
        c["L"] = _log(rng, 64, 131072)
        c["n_select"] = _log(rng, FIRST + LAST, 128)
    elif kind == "weights":
        c["L"] = _log(rng, 1, 32768)
    else:
        c["L"] = _log(rng, 16, 32768)
        c["keep"] = _log(rng, 1, c["L"]) if kind == "evict" else 0
    # No more than the kind's largest listed one; and what the plain forms hold at a time stays small:
    # scores of 32 bits, the rows of a cache's positions.
    most = max(_cost(x) for x in listed() if x["kind"] == kind)
    s = MODELS[model]

    def too_large():
        rows = {"prefix": c["b"] * c["P"], "prompt": c["L"] * (c["P"] + c["L"]),
                "weights": c["b"] * c["L"]}.get(kind, 0)
        held = 4.0 * c["g"] * s["d"] * (c["b"] * c["L"] + c["n_prefix"] * c["P"])
        return rows * s["h"] > 1.2e9 or held > 4.5e9 or _cost(c) > most

    while too_large():
        if c["b"] > 1:
            c["b"] = max(1, c["b"] * 2 // 3)
        elif c["P"] > 16:
            c["P"] = max(16, c["P"] * 2 // 3)
        else:
            c["L"] = max(1, c["L"] * 2 // 3)
    c["keep"] = min(c["keep"], c["L"])
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------


def _random(case, what):
    return random.Random("%s %d %d %d %s" % (case["model"], case["b"], case["L"], case["P"], what))


def _lens(case):
    """The sequences' lengths: part of the case, not of its inputs."""
    if not case["ragged"]:
        return [case["L"]] * case["b"]
    r = _random(case, "lens")
    return [r.randint(1, case["L"]) for _ in range(case["b"])]


def _prefixes(case):
    """Each sequence's beginning (-1: none) and the beginnings' lengths."""
    n, P = case["n_prefix"], case["P"]
    if n <= 1:
        return [0] * case["b"], [P] * n
    r = _random(case, "prefixes")
    return ([r.choice([-1] + 2 * list(range(n))) for _ in range(case["b"])],
            [r.randint((P + 1) // 2, P) for _ in range(n)])


def _keeps(case):
    return case["keep"], case["keep"] // 4


def _normal(seed, what, shape, sigma=1.0, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed((seed * 1000003 + what) % (1 << 62))
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=gen)


def _kv(case, seed, n, b, what):
    s = MODELS[case["model"]]
    shape = (b, case["g"], n, s["d"])
    K, V = _normal(seed, what, shape, s["sigma_k"]), _normal(seed, what + 1, shape)
    if case["kind"] in ("blocks", "bounds"):
        K += _normal(seed, what + 2, (1, case["g"], 1, s["d"]))
    return K, V


def _log_normal(case, seed):
    return _normal(seed, 8, (case["b"], case["g"], case["L"]), 1.5, torch.float32).exp_()


def prepare(case, seed):
    s = MODELS[case["model"]]
    h, d, g, b, L, kind = s["h"], s["d"], case["g"], case["b"], case["L"], case["kind"]
    state = {"case": case}
    lens = _lens(case)
    K, V = _kv(case, seed, L, b, 2)
    Q = _normal(seed, 1, ((b, L) if kind == "prompt" else (b,)) + (h, d))
    state.update(Q=Q, out=torch.zeros_like(Q), K=K, V=V)
    n_blocks = (L + BLOCK - 1) // BLOCK
    if kind in ("prefix", "prompt"):
        prefix_of, prefix_lens = _prefixes(case)
        P_K, P_V = _kv(case, seed, case["P"], case["n_prefix"], 5)
        state.update(P_K=P_K, P_V=P_V, prefix_of=prefix_of, prefix_lens=prefix_lens)
    if kind in ("bounds", "blocks"):
        state.update(bounds=torch.zeros((b, g, n_blocks, 2, d), dtype=torch.int8, device="cuda"),
                     scales=torch.zeros((b, g, n_blocks), dtype=torch.float32, device="cuda"),
                     blocks=torch.zeros((b, g, case["n_select"]), dtype=torch.int32, device="cuda"))
    if kind == "weights":
        state.update(before=_log_normal(case, seed), after=torch.zeros((b, g, L), device="cuda"))
    if kind == "evict":
        keep, recent = _keeps(case)
        state.update(before=_log_normal(case, seed), after=torch.zeros((b, g, keep), device="cuda"),
                     kept=torch.zeros((b, g, keep), dtype=torch.int32, device="cuda"), keep=[keep] * b,
                     recent=recent)
    # What a program keeps from call to call: with the library caches (their memory is the library's own),
    # for the plain forms the same contents as tensors.
    if own:
        _prepare_own(state, case, lens)
    else:
        state["lens"] = torch.tensor(lens, device="cuda")
        if kind == "prompt":
            state["stored"] = [torch.zeros_like(K), torch.zeros_like(V)]
        if kind == "blocks":
            state["bounds"], state["scales"] = _bounds(K, state["lens"])
        if kind == "evict":
            state["rows"] = [torch.zeros((b, g, case["keep"], d), dtype=torch.bfloat16, device="cuda")
                             for _ in range(2)]
    return state


def _prepare_own(state, case, lens):
    import paper_2406_09297_gb300 as mlkv
    s, kind = MODELS[case["model"]], case["kind"]

    def cache(b, n):
        return mlkv.MLKVCache(2, s["h"], s["d"], [0, 0], case["g"], b, n)   # an owner and a reader

    c = state["cache"] = cache(case["b"], case["L"])
    state["lens"] = mlkv.as_seq_lens(lens)
    if kind in ("prefix", "prompt"):
        state["prefix"] = cache(case["n_prefix"], case["P"])
        state["prefix"].load_prefix(0, state["P_K"], state["P_V"], case["P"])
        state["prefix_of"] = mlkv.as_seq_lens(state["prefix_of"])
        state["prefix_lens"] = mlkv.as_seq_lens(state["prefix_lens"])
    if kind == "prompt":
        state["stored"] = _stored(c)
    else:
        c.load_prefix(0, state["K"], state["V"], case["L"])
    if kind == "blocks":
        c.block_bounds(0, state["lens"], state["bounds"], state["scales"])
    if kind == "evict":
        state["to"] = cache(case["b"], case["keep"])
        state["rows"], state["keep"] = _stored(state["to"]), mlkv.as_seq_lens(state["keep"])
    torch.cuda.synchronize()   # the caches copy from tensors that end here
    for k in ("P_K", "P_V") if kind == "prompt" else ("K", "V", "P_K", "P_V"):
        state.pop(k, None)


class _DeviceMemory:
    """A view of cache memory for torch; it keeps the cache alive as long as a tensor uses it."""

    def __init__(self, cache, ptr, shape, strides):
        self.cache = cache
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": shape, "typestr": "<i2",
                                         "strides": tuple(2 * x for x in strides), "version": 3}


def _stored(cache):
    """The owner's keys and values where they lie in the cache."""
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
    cache, Q, out, lens = state["cache"], state["Q"], state["out"], state["lens"]
    if kind == "prefix":
        cache.decode_attention_prefix(1, state["prefix"], state["prefix_of"], state["prefix_lens"], Q, out,
                                      lens)
        return out
    if kind == "prompt":
        cache.prefill_prefix(0, state["prefix"], state["prefix_of"], state["prefix_lens"], Q, state["K"],
                             state["V"], out, lens)
        return {"out": out, "stored": state["stored"]}
    if kind == "bounds":
        cache.block_bounds(0, lens, state["bounds"], state["scales"])
        return {"bounds": _values(state["bounds"], state["scales"]), "scales": state["scales"]}
    if kind == "blocks":
        cache.select_blocks(1, Q, state["bounds"], state["scales"], lens, state["blocks"], FIRST, LAST)
        cache.decode_attention_blocks(1, Q, out, lens, state["blocks"])
        return {"blocks": state["blocks"], "out": out}
    if kind == "weights":
        cache.decode_attention_weights(1, Q, out, lens, state["before"], state["after"])
        return {"out": out, "weights": state["after"]}
    cache.evict(0, state["before"], state["after"], lens, state["keep"], state["recent"], state["kept"],
                state["to"])
    return {"rows": state["rows"], "weights": state["after"], "kept": state["kept"]}


def _run_plain(state, case, kind):
    Q, K, V, lens = state["Q"], state["K"], state["V"], state["lens"]
    if kind == "prefix":
        return _with_prefix(state, Q, K, V, lens)
    if kind == "prompt":
        return _prompt(state, case, Q, K, V)
    if kind == "bounds":
        bounds, scales = _bounds(K, lens)
        return {"bounds": _values(bounds, scales), "scales": scales}
    if kind == "blocks":
        blocks = _select(Q, state["bounds"], state["scales"], lens, case["n_select"])
        at = (blocks[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(-2).long()
        seen = (blocks >= 0).repeat_interleave(BLOCK, -1) & (at < lens[:, None, None])
        at = at.clamp(0, K.shape[2] - 1)[..., None].expand(-1, -1, -1, K.shape[3])
        p = _weights(_scores(Q, K.gather(2, at)), seen[:, :, None])
        return {"blocks": blocks,
                "out": torch.matmul(p, V.gather(2, at).float()).reshape(Q.shape).bfloat16()}
    seen = torch.arange(case["L"], device="cuda")[None] < lens[:, None]
    if kind == "weights":
        p = _weights(_scores(Q, K), seen[:, None, None])
        return {"out": torch.matmul(p, V.float()).reshape(Q.shape).bfloat16(),
                "weights": state["before"] + p.sum(2)}
    keep, recent = _keeps(case)
    kept = _heaviest(state["before"], lens, keep, recent)
    valid = torch.arange(keep, device="cuda") < lens[:, None, None].clamp(max=keep)
    at = kept.clamp(min=0).long()
    # what lies behind a sequence's kept positions stays as it was
    for to, x in zip(state["rows"], (K, V)):
        to.copy_(torch.where(valid[..., None], x.gather(2, at[..., None].expand(-1, -1, -1, x.shape[3])), to))
    state["kept"].copy_(torch.where(valid, kept, state["kept"]))
    return {"rows": state["rows"], "kept": state["kept"],
            "weights": torch.where(valid, state["before"].gather(2, at), 0.0)}


def _scores(Q, K):
    """Q [b][h][d], K [b][g][n][d] -> [b][g][G][n] in 32 bits."""
    q = Q.float().view(Q.shape[0], K.shape[1], -1, Q.shape[2])
    return torch.matmul(q, K.float().transpose(-1, -2)) / math.sqrt(Q.shape[-1])


def _weights(s, seen):
    """softmax over the seen positions."""
    s = s.masked_fill(~seen, -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    return e / e.sum(-1, keepdim=True)


def _with_prefix(state, Q, K, V, lens):
    b, h, d = Q.shape
    g, P = K.shape[1], state["P_K"].shape[2]
    own_s = _scores(Q, K).masked_fill((torch.arange(K.shape[2], device="cuda") >= lens[:, None])[:, None, None],
                                      -math.inf)
    out = torch.empty_like(Q)
    prefix_of = torch.tensor(state["prefix_of"])
    for p in range(-1, len(state["prefix_lens"])):
        of = (prefix_of == p).nonzero()[:, 0].to("cuda")
        n = len(of)
        if n == 0:
            continue
        s, v = own_s[of], V[of].float()
        if p < 0:
            out[of] = torch.matmul(_weights(s, s > -math.inf), v).reshape(n, h, d).bfloat16()
            continue
        # all the queries of a KV head against the prefix's keys at once
        m = state["prefix_lens"][p]
        q = Q[of].float().view(n, g, -1, d).transpose(0, 1).reshape(g, -1, d)
        ps = torch.matmul(q, state["P_K"][p, :, :m].float().transpose(-1, -2)) / math.sqrt(d)
        own = s.transpose(0, 1).reshape(g, ps.shape[1], -1)
        top = torch.maximum(ps.amax(-1, keepdim=True), own.amax(-1, keepdim=True))
        e, f = torch.exp(ps - top), torch.exp(own - top)
        o = torch.matmul(e, state["P_V"][p, :, :m].float()).view(g, n, -1, d).transpose(0, 1)
        total = (e.sum(-1, keepdim=True) + f.sum(-1, keepdim=True)).view(g, n, -1, 1).transpose(0, 1)
        o = o + torch.matmul(f.view(g, n, -1, f.shape[-1]).transpose(0, 1), v)
        out[of] = (o / total).reshape(n, h, d).bfloat16()
    return out


def _prompt(state, case, Q, K, V):
    b, L, h, d = Q.shape
    g = K.shape[1]
    t = torch.arange(L, device="cuda")
    for i, n in enumerate(_lens(case)):
        p = state["prefix_of"][i]
        m = state["prefix_lens"][p] if p >= 0 else 0
        k = torch.cat([state["P_K"][p, :, :m], K[i, :, :n]], 1).float()[:, None]
        v = torch.cat([state["P_V"][p, :, :m], V[i, :, :n]], 1).float()[:, None]
        q = Q[i, :n].float().view(n, g, -1, d).permute(1, 2, 0, 3)            # [g][G][n][d]
        seen = torch.arange(m + n, device="cuda")[None] <= m + t[:n, None]
        o = torch.matmul(_weights(torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d), seen), v)
        state["out"][i, :n] = o.permute(2, 0, 1, 3).reshape(n, h, d).bfloat16()
    for to, x in zip(state["stored"], (K, V)):
        to.copy_(x)
    return {"out": state["out"], "stored": state["stored"]}


def _power(amax):
    """2^e, e the least whole number in [-60, 40] with amax <= 127 * 2^e."""
    m, e = torch.frexp(amax.double() / 127)
    return torch.ldexp(torch.ones_like(m), (e - (m == 0.5).int()).clamp(-60, 40)).float()


def _bounds(K, lens):
    """(codes [b][g][n][2][d], scales [b][g][n]) of the blocks that hold positions below the lengths; zeros
    elsewhere."""
    b, g, L, d = K.shape
    n = (L + BLOCK - 1) // BLOCK
    seen = (torch.arange(n * BLOCK, device="cuda") < lens[:, None]).view(b, 1, n, BLOCK, 1)
    x = torch.nn.functional.pad(K, (0, 0, 0, n * BLOCK - L)).view(b, g, n, BLOCK, d).float()
    lo = x.masked_fill(~seen, math.inf).amin(3)
    hi = x.masked_fill(~seen, -math.inf).amax(3)
    live = seen.any(3)                                           # [b][1][n][1]
    lo, hi = torch.where(live, lo, 0.0), torch.where(live, hi, 0.0)
    scale = _power(torch.maximum(lo.abs(), hi.abs()).amax(-1))
    codes = torch.stack([torch.floor(lo / scale[..., None]), torch.ceil(hi / scale[..., None])], 3)
    return codes.to(torch.int8), torch.where(live[..., 0], scale, 0.0)


def _values(codes, scales):
    return codes * scales[..., None, None]


def _select(Q, codes, scales, lens, n_select):
    """The selected blocks in rising order, -1 behind them."""
    b, h, d = Q.shape
    g, n = codes.shape[1], codes.shape[2]
    q = Q.float().view(b, g, -1, d)
    power = _power(q.abs().amax(-1))
    q8 = torch.round(q / power[..., None])
    lo, hi = codes[:, :, :, 0].float(), codes[:, :, :, 1].float()
    s = (torch.matmul(q8.clamp(min=0), hi.transpose(-1, -2)) +
         torch.matmul(q8.clamp(max=0), lo.transpose(-1, -2)))                # whole numbers below 2^24
    s = (s * (power[..., None] * scales[:, :, None])).amax(2)
    at = torch.arange(n, device="cuda")
    count = ((lens + BLOCK - 1) // BLOCK)[:, None, None]
    s = torch.where((at < FIRST) | (at >= count - LAST), math.inf, s)
    s = torch.where(at < count, s, -math.inf)
    first = torch.sort(s, dim=-1, descending=True, stable=True).indices[..., :n_select]
    first = torch.where(first < count, first, n).sort(-1).values
    first = torch.nn.functional.pad(first, (0, n_select - first.shape[-1]), value=n)
    return torch.where(first < n, first, -1).int()


def _heaviest(w, lens, keep, recent):
    """The `recent` newest positions of each sequence and the heaviest others, `keep` in all, in rising
    order; -1 behind a shorter sequence's."""
    at = torch.arange(w.shape[-1], device="cuda")
    n = lens[:, None, None]
    w = torch.where(at >= n - recent, math.inf, w).masked_fill(at >= n, -math.inf)
    first = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    first = torch.where(first < n, first, w.shape[-1]).sort(-1).values
    return torch.where(first < n, first, -1).int()


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------


def work(case):
    s = MODELS[case["model"]]
    h, d, g, b, L, kind = s["h"], s["d"], case["g"], case["b"], case["L"], case["kind"]
    lens = _lens(case)
    total = float(sum(lens))
    row = 4.0 * g * d            # a position's keys and values
    qo = 4.0 * h * d             # a token's queries and outputs
    if kind in ("prefix", "prompt"):
        prefix_of, prefix_lens = _prefixes(case)
        shared = row * sum(prefix_lens[p] for p in set(prefix_of) if p >= 0)
        behind = [prefix_lens[p] if p >= 0 else 0 for p in prefix_of]
        if kind == "prefix":
            return {"bytes": shared + row * total + qo * b, "flops": 4.0 * h * d * (sum(behind) + total)}
        # the prompts' keys and values in and into the cache
        return {"bytes": shared + row * (total + b * L) + qo * total,
                "flops": 4.0 * h * d * sum(n * m + n * (n + 1) / 2 for n, m in zip(lens, behind))}
    blocks = [(n + BLOCK - 1) // BLOCK for n in lens]
    per_block = 2.0 * d + 4      # codes and scale
    if kind == "bounds":
        # a magnitude, a minimum and a maximum a key channel; every block's bounds written
        return {"bytes": row / 2 * total + g * per_block * sum(blocks), "flops": 3.0 * g * d * total}
    if kind == "blocks":
        took = float(sum(min(n, BLOCK * case["n_select"]) for n in lens))
        return {"bytes": g * per_block * sum(blocks) + row * took + qo * b + 4.0 * b * g * case["n_select"],
                "flops": 4.0 * h * d * (sum(blocks) + took)}
    if kind == "weights":
        return {"bytes": row * total + qo * b + 8.0 * b * g * L, "flops": 4.0 * h * d * total}
    # weights in, the kept positions' keys, values and weights in and out, their numbers out
    kept = float(sum(min(n, case["keep"]) for n in lens))
    return {"bytes": 4.0 * g * total + kept * (2 * row + 8.0 * g), "flops": 2.0 * g * total}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits
# ------------------------------------------------------------------------------------------------


def _soft(x):
    x = torch.exp(x - x.max(-1, keepdim=True).values)
    return x / x.sum(-1, keepdim=True)


def exact(case, seed):
    s = MODELS[case["model"]]
    h, d, g, b, L, kind = s["h"], s["d"], case["g"], case["b"], case["L"], case["kind"]
    G, lens = h // g, _lens(case)
    K, V = _kv(case, seed, L, b, 2)
    Q = _normal(seed, 1, ((b, L) if kind == "prompt" else (b,)) + (h, d))
    out = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    if kind in ("prefix", "prompt"):
        prefix_of, prefix_lens = _prefixes(case)
        P_K, P_V = _kv(case, seed, case["P"], case["n_prefix"], 5)
        for i, n in enumerate(lens):
            p = prefix_of[i]
            m = prefix_lens[p] if p >= 0 else 0
            for j in range(g):
                k, v = K[i, j, :n].double(), V[i, j, :n].double()
                if m > 0:
                    k = torch.cat([P_K[p, j, :m].double(), k])
                    v = torch.cat([P_V[p, j, :m].double(), v])
                for a in range(j * G, (j + 1) * G) if kind == "prompt" else [slice(j * G, (j + 1) * G)]:
                    q = Q[i, :n, a] if kind == "prompt" else Q[i, a]
                    sc = q.double() @ k.T / math.sqrt(d)
                    if kind == "prompt":
                        late = torch.ones(n, m + n, dtype=torch.bool, device="cuda").triu(m + 1)
                        out[i, :n, a] = _soft(sc.masked_fill_(late, -math.inf)) @ v
                    else:
                        out[i, a] = _soft(sc) @ v
        return {"out": out, "stored": [K.double(), V.double()]} if kind == "prompt" else out
    if kind in ("bounds", "blocks"):
        n_blocks = (L + BLOCK - 1) // BLOCK
        lo = torch.zeros((b, g, n_blocks, d), dtype=torch.float64, device="cuda")
        hi, scale = torch.zeros_like(lo), torch.zeros_like(lo[..., 0])
        for i, n in enumerate(lens):
            for u in range((n + BLOCK - 1) // BLOCK):
                k = K[i, :, u * BLOCK:min(n, (u + 1) * BLOCK)]
                lo[i, :, u], hi[i, :, u] = k.amin(1).double(), k.amax(1).double()
            live = slice(0, (n + BLOCK - 1) // BLOCK)
            amax = torch.maximum(hi[i, :, live], -lo[i, :, live]).max(-1).values
            scale[i, :, live] = torch.exp2(torch.ceil(torch.log2(amax / 127)).clamp(-60, 40))
            lo[i, :, live] = torch.floor(lo[i, :, live] / scale[i, :, live, None])
            hi[i, :, live] = torch.ceil(hi[i, :, live] / scale[i, :, live, None])
        if kind == "bounds":
            return {"bounds": torch.stack([lo, hi], 3) * scale[..., None, None], "scales": scale}
        blocks = torch.full((b, g, case["n_select"]), -1, dtype=torch.int32, device="cuda")
        for i, n in enumerate(lens):
            q = Q[i].double().view(g, G, 1, d)
            f = torch.exp2(torch.ceil(torch.log2(q.abs().amax(-1, keepdim=True) / 127)).clamp(-60, 40))
            q8 = torch.round(q / f)
            count = (n + BLOCK - 1) // BLOCK
            inner = max(0, count - FIRST - LAST)       # blocks that are not selected in any case
            sc = torch.stack([torch.maximum(q8[j] * lo[i, j, :count], q8[j] * hi[i, j, :count]).sum(-1)
                              for j in range(g)]) * f[..., 0] * scale[i, :, None, :count]
            sc = sc.amax(1)[:, FIRST:FIRST + inner]
            by = torch.argsort(-sc, dim=-1, stable=True)[:, :max(0, case["n_select"] - FIRST - LAST)] + FIRST
            always = [u for u in range(count) if u < FIRST or u >= count - LAST]
            always = torch.tensor(always, device="cuda").expand(g, -1)
            took = torch.cat([by, always], -1).sort(-1).values
            blocks[i, :, :took.shape[-1]] = took
            for j in range(g):
                at = (took[j, :, None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten()
                at = at[at < n]
                sc = Q[i, j * G:(j + 1) * G].double() @ K[i, j, at].double().T / math.sqrt(d)
                out[i, j * G:(j + 1) * G] = _soft(sc) @ V[i, j, at].double()
        return {"blocks": blocks, "out": out}
    w = _log_normal(case, seed)
    if kind == "weights":
        w = w.double()
        for i, n in enumerate(lens):
            p = _soft(torch.einsum("gqd,gtd->gqt", Q[i].double().view(g, G, d), K[i, :, :n].double()) /
                      math.sqrt(d))
            w[i, :, :n] += p.sum(1)
            out[i] = (p @ V[i, :, :n].double()).reshape(h, d)
        return {"out": out, "weights": w}
    keep, recent = _keeps(case)
    rows = [torch.zeros((b, g, keep, d), dtype=torch.float64, device="cuda") for _ in range(2)]
    kept = torch.zeros((b, g, keep), dtype=torch.int32, device="cuda")
    after = torch.zeros((b, g, keep), dtype=torch.float64, device="cuda")
    for i, n in enumerate(lens):
        new = min(n, recent)
        by = torch.argsort(-w[i, :, :n - new].double(), dim=-1, stable=True)[:, :min(n, keep) - new]
        at = torch.cat([by, torch.arange(n - new, n, device="cuda").expand(g, -1)], -1).sort(-1).values
        m = at.shape[-1]
        kept[i, :, :m] = at
        after[i, :, :m] = w[i].gather(1, at).double()
        for to, x in zip(rows, (K, V)):
            to[i, :, :m] = x[i].gather(1, at[..., None].expand(-1, -1, d)).double()
    return {"rows": rows, "weights": after, "kept": kept}

"""The calls for long caches together, as a decoder makes them: behind a shared prefix, over selected blocks, with
eviction; in a captured graph; on other streams; two caches at once."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend  # noqa: E402

pytestmark = pytest.mark.gpu
ROUNDINGS = 2   # a few visible keys: see test_gpu_shared_prefix


def _randn(*shape):
    return torch.randn(shape, device="cuda").bfloat16()


def _check(out, Q, k, v):
    """One KV head's group: out and Q [G][d], k and v [n][d]."""
    want, spread = attend(Q.double()[:, None], k.double()[None], v.double()[None],
                          torch.ones(1, k.shape[0], dtype=torch.bool, device="cuda"))
    assert_attention(out, want[:, 0], spread[:, 0], ROUNDINGS)


@pytest.mark.parametrize("d,h,g", [(64, 12, 4), (128, 16, 2)])
def test_decoder_that_evicts(d, h, g):
    """A cache of 192 positions: prompts of up to 150 fill it, every step adds one and its weights (two layers of one
    block), and a full cache goes back to 100, the 20 newest among them."""
    torch.manual_seed(d)
    b, cap, G = 3, 192, h // g
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap)
    lens = [150, 40, 101]
    K, V, P = _randn(b, g, 150, d), _randn(b, g, 150, d), _randn(b, 150, h, d)
    out = torch.zeros_like(P)
    cache.prefill(0, P, K, V, out, lens)
    held = [[(K[i, j, :lens[i]], V[i, j, :lens[i]]) for j in range(g)] for i in range(b)]
    w = torch.zeros(b, g, cap, device="cuda")
    total = torch.zeros(b, g, cap, device="cuda", dtype=torch.float64)
    kept = torch.zeros(b, g, 100, dtype=torch.int32, device="cuda")
    evictions = 0
    for step in range(120):
        k, v = _randn(b, g, d), _randn(b, g, d)
        lens = [n + 1 for n in lens]
        cache.append(0, k, v, lens)
        for i in range(b):
            for j in range(g):
                a, c = held[i][j]
                held[i][j] = torch.cat([a, k[i, j][None]]), torch.cat([c, v[i, j][None]])
        for layer in (0, 1):
            Q = _randn(b, h, d)
            out = torch.zeros_like(Q)
            cache.decode_attention_weights(layer, Q, out, lens, w, w)
            for i in range(b):
                for j in range(g):
                    q = Q[i, j * G:(j + 1) * G]
                    s = q.double() @ held[i][j][0].double().T / math.sqrt(d)
                    total[i, j, :lens[i]] += torch.softmax(s, -1).sum(0)
                    if step % 10 == 0:
                        _check(out[i, j * G:(j + 1) * G], q, *held[i][j])
        # fp32 sums of up to 2 G weights a step, each to about 1e-4 (see test_gpu_evict) and each sum to 2^-24
        assert torch.allclose(w.double(), total, rtol=2e-4, atol=1e-6)
        if max(lens) == cap:
            evictions += 1
            cache.evict(0, w, w, lens, [100] * b, 20, kept)
            at = kept.cpu().long()
            for i in range(b):
                n = min(lens[i], 100)
                for j in range(g):
                    pos = at[i, j, :n].cuda()
                    assert (pos[1:] > pos[:-1]).all() and (pos[-20:] == torch.arange(lens[i] - 20, lens[i],
                                                                                      device="cuda")).all()
                    held[i][j] = held[i][j][0][pos], held[i][j][1][pos]
                    t = total[i, j, pos]
                    total[i, j] = 0
                    total[i, j, :n] = t
                lens[i] = n
    cache.sync_status()
    assert evictions == 1


@pytest.mark.parametrize("d,h,g", [(64, 12, 1), (128, 32, 8)])
def test_decoder_over_blocks(d, h, g):
    torch.manual_seed(d)
    b, cap, G, n = 2, 64 * 30, h // g, 6
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap)
    K, V = _randn(b, g, cap, d), _randn(b, g, cap, d)
    lens = [1500, 63]
    for i in range(b):
        K[i, :, lens[i]:], V[i, :, lens[i]:] = 0, 0
    cache.load_prefix(0, K, V, cap)
    bounds = torch.zeros(b, g, 30, 2, d, dtype=torch.int8, device="cuda")
    scales = torch.zeros(b, g, 30, device="cuda")
    blocks = torch.zeros(b, g, n, dtype=torch.int32, device="cuda")
    cache.block_bounds(0, lens, bounds, scales)
    for step in range(70):
        k, v = _randn(b, g, d), _randn(b, g, d)
        lens = [x + 1 for x in lens]
        cache.append(0, k, v, lens)
        for i in range(b):
            K[i, :, lens[i] - 1], V[i, :, lens[i] - 1] = k[i], v[i]
        cache.block_bounds(0, lens, bounds, scales, first=[x - 1 for x in lens])
        for layer in (0, 1):
            Q = _randn(b, h, d)
            out = torch.zeros_like(Q)
            cache.select_blocks(layer, Q, bounds, scales, lens, blocks, 1, 1)
            cache.decode_attention_blocks(layer, Q, out, lens, blocks)
            if step % 9:
                continue
            at = blocks.cpu().tolist()
            for i in range(b):
                for j in range(g):
                    took = [u for u in at[i][j] if u >= 0]
                    assert took[0] == 0 and took[-1] == (lens[i] - 1) // 64 and len(took) == min(
                        n, (lens[i] + 63) // 64)
                    pos = [u for x in took for u in range(64 * x, min(lens[i], 64 * x + 64))]
                    _check(out[i, j * G:(j + 1) * G], Q[i, j * G:(j + 1) * G], K[i, j, pos], V[i, j, pos])
    cache.sync_status()


def _steps(d=128, h=16, g=4, b=6, cap=700, P=600):
    """A cache behind a shared prefix, and one step of every call over it, as functions of what a step reads."""
    cache, prefix = mlkv.MLKVCache(1, h, d, [0], g, b, cap), mlkv.MLKVCache(1, h, d, [0], g, 2, P)
    to = mlkv.MLKVCache(1, h, d, [0], g, b, 64)
    K, V, PK = _randn(b, g, cap, d), _randn(b, g, cap, d), _randn(2, g, P, d)
    cache.load_prefix(0, K, V, cap)
    prefix.load_prefix(0, PK, PK, P)
    n = (cap + 63) // 64
    x = {"Q": _randn(b, h, d), "w": torch.rand(b, g, cap, device="cuda"),
         "bounds": torch.zeros(b, g, n, 2, d, dtype=torch.int8, device="cuda"),
         "scales": torch.zeros(b, g, n, device="cuda"),
         "blocks": torch.zeros(b, g, 4, dtype=torch.int32, device="cuda"),
         "kept": torch.zeros(b, g, 50, dtype=torch.int32, device="cuda"),
         "after": torch.zeros(b, g, cap, device="cuda"), "small": torch.zeros(b, g, 64, device="cuda"),
         "prompt": _randn(b, 9, h, d), "kv": _randn(b, g, 9, d)}
    for name in ("o1", "o2", "o3"):
        x[name] = torch.zeros(b, h, d, dtype=torch.bfloat16, device="cuda")
    x["o4"] = torch.zeros_like(x["prompt"])
    lens = [cap, 3, 64, 333, 65, 699]

    def run():
        cache.decode_attention_prefix(0, prefix, [0, 1, 0, -1, 0, 1], [P, P - 70], x["Q"], x["o1"], lens)
        cache.block_bounds(0, lens, x["bounds"], x["scales"])
        cache.select_blocks(0, x["Q"], x["bounds"], x["scales"], lens, x["blocks"])
        cache.decode_attention_blocks(0, x["Q"], x["o2"], lens, x["blocks"])
        cache.decode_attention_weights(0, x["Q"], x["o3"], lens, x["w"], x["after"])
        cache.evict(0, x["after"], x["small"], lens, [50] * b, 10, x["kept"], to)
        to.prefill_prefix(0, prefix, [0] * b, [P, P], x["prompt"], x["kv"], x["kv"], x["o4"], [9] * b)

    def results():
        cache.sync_status()
        to.sync_status()
        return [x[k].clone() for k in ("o1", "o2", "o3", "o4", "bounds", "scales", "blocks", "kept", "after", "small")]
    return x, run, results


def test_captured_and_replayed():
    torch.manual_seed(0)
    x, run, results = _steps()
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        torch.manual_seed(seed + 5)
        x["Q"].copy_(_randn(*x["Q"].shape))
        x["w"].copy_(torch.rand_like(x["w"]))
        x["prompt"].copy_(_randn(*x["prompt"].shape))
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        replayed = results()
        run()
        for a, b in zip(replayed, results()):
            assert torch.equal(a, b)


def test_scratch_does_not_grow_under_capture():
    torch.manual_seed(0)
    d, h, g, b, cap = 64, 8, 2, 2, 300
    cache = mlkv.MLKVCache(1, h, d, [0], g, b, cap)
    Q, out, w = _randn(b, h, d), _randn(b, h, d), torch.zeros(b, g, cap, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with pytest.raises(mlkv.MLKVError) as e:
            cache.decode_attention_weights(0, Q, out, [300, 100], w, w)
        assert e.value.code == mlkv.MLKV_ERR_UNSUPPORTED
        cache.decode_attention(0, Q, out, [300, 100])   # the capture goes on
    graph.replay()
    cache.sync_status()
    cache.decode_attention_weights(0, Q, out, [300, 100], w, w)   # outside it grows
    with torch.cuda.graph(graph2 := torch.cuda.CUDAGraph()):
        cache.decode_attention_weights(0, Q, out, [300, 100], None, w)
    graph2.replay()
    cache.sync_status()
    assert torch.allclose(w.sum(-1), torch.full((b, g), h / g, device="cuda"), rtol=1e-4)


def test_prompts_do_without_scratch_under_capture():
    """Short prompts are rows of a decode, whose records lie in scratch; a first call of a captured stream takes none
    and is the prefill's kernel, with its store."""
    torch.manual_seed(0)
    d, h, g, b, p = 64, 12, 1, 66, 2000
    Q, out = _randn(b, 1, h, d), _randn(b, 1, h, d)
    K, V, PK, PV = _randn(b, g, 1, d), _randn(b, g, 1, d), _randn(1, g, p, d), _randn(1, g, p, d)
    step, own = _randn(b, h, d), _randn(b, h, d)
    prefix = mlkv.MLKVCache(1, h, d, [0], g, 1, p)
    prefix.load_prefix(0, PK, PV, p)
    torch.cuda.synchronize()
    got = []
    for captured in (False, True):
        cache = mlkv.MLKVCache(1, h, d, [0], g, b, 4)
        call = lambda: cache.prefill_prefix(0, prefix, [0] * b, [p], Q, K, V, out, [1] * b)
        if captured:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                call()
            out.zero_()
            graph.replay()
        else:
            call()
        for i in (0, 31, 65):
            _check(out[i, 0], Q[i, 0], torch.cat([PK[0, 0], K[i, 0]]), torch.cat([PV[0, 0], V[i, 0]]))
        cache.decode_attention(0, step, own, [1] * b)   # what was stored
        cache.sync_status()
        got.append(own.clone())
        assert torch.equal(own, V[:, 0].expand_as(own))
    assert torch.equal(*got)


def test_scratch_that_is_outgrown_lives_on():
    """A graph recorded over a smaller scratch replays after a larger call has replaced it."""
    torch.manual_seed(0)
    d, h, g, b, cap = 64, 8, 2, 2, 4000
    cache = mlkv.MLKVCache(1, h, d, [0], g, b, cap)
    K = _randn(b, g, cap, d)
    cache.load_prefix(0, K, K, cap)
    Q, out, w = _randn(b, h, d), _randn(b, h, d), torch.zeros(b, g, cap, device="cuda")
    cache.decode_attention_weights(0, Q, out, [100, 50], None, w)
    first = w.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.decode_attention_weights(0, Q, out, [100, 50], None, w)
    cache.decode_attention_weights(0, Q, out, [4000, 3999], None, w)
    graph.replay()
    cache.sync_status()
    assert torch.equal(w, first)


def test_other_streams():
    torch.manual_seed(0)
    x, run, results = _steps()
    run()
    want = results()
    for k in ("o1", "o2", "o3", "o4", "after", "small", "kept", "blocks"):
        x[k].zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(results(), want):
        assert torch.equal(a, b)


def test_two_caches_at_once():
    torch.manual_seed(0)
    one, two = _steps(), _steps(d=64, h=12, g=12, P=3000)
    want = []
    for _, run, results in (one, two):
        run()
        want.append(results())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for s, (_, run, _) in zip(streams, (one, two)):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, _, results), w in zip((one, two), want):
        for a, b in zip(results(), w):
            assert torch.equal(a, b)


def test_what_ran_before_shares_the_scratch():
    """The fused decode step and the calls here use one scratch of a cache in turn."""
    torch.manual_seed(0)
    d, h, g, b, cap, l = 64, 12, 1, 4, 2048, 6
    cache = mlkv.MLKVCache(l, h, d, [0] * l, g, b, cap)
    K = _randn(b, g, cap, d)
    cache.load_prefix(0, K, K, cap)
    Q, k = _randn(l, b, h, d), _randn(1, b, g, d)
    out, o, w = torch.zeros_like(Q), torch.zeros_like(Q[0]), torch.zeros(b, g, cap, device="cuda")
    cache.set_option("step_fused", 2)
    lens = [2048, 1000, 1, 1999]
    cache.decode_step(Q, k, k, out, lens)
    want = out.clone()
    cache.decode_attention_weights(0, Q[0], o, lens, None, w)
    want_w = w.clone()
    for _ in range(5):
        cache.decode_step(Q, k, k, out, lens)
        cache.decode_attention_weights(0, Q[0], o, lens, None, w)
    cache.sync_status()
    assert torch.equal(out, want) and torch.equal(w, want_w)


def test_offsets_beyond_32_bits():
    """Two caches of 2.4e9 elements a side; what is asked for lies in the last sequence."""
    torch.manual_seed(0)
    d, h, g, b, cap = 128, 16, 8, 9, 262144
    G, i, n = h // g, b - 1, cap - 44
    lens = [70] * i + [n]
    K = torch.empty(b, g, cap, d, dtype=torch.bfloat16, device="cuda").normal_()
    V = torch.empty_like(K).normal_()
    cache, other = (mlkv.MLKVCache(1, h, d, [0], g, b, cap) for _ in range(2))
    cache.load_prefix(0, K, V, cap)
    Q, out = _randn(b, h, d), _randn(b, h, d)

    def check(to, k, v, j):
        _check(to[j * G:(j + 1) * G], Q[i, j * G:(j + 1) * G], k, v)

    # behind its positions as a prefix
    small = mlkv.MLKVCache(1, h, d, [0], g, 2, 64)
    own = _randn(2, g, 64, d)
    small.load_prefix(0, own, own, 64)
    two = _randn(2, h, d)
    small.decode_attention_prefix(0, cache, [i, -1], lens, Q[i - 1:].contiguous(), two, [5, 64])
    for j in (0, 7):
        q = Q[i - 1, j * G:(j + 1) * G]
        _check(two[0, j * G:(j + 1) * G], q, torch.cat([K[i, j, :n], own[0, j, :5]]), torch.cat([V[i, j, :n], own[0, j, :5]]))
    # blocks
    blk = (cap + 63) // 64
    bounds = torch.zeros(b, g, blk, 2, d, dtype=torch.int8, device="cuda")
    scales = torch.zeros(b, g, blk, device="cuda")
    blocks = torch.zeros(b, g, 50, dtype=torch.int32, device="cuda")
    cache.block_bounds(0, lens, bounds, scales)
    cache.select_blocks(0, Q, bounds, scales, lens, blocks, 1, 2)
    cache.decode_attention_blocks(0, Q, out, lens, blocks)
    last = (n + 63) // 64 - 1
    for j in (0, 7):
        for u in (0, 1000, last):
            k = K[i, j, 64 * u:min(n, 64 * u + 64)].float()
            assert scales[i, j, u] == 2.0 ** math.ceil(math.log2(float(k.abs().max()) / 127))
            assert torch.equal(bounds[i, j, u, 0].float(), (k.amin(0) / scales[i, j, u]).floor())
            assert torch.equal(bounds[i, j, u, 1].float(), (k.amax(0) / scales[i, j, u]).ceil())
        took = blocks[i, j].tolist()
        assert took == sorted(set(took)) and took[0] == 0 and took[-2:] == [last - 1, last]
        pos = [u for x in took for u in range(64 * x, min(n, 64 * x + 64))]
        check(out[i], K[i, j, pos], V[i, j, pos], j)
    # weights, and eviction to another cache and in place
    w, after = torch.zeros(b, g, cap, device="cuda"), torch.zeros(b, g, cap, device="cuda")
    cache.decode_attention_weights(0, Q, out, lens, None, w)
    kept = torch.zeros(b, g, 200000, dtype=torch.int32, device="cuda")
    keep = [100] * i + [200000]   # (all there are of the short ones)
    cache.evict(0, w, after, lens, keep, 100, kept, other)
    for j in (0, 7):
        check(out[i], K[i, j, :n], V[i, j, :n], j)
        assert abs(float(w[i, j, :n].double().sum()) - G) < 1e-3
        order = torch.sort(w[i, j, :n - 100], descending=True, stable=True).indices[:200000 - 100]
        want = torch.cat([order.sort().values, torch.arange(n - 100, n, device="cuda")])
        assert torch.equal(kept[i, j].long(), want)
        assert torch.equal(after[i, j, :200000], w[i, j, want]) and not after[i, j, 200000:].any()
    again = kept.clone().zero_()
    cache.evict(0, w, w, lens, keep, 100, again)
    assert torch.equal(again, kept) and torch.equal(w, after)
    for c in (other, cache):
        c.decode_attention(0, Q, out, [70] * i + [200000])
        for j in (0, 7):
            at = kept[i, j].long()
            check(out[i], K[i, j, at], V[i, j, at], j)
        c.sync_status()

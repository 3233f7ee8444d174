"""Decode attention that adds up its weights, and the eviction that goes by them, against 64-bit forms."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend  # noqa: E402

pytestmark = pytest.mark.gpu

# Of a few visible keys no roundings average out.  A weight rounded to bf16 is off by at most 2^-8 of itself, its sum is
# not rounded, so that an output before its own rounding is off by at most 2^-8 A (A = sum p |v| / sum p), its own
# rounding is 2^-8 |want|, and |want| <= A: 2^-8 A + 2^-8 |want| <= (2 + 1) 2^-9 A + 2^-9 |want|, assert_attention's
# bound for two.
ROUNDINGS = 2


def _randn(*shape, sigma=1.0):
    return (torch.randn(shape, device="cuda") * sigma).bfloat16()


def _weights(d, h, g, lens, cap, mode="apart", sigma=1.0, seed=0):
    torch.manual_seed(seed)
    b, G = len(lens), h // g
    K, V, Q = _randn(b, g, cap, d), _randn(b, g, cap, d), _randn(b, h, d, sigma=sigma)
    for i, n in enumerate(lens):
        K[i, :, n:], V[i, :, n:] = math.nan, math.inf
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap)
    cache.load_prefix(0, K, V, cap)
    out = torch.full_like(Q, 9.0)
    before = None if mode == "none" else torch.rand(b, g, cap, device="cuda")
    old = torch.zeros(b, g, cap, device="cuda") if before is None else before.clone()
    after = before if mode == "same" else torch.full((b, g, cap), 7.0, device="cuda")
    cache.decode_attention_weights(1, Q, out, lens, before, after)
    cache.sync_status()
    for i, n in enumerate(lens):
        q, k = Q[i].double().view(g, G, d), K[i, :, :n].double()
        s = torch.einsum("gqd,gtd->gqt", q, k) / math.sqrt(d)
        got = torch.softmax(s, -1).sum(1)
        # A score in units of log2 is off by at most d 2^-24 sum |q k| log2(e) / sqrt(d) (a sum of d products in
        # 32 bits) and the rounding of its product; the log of the sum by as much again; their difference's
        # exponential, relatively, by ln 2 times both.
        size = torch.einsum("gqd,gtd->gqt", q.abs(), k.abs()).amax() / math.sqrt(d) * math.log2(math.e)
        rel = 2 * math.log(2) * (float(size) * (d + 2) * 2.0 ** -24) + 8 * 2.0 ** -23
        want = old[i, :, :n].double() + got
        err = (after[i, :, :n].double() - want).abs()
        assert (err <= rel * got + 2.0 ** -24 * want + 1e-30).all(), float((err / (rel * got)).max())
        assert torch.equal(after[i, :, n:], old[i, :, n:])
        want, spread = attend(Q[i].double()[:, None], k, V[i, :, :n].double(),
                              torch.ones(1, n, dtype=torch.bool, device="cuda"))
        assert_attention(out[i], want[:, 0], spread[:, 0], ROUNDINGS)
    return out, after


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(12, 1), (8, 2), (16, 1), (3, 3)])
@pytest.mark.parametrize("mode", ["none", "same", "apart"])
def test_weights(d, h, g, mode):
    _weights(d, h, g, [1, 63, 64, 65, 128, 300, 1001], 1003, mode)
    _weights(d, h, g, [257] * 3, 257, mode, sigma=6.0, seed=1)


@pytest.mark.parametrize("d,h,g,lens", [(64, 12, 1, [100000]), (128, 32, 8, [9000, 1, 20000]),
                                        (128, 32, 8, [2000] * 64), (64, 12, 12, [700] * 50)])
def test_weights_long(d, h, g, lens):
    first = _weights(d, h, g, lens, max(lens) + 1)
    for a, b in zip(first, _weights(d, h, g, lens, max(lens) + 1)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_scores_that_are_all_minus_infinity(d):
    """KV head 0 has no finite score: zeros, and no weight."""
    n, cap = 70, 200
    cache = mlkv.MLKVCache(1, 4, d, [0], 2, 1, cap)
    K, V, Q = torch.zeros(1, 2, cap, d).bfloat16().cuda(), _randn(1, 2, cap, d), torch.zeros(1, 4, d).bfloat16().cuda()
    K[0, 0, :, 0] = -math.inf
    Q[0, :, 0] = 1
    cache.load_prefix(0, K, V, cap)
    out, w = torch.full_like(Q, 9.0), torch.full((1, 2, cap), 7.0, device="cuda")
    cache.decode_attention_weights(0, Q, out, [n], None, w)
    cache.sync_status()
    assert (out[0, :2] == 0).all() and (w[0, 0] == 0).all()
    assert torch.allclose(w[0, 1, :n], torch.full((n,), 2 / n, device="cuda"), rtol=1e-5) and (w[0, 1, n:] == 0).all()


def _evict(d, h, g, lens, cap, keep, recent, w, where="same", cap_to=None, seed=0, owners=(0, 0)):
    torch.manual_seed(seed)
    b = len(lens)
    K, V = _randn(b, g, cap, d), _randn(b, g, cap, d)
    cache = mlkv.MLKVCache(len(owners), h, d, list(owners), g, b, cap)
    layer = max(owners)
    cache.load_prefix(layer, K, V, cap)
    to = cache if where == "same" else mlkv.MLKVCache(len(owners), h, d, list(owners), g, b, cap_to or cap)
    k_max = max(min(k, n) for k, n in zip(keep, lens))
    kept = torch.full((b, g, k_max), -5, dtype=torch.int32, device="cuda")
    old = w.clone()
    # `where`: rows and weights in place, both elsewhere, or one of the two
    after = w if where in ("same", "weights") else torch.full((b, g, to.max_seq), 3.0, device="cuda")
    cache.evict(layer, w, after, lens, keep, recent, kept, None if where == "same" else to)
    cache.sync_status()
    G = to
    ptr = G.kv_ptr(G.owner_slot(layer)[1])
    rows = [torch.as_tensor(_Memory(p, (b, g, G.max_seq, d)), device="cuda").view(torch.bfloat16)
            for p in ptr[:2]]
    wn, got = old.cpu().numpy(), kept.cpu().tolist()
    for i, n in enumerate(lens):
        m = min(n, keep[i])
        for j in range(g):
            x = np.where(np.isnan(wn[i, j, :n]), np.inf, wn[i, j, :n])
            nan = np.isnan(wn[i, j, :n])
            new = min(recent, m)
            order = sorted(range(n - new), key=lambda u: (not nan[u], -x[u], u))
            want = sorted(order[:m - new]) + list(range(n - new, n))
            assert got[i][j][:m] == want, (i, j)
            assert got[i][j][m:] == [-5] * (k_max - m)
            for r, src in zip(rows, (K, V)):
                assert torch.equal(r[i, j, :m], src[i, j, want])
                if where == "same" or where == "weights":
                    pass
                else:
                    assert (r[i, j, m:] == 0).all()
            at = after[i, j].cpu().numpy()
            assert np.array_equal(at[:m], wn[i, j, want], equal_nan=True) and (at[m:] == 0).all()
            if where == "same":   # what lies behind is as it was
                for r, src in zip(rows, (K, V)):
                    assert torch.equal(r[i, j, m:], src[i, j, m:])
    return cache


class _Memory:
    def __init__(self, ptr, shape):
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": shape, "typestr": "<i2", "version": 3}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 3])
@pytest.mark.parametrize("where", ["same", "apart", "weights", "rows"])
def test_evict(d, g, where):
    lens, cap = [1, 5, 64, 500, 1000, 1000, 777], 1000
    b = len(lens)
    for keep, recent in ([3, 5, 64, 100, 1000, 999, 300], 2), ([1] * b, 0), ([700] * b, 700), ([130] * b, 5):
        torch.manual_seed(keep[0])
        w = torch.randn(b, g, cap, device="cuda").exp()
        if where == "rows":
            _evict_rows_in_place(d, 3 * g, g, lens, cap, keep, min(recent, min(keep)), w)
        else:
            _evict(d, 3 * g, g, lens, cap, keep, min(recent, min(keep)), w, where)


def _evict_rows_in_place(d, h, g, lens, cap, keep, recent, w):
    torch.manual_seed(0)
    b = len(lens)
    K, V = _randn(b, g, cap, d), _randn(b, g, cap, d)
    cache = mlkv.MLKVCache(1, h, d, [0], g, b, cap)
    cache.load_prefix(0, K, V, cap)
    kept = torch.zeros((b, g, max(keep)), dtype=torch.int32, device="cuda")
    after = torch.zeros_like(w)
    old = w.clone()
    cache.evict(0, w, after, lens, keep, recent, kept)
    cache.sync_status()
    assert torch.equal(w, old)
    rows = [torch.as_tensor(_Memory(p, (b, g, cap, d)), device="cuda").view(torch.bfloat16)
            for p in cache.kv_ptr(0)[:2]]
    for i, n in enumerate(lens):
        m = min(n, keep[i])
        for j in range(g):
            at = kept[i, j, :m].long()
            assert torch.equal(rows[0][i, j, :m], K[i, j, at]) and torch.equal(rows[1][i, j, :m], V[i, j, at])
            assert torch.equal(after[i, j, :m], old[i, j, at]) and (after[i, j, m:] == 0).all()


@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "strange"])
@pytest.mark.parametrize("where", ["same", "apart"])
def test_evict_orders(kind, where):
    d, g, n, cap = 64, 2, 3000, 3001
    w = torch.ones(2, g, cap, device="cuda")
    if kind in ("rising", "falling"):
        w = w * torch.arange(cap, device="cuda")
        w = w if kind == "rising" else -w
    if kind == "strange":
        torch.manual_seed(0)
        w = torch.randn(2, g, cap, device="cuda").round()
        w[0, 0, 10::50] = math.nan
        w[0, 1, 5::500] = math.inf
        w[1, 0, ::3] = -0.0
        w[1, 1, ::2] = -math.inf
    _evict(d, 2 * g, g, [n, n - 999], cap, [1024, 1000], 10, w, where)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,g,n,keep", [(1, 1, 700, 600), (2, 2, 1000, 130), (5, 1, 9000, 300), (40, 3, 600, 400),
                                        (50, 4, 500, 30), (50, 4, 500, 260), (50, 4, 9000, 60), (170, 1, 300, 299)])
@pytest.mark.parametrize("where", ["same", "apart", "weights"])
def test_evict_forms(d, b, g, n, keep, where):
    """Moved by the selecting CTA in one round or several, by one of many, by a cluster, or by units."""
    lens = [n - 3 * i for i in range(b)] if 3 * b < n else [n - i for i in range(b)]
    torch.manual_seed(b)
    w = torch.rand(b, g, n, device="cuda")
    _evict(d, g, g, lens, n, [max(1, keep - i % 50) for i in range(b)], 1, w, where)


@pytest.mark.parametrize("largest", [math.nan, math.inf, 3.4028234663852886e38])
@pytest.mark.parametrize("n", [609, 20000])
@pytest.mark.parametrize("sign", [1, -1])
def test_evict_more_largest_than_stay(largest, n, sign):
    """More positions of the largest weight, at the end of the keys' range, than are kept."""
    torch.manual_seed(n)
    w = torch.rand(2, 2, n, device="cuda") * sign
    w[torch.rand_like(w) < 0.1] = largest
    _evict(64, 4, 2, [n, n - 7], n, [2, 30], 1, w, "apart")


@pytest.mark.parametrize("d,g,b,n,keep", [(64, 1, 1, 131072, 40000), (128, 8, 2, 20000, 5000),
                                          (128, 8, 16, 3000, 2999), (64, 1, 1, 300000, 1000)])
@pytest.mark.parametrize("where", ["same", "apart"])
def test_evict_long(d, g, b, n, keep, where):
    torch.manual_seed(1)
    w = torch.randn(b, g, n, device="cuda").exp()
    cap_to = None if where == "same" else keep
    _evict(d, g, g, [n] * b, n, [keep] * b, keep // 4, w, where, cap_to)


def test_evict_later_owner():
    torch.manual_seed(1)
    _evict(64, 4, 2, [100, 50], 100, [30, 30], 5, torch.rand(2, 2, 100, device="cuda"), owners=(0, 0, 2, 2))
    cache = mlkv.MLKVCache(2, 4, 64, [0, 0], 2, 1, 100)   # not an owner: nothing happens
    w, kept = torch.rand(1, 2, 100, device="cuda"), torch.zeros(1, 2, 9, dtype=torch.int32, device="cuda")
    old = w.clone()
    cache.evict(1, w, w, [100], [9], 1, kept)
    torch.cuda.synchronize()
    assert torch.equal(w, old) and (kept == 0).all()


def test_evict_again_and_again():
    """The same call repeated: what is kept stays, nothing moves."""
    d, g = 128, 2
    torch.manual_seed(0)
    w = torch.rand(3, g, 500, device="cuda")
    cache = _evict(d, 4, g, [500, 400, 300], 500, [200] * 3, 50, w)
    rows = [torch.as_tensor(_Memory(p, (3, g, 500, d)), device="cuda").clone() for p in cache.kv_ptr(0)[:2]]
    kept = torch.zeros(3, g, 200, dtype=torch.int32, device="cuda")
    old = w.clone()
    cache.evict(0, w, w, [200] * 3, [200] * 3, 50, kept)
    cache.sync_status()
    assert (kept == torch.arange(200, device="cuda")).all() and torch.equal(w, old)
    for p, r in zip(cache.kv_ptr(0)[:2], rows):
        assert torch.equal(torch.as_tensor(_Memory(p, (3, g, 500, d)), device="cuda"), r)


def test_rejections():
    d, h, g, cap = 64, 4, 2, 100
    cache, small = mlkv.MLKVCache(2, h, d, [0, 0], g, 1, cap), mlkv.MLKVCache(2, h, d, [0, 0], g, 1, 20)
    Q, out = _randn(1, h, d), torch.zeros(1, h, d, dtype=torch.bfloat16, device="cuda")
    w, w2 = torch.rand(1, g, cap, device="cuda"), torch.rand(1, g, cap, device="cuda")
    kept = torch.zeros(1, g, 50, dtype=torch.int32, device="cuda")
    RANGE, BAD, MAP = mlkv.MLKV_ERR_RANGE, mlkv.MLKV_ERR_INVALID_ARG, mlkv.MLKV_ERR_MAP

    def refused(call, good, *changes):
        call(**good)
        for change, code in changes:
            with pytest.raises(mlkv.MLKVError) as e:
                call(**dict(good, **change))
            assert e.value.code == code, change

    both = torch.rand(g * cap + 8, device="cuda")
    part = [both[i:i + g * cap].view(1, g, cap) for i in (0, 8)]
    refused(cache.decode_attention_weights, dict(layer=1, Q=Q, out=out, seq_lens=[cap], weights_in=w, weights_out=w2),
            (dict(layer=2), BAD), (dict(Q=None), BAD), (dict(out=Q), BAD), (dict(seq_lens=[0]), RANGE),
            (dict(weights_in=w.double()), BAD), (dict(weights_out=w2[:, :1]), BAD),
            (dict(weights_in=part[0], weights_out=part[1]), BAD))
    refused(cache.evict, dict(layer=0, weights_in=w, weights_out=w, seq_lens=[cap], keep=[50], recent=5, kept=kept),
            (dict(layer=2), BAD), (dict(seq_lens=[101]), RANGE), (dict(keep=[0]), BAD), (dict(recent=51), BAD),
            (dict(recent=-1), BAD), (dict(keep=[51]), RANGE), (dict(kept=kept.long()), BAD),
            (dict(kept=kept[:, :, :0]), BAD), (dict(weights_in=part[0], weights_out=part[1]), BAD),
            (dict(weights_out=w2[:, :, :20].contiguous(), to=small), RANGE),
            (dict(weights_out=w2, to=mlkv.MLKVCache(2, h, d, [0, 1], g, 1, cap)), MAP),
            (dict(to=mlkv.MLKVCache(2, h, d, [0, 0], g, 2, cap),
                  weights_out=torch.zeros(2, g, cap, device="cuda")), MAP),
            (dict(to=small, keep=[20]), BAD))
    cache.evict(0, w, w2[:, :, :20].contiguous(), [cap], [20], 3, kept, small)

"""Decode and prefill behind beginnings that sequences share, against a 64-bit reference."""
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


def _ends(K, V, lens):
    """What lies behind the ends is never used."""
    for i, n in enumerate(lens):
        K[i, :, n:] = math.nan
        V[i, :, n:] = math.inf


def _caches(d, h, g, lens, prefix_lens, owners=(0, 0), seed=0, room=3):
    torch.manual_seed(seed)
    b, n = len(lens), len(prefix_lens)
    cap, pcap = max(lens) + room, max(1, max(prefix_lens) + room)
    cache = mlkv.MLKVCache(len(owners), h, d, list(owners), g, b, cap)
    prefix = mlkv.MLKVCache(len(owners), h, d, list(owners), g, n, pcap)
    K, V = _randn(b, g, cap, d), _randn(b, g, cap, d)
    PK, PV = _randn(n, g, pcap, d), _randn(n, g, pcap, d)
    _ends(K, V, lens)
    _ends(PK, PV, prefix_lens)
    layer = max(owners)
    cache.load_prefix(layer, K, V, cap)
    prefix.load_prefix(layer, PK, PV, pcap)
    return cache, prefix, K, V, PK, PV, layer


def _joined(i, n, x, m, K, V, PK, PV):
    k, v = K[i, :, :n], V[i, :, :n]
    if x >= 0:
        k, v = torch.cat([PK[x, :, :m], k], 1), torch.cat([PV[x, :, :m], v], 1)
    return k.double(), v.double()


def _decode(d, h, g, lens, prefix_of, prefix_lens, owners=(0, 0), seed=0, sigma=1.0):
    cache, prefix, K, V, PK, PV, layer = _caches(d, h, g, lens, prefix_lens, owners, seed)
    Q = _randn(len(lens), h, d, sigma=sigma)
    out = torch.full_like(Q, 9.0)
    cache.decode_attention_prefix(layer, prefix, prefix_of, prefix_lens, Q, out, lens)
    cache.sync_status()
    for i, n in enumerate(lens):
        x = prefix_of[i]
        k, v = _joined(i, n, x, prefix_lens[x] if x >= 0 else 0, K, V, PK, PV)
        see = torch.ones(1, k.shape[1], dtype=torch.bool, device="cuda")
        want, spread = attend(Q[i].double()[:, None], k, v, see)
        assert_attention(out[i], want[:, 0], spread[:, 0], ROUNDINGS)
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(8, 2), (12, 1), (16, 1), (3, 3), (20, 4)])
def test_decode_small(d, h, g):
    # neighbours; sequences in no order; an empty prefix; sequences without any; a prefix without sequences
    _decode(d, h, g, [1, 7, 64], [0, 0, 0], [130])
    _decode(d, h, g, [1, 65, 3, 200, 64, 128, 9], [1, 0, -1, 1, 2, 0, 1], [100, 257, 0, 40], seed=1)
    _decode(d, h, g, [5, 6], [-1, -1], [10], seed=2)
    _decode(d, h, g, [5, 6], [0, 0], [0], seed=3)
    _decode(d, h, g, [1], [0], [1], seed=4)
    _decode(d, h, g, [70] * 5, [2, 2, 0, 0, 1], [64, 128, 129], seed=5)


@pytest.mark.parametrize("d,h,g,b,lens,n", [
    (64, 12, 1, 40, 30, 1),         # 480 rows of a KV head: two pairs of tiles
    (64, 12, 4, 130, 5, 1),         # 390 rows
    (128, 32, 8, 100, 300, 3),
    (128, 16, 1, 33, 100, 2),       # eight sequences a tile
    (64, 12, 12, 300, 3, 2),        # one head a row: 128 sequences a tile
    (128, 14, 2, 50, 64, 1),        # 18 sequences of 7 heads: 126 rows of a tile
    (128, 32, 8, 24, 1500, 4),      # four to seven sequences a prefix
    (64, 12, 4, 21, 2500, 3),       # groups of five sequences of 3 heads, and what is left
    (64, 14, 2, 12, 2500, 2),       # of two of 7
    (128, 16, 1, 6, 3000, 2),       # of one of 16
])
@pytest.mark.parametrize("p", [1, 127, 128, 1000, 5000])
def test_decode_many_sequences(d, h, g, b, lens, n, p):
    rng = np.random.default_rng(b + p)
    prefix_of = [int(x) for x in rng.integers(0 if n == 1 else -1, n, b)]
    seq = [int(x) for x in rng.integers(1, lens + 1, b)]
    _decode(d, h, g, seq, prefix_of, [max(1, p - 77 * x) for x in range(n)], seed=p)


@pytest.mark.parametrize("d,h,g", [(64, 12, 1), (128, 32, 8)])
def test_decode_long(d, h, g):
    out = _decode(d, h, g, [3000, 20, 9000], [0, 0, 0], [40001])
    assert torch.equal(out, _decode(d, h, g, [3000, 20, 9000], [0, 0, 0], [40001]))


def test_decode_many_prefixes():
    """More units than a launch takes."""
    b = 700
    _decode(64, 12, 12, [1 + i % 5 for i in range(b)], [(i * 7) % b for i in range(b)],
            [1 + i % 260 for i in range(b)])


def test_decode_later_owner():
    _decode(128, 8, 2, [33, 65], [1, 0], [200, 100], owners=(0, 0, 2, 2))
    _decode(64, 8, 2, [33, 65], [1, 0], [200, 100], owners=(0, 1, 2))


def test_decode_prefix_in_the_same_cache():
    """Sequences that branch from sequence 2 of their own cache."""
    torch.manual_seed(0)
    d, h, g, lens = 128, 8, 2, [40, 3, 500, 66]
    cache = mlkv.MLKVCache(1, h, d, [0], g, 4, 512)
    K, V, Q = _randn(4, g, 512, d), _randn(4, g, 512, d), _randn(4, h, d)
    cache.load_prefix(0, K, V, 512)
    out = torch.zeros_like(Q)
    cache.decode_attention_prefix(0, cache, [2, 2, -1, 2], [0, 0, 333, 0], Q, out, lens)
    for i, n in enumerate(lens):
        k, v = _joined(i, n, -1 if i == 2 else 2, 333, K, V, K, V)
        want, spread = attend(Q[i].double()[:, None], k, v,
                              torch.ones(1, k.shape[1], dtype=torch.bool, device="cuda"))
        assert_attention(out[i], want[:, 0], spread[:, 0], ROUNDINGS)


def test_decode_peaked_scores():
    _decode(128, 32, 8, [100] * 20, [0] * 20, [3000], sigma=8.0)
    _decode(64, 12, 4, [100] * 20, [0] * 20, [3000], sigma=8.0)


def test_decode_nan_stays_with_its_sequence():
    torch.manual_seed(0)
    d, h, g, b = 64, 12, 4, 6
    cache, prefix, K, V, PK, PV, _ = _caches(d, h, g, [20] * b, [300, 300])
    Q = _randn(b, h, d)
    Q[3, 5] = math.nan
    out, clean = torch.zeros_like(Q), torch.zeros_like(Q)
    where = [0, 0, 0, 0, 1, 1]
    cache.decode_attention_prefix(0, prefix, where, [300, 300], Q, out, [20] * b)
    cache.decode_attention_prefix(0, prefix, where, [300, 300], torch.nan_to_num(Q), clean, [20] * b)
    bad = torch.isnan(out.float())
    assert bad[3, 5].all() and bad.sum() == d
    assert torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("d,h,g", [(64, 12, 4), (64, 12, 12), (128, 32, 8), (128, 6, 2), (128, 12, 1)])
@pytest.mark.parametrize("lens,prefix_of,prefix_lens", [
    ([1, 2, 130], [0, 0, 0], [1]),
    ([128, 257, 5, 129], [0, 1, -1, 1], [128, 200]),
    ([300, 1], [1, 0], [0, 1025]),
    ([64, 500, 333], [0, 0, 1], [127, 700]),
])
@pytest.mark.parametrize("owner", [True, False])
def test_prefill(d, h, g, lens, prefix_of, prefix_lens, owner):
    torch.manual_seed(len(lens))
    b, s = len(lens), max(lens) + 3
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, s + 5)
    prefix = mlkv.MLKVCache(2, h, d, [0, 0], g, len(prefix_lens), max(prefix_lens) + 3)
    n, pcap = len(prefix_lens), max(prefix_lens) + 3
    K, V, Q = _randn(b, g, s, d), _randn(b, g, s, d), _randn(b, s, h, d)
    PK, PV = _randn(n, g, pcap, d), _randn(n, g, pcap, d)
    _ends(PK, PV, prefix_lens)
    prefix.load_prefix(0, PK, PV, pcap)
    out = torch.full_like(Q, 9.0)
    if not owner:
        cache.load_prefix(0, K, V, s)
    cache.prefill_prefix(0 if owner else 1, prefix, prefix_of, prefix_lens, Q, K if owner else None,
                         V if owner else None, out, lens)
    cache.sync_status()
    for i, m in enumerate(lens):
        x = prefix_of[i]
        p = prefix_lens[x] if x >= 0 else 0
        k, v = _joined(i, m, x, p, K, V, PK, PV)
        t, u = torch.arange(m, device="cuda")[:, None], torch.arange(p + m, device="cuda")[None]
        want, spread = attend(Q[i, :m].transpose(0, 1).double(), k, v, u <= p + t)
        assert_attention(out[i, :m].transpose(0, 1), want, spread, ROUNDINGS)
        assert (out[i, m:] == 9.0).all()
    # the prompt is stored, and a step goes on from there
    q, one = _randn(b, h, d), torch.zeros(b, h, d, dtype=torch.bfloat16, device="cuda")
    cache.decode_attention_prefix(1, prefix, prefix_of, prefix_lens, q, one, lens)
    for i, m in enumerate(lens):
        x = prefix_of[i]
        k, v = _joined(i, m, x, prefix_lens[x] if x >= 0 else 0, K, V, PK, PV)
        want, spread = attend(q[i].double()[:, None], k, v,
                              torch.ones(1, k.shape[1], dtype=torch.bool, device="cuda"))
        assert_attention(one[i], want[:, 0], spread[:, 0], ROUNDINGS)


@pytest.mark.parametrize("d,h,g", [(64, 12, 4), (64, 12, 1), (128, 32, 8), (128, 6, 2), (128, 16, 1)])
@pytest.mark.parametrize("b,s,p", [(66, 1, 2000), (40, 13, 700), (3, 300, 40), (9, 100, 5000), (1000, 1, 129)])
def test_prefill_short_prompts(d, h, g, b, s, p):
    """Prompts whose positions leave most of a tile empty; neighbours and others, uneven."""
    torch.manual_seed(b)
    rng = np.random.default_rng(b + s)
    lens = [int(x) for x in rng.integers(max(1, s // 2), s + 1, b)]
    lens[-1] = s
    prefix_of = [int(x) for x in rng.integers(-1, 2, b)]
    prefix_lens = [p, max(1, p - 70)]
    cap = s + 2
    cache, prefix = mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap), mlkv.MLKVCache(2, h, d, [0, 0], g, 2, p)
    K, V, Q = _randn(b, g, s, d), _randn(b, g, s, d), _randn(b, s, h, d)
    for i, n in enumerate(lens):
        K[i, :, n:], V[i, :, n:] = math.nan, math.inf
    PK, PV = _randn(2, g, p, d), _randn(2, g, p, d)
    prefix.load_prefix(0, PK, PV, p)
    out = torch.full_like(Q, 9.0)
    cache.prefill_prefix(0, prefix, prefix_of, prefix_lens, Q, K, V, out, lens)
    again = torch.full_like(Q, 9.0)
    cache.prefill_prefix(1, prefix, prefix_of, prefix_lens, Q, None, None, again, lens)
    cache.sync_status()
    for i in sorted(set([0, b - 1] + [int(x) for x in rng.integers(0, b, 10)])):
        m, x = lens[i], prefix_of[i]
        n = prefix_lens[x] if x >= 0 else 0
        k, v = _joined(i, m, x, n, K, V, PK, PV)
        t, u = torch.arange(m, device="cuda")[:, None], torch.arange(n + m, device="cuda")[None]
        want, spread = attend(Q[i, :m].transpose(0, 1).double(), k, v, u <= n + t)
        assert_attention(out[i, :m].transpose(0, 1), want, spread, ROUNDINGS)
        assert_attention(again[i, :m].transpose(0, 1), want, spread, ROUNDINGS)
    for i, m in enumerate(lens):
        assert (out[i, m:] == 9.0).all() and (again[i, m:] == 9.0).all()


def test_prefill_without_anything_in_front_is_the_plain_one():
    torch.manual_seed(0)
    d, h, g, lens = 128, 8, 2, [100, 333]
    Q, K, V = _randn(2, 333, h, d), _randn(2, g, 333, d), _randn(2, g, 333, d)
    got = []
    for shared in (False, True):
        cache = mlkv.MLKVCache(1, h, d, [0], g, 2, 400)
        prefix = mlkv.MLKVCache(1, h, d, [0], g, 1, 10)
        out = torch.zeros_like(Q)
        if shared:
            cache.prefill_prefix(0, prefix, [-1, 0], [0], Q, K, V, out, lens)
        else:
            cache.prefill(0, Q, K, V, out, lens)
        got.append(out)
    assert torch.equal(*got)


def test_prefill_more_units_than_a_launch():
    torch.manual_seed(0)
    d, h, g, b, s = 64, 12, 1, 90, 600
    cache = mlkv.MLKVCache(1, h, d, [0], g, b, s)
    prefix = mlkv.MLKVCache(1, h, d, [0], g, 2, 200)
    K, V, Q = _randn(b, g, s, d), _randn(b, g, s, d), _randn(b, s, h, d)
    PK, PV = _randn(2, g, 200, d), _randn(2, g, 200, d)
    prefix.load_prefix(0, PK, PV, 200)
    out = torch.zeros_like(Q)
    lens = [s - i % 7 for i in range(b)]
    cache.prefill_prefix(0, prefix, [i % 3 - 1 for i in range(b)], [200, 90], Q, K, V, out, lens)
    for i in (0, 1, 2, 44, 88, 89):
        x, p = i % 3 - 1, [200, 90, 0][i % 3 - 1]
        k, v = _joined(i, lens[i], x, p, K, V, PK, PV)
        t, u = torch.arange(lens[i], device="cuda")[:, None], torch.arange(p + lens[i], device="cuda")[None]
        want, spread = attend(Q[i, :lens[i]].transpose(0, 1).double(), k, v, u <= p + t)
        assert_attention(out[i, :lens[i]].transpose(0, 1), want, spread, ROUNDINGS)


def test_rejections():
    d, h, g = 64, 8, 2
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, 2, 100)
    prefix = mlkv.MLKVCache(2, h, d, [0, 0], g, 1, 50)
    Q, out = _randn(2, h, d), torch.zeros(2, h, d, dtype=torch.bfloat16, device="cuda")
    good = dict(layer=0, prefix=prefix, prefix_of=[0, -1], prefix_lens=[50], Q=Q, out=out, seq_lens=[1, 100])
    cache.decode_attention_prefix(**good)
    other = [mlkv.MLKVCache(2, h, d, [0, 1], g, 1, 50), mlkv.MLKVCache(2, 4, d, [0, 0], g, 1, 50),
             mlkv.MLKVCache(1, h, d, [0], g, 1, 50), mlkv.MLKVCache(2, h, 128, [0, 0], g, 1, 50)]
    for change, code in [(dict(prefix=o), mlkv.MLKV_ERR_MAP) for o in other] + [
            (dict(prefix_of=[1, 0]), mlkv.MLKV_ERR_RANGE), (dict(prefix_of=[-2, 0]), mlkv.MLKV_ERR_RANGE),
            (dict(prefix_lens=[51]), mlkv.MLKV_ERR_RANGE), (dict(prefix_lens=[-1]), mlkv.MLKV_ERR_RANGE),
            (dict(seq_lens=[0, 1]), mlkv.MLKV_ERR_RANGE), (dict(seq_lens=[1, 101]), mlkv.MLKV_ERR_RANGE),
            (dict(layer=2), mlkv.MLKV_ERR_INVALID_ARG), (dict(Q=None), mlkv.MLKV_ERR_INVALID_ARG),
            (dict(out=Q), mlkv.MLKV_ERR_INVALID_ARG), (dict(prefix_of=[0]), mlkv.MLKV_ERR_INVALID_ARG),
            (dict(prefix_lens=[1, 1]), mlkv.MLKV_ERR_INVALID_ARG)]:
        with pytest.raises(mlkv.MLKVError) as e:
            cache.decode_attention_prefix(**dict(good, **change))
        assert e.value.code == code, change
    K, P = _randn(2, g, 30, d), _randn(2, 30, h, d)
    for change, code in [(dict(prefix=cache, prefix_lens=[1, 1]), mlkv.MLKV_ERR_INVALID_ARG),
                         (dict(prefix=other[0]), mlkv.MLKV_ERR_MAP), (dict(K=None), mlkv.MLKV_ERR_INVALID_ARG),
                         (dict(prefix_of=[0, 3]), mlkv.MLKV_ERR_RANGE),
                         (dict(prompt_lens=[31, 1]), mlkv.MLKV_ERR_RANGE)]:
        with pytest.raises(mlkv.MLKVError) as e:
            cache.prefill_prefix(**dict(dict(layer=0, prefix=prefix, prefix_of=[0, 0], prefix_lens=[9], Q=P, K=K,
                                             V=K, out=torch.zeros_like(P), prompt_lens=[30, 1]), **change))
        assert e.value.code == code, change

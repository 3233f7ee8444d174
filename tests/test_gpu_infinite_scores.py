"""Scores of -infinity: keys with an infinity that every query has a positive product with.

A softmax gives such keys the weight 0, wherever they lie: in the first tile, in a whole chunk of the context, in all
of a prefix.  Against 64-bit forms, with the bounds of the operators' tests.
"""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend  # noqa: E402

pytestmark = pytest.mark.gpu
ROUNDINGS = 2


def _randn(*shape):
    return torch.randn(shape, device="cuda").bfloat16()


def _queries(*shape):
    """Channel 0 positive, so that -infinity there makes the score -infinity (and not NaN)."""
    q = _randn(*shape)
    q[..., 0] = q[..., 0].abs() + 0.5
    return q


def _see(rows, n):
    return torch.ones(rows, n, dtype=torch.bool, device="cuda")


# (64, 12, 4): three heads a KV head; (128, 32, 8): four; (128, 6, 6): one; (64, 32, 2): sixteen
SHAPES = [(64, 12, 4), (128, 32, 8), (128, 6, 6), (64, 32, 2)]


@pytest.mark.parametrize("d,h,g", SHAPES)
@pytest.mark.parametrize("b", [2, 8, 128])
@pytest.mark.parametrize("p,dead", [(128, 128), (500, 128), (4000, 64), (4000, 128), (4000, 2500), (4000, 4000)])
def test_decode_behind_a_prefix(d, h, g, b, p, dead):
    """The first `dead` positions of the prefix, for few sequences and many."""
    torch.manual_seed(b + p)
    cache, prefix = mlkv.MLKVCache(1, h, d, [0], g, b, 70), mlkv.MLKVCache(1, h, d, [0], g, 1, p)
    K, V, PK, PV = _randn(b, g, 70, d), _randn(b, g, 70, d), _randn(1, g, p, d), _randn(1, g, p, d)
    PK[:, :, :dead, 0] = -math.inf
    cache.load_prefix(0, K, V, 70)
    prefix.load_prefix(0, PK, PV, p)
    lens = [1 + (i * 13) % 70 for i in range(b)]
    Q = _queries(b, h, d)
    out = torch.full_like(Q, 9.0)
    cache.decode_attention_prefix(0, prefix, [0] * b, [p], Q, out, lens)
    cache.sync_status()
    for i in sorted({0, 1, b // 2, b - 1}):
        k = torch.cat([PK[0], K[i, :, :lens[i]]], 1).double()
        v = torch.cat([PV[0], V[i, :, :lens[i]]], 1).double()
        want, spread = attend(Q[i].double()[:, None], k, v, _see(1, k.shape[1]))
        assert_attention(out[i], want[:, 0], spread[:, 0], ROUNDINGS)
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("d,h,g", SHAPES)
@pytest.mark.parametrize("b,s,p", [(2, 300, 700), (3, 130, 128), (40, 1, 2000), (4, 12, 3582)])
@pytest.mark.parametrize("dead,own", [(128, 0), (-1, 0), (128, 129), (0, 128)])
def test_prefill_behind_a_prefix(d, h, g, b, s, p, dead, own):
    """The first `dead` positions of the prefix (-1: all), and `own` of the prompts behind them."""
    torch.manual_seed(b + s)
    dead = p if dead < 0 else dead
    cache, prefix = mlkv.MLKVCache(1, h, d, [0], g, b, s), mlkv.MLKVCache(1, h, d, [0], g, 1, p)
    K, V, PK, PV = _randn(b, g, s, d), _randn(b, g, s, d), _randn(1, g, p, d), _randn(1, g, p, d)
    PK[:, :, :dead, 0] = -math.inf
    K[:, :, :own, 0] = -math.inf
    prefix.load_prefix(0, PK, PV, p)
    Q = _queries(b, s, h, d)
    out = torch.full_like(Q, 9.0)
    cache.prefill_prefix(0, prefix, [0] * b, [p], Q, K, V, out, [s] * b)
    cache.sync_status()
    t, u = torch.arange(s, device="cuda")[:, None], torch.arange(p + s, device="cuda")[None]
    see = u <= p + t
    alive = (u >= dead) & ((u < p) | (u >= p + own))
    some = (see & alive).any(1)   # rows with a score above -infinity
    for i in (0, b - 1):
        k, v = torch.cat([PK[0], K[i]], 1).double(), torch.cat([PV[0], V[i]], 1).double()
        want, spread = attend(Q[i, some].transpose(0, 1).double(), k, v, see[some])
        assert_attention(out[i, some].transpose(0, 1), want, spread, ROUNDINGS)
    # every form gives zeros where a row has nothing but such scores, as the decode behind a prefix does
    assert (out[:, ~some] == 0).all()


@pytest.mark.parametrize("d,h,g", SHAPES)
@pytest.mark.parametrize("dead", [1, 128, 200, 256])
@pytest.mark.parametrize("window", [0, 450])
def test_prefill(d, h, g, dead, window):
    torch.manual_seed(dead)
    b, s = 2, 600
    cache = mlkv.MLKVCache(1, h, d, [0], g, b, s)
    K, V, Q = _randn(b, g, s, d), _randn(b, g, s, d), _queries(b, s, h, d)
    K[:, :, :dead, 0] = -math.inf
    out = torch.full_like(Q, 9.0)
    if window:
        cache.prefill_window(0, Q, K, V, out, [s, s - 1], window, 4)
    else:
        cache.prefill(0, Q, K, V, out, [s, s - 1])
    cache.sync_status()
    t, u = torch.arange(s, device="cuda")[:, None], torch.arange(s, device="cuda")[None]
    see = u <= t
    if window:
        see &= (u < 4) | (u > t - window)
    for i, n in enumerate([s, s - 1]):
        want, spread = attend(Q[i, dead:n].transpose(0, 1).double(), K[i].double(), V[i].double(), see[dead:n])
        assert_attention(out[i, dead:n].transpose(0, 1), want, spread, ROUNDINGS)


@pytest.mark.parametrize("d,h,g,layers", [(64, 12, 1, 6), (64, 12, 1, 12), (128, 32, 8, 4), (128, 16, 1, 12)])
@pytest.mark.parametrize("b,n,dead", [(2, 300, 128), (2, 3000, 128), (3, 5000, 3000), (64, 2000, 256)])
def test_decode_of_a_block_of_layers(d, h, g, layers, b, n, dead):
    torch.manual_seed(n)
    cache = mlkv.MLKVCache(layers, h, d, [0] * layers, g, b, n)
    K, V, Q = _randn(b, g, n, d), _randn(b, g, n, d), _queries(layers, b, h, d)
    K[:, :, :dead, 0] = -math.inf
    cache.load_prefix(0, K, V, n)
    out = torch.full_like(Q, 9.0)
    lens = [n - i % 3 for i in range(b)]
    cache.decode_block_fused(0, Q, out, lens)
    cache.sync_status()
    for i in sorted({0, 1, b - 1}):
        want, spread = attend(Q[:, i].transpose(0, 1).double(), K[i].double(), V[i].double(),
                              (torch.arange(n, device="cuda") < lens[i]).expand(layers, n))
        assert_attention(out[:, i].transpose(0, 1), want, spread, ROUNDINGS)

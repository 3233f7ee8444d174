"""Decode over the 4-bit cache where values differ by magnitude: between positions, between groups of
channels, together with logits that differ too.  Every channel is judged by its own values.

The bound, relative to the spread A = sum p |v| / sum p of the channel over what the cache holds: a weight
times a scale is rounded once to fp16 (2^-11), scores are fp32 (1e-3 covers weights and their sum), the output
is rounded to bf16 (HALF_ULP of itself).  What falls below fp16's normal range, up to 2^-27 of the largest such
product of the group of channels a position, gets 2^-34: no input here leans on it.
"""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import HALF_ULP, held, visible  # noqa: E402

pytestmark = pytest.mark.gpu


def _uneven(n, most):
    return [1 + (7919 * i * i + 13 * i) % most for i in range(n)]


def _inputs(d, h, g, lens, seed):
    """Queries that share a direction u, keys with small logits, values around 1; logit(x): the key whose
    logit is about x for every head."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b, cap = len(lens), max(lens)
    u = torch.randint(0, 2, (d,), device="cuda", generator=gen) * 2.0 - 1

    def normal(*shape):
        return torch.empty(shape, device="cuda").normal_(generator=gen)

    Q = (u + 0.3 * normal(b, h, d)).bfloat16()
    K, V = 0.5 * normal(b, g, cap, d), 1 + 0.25 * normal(b, g, cap, d)
    return Q, K, V, lambda x: u * (x / math.sqrt(d)), normal


def _check(d, h, g, lens, Q, K, V, window=0, sinks=0):
    K, V = K.bfloat16(), V.bfloat16()
    b, cap = len(lens), max(lens)
    cache = mlkv.MLKVQ4Cache(1, h, d, [0], g, b, cap)
    cache.load_prefix(0, K, V, cap)
    out = torch.full_like(Q, 9.0)
    cache.decode_attention(0, Q, out, lens, window, sinks)
    cache.sync_status()
    worst = 0.0
    for i in range(0, b, max(1, b // 8)):
        see = visible(lens[i], window, sinks)
        k, v = held(K[i, :, :lens[i]][:, see]), held(V[i, :, :lens[i]][:, see])
        n = k.shape[1]
        q = Q[i].double().view(g, h // g, d)
        p = torch.softmax(q @ k.transpose(1, 2) / math.sqrt(d), -1)          # [g][G][n]
        want, spread = p @ v, p @ v.abs()
        largest = v.abs().unflatten(-1, (-1, 32)).amax(-1)                   # [g][n][groups]
        top = (p[..., None] * largest[:, None]).amax(2).repeat_interleave(32, -1)
        bound = ((2.0 ** -11 + 1e-3) * spread + HALF_ULP * 1.01 * want.abs() + n * 2.0 ** -34 * top)
        got = out[i].double().view(want.shape)
        assert torch.isfinite(got).all()
        worst = max(worst, float(((got - want).abs() / bound).max()))
    assert worst <= 1.0, worst


FORMS = [   # runs of CTAs: few tiles; runs of warps: many
    (128, 8, 2, [700, 257, 64], 0, 0), (64, 12, 4, [1000, 300], 0, 0), (128, 16, 1, [4000], 0, 0),
    (64, 12, 1, [3000, 2000], 0, 0), (128, 8, 2, [2000, 900], 300, 4),
    (128, 32, 8, _uneven(64, 8000), 0, 0), (64, 12, 4, [5000] * 40 + [3000] * 60, 0, 0),
    (128, 32, 2, _uneven(100, 16000), 0, 0), (64, 12, 1, _uneven(90, 60000), 0, 0),
    (128, 8, 2, _uneven(300, 9000), 3000, 70),
]


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
@pytest.mark.parametrize("nats,group", [(10, 4), (12, 4), (10, 6), (8, 8), (14, 12), (0, 20)])
def test_sink_of_small_value_and_smaller_groups(d, h, g, lens, window, sinks, nats, group):
    """The first token takes most of the weight and holds little; the channels past the first 32 are
    2^-group of those."""
    Q, K, V, logit, _ = _inputs(d, h, g, lens, nats + group)
    K[:, :, 0] = logit(nats)
    V[:, :, 0] *= 0.02
    V[..., 32:] *= 2.0 ** -group
    _check(d, h, g, lens, Q, K, V, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
@pytest.mark.parametrize("nats,power", [(-40, 12), (-40, 16), (-40, 20), (-40, 24), (-40, 40), (-8, 10),
                                        (-20, 30)])
def test_one_larger_value_of_little_weight(d, h, g, lens, window, sinks, nats, power):
    """One visible position (of the sinks, where there are some) holds values 2^power larger."""
    Q, K, V, logit, _ = _inputs(d, h, g, lens, power - nats)
    at = 1 if sinks else min(lens) // 2
    K[:, :, at] = logit(nats)
    V[:, :, at] *= 2.0 ** power
    _check(d, h, g, lens, Q, K, V, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
def test_sink_without_value_and_a_larger_one(d, h, g, lens, window, sinks):
    Q, K, V, logit, _ = _inputs(d, h, g, lens, 3)
    K[:, :, 0] = logit(14)
    V[:, :, 0] *= 0.001
    V[::2, :, 0] = 0
    V[:, :, 1 if sinks else min(lens) // 2] *= 64
    _check(d, h, g, lens, Q, K, V, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
def test_every_magnitude(d, h, g, lens, window, sinks):
    """Positions, groups and both together spread over 2^40, logits over tens."""
    Q, K, V, _, normal = _inputs(d, h, g, lens, 4)
    K *= 8
    for shape in ((*V.shape[:3], 1), (1, 1, 1, d // 32), (*V.shape[:3], d // 32)):
        V *= torch.exp2(normal(*shape).mul(7).clamp(-20, 20)).repeat_interleave(d // shape[3] if shape[3] > 1
                                                                              else 1, -1)
    _check(d, h, g, lens, Q, K, V, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
@pytest.mark.parametrize("power", [120, 100, -60, -100, -112])
def test_huge_and_tiny_values(d, h, g, lens, window, sinks, power):
    Q, K, V, _, _ = _inputs(d, h, g, lens, 5)
    _check(d, h, g, lens, Q, K, V * 2.0 ** power, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
@pytest.mark.parametrize("nats", [10, 25, 60])
def test_weight_moves_to_a_position_without_values(d, h, g, lens, window, sinks, nats):
    """A late position takes the weight and holds zeros: the others' sum is all there is."""
    Q, K, V, logit, _ = _inputs(d, h, g, lens, nats)
    for i, n in enumerate(lens):
        K[i, :, n - 1 - n // 5 if not window else n - 1 - min(n, window) // 5] = logit(nats)
        V[i, :, n - 1 - n // 5 if not window else n - 1 - min(n, window) // 5] = 0
    _check(d, h, g, lens, Q, K, V, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
def test_logits_that_rise_as_values_fall(d, h, g, lens, window, sinks):
    """Every position outweighs the last and holds less."""
    Q, K, V, logit, _ = _inputs(d, h, g, lens, 6)
    cap = max(lens)
    at = torch.arange(cap, device="cuda") * (80.0 / cap)          # nats
    K[:] = K * 0.2 + at[:, None] * logit(1.0)
    V *= torch.exp(-at)[:, None]
    _check(d, h, g, lens, Q, K, V, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", FORMS)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bad_value_stays_in_its_group(d, h, g, lens, window, sinks, bad):
    """A visible value that is none spoils its 32 channels, of its KV head and sequence alone."""
    Q, K, V, _, _ = _inputs(d, h, g, lens, 7)
    K, V = K.bfloat16(), V.bfloat16()
    i = len(lens) - 1
    V[i, g - 1, lens[i] - 1, 33] = bad
    cache = mlkv.MLKVQ4Cache(1, h, d, [0], g, len(lens), max(lens))
    cache.load_prefix(0, K, V, max(lens))
    out = torch.zeros_like(Q)
    cache.decode_attention(0, Q, out, lens, window, sinks)
    cache.sync_status()
    want = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    want[i, (g - 1) * (h // g):, 32:64] = True
    assert torch.equal(torch.isnan(out), want) and torch.isfinite(out[~want]).all()

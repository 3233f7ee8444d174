"""The 4-bit cache: what it holds (exactly), decode attention over it (64-bit reference over the held
values), prefill into it, and its refusals."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend, held, visible  # noqa: E402

pytestmark = pytest.mark.gpu


def _randn(*shape, sigma=1.0):
    return (torch.randn(shape, device="cuda") * sigma).bfloat16()


def _read(cache, layer, start, n):
    k = torch.full((cache.b, cache.g, n, cache.d), 9.0, device="cuda").bfloat16()
    v = torch.full_like(k, 9.0)
    cache.read(layer, k, v, start, n)
    return k, v


def _same(got, want):
    want = want.bfloat16()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 200])
def test_prefix_and_read_are_exact(d, n):
    torch.manual_seed(n)
    b, g, cap = 3, 2, 205
    cache = mlkv.MLKVQ4Cache(4, 4, d, [0, 0, 2, 2], g, b, cap)
    K, V = _randn(b, g, n, d), _randn(b, g, n, d, sigma=30.0)
    cache.load_prefix(2, K, V, n)
    k, v = _read(cache, 3, 0, n)     # a reader of layer 2's slot
    _same(k, held(K))
    _same(v, held(V))
    assert float(torch.stack(_read(cache, 0, 0, n)).abs().max()) == 0   # the other slot
    for start, m in ((0, 1), (n - 1, 1), (n // 2, n - n // 2), (n // 3, 1)):
        k, v = _read(cache, 2, start, m)
        _same(k, held(K[:, :, start:start + m]))
        _same(v, held(V[:, :, start:start + m]))
    # a shorter prefix leaves the positions behind it alone
    K2, V2 = _randn(b, g, max(1, n // 2), d), _randn(b, g, max(1, n // 2), d)
    cache.load_prefix(2, K2, V2, K2.shape[2])
    k, v = _read(cache, 2, 0, n)
    _same(k, held(torch.cat([K2, K[:, :, K2.shape[2]:]], 2)))
    _same(v, held(torch.cat([V2, V[:, :, V2.shape[2]:]], 2)))
    cache.load_prefix(3, K, V, n)     # not an owner: nothing is stored
    assert torch.equal(_read(cache, 2, 0, n)[0], k)


@pytest.mark.parametrize("d", [64, 128])
def test_values_at_their_limits(d):
    """Every tie between two codes, signs, zeros, tiny and huge groups, NaN and infinities."""
    rows = []
    for scale in (1.0, 0.5, 3.0, 1.4921875, 2.0 ** -100, 2.0 ** 100):
        top = 7.0 * scale
        for k in range(4):
            row = torch.zeros(d)
            row[::32] = top if k % 2 else -top
            for i in range(1, 32):
                x = (i % 8 + 0.5) * scale if k < 2 else (i % 8 + 0.5) * scale * 0.996
                row[i::32] = (x if i % 3 else -x) if abs(x) <= top else 0.0
            rows.append(row)
    rows += [torch.zeros(d), torch.full((d,), 1e-39), torch.full((d,), 8.3e-38),
             torch.full((d,), 3.38e38), torch.full((d,), -3.38e38)]
    for bad in (math.nan, math.inf, -math.inf):
        row = torch.randn(d)
        row[5] = bad
        rows.append(row)
    x = torch.stack(rows).cuda().bfloat16()[None, None]
    n = x.shape[2]
    cache = mlkv.MLKVQ4Cache(1, 1, d, [0], 1, 1, n)
    cache.load_prefix(0, x, x.flip(3).contiguous(), n)
    k, v = _read(cache, 0, 0, n)
    _same(k, held(x))
    _same(v, held(x.flip(3)))
    assert torch.isnan(k[0, 0, -3:, :32]).all() and torch.isfinite(k[0, 0, -3:, 32:]).all()


def test_random_bit_patterns():
    torch.manual_seed(11)
    bits = torch.randint(-32768, 32768, (2, 2, 640, 64), device="cuda", dtype=torch.int16)
    x = bits.view(torch.bfloat16)
    # groups of one magnitude, so that few codes are zero
    y = (_randn(2, 2, 640, 64) * torch.exp2(torch.randint(-90, 90, (2, 2, 640, 1), device="cuda").float())
         ).bfloat16()
    cache = mlkv.MLKVQ4Cache(1, 2, 64, [0], 2, 2, 640)
    cache.load_prefix(0, x, y, 640)
    k, v = _read(cache, 0, 0, 640)
    _same(k, held(x))
    _same(v, held(y))


@pytest.mark.parametrize("d", [64, 128])
def test_append_places_each_token(d):
    torch.manual_seed(2)
    b, g, n = 5, 3, 50
    cache = mlkv.MLKVQ4Cache(2, 3, d, [0, 0], g, b, n)
    K, V = _randn(b, g, n, d), _randn(b, g, n, d)
    cache.load_prefix(0, K, V, n)
    want_k, want_v = K.clone(), V.clone()
    for lens in ([1, 2, 16, 17, 50], [33, 32, 31, 8, 9]):
        k, v = _randn(b, g, d), _randn(b, g, d)
        cache.append(1, _randn(b, g, d), _randn(b, g, d), lens)   # not an owner
        cache.append(0, k, v, lens)
        for i, L in enumerate(lens):
            want_k[i, :, L - 1], want_v[i, :, L - 1] = k[i], v[i]
    k, v = _read(cache, 0, 0, n)
    _same(k, held(want_k))
    _same(v, held(want_v))


def _decode(d, h, g, lens, window=0, sinks=0, sigma=1.0, cap=None, seed=0, poison=True):
    torch.manual_seed(seed)
    b, cap = len(lens), cap or max(lens)
    cache = mlkv.MLKVQ4Cache(2, h, d, [0, 0], g, b, cap)
    K, V, Q = _randn(b, g, cap, d), _randn(b, g, cap, d), _randn(b, h, d, sigma=sigma)
    see = [visible(cap, window, sinks, t=L - 1) for L in lens]
    if poison:   # what is not visible holds NaN, in scales too
        for i in range(b):
            K[i, :, ~see[i]] = math.nan
            V[i, :, ~see[i]] = math.nan
    cache.load_prefix(0, K, V, cap)
    out = torch.full_like(Q, 9.0)
    cache.decode_attention(1, Q, out, lens, window, sinks)
    cache.sync_status()
    hk, hv = held(K), held(V)
    for i in range(b):
        want, spread = attend(Q[i].double()[:, None], hk[i], hv[i], see[i][None])
        # the offset of 136 a code cancels in fp32 over a tile: 1e-4 of the largest magnitudes' mean
        top = V[i][:, see[i]].double().abs().amax()
        assert_attention(out[i], want[:, 0], spread[:, 0], 2, floor=1e-4 * float(top))
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(1, 1), (12, 4), (16, 2), (12, 1), (32, 2), (9, 1)])
def test_decode_head_layouts(d, h, g):
    _decode(d, h, g, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 257], cap=300)
    _decode(d, h, g, [77, 77, 77], cap=77)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(8, 2), (12, 1)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 16), (33, 0), (64, 5), (100, 130),
                                          (250, 64), (1000, 3)])
def test_decode_window(d, h, g, window, sinks):
    lens = [1, 2, 8, 33, 64, 65, 100, 131, 200, 255, 256, 390, 400]
    _decode(d, h, g, lens, window, sinks, cap=400)
    _decode(d, h, g, [333] * 3, window, sinks, cap=400, seed=1)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (128, 32, 8, [1 + 61 * i % 997 for i in range(40)], 0, 0),     # more segments than CTAs at a time
    (64, 12, 4, [1 + 37 * i % 300 for i in range(200)], 0, 0),
    (64, 12, 1, [20000] + [5] * 63, 0, 0),                         # one long one among short ones
    (128, 32, 2, [4000 - 9 * i for i in range(64)], 0, 0),         # two records a segment, 16 heads
    (128, 32, 2, [4000, 1, 2500, 257], 0, 0),                      # many records, 16 heads
    (64, 12, 1, [8192], 0, 0), (128, 4, 1, [8192, 33], 0, 0),
    (128, 32, 8, [900 + i for i in range(20)], 700, 5),            # equal windows
    (64, 12, 1, [385 * (1 + i % 7) for i in range(300)], 0, 0),    # runs just passed by a tile
])
def test_decode_deals(d, h, g, lens, window, sinks):
    _decode(d, h, g, lens, window, sinks)


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (64, 12, 1, [70001], 0, 0),                  # hundreds of pieces: the separate merge
    (128, 8, 1, [40000], 0, 0),
    (128, 32, 8, [3000, 1, 2999, 700], 0, 0),    # a few pieces a segment: merged in the launch
    (64, 12, 4, [5000] * 40, 0, 0),              # several segments a CTA
    (128, 32, 8, [5000] * 20, 0, 0),
    (128, 32, 8, [9000, 100, 5000, 4200], 4096, 4),
    (64, 12, 1, [30000] * 2, 20000, 300),
])
def test_decode_splits(d, h, g, lens, window, sinks):
    out = _decode(d, h, g, lens, window, sinks)
    # the same bits again, whichever CTA finishes a segment last
    assert torch.equal(out, _decode(d, h, g, lens, window, sinks))


def _uneven(n, most):
    return [1 + (7919 * i * i + 13 * i) % most for i in range(n)]


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (64, 12, 4, [5000] * 40 + [3000] * 60, 0, 0),   # every warp has a run, of few tiles
    (128, 32, 8, [9000] * 32, 0, 0),             # equal lengths
    (64, 12, 1, _uneven(90, 60000), 0, 0),
    (128, 32, 8, _uneven(64, 8000), 0, 0),
    (128, 32, 2, _uneven(100, 16000), 0, 0),     # groups of 16
    (128, 8, 2, _uneven(300, 9000), 3000, 70),
    (64, 16, 1, [131072] * 22, 0, 0),            # dozens of runs a segment
])
def test_decode_warp_runs(d, h, g, lens, window, sinks):
    out = _decode(d, h, g, lens, window, sinks)
    assert torch.equal(out, _decode(d, h, g, lens, window, sinks))


@pytest.mark.parametrize("d", [64, 128])
def test_decode_sharp_scores(d):
    """Scores that differ by hundreds: the running maximum moves all the time."""
    _decode(d, 12, 2, [300, 1000, 77], sigma=30.0)


def test_decode_batch_limit_and_large_cache():
    """Every sequence slot, and rows past 2^32 bytes from the cache's start."""
    _decode(64, 1, 1, [(7 * i) % 40 + 1 for i in range(1024)])
    d, g, cap = 128, 8, 262144
    cache = mlkv.MLKVQ4Cache(1, 8, d, [0], g, 16, cap)
    assert cache.cache_bytes() == 16 * g * cap * 144 > 2 ** 32
    K, V, Q = _randn(16, g, d), _randn(16, g, d), _randn(16, 8, d)
    lens = [cap - 5] * 16
    cache.append(0, K, V, lens)
    out = torch.empty_like(Q)
    cache.decode_attention(0, Q, out, lens, 1, 0)    # sees the new token alone
    want = held(V)
    assert float((out.double() - want).abs().max()) <= 2 ** -7 * float(want.abs().max())
    cache.sync_status()


def test_nan_stays_in_its_rows():
    """A NaN query row, and a NaN key of one sequence, spoil what they enter and nothing else."""
    torch.manual_seed(4)
    cache = mlkv.MLKVQ4Cache(1, 8, 64, [0], 2, 2, 100)
    K, V, Q = _randn(2, 2, 100, 64), _randn(2, 2, 100, 64), _randn(2, 8, 64)
    K[1, 0, 50, 3] = math.nan
    Q[0, 5] = math.nan
    cache.load_prefix(0, K, V, 100)
    out = torch.empty_like(Q)
    cache.decode_attention(0, Q, out, [100, 100])
    bad = torch.isnan(out.float()).all(-1).cpu()
    assert bad[0].tolist() == [False] * 5 + [True] + [False] * 2
    assert bad[1].tolist() == [True] * 4 + [False] * 4
    assert torch.isfinite(out[0, :5]).all() and torch.isfinite(out[1, 4:]).all()


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (64, 12, 4, [1, 100, 128, 300], 0, 0), (128, 8, 2, [257, 64], 100, 3), (128, 3, 1, [300], 64, 0)])
def test_prefill_then_decode(d, h, g, lens, window, sinks):
    """Prefill attends over the bf16 prompt, an owner stores it, a reader does not; the next tokens are
    appended and attended to by both layers."""
    torch.manual_seed(8)
    b, s = len(lens), max(lens)
    cache = mlkv.MLKVQ4Cache(2, h, d, [0, 0], g, b, s + 2)
    K, V = _randn(b, g, s, d), _randn(b, g, s, d)
    for layer in (0, 1):
        Q = _randn(b, s, h, d)
        out = torch.full_like(Q, 9.0)
        cache.prefill(layer, Q, K, V, out, lens, window, sinks)
        for i, n in enumerate(lens):
            see = torch.stack([visible(n, window, sinks, t) for t in range(n)])
            want, spread = attend(Q[i, :n].double().transpose(0, 1), K[i, :, :n].double(),
                                  V[i, :, :n].double(), see)
            assert_attention(out[i, :n].transpose(0, 1), want, spread, 1)
            assert (out[i, n:] == 9).all()
    _same(_read(cache, 1, 0, s)[0], held(K))
    for step in range(2):
        now = [n + 1 + step for n in lens]
        k, v = _randn(b, g, d), _randn(b, g, d)
        cache.append(0, k, v, now)
        Q = _randn(b, h, d)
        out = torch.empty_like(Q)
        cache.decode_attention(1, Q, out, now, window, sinks)
        hk, hv = (x.double() for x in _read(cache, 0, 0, s + 2))
        for i, n in enumerate(now):
            want, spread = attend(Q[i].double()[:, None], hk[i, :, :n], hv[i, :, :n],
                                  visible(n, window, sinks)[None])
            assert_attention(out[i], want[:, 0], spread[:, 0], 2, floor=1e-3)
    cache.sync_status()


def test_refusals():
    cache = mlkv.MLKVQ4Cache(2, 8, 64, [0, 0], 2, 2, 100)
    K, Q = _randn(2, 2, 100, 64), _randn(2, 8, 64)
    out = torch.empty_like(Q)
    one = K[:, :, 0].contiguous()
    odd = torch.empty(K.numel() + 8, device="cuda", dtype=torch.bfloat16)[1:]

    def refused(code, fn, *args):
        with pytest.raises(mlkv.MLKVError) as e:
            fn(*args)
        assert e.value.code == code, e.value

    bad, rng = mlkv.MLKV_ERR_INVALID_ARG, mlkv.MLKV_ERR_RANGE
    refused(bad, cache.decode_attention, 2, Q, out, [1, 1])
    refused(bad, cache.decode_attention, 0, Q, Q, [1, 1])
    refused(bad, cache.decode_attention, 0, None, out, [1, 1])
    refused(bad, cache.decode_attention, 0, Q, odd, [1, 1])
    refused(bad, cache.decode_attention, 0, Q, out, [1, 1], -1, 0)
    refused(bad, cache.decode_attention, 0, Q, out, [1, 1], 4, -1)
    for lens in ([0, 1], [1, 101], [-3, 1]):
        refused(rng, cache.decode_attention, 0, Q, out, lens)
        refused(rng, cache.append, 0, one, one, lens)
    refused(bad, cache.append, 0, None, one, [1, 1])
    refused(bad, cache.append, -1, one, one, [1, 1])
    refused(bad, cache.load_prefix, 0, odd, K, 100)
    refused(rng, cache.load_prefix, 0, K, K, 101)
    refused(rng, cache.read, 0, K, K.clone(), 50, 51)
    refused(rng, cache.read, 0, K, K.clone(), -1, 5)
    refused(bad, cache.read, 0, K, K, 0, 100)
    P = _randn(2, 100, 8, 64)
    refused(bad, cache.prefill, 1, P, None, None, torch.empty_like(P), [5, 5])
    refused(rng, cache.prefill, 0, P, K, K, torch.empty_like(P), [5, 101])
    refused(bad, cache.prefill, 0, P, K, K, P, [5, 5])
    refused(bad, cache.prefill, 0, P, K, P.view(-1)[:K.numel()], P.clone()[:0], [5, 5])
    cache.load_prefix(0, K, K, 0)
    cache.read(0, None, None, 3, 0)
    assert torch.isfinite(out[:0]).all()
    assert np.array_equal(cache.owner, [0, 0])

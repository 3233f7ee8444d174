"""Sliding window and sinks over the bf16 cache: decode and prefill against a 64-bit reference."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend, visible  # noqa: E402

pytestmark = pytest.mark.gpu


def _randn(*shape, sigma=1.0):
    return (torch.randn(shape, device="cuda") * sigma).bfloat16()


def _decode(d, h, g, lens, window, sinks, cap=None, options=(), seed=0, sigma=1.0):
    torch.manual_seed(seed)
    b, cap = len(lens), cap or max(lens)
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap)
    for key, value in options:
        cache.set_option(key, value)
    K, V, Q = _randn(b, g, cap, d), _randn(b, g, cap, d), _randn(b, h, d, sigma=sigma)
    see = [visible(cap, window, sinks, t=L - 1) for L in lens]
    for i in range(b):   # what is not visible is never used
        K[i, :, ~see[i]] = math.nan
        V[i, :, ~see[i]] = math.inf
    cache.load_prefix(0, K, V, cap)
    out = torch.full_like(Q, 9.0)
    cache.decode_attention_window(1, Q, out, lens, window, sinks)
    cache.sync_status()
    for i in range(b):
        want, spread = attend(Q[i].double()[:, None], K[i].double(), V[i].double(), see[i][None])
        assert_attention(out[i], want[:, 0], spread[:, 0], 1)
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(8, 2), (12, 1)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (64, 64), (65, 0), (128, 5), (100, 130),
                                          (250, 64), (300, 257), (1000, 3), (0, 5)])
def test_decode_window(d, h, g, window, sinks):
    lens = [1, 2, 8, 33, 64, 65, 100, 131, 200, 255, 256, 257, 390, 700]
    _decode(d, h, g, lens, window, sinks, cap=701)
    _decode(d, h, g, [613] * 3, window, sinks, cap=640, seed=1)


@pytest.mark.parametrize("d,tile", [(64, 64), (64, 128), (64, 256), (128, 64), (128, 128)])
@pytest.mark.parametrize("g", [1, 3])
def test_decode_every_tile_length(d, tile, g):
    _decode(d, 12, g, [1, 500, 900, 333], 300, 70, options=[("tile_tokens", tile)])
    _decode(d, 12, g, [900] * 4, 300, 70, options=[("tile_tokens", tile), ("tc", 1)])


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (64, 12, 1, [100000], 60000, 100),            # many pieces: the separate merge
    (128, 32, 8, [9000, 100, 5000, 4200], 2048, 16),
    (64, 12, 1, [6000] * 64, 511, 4),
    (128, 8, 1, [4096] * 8, 1024, 0),             # equal pieces: clusters
])
def test_decode_splits(d, h, g, lens, window, sinks):
    out = _decode(d, h, g, lens, window, sinks)
    assert torch.equal(out, _decode(d, h, g, lens, window, sinks))


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (64, 12, 1, [600 + 7 * i for i in range(64)], 511, 4),     # the same tiles, other lengths
    (64, 12, 4, [1300 + i for i in range(32)], 1020, 0),
    (64, 3, 1, [512] + [900] * 63, 508, 4),                    # one just inside its window: fewer tiles
    (64, 12, 1, [2500 + 3 * i for i in range(33)], 2040, 300),
    (128, 32, 8, [1100 + i for i in range(16)], 1000, 16),
])
def test_decode_even_windows_of_uneven_lengths(d, h, g, lens, window, sinks):
    _decode(d, h, g, lens, window, sinks)


def test_decode_no_window_is_the_plain_call():
    """window 0, or one that no length outgrows, gives mlkv_decode_attention's bits."""
    torch.manual_seed(3)
    cache = mlkv.MLKVCache(1, 8, 128, [0], 2, 3, 500)
    K, V, Q = _randn(3, 2, 500, 128), _randn(3, 2, 500, 128), _randn(3, 8, 128)
    cache.load_prefix(0, K, V, 500)
    lens = [500, 17, 300]
    want, got = torch.empty_like(Q), torch.empty_like(Q)
    cache.decode_attention(0, Q, want, lens)
    for window in (0, 500, 2 ** 31 - 1):
        cache.decode_attention_window(0, Q, got, lens, window, 2 ** 31 - 1)
        assert torch.equal(want, got)
    cache.decode_attention_window(0, Q, got, lens, 1, 2 ** 31 - 1)   # every position is a sink
    assert (want.float() - got.float()).abs().max() <= 2 ** -7


def test_decode_sharp_scores():
    _decode(64, 12, 2, [1000, 77, 650], 200, 30, sigma=30.0)


@pytest.mark.parametrize("d,h,g", [(64, 12, 4), (64, 3, 1), (128, 8, 2), (128, 3, 1), (128, 6, 2)])
@pytest.mark.parametrize("lens,window,sinks", [
    ([1, 700, 128, 300], 1, 0), ([513], 64, 0), ([640, 129], 128, 1), ([777, 500], 200, 130),
    ([900], 127, 256), ([1000, 385], 300, 4), ([400], 399, 0), ([260, 256], 0, 7),
])
def test_prefill_window(d, h, g, lens, window, sinks):
    torch.manual_seed(len(lens) + window)
    b, s = len(lens), max(lens)
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, s)
    K, V = _randn(b, g, s, d), _randn(b, g, s, d)
    for layer in (0, 1):   # over the prompt's own tensors, then over the slot
        Q = _randn(b, s, h, d)
        out = torch.full_like(Q, 9.0)
        cache.prefill_window(layer, Q, K, V, out, lens, window, sinks)
        cache.sync_status()
        for i, n in enumerate(lens):
            see = torch.stack([visible(n, window, sinks, t) for t in range(n)])
            want, spread = attend(Q[i, :n].double().transpose(0, 1), K[i, :, :n].double(),
                                  V[i, :, :n].double(), see)
            assert_attention(out[i, :n].transpose(0, 1), want, spread, 1)
            assert (out[i, n:] == 9).all()


def test_prefill_window_leaves_hidden_tiles_unread():
    """Keys and values in tiles that no query sees may hold anything; what lies past a prompt too."""
    torch.manual_seed(1)
    d, n, window, sinks = 64, 1000, 128, 4
    cache = mlkv.MLKVCache(1, 4, d, [0], 1, 2, n)
    K, V, Q = _randn(2, 1, n, d), _randn(2, 1, n, d), _randn(2, n, 4, d)
    out = torch.empty_like(Q)
    clean = torch.empty_like(Q)
    cache.prefill_window(0, Q, K, V, clean, [n, n], window, sinks)
    K[:, :, 128:256] = math.nan
    V[:, :, 128:256] = math.nan
    cache.prefill_window(0, Q, K, V, out, [n, n], window, sinks)
    rows = slice(3 * 128, n)   # their windows start behind position 256
    assert torch.equal(out[:, rows], clean[:, rows])
    K[1, :, 450:], V[1, :, 450:] = math.nan, math.nan
    cache.prefill_window(0, Q, K, V, out, [n, 450], window, sinks)
    assert torch.equal(out[1, 384:450], clean[1, 384:450])


def test_refusals():
    cache = mlkv.MLKVCache(1, 8, 64, [0], 2, 1, 100)
    K, Q, P = _randn(1, 2, 100, 64), _randn(1, 8, 64), _randn(1, 100, 8, 64)
    for window, sinks in ((-1, 0), (5, -1)):
        for call in (lambda: cache.decode_attention_window(0, Q, Q.clone(), [5], window, sinks),
                     lambda: cache.prefill_window(0, P, K, K, P.clone(), [5], window, sinks)):
            with pytest.raises(mlkv.MLKVError) as e:
                call()
            assert e.value.code == mlkv.MLKV_ERR_INVALID_ARG
    with pytest.raises(mlkv.MLKVError) as e:
        cache.decode_attention_window(0, Q, Q.clone(), [101], 5, 0)
    assert e.value.code == mlkv.MLKV_ERR_RANGE

"""Blocks' bounds, the selection of blocks and the decode over listed blocks, against 64-bit forms of their
definitions.  Codes, scales and block numbers have one right value each: they are compared exactly."""
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


def _scale(amax):
    """2^e for the least e in [-60, 40] with amax <= 127 * 2^e."""
    for e in range(-60, 41):
        if amax <= 127.0 * 2.0 ** e:
            return 2.0 ** e
    return math.inf


def _bounds(K, n):
    """Codes [blocks][2][d] and scales of K [n][d], a block after the other."""
    codes, scales = [], []
    for u in range(0, n, 64):
        x = K[u:min(n, u + 64)].double().cpu().numpy()
        amax = np.abs(x).max()
        s = _scale(amax) if np.isfinite(amax) else math.inf
        if math.isinf(s):
            codes.append(np.stack([np.full(x.shape[1], -127), np.full(x.shape[1], 127)]))
        else:
            codes.append(np.stack([np.floor(x.min(0) / s), np.ceil(x.max(0) / s)]))
        scales.append(s)
    return np.stack(codes), np.array(scales)


def _cache(d, h, g, b, cap, K, V=None, owners=(0, 0)):
    cache = mlkv.MLKVCache(len(owners), h, d, list(owners), g, b, cap)
    cache.load_prefix(max(owners), K, K if V is None else V, cap)
    return cache


def _empty(b, g, cap, d):
    n = (cap + 63) // 64
    return (torch.full((b, g, n, 2, d), 77, dtype=torch.int8, device="cuda"),
            torch.full((b, g, n), -1.0, device="cuda"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 3])
def test_bounds(d, g):
    torch.manual_seed(d + g)
    lens, cap = [1, 63, 64, 65, 200, 301], 301
    K = _randn(len(lens), g, cap, d)
    K[1] *= 1e-3
    K[2] = 127.0                     # a power of two of 127 exactly
    K[3, :, :, 5] = 127.5 * 2 ** 8   # just above one
    K[4, 0] = 0.0
    K[4, -1, 70, 3] = 3e13           # near the largest magnitude that has a scale
    K[5, :, :64] *= 1e-25            # below the least scale
    for i, n in enumerate(lens):
        K[i, :, n:] = math.nan       # not visible
    cache = _cache(d, 3 * g, g, len(lens), cap, K, owners=(0, 1))
    bounds, scales = _empty(len(lens), g, cap, d)
    cache.block_bounds(1, lens, bounds, scales)
    for i, n in enumerate(lens):
        m = (n + 63) // 64
        for j in range(g):
            codes, s = _bounds(K[i, j], n)
            assert np.array_equal(bounds[i, j, :m].cpu().numpy(), codes)
            assert np.array_equal(scales[i, j, :m].double().cpu().numpy(), s)
        assert (bounds[i, :, m:] == 77).all() and (scales[i, :, m:] == -1).all()
    cache.block_bounds(0, lens, *_empty(len(lens), g, cap, d))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 2e14, -3e38])
def test_bounds_of_what_has_none(bad):
    K = _randn(1, 2, 192, 128)
    K[0, 1, 100, 17] = bad
    cache = _cache(128, 2, 2, 1, 192, K)
    bounds, scales = _empty(1, 2, 192, 128)
    cache.block_bounds(0, [192], bounds, scales)
    assert torch.isinf(scales).nonzero().tolist() == [[0, 1, 1]]
    assert (bounds[0, 1, 1, 0] == -127).all() and (bounds[0, 1, 1, 1] == 127).all()


def test_bounds_token_by_token():
    torch.manual_seed(3)
    d, g, cap, lens = 64, 2, 200, [62, 1, 127]
    K = _randn(3, g, cap, d)
    cache = mlkv.MLKVCache(1, 4, d, [0], g, 3, cap)
    bounds, scales = _empty(3, g, cap, d)
    for i, n in enumerate(lens):
        K[i, :, n:] = 0
    cache.load_prefix(0, K, K, cap)
    cache.block_bounds(0, lens, bounds, scales)
    for step in range(70):
        new = _randn(3, g, d, sigma=1.0 + step)
        lens = [n + 1 for n in lens]
        for i, n in enumerate(lens):
            K[i, :, n - 1] = new[i]
        cache.append(0, new, new, lens)
        cache.block_bounds(0, lens, bounds, scales, first=[n - 1 for n in lens])
    whole = _empty(3, g, cap, d)
    cache.block_bounds(0, lens, *whole)
    assert torch.equal(bounds, whole[0]) and torch.equal(scales, whole[1])
    codes, s = _bounds(K[1, 1], lens[1])
    assert np.array_equal(bounds[1, 1, :2].cpu().numpy(), codes)
    # nothing new: nothing is touched
    cache.block_bounds(0, [128, 64, 192], bounds.fill_(5), scales, first=[128, 64, 192])
    assert (bounds == 5).all()


def _scores(Q, bounds, scales, G):
    """[g][blocks] of Q [h][d], codes [g][blocks][2][d]: whole numbers times powers of two, exact."""
    g = bounds.shape[0]
    out = np.full(bounds.shape[:2], -math.inf)
    for j in range(g):
        lo, hi = bounds[j, :, 0].astype(np.int64), bounds[j, :, 1].astype(np.int64)
        for i in range(j * G, (j + 1) * G):
            q = Q[i].double().cpu().numpy()
            amax = np.abs(q).max()
            f = _scale(amax) if np.isfinite(amax) else math.inf
            if math.isinf(f):
                continue
            q8 = np.rint(q / f).astype(np.int64)
            s = np.maximum(q8 * lo, q8 * hi).sum(-1) * f
            out[j] = np.maximum(out[j], s * np.where(np.isinf(scales[j]), 0.0, scales[j]))
        out[j][np.isinf(scales[j])] = math.inf
    return out


def _selected(score, n, n_select, n_first, n_last):
    count = (n + 63) // 64
    always = [u for u in range(count) if u < n_first or u >= count - n_last]
    others = [u for u in range(count) if u not in set(always)]
    others.sort(key=lambda u: -score[u])          # stable: the first of equal ones
    if count <= n_select:
        took = list(range(count))
    else:
        took = sorted(always + others[:n_select - len(always)])
    return took + [-1] * (n_select - len(took))


def _select(d, h, g, lens, cap, n_select, n_first, n_last, K, Q):
    b = len(lens)
    cache = _cache(d, h, g, b, cap, K)
    bounds, scales = _empty(b, g, cap, d)
    cache.block_bounds(0, lens, bounds, scales)
    blocks = torch.full((b, g, n_select), 99, dtype=torch.int32, device="cuda")
    cache.select_blocks(1, Q, bounds, scales, lens, blocks, n_first, n_last)
    cache.sync_status()
    bn, sn, got = bounds.cpu().numpy(), scales.double().cpu().numpy(), blocks.cpu().numpy()
    for i, n in enumerate(lens):
        m = (n + 63) // 64
        score = _scores(Q[i], bn[i, :, :m], sn[i, :, :m], h // g)
        for j in range(g):
            assert got[i, j].tolist() == _selected(score[j], n, n_select, n_first, n_last), (i, j)
    return cache, blocks


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(12, 1), (8, 2), (16, 1), (3, 3)])
@pytest.mark.parametrize("n_select,n_first,n_last", [(1, 0, 0), (1, 0, 1), (3, 1, 2), (8, 0, 0), (17, 2, 3),
                                                     (40, 1, 1)])
def test_select(d, h, g, n_select, n_first, n_last):
    torch.manual_seed(n_select)
    lens, cap = [1, 64, 65, 500, 1000, 2303, 2304], 2304
    K, Q = _randn(len(lens), g, cap, d), _randn(len(lens), h, d)
    _select(d, h, g, lens, cap, n_select, n_first, n_last, K, Q)


@pytest.mark.parametrize("d,h,g,lens,n_select", [
    (64, 12, 1, [131072], 64), (64, 12, 1, [70000, 131072], 500), (128, 32, 8, [40000, 9000, 20001], 64),
    (128, 4, 2, [64 * 515] * 3, 300)])
def test_select_long(d, h, g, lens, n_select):
    torch.manual_seed(1)
    K = _randn(len(lens), g, max(lens), d) + _randn(1, g, 1, d)
    _select(d, h, g, lens, max(lens), n_select, 1, 2, K, _randn(len(lens), h, d))


def test_select_ties_go_to_the_first():
    d, h, g, cap = 64, 4, 2, 64 * 600
    K = torch.ones(2, g, cap, d, dtype=torch.bfloat16, device="cuda")
    K[1, :, 64 * 300:] = 2.0                       # two values, 300 blocks each
    Q = torch.ones(2, h, d, dtype=torch.bfloat16, device="cuda")
    _, blocks = _select(d, h, g, [cap, cap], cap, 20, 1, 1, K, Q)
    assert blocks[0, 0].tolist() == list(range(19)) + [599]
    assert blocks[1, 1].tolist() == [0] + list(range(300, 318)) + [599]
    _select(d, h, g, [cap, cap], cap, 320, 0, 0, K, Q)
    _select(d, h, g, [cap, cap], cap, 20, 0, 0, K, -Q)


def test_select_extremes():
    torch.manual_seed(5)
    d, h, g, cap = 128, 8, 2, 64 * 40
    K, Q = _randn(3, g, cap, d), _randn(3, h, d)
    K[0, 0, 64 * 7 + 3, 9] = math.nan              # taken before all
    K[0, 1, 64 * 30, 0] = math.inf
    K[1] *= 1e30                                   # infinite everywhere
    K[2, :, ::2] = 0
    Q[0, 1] = math.nan                             # no say
    Q[0, 4:] = math.inf                            # no head of KV head 1 has
    Q[1, 0] = 0
    Q[2, 3] *= 1e-30
    _select(d, h, g, [cap] * 3, cap, 5, 1, 1, K, Q)
    _select(d, h, g, [cap] * 3, cap, 1, 0, 0, K, Q)


@pytest.mark.parametrize("n_select", [1, 5, 20])
@pytest.mark.parametrize("sigma", [1.0, -1.0])
def test_select_more_unknown_than_stay(n_select, sigma):
    """More blocks of which nothing is known than are selected."""
    torch.manual_seed(n_select)
    K, Q = _randn(2, 2, 6400, 64), _randn(2, 4, 64)
    K[:, :, ::160, 3] = math.nan
    K[..., 5] = 30.0
    Q[..., 5] = 30.0 * sigma   # all other scores of one sign
    _select(64, 4, 2, [6400, 6000], 6400, n_select, 0, 0, K, Q)


def _listed(cache, d, h, g, lens, K, V, Q, blocks):
    out = torch.full_like(Q, 9.0)
    cache.decode_attention_blocks(1, Q, out, lens, blocks)
    cache.sync_status()
    at = blocks.cpu().tolist()
    G = h // g
    for i, n in enumerate(lens):
        for j in range(g):
            pos = [u for x in at[i][j] if 0 <= x < (n + 63) // 64 for u in range(64 * x, min(n, 64 * x + 64))]
            q = Q[i, j * G:(j + 1) * G]
            if not pos:
                assert (out[i, j * G:(j + 1) * G] == 0).all()
                continue
            want, spread = attend(q.double()[:, None], K[i, j, pos].double()[None], V[i, j, pos].double()[None],
                                  torch.ones(1, len(pos), dtype=torch.bool, device="cuda"))
            assert_attention(out[i, j * G:(j + 1) * G], want[:, 0], spread[:, 0], ROUNDINGS)
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h,g", [(12, 1), (8, 2), (16, 1), (3, 3)])
@pytest.mark.parametrize("n", [1, 4, 5, 33, 70])
def test_listed_blocks(d, h, g, n):
    rng = np.random.default_rng(n)
    torch.manual_seed(n)
    lens, cap = [1, 64, 130, 1000, 2001, 500], 2005
    b = len(lens)
    K, V, Q = _randn(b, g, cap, d), _randn(b, g, cap, d), _randn(b, h, d)
    for i, m in enumerate(lens):
        K[i, :, m:], V[i, :, m:] = math.nan, math.inf
    cache = _cache(d, h, g, b, cap, K, V)
    blocks = torch.from_numpy(rng.integers(-3, 36, (b, g, n)).astype(np.int32)).cuda()   # some not there
    blocks[5] = -1                                                                       # none at all
    if n > 4:
        blocks[3, :, 1] = blocks[3, :, 4] = 2                                            # one twice
        blocks[4, :, 0], blocks[4, :, 2] = 31, 2 ** 31 - 1
        blocks[4, :, 3] = -2 ** 31
    _listed(cache, d, h, g, lens, K, V, Q, blocks)


@pytest.mark.parametrize("d,h,g,lens,n", [(64, 12, 1, [131072], 600), (128, 32, 8, [30000, 10, 9000, 20001], 200),
                                          (128, 32, 8, [6000] * 60, 64), (64, 12, 12, [3000] * 40, 30)])
def test_select_and_attend(d, h, g, lens, n):
    torch.manual_seed(2)
    b, cap = len(lens), max(lens)
    K, V, Q = _randn(b, g, cap, d) + _randn(1, g, 1, d), _randn(b, g, cap, d), _randn(b, h, d)
    cache = _cache(d, h, g, b, cap, K, V)
    bounds, scales = _empty(b, g, cap, d)
    cache.block_bounds(0, lens, bounds, scales)
    blocks = torch.zeros((b, g, n), dtype=torch.int32, device="cuda")
    cache.select_blocks(1, Q, bounds, scales, lens, blocks)
    out = _listed(cache, d, h, g, lens, K, V, Q, blocks)
    assert torch.equal(out, _listed(cache, d, h, g, lens, K, V, Q, blocks))


def test_all_blocks_are_the_plain_decode():
    torch.manual_seed(0)
    d, h, g, lens, cap = 128, 32, 8, [777, 64, 1000], 1000
    K, V, Q = _randn(3, g, cap, d), _randn(3, g, cap, d), _randn(3, h, d)
    cache = _cache(d, h, g, 3, cap, K, V)
    bounds, scales = _empty(3, g, cap, d)
    cache.block_bounds(0, lens, bounds, scales)
    blocks = torch.zeros((3, g, 20), dtype=torch.int32, device="cuda")
    cache.select_blocks(1, Q, bounds, scales, lens, blocks)
    _listed(cache, d, h, g, lens, K, V, Q, blocks)
    for i, n in enumerate(lens):
        assert blocks[i, 0].tolist() == [u if u < (n + 63) // 64 else -1 for u in range(20)]


def test_rejections():
    d, h, g, cap = 64, 4, 2, 200
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, 1, cap)
    Q, out = _randn(1, h, d), torch.zeros(1, h, d, dtype=torch.bfloat16, device="cuda")
    bounds, scales = _empty(1, g, cap, d)
    blocks = torch.zeros((1, g, 3), dtype=torch.int32, device="cuda")
    RANGE, BAD = mlkv.MLKV_ERR_RANGE, mlkv.MLKV_ERR_INVALID_ARG

    def refused(call, good, *changes):
        call(**good)
        for change, code in changes:
            with pytest.raises(mlkv.MLKVError) as e:
                call(**dict(good, **change))
            assert e.value.code == code, change

    refused(cache.block_bounds, dict(layer=0, seq_lens=[cap], bounds=bounds, scales=scales),
            (dict(layer=2), BAD), (dict(layer=-1), BAD), (dict(seq_lens=[0]), RANGE),
            (dict(seq_lens=[cap + 1]), RANGE), (dict(first=[-1]), RANGE), (dict(first=[cap + 1]), RANGE),
            (dict(bounds=bounds.float()), BAD), (dict(scales=scales.double()), BAD),
            (dict(bounds=bounds[:, :, :3]), BAD), (dict(scales=scales[:, :1]), BAD), (dict(seq_lens=[1, 1]), BAD))
    refused(cache.select_blocks, dict(layer=1, Q=Q, bounds=bounds, scales=scales, seq_lens=[cap], blocks=blocks),
            (dict(layer=2), BAD), (dict(Q=None), BAD), (dict(n_first=-1), BAD), (dict(n_last=-1), BAD),
            (dict(n_first=2, n_last=2), BAD), (dict(n_first=2 ** 31 - 1, n_last=1), BAD),
            (dict(blocks=blocks.long()), BAD), (dict(blocks=blocks[:, :, :0]), BAD), (dict(seq_lens=[0]), RANGE),
            (dict(blocks=blocks.expand(2, g, 3)), BAD))
    refused(cache.decode_attention_blocks, dict(layer=1, Q=Q, out=out, seq_lens=[cap], blocks=blocks),
            (dict(layer=2), BAD), (dict(Q=None), BAD), (dict(out=None), BAD), (dict(out=Q), BAD),
            (dict(blocks=blocks[:, :, :0]), BAD), (dict(blocks=blocks.float()), BAD),
            (dict(blocks=blocks[:, :1]), BAD), (dict(seq_lens=[201]), RANGE))
    many = torch.empty((1, g, 2 ** 29), dtype=torch.int32, device="cuda")
    with pytest.raises(mlkv.MLKVError) as e:
        cache.decode_attention_blocks(1, Q, out, [cap], many)
    assert e.value.code == mlkv.MLKV_ERR_UNSUPPORTED

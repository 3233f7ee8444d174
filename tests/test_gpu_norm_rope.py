"""mlkv_qk_norm_rope against the formula in 64 bits, its layouts and its refusals."""
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import HALF_ULP  # noqa: E402

pytestmark = pytest.mark.gpu
N_POS = 64


def _tables(rot, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.rand((N_POS, rot // 2), device="cuda", generator=g) * 6.3
    return a.cos(), a.sin()


def _want(x, gain, cos, sin, pos, eps, interleaved):
    """(y, magnitude of the two products behind every channel)."""
    y = x.double()
    y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt()
    if gain is not None:
        y = y * gain.double()
    mag = y.abs().clone()
    if cos is None:
        return y, mag
    rot = 2 * cos.shape[1]
    c, s = cos.double()[pos.long()][:, :, None], sin.double()[pos.long()][:, :, None]
    r = y[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    lo, hi, m = a * c - b * s, b * c + a * s, a.abs() + b.abs()
    if interleaved:
        out, mm = torch.stack([lo, hi], -1).flatten(-2), torch.stack([m, m], -1).flatten(-2)
    else:
        out, mm = torch.cat([lo, hi], -1), torch.cat([m, m], -1)
    return torch.cat([out, y[..., rot:]], -1), torch.cat([mm, mag[..., rot:]], -1)


def _check(got, want, mag):
    # half a unit of the bf16 output, and fp32 arithmetic: a sum of up to 128 squares, a reciprocal
    # root, three products
    bound = HALF_ULP * want.abs() * 1.004 + 32 * 2.0 ** -24 * mag + 1e-38
    assert float(((got.double() - want).abs() / bound).max()) <= 1.0


@pytest.mark.parametrize("b,s,h,g,d,rot", [
    (1, 1, 12, 4, 64, 16), (3, 7, 12, 1, 64, 64), (2, 33, 32, 8, 128, 128), (64, 1, 32, 8, 128, 48),
    (1, 5, 1, 1, 128, 0), (5, 129, 3, 3, 64, 32), (2, 1000, 16, 2, 128, 96),
])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("gains", [True, False])
def test_matches_formula(b, s, h, g, d, rot, interleaved, gains):
    torch.manual_seed(b * 1000 + s)
    fused = torch.randn((b, s, h + 2 * g, d), device="cuda").bfloat16()
    fused[0, 0, 0] = 0          # a head of zeros
    fused[-1, -1, -1] *= 1e4
    Q, K, V = fused[:, :, :h], fused[:, :, h:h + g], fused[:, :, h + g:]
    gq = torch.randn(d, device="cuda").bfloat16() if gains else None
    gk = torch.randn(d, device="cuda").bfloat16() if gains else None
    cos, sin = _tables(rot) if rot else (None, None)
    pos = torch.randint(0, N_POS, (b, s), device="cuda", dtype=torch.int32) if rot else None
    qo = torch.full((b, s, h, d), 7.0, device="cuda").bfloat16()
    ko = torch.full((b, g, s, d), 7.0, device="cuda").bfloat16()
    vo = torch.full((b, g, s, d), 7.0, device="cuda").bfloat16()
    mlkv.mlkv_qk_norm_rope(Q, K, V, gq, gk, cos, sin, pos, qo, ko, vo, eps=1e-5,
                           interleaved=interleaved)
    _check(qo, *_want(Q, gq, cos, sin, pos, 1e-5, interleaved))
    want, mag = _want(K, gk, cos, sin, pos, 1e-5, interleaved)
    _check(ko, want.transpose(1, 2), mag.transpose(1, 2))
    assert torch.equal(vo, V.transpose(1, 2))


def test_many_tokens_take_the_wide_form():
    """Enough heads for the form with several loads in flight, with heads that do not fill its last."""
    b, s, h, g, d = 2, 9000, 5, 1, 64
    torch.manual_seed(3)
    Q = torch.randn((b, s, h, d), device="cuda").bfloat16()
    K = torch.randn((b, s, g, d), device="cuda").bfloat16()
    cos, sin = _tables(16)
    pos = torch.randint(0, N_POS, (b, s), device="cuda", dtype=torch.int32)
    qo, ko = torch.empty_like(Q), torch.empty((b, g, s, d), device="cuda").bfloat16()
    mlkv.mlkv_qk_norm_rope(Q, K, None, None, None, cos, sin, pos, qo, ko, None)
    _check(qo, *_want(Q, None, cos, sin, pos, 1e-6, False))
    want, mag = _want(K, None, cos, sin, pos, 1e-6, False)
    _check(ko, want.transpose(1, 2), mag.transpose(1, 2))


@pytest.mark.parametrize("h,g", [(12, 4), (16, 2), (3, 1), (32, 12)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_many_tokens_of_every_grouping(h, g, interleaved):
    b, s, d = 3, 4001, 64
    torch.manual_seed(h)
    fused = torch.randn((b, s, h + 2 * g, d), device="cuda").bfloat16()
    Q, K, V = fused[:, :, :h], fused[:, :, h:h + g], fused[:, :, h + g:]
    gq, gk = torch.randn(d, device="cuda").bfloat16(), torch.randn(d, device="cuda").bfloat16()
    cos, sin = _tables(16)
    pos = torch.randint(0, N_POS, (b, s), device="cuda", dtype=torch.int32)
    qo = torch.full((b, s, h, d), 7.0, device="cuda").bfloat16()
    ko = torch.full((b, g, s, d), 7.0, device="cuda").bfloat16()
    vo = torch.full((b, g, s, d), 7.0, device="cuda").bfloat16()
    mlkv.mlkv_qk_norm_rope(Q, K, V, gq, gk, cos, sin, pos, qo, ko, vo, interleaved=interleaved)
    _check(qo, *_want(Q, gq, cos, sin, pos, 1e-6, interleaved))
    want, mag = _want(K, gk, cos, sin, pos, 1e-6, interleaved)
    _check(ko, want.transpose(1, 2), mag.transpose(1, 2))
    assert torch.equal(vo, V.transpose(1, 2))


def test_in_place_and_other_stream():
    b, h, g, d = 9, 12, 4, 64
    torch.manual_seed(5)
    Q = torch.randn((b, 1, h, d), device="cuda").bfloat16()
    K = torch.randn((b, 1, g, d), device="cuda").bfloat16()
    cos, sin = _tables(16)
    pos = torch.arange(b, device="cuda", dtype=torch.int32).view(b, 1)
    wq, mq = _want(Q, None, cos, sin, pos, 1e-6, False)
    wk, mk = _want(K, None, cos, sin, pos, 1e-6, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mlkv.mlkv_qk_norm_rope(Q, K, None, None, None, cos, sin, pos, Q, K.view(b, g, 1, d), None,
                           stream=side)
    torch.cuda.current_stream().wait_stream(side)
    _check(Q, wq, mq)
    _check(K, wk, mk)


def test_position_outside_the_table():
    """Only the token's rotated channels are NaN."""
    torch.manual_seed(7)
    Q = torch.randn((1, 4, 2, 64), device="cuda").bfloat16()
    K = torch.randn((1, 4, 1, 64), device="cuda").bfloat16()
    cos, sin = _tables(16)
    pos = torch.tensor([[0, -1, N_POS, N_POS - 1]], device="cuda", dtype=torch.int32)
    qo, ko = torch.empty_like(Q), torch.empty((1, 1, 4, 64), device="cuda").bfloat16()
    mlkv.mlkv_qk_norm_rope(Q, K, None, None, None, cos, sin, pos, qo, ko, None)
    for out in (qo, ko.transpose(1, 2)):
        assert torch.isnan(out[:, 1:3, :, :16]).all()
        assert torch.isfinite(out[:, 1:3, :, 16:]).all()
        assert torch.isfinite(out[:, [0, 3]]).all()


@pytest.mark.parametrize("s", [1, 700])
def test_queries_alone(s):
    """A layer that reads another's cache has no keys of its own."""
    torch.manual_seed(11)
    Q = torch.randn((3, s, 12, 64), device="cuda").bfloat16()
    gain = torch.randn(64, device="cuda").bfloat16()
    cos, sin = _tables(32)
    pos = torch.randint(0, N_POS, (3, s), device="cuda", dtype=torch.int32)
    out = torch.empty_like(Q)
    mlkv.mlkv_qk_norm_rope(Q, None, None, gain, None, cos, sin, pos, out, None, None)
    _check(out, *_want(Q, gain, cos, sin, pos, 1e-6, False))

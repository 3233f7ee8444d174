"""What the entry points around the decode step take, and refuse, by where tensors lie."""
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h,g,d", [(12, 4, 64), (32, 8, 128), (1, 1, 64)])
def test_norm_rope_of_one_fused_row_in_place(h, g, d):
    torch.manual_seed(h)
    rows = torch.randn((1, 1, h + 2 * g, d), device="cuda").bfloat16()
    Q, K, V = rows[:, :, :h], rows[:, :, h:h + g], rows[:, :, h + g:]
    want = rows.clone()
    heads = want[:, :, :h + g].double()
    heads = heads / (heads.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    mlkv.mlkv_qk_norm_rope(Q, K, V, None, None, None, None, None, Q, K.view(1, g, 1, d),
                           V.view(1, g, 1, d))
    assert torch.equal(V, want[:, :, h + g:])
    # half a unit of bf16, fp32 before it
    assert float(((rows[:, :, :h + g].double() - heads).abs() / heads.abs()).max()) <= 2.0 ** -8 * 1.01

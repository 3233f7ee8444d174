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


def test_q4_prompts_outside_the_device_are_refused():
    """The kernels read a prompt's keys and values where they lie: the host's memory may not be readable to
    them (mlkv_prefill copies such prompts, a 4-bit cache has no bf16 place to copy them to)."""
    b, g, h, s, d = 2, 2, 4, 70, 64
    cache = mlkv.MLKVQ4Cache(2, h, d, [0, 0], g, b, s)
    K = torch.randn((b, g, s, d), device="cuda").bfloat16()
    Q = torch.randn((b, s, h, d), device="cuda").bfloat16()
    out = torch.zeros_like(Q)
    for far in (K.cpu(), K.cpu().pin_memory()):
        for k, v in ((far, K), (K, far)):
            for layer in (0, 1):   # an owner and a reader
                with pytest.raises(mlkv.MLKVError) as e:
                    cache.prefill(layer, Q, k, v, out, [s, 5])
                assert e.value.code == mlkv.MLKV_ERR_INVALID_ARG
            with pytest.raises(mlkv.MLKVError) as e:
                cache.load_prefix(0, k, v, s)
            assert e.value.code == mlkv.MLKV_ERR_INVALID_ARG
    cache.sync_status()
    assert not out.any()
    cache.prefill(0, Q, K, K, out, [s, 5])
    cache.load_prefix(0, K, K, s)
    cache.sync_status()
    assert out[0].any(-1).all()


def test_q4_prompts_in_a_graph():
    """Where a prompt lies is asked while a graph records, too."""
    b, g, h, s, d = 2, 2, 4, 70, 64
    cache = mlkv.MLKVQ4Cache(1, h, d, [0], g, b, s)
    K = torch.randn((b, g, s, d), device="cuda").bfloat16()
    Q = torch.randn((b, s, h, d), device="cuda").bfloat16()
    out = torch.zeros_like(Q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.prefill(0, Q, K, K, out, [s, s])
    torch.cuda.current_stream().wait_stream(side)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.prefill(0, Q, K, K, out, [s, s])
        cache.load_prefix(0, K, K, s)
    out.zero_()
    graph.replay()
    cache.sync_status()
    assert torch.equal(out, want)

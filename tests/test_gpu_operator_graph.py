"""The operators around the decode step inside a CUDA graph: a replay gives what the calls give."""
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,h,g,lens,window,sinks", [
    (64, 12, 1, [30000], 0, 0),                      # the merge is a launch of its own
    (128, 32, 8, [700, 33, 1, 512], 300, 4),
])
def test_step(d, h, g, lens, window, sinks):
    torch.manual_seed(1)
    b, n = len(lens), max(lens)
    q4 = mlkv.MLKVQ4Cache(1, h, d, [0], g, b, n)
    bf = mlkv.MLKVCache(1, h, d, [0], g, b, n)
    K = torch.randn((b, g, n, d), device="cuda").bfloat16()
    q4.load_prefix(0, K, K, n)
    bf.load_prefix(0, K, K, n)
    rows = torch.randn((b, 1, h + 2 * g, d), device="cuda").bfloat16()
    cos, sin = torch.rand((2, n, d // 2), device="cuda")
    pos = torch.tensor([[x - 1] for x in lens], dtype=torch.int32, device="cuda")
    Q, out4, out16 = (torch.zeros((b, 1, h, d), device="cuda").bfloat16() for _ in range(3))
    k, v = (torch.zeros((b, g, 1, d), device="cuda").bfloat16() for _ in range(2))
    host = mlkv.as_seq_lens(lens)

    def step():
        mlkv.mlkv_qk_norm_rope(rows[:, :, :h], rows[:, :, h:h + g], rows[:, :, h + g:], None, None, cos,
                               sin, pos, Q, k, v)
        q4.append(0, k, v, host)
        q4.decode_attention(0, Q, out4, host, window, sinks)
        bf.append(0, k, v, host)
        bf.decode_attention_window(0, Q, out16, host, window, sinks)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 3):
        rows.copy_(torch.randn(rows.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
        step()
        want = [x.clone() for x in (Q, k, v, out4, out16)]
        for x in (Q, k, v, out4, out16):
            x.zero_()
        graph.replay()
        for x, y in zip((Q, k, v, out4, out16), want):
            assert torch.equal(x, y)
    q4.sync_status()
    bf.sync_status()

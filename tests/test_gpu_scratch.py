"""How much device memory the scratch of the calls for long caches takes, as the header states it."""
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402

pytestmark = pytest.mark.gpu
PAGE = 2 << 20   # what a device allocation is rounded up to


def _used():
    torch.cuda.synchronize()
    free, total = torch.cuda.mem_get_info()
    return total - free


def _weights(b, h, g, d, cap):
    cache = mlkv.MLKVCache(1, h, d, [0], g, b, cap)
    Q = torch.zeros(b, h, d, dtype=torch.bfloat16, device="cuda")
    out, w = torch.zeros_like(Q), torch.zeros(b, g, cap, device="cuda")

    def call(n):
        cache.decode_attention_weights(0, Q, out, [n] * b, None, w)
    return cache, call, lambda n: b * h * ((n + 63) // 64 * 64) * 4


def test_scores_of_growing_sequences():
    """Up to twice the scores' bytes, and as much again that was outgrown."""
    cache, call, need = _weights(32, 32, 8, 128, 6000)
    call(64)
    before = _used()
    most, sizes = 0, 0
    for n in range(64, 6000, 64):
        call(n)
        used = _used() - before
        if used > most:
            most, sizes = used, sizes + 1
        assert used <= 4 * need(n) + 16 * PAGE, n
    assert most >= need(5900) - PAGE   # (the scores of 6000 positions are 786 MB: they are what is measured)
    assert sizes <= 8                  # grown by doubling
    cache.sync_status()


def test_the_longest_first_makes_room_for_all():
    cache, call, need = _weights(16, 32, 8, 128, 5000)
    call(5000)
    before = _used()
    for n in (1, 64, 65, 4999, 5000):
        call(n)
    assert _used() <= before
    # (under capture scratch that would have to grow is refused; what a graph itself takes is not looked at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for n in (3000, 4999, 5000):
            call(n)
    graph.replay()
    cache.sync_status()


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")


def test_calls_without_scratch_allocate_nothing():
    b, h, g, d, cap, s = 8, 32, 8, 128, 3000, 2000
    Q, out, K = _bf16(b, h, d), _bf16(b, h, d), _bf16(b, g, s, d)
    P, pout = _bf16(b, s, h, d), _bf16(b, s, h, d)
    new, n = _bf16(b, g, d), (cap + 63) // 64
    bounds, scales = torch.zeros(b, g, n, 2, d, dtype=torch.int8, device="cuda"), torch.zeros(b, g, n, device="cuda")
    blocks = torch.zeros(b, g, 9, dtype=torch.int32, device="cuda")
    lens = [s + 1] * b

    def calls(cache):
        cache.load_prefix(0, K, K, s)
        cache.prefill(0, P, K, K, pout, [s] * b)
        cache.prefill_window(0, P, K, K, pout, [s] * b, 500, 4)
        cache.append(0, new, new, lens)
        cache.decode_attention(0, Q, out, lens)
        cache.append_decode_attention(0, new, new, Q, out, lens)
        cache.decode_attention_window(0, Q, out, lens, 500, 4)
        cache.block_bounds(0, lens, bounds, scales)
        cache.select_blocks(0, Q, bounds, scales, lens, blocks)
        cache.decode_attention_blocks(0, Q, out, lens, blocks)
        cache.sync_status()

    calls(mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap))   # (kernels are loaded when they first run)
    cache = mlkv.MLKVCache(2, h, d, [0, 0], g, b, cap)
    before = _used()
    calls(cache)
    assert _used() <= before

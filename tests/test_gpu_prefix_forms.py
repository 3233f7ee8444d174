"""The decode behind shared prefixes in each of its forms, against a 64-bit reference."""
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend  # noqa: E402

pytestmark = pytest.mark.gpu
ROUNDINGS = 2


def _randn(*shape):
    return torch.randn(shape, device="cuda").bfloat16()


def _decode(d, h, g, prefix_of, prefix_lens, lens, check):
    """One decode; the sequences in `check` against the reference."""
    torch.manual_seed(len(lens))
    b, n, cap, pcap = len(lens), len(prefix_lens), max(lens), max(prefix_lens)
    cache, prefix = mlkv.MLKVCache(1, h, d, [0], g, b, cap), mlkv.MLKVCache(1, h, d, [0], g, n, pcap)
    K, V, PK, PV = _randn(b, g, cap, d), _randn(b, g, cap, d), _randn(n, g, pcap, d), _randn(n, g, pcap, d)
    cache.load_prefix(0, K, V, cap)
    prefix.load_prefix(0, PK, PV, pcap)
    Q = _randn(b, h, d)
    out = torch.full_like(Q, 9.0)
    cache.decode_attention_prefix(0, prefix, prefix_of, prefix_lens, Q, out, lens)
    cache.sync_status()
    for i in check:
        x, m = prefix_of[i], lens[i]
        p = prefix_lens[x] if x >= 0 else 0
        k = torch.cat([PK[max(x, 0), :, :p], K[i, :, :m]], 1).double()
        v = torch.cat([PV[max(x, 0), :, :p], V[i, :, :m]], 1).double()
        want, spread = attend(Q[i].double()[:, None], k, v, torch.ones(1, p + m, dtype=torch.bool, device="cuda"))
        assert_attention(out[i], want[:, 0], spread[:, 0], ROUNDINGS)
    return cache


@pytest.mark.parametrize("d,h,g,n,per,p", [
    (128, 32, 8, 80, 12, 1024),     # more units than four rounds on the SMs, each a whole prefix
    (64, 12, 12, 100, 10, 1500),
    (64, 1024, 64, 64, 16, 1024),   # 4096 of them: two launches
])
def test_decode_of_many_prefixes_and_sequences(d, h, g, n, per, p):
    b = n * per
    _decode(d, h, g, [i // per for i in range(b)], [p - x % 7 for x in range(n)], [1 + i % 70 for i in range(b)],
            [0, 1, b // 2, b - per - 1, b - 1])

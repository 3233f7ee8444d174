"""The calls behind shared prefixes in each of their forms, which are asserted, against a 64-bit reference."""
import pytest

torch = pytest.importorskip("torch")
import paper_2406_09297_gb300 as mlkv  # noqa: E402
from tests.operator_refs import assert_attention, attend  # noqa: E402

pytestmark = pytest.mark.gpu
ROUNDINGS = 2
JOINED, GROUPS, KERNEL, BESIDE, PROMPT = 1, 2, 3, 4, 5   # option "last_prefix_form"


def _took(cache):
    return cache.get_option("last_prefix_form"), cache.get_option("last_prefix_launches")


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


@pytest.mark.parametrize("d,h,g,n,per,p,launches", [
    (128, 32, 8, 80, 12, 1024, 2),     # more units than four rounds on the SMs, each a whole prefix
    (64, 12, 12, 100, 10, 1500, 2),
    (64, 1024, 64, 64, 16, 1024, 3),   # 4096 of them: two launches, and the suffixes start beside the second
    (64, 1024, 64, 64, 16, 256, 3),
])
def test_decode_of_many_prefixes_and_sequences(d, h, g, n, per, p, launches):
    b = n * per
    cache = _decode(d, h, g, [i // per for i in range(b)], [p - x % 7 for x in range(n)],
                    [1 + i % 70 for i in range(b)], [0, 1, b // 2, b - per - 1, b - 1])
    form, took = _took(cache)
    assert form in (KERNEL, BESIDE) and took == launches + (form == BESIDE)


@pytest.mark.parametrize("d,h,g,n,b,p,own,form", [
    (64, 12, 4, 1, 3, 130, 60, JOINED), (128, 32, 8, 1, 2, 5000, 70, JOINED), (64, 12, 4, 3, 21, 2500, 2500, JOINED),
    (128, 32, 8, 1, 4, 16000, 300, GROUPS), (64, 12, 12, 1, 16, 4000, 100, GROUPS),
    (64, 1024, 64, 64, 1024, 256, 5, KERNEL),
    (128, 32, 8, 1, 64, 8192, 256, BESIDE), (64, 12, 1, 1, 64, 32768, 1000, BESIDE),
    (128, 32, 8, 1, 100, 3000, 100, BESIDE),
])
@pytest.mark.parametrize("order", ["neighbours", "scattered"])
def test_decode_form(d, h, g, n, b, p, own, form, order):
    """A shape of each form, the sequences of a prefix side by side or not."""
    where = [i * n // b for i in range(b)] if order == "neighbours" else [(i * 5) % n for i in range(b)]
    if order == "scattered":
        where[b // 3] = -1
    cache = _decode(d, h, g, where, [p] * n, [own] * b, [0, b // 3, b // 2, b - 1])
    took, launches = _took(cache)
    assert took == form
    assert launches in {JOINED: (1, 2), GROUPS: (2,), KERNEL: (3,), BESIDE: (3,)}[form]


@pytest.mark.parametrize("d,h,g,b,s,p,form,launches", [
    (64, 12, 4, 3, 300, 40, PROMPT, 1), (128, 32, 8, 9, 100, 5000, PROMPT, 1),
    (64, 12, 1, 90, 600, 200, PROMPT, 2),           # 5400 units
    (64, 12, 4, 66, 1, 2000, KERNEL, 3), (128, 32, 8, 4, 12, 3582, KERNEL, 3),
    (64, 12, 4, 9, 100, 5000, BESIDE, 3), (128, 32, 8, 2, 1, 3000, JOINED, 2),
])
def test_prefill_form(d, h, g, b, s, p, form, launches):
    torch.manual_seed(b)
    cache, prefix = mlkv.MLKVCache(1, h, d, [0], g, b, s), mlkv.MLKVCache(1, h, d, [0], g, 1, p)
    K, V, PK, PV = _randn(b, g, s, d), _randn(b, g, s, d), _randn(1, g, p, d), _randn(1, g, p, d)
    prefix.load_prefix(0, PK, PV, p)
    Q = _randn(b, s, h, d)
    out = torch.full_like(Q, 9.0)
    cache.prefill_prefix(0, prefix, [0] * b, [p], Q, K, V, out, [s] * b)
    cache.sync_status()
    assert _took(cache) == (form, launches)
    t, u = torch.arange(s, device="cuda")[:, None], torch.arange(p + s, device="cuda")[None]
    for i in (0, b // 2, b - 1):
        k, v = torch.cat([PK[0], K[i]], 1).double(), torch.cat([PV[0], V[i]], 1).double()
        want, spread = attend(Q[i].transpose(0, 1).double(), k, v, u <= p + t)
        assert_attention(out[i].transpose(0, 1), want, spread, ROUNDINGS)

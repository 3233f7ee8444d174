"""The long-context example: its logits against a plain 64-bit decoder over the same weights."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
from tests.operator_refs import held  # noqa: E402

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "long_context.py")
    spec = importlib.util.spec_from_file_location("long_context", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _norm(x):
    return x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()


def _rope(x, cos, sin):
    half = cos.shape[1]
    a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    cos, sin = cos[:, None], sin[:, None]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _plain(m, tokens, prompt, window, sinks):
    """Logits after every token of one sequence [n]: tokens from `prompt` on read 4-bit keys and values."""
    n = tokens.shape[0]
    t, u = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    visible = (u <= t) & ((u < sinks) | (u > t - window))
    coded = t[:, 0] >= prompt
    cos, sin = m.cos.double()[:n], m.sin.double()[:n]
    x = m.embed[tokens].double()
    for layer in range(m.l):
        rows = (_norm(x) @ m.w_in[layer].double().T).view(n, -1, m.d)
        q = _rope(_norm(rows[:, :m.h]) * m.q_gain[layer].double(), cos, sin)
        if m.owner[layer] == layer:
            k = _rope(_norm(rows[:, m.h:m.h + m.g]) * m.k_gain[layer].double(), cos, sin)
            v = rows[:, m.h + m.g:]
            k4, v4 = held(k.bfloat16()), held(v.bfloat16())
        out = []
        for kk, vv in ((k, v), (k4, v4)):
            heads = m.h // m.g
            s = torch.einsum("thd,uhd->htu", q, kk.repeat_interleave(heads, 1)) / math.sqrt(m.d)
            p = s.masked_fill(~visible, -math.inf).softmax(-1)
            out.append(torch.einsum("htu,uhd->thd", p, vv.repeat_interleave(heads, 1)))
        x = x + torch.where(coded[:, None, None], out[1], out[0]).flatten(1) @ m.w_out[layer].double().T
        up = torch.nn.functional.gelu(_norm(x) @ m.w_up[layer].double().T)
        x = x + up @ m.w_down[layer].double().T
    return _norm(x) @ m.embed.double().T


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("size", [
    dict(n_layers=4, hidden=192, n_q_heads=6, head_dim=64, n_owners=2, kv_heads=2, rot_dim=16),
    dict(n_layers=3, hidden=256, n_q_heads=4, head_dim=128, n_owners=1, kv_heads=1, rot_dim=128),
])
def test_logits(size):
    """bf16 steps (relative 2^-9 each on average, some ten a layer, four layers at most: 1e-2) and codes
    that such a step moves to the next number (about one in forty, a seventh of the group's largest value:
    a relative 5e-2 of a key or value, which the mean over the visible positions lessens): 5e-2 of the
    logits' norm.  Without the window they differ by more than that."""
    window, sinks, lens, new = 40, 3, [133, 70, 1], 12
    m = _example().Decoder(vocab=500, window=window, sinks=sinks, batch=3, max_seq=160, seed=3, **size)
    torch.manual_seed(5)
    tokens = torch.randint(0, 500, (3, 160), device="cuda")
    want = [_plain(m, tokens[i, :lens[i] + new], lens[i], window, sinks) for i in range(3)]
    free = [_plain(m, tokens[i, :lens[i] + new], lens[i], 1000, 0) for i in range(3)]
    got = m.prefill(tokens[:, :max(lens)], lens)
    for i in range(3):
        assert _off(got[i], want[i][lens[i] - 1]) < 5e-2
    for k in range(new):
        at = [n + k for n in lens]
        got = m.step(torch.stack([tokens[i, at[i]] for i in range(3)]), [n + 1 for n in at])
        for i in range(3):
            assert _off(got[i], want[i][at[i]]) < 5e-2
        assert _off(got[0], free[0][at[0]]) > 5e-2
    m.cache.sync_status()

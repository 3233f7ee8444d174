"""Sizes and layouts at which the entry points around the decode step must refuse, or must not."""
import pytest

import paper_2406_09297_gb300 as mlkv


@pytest.mark.parametrize("g,d,max_seq,owners", [
    (16384, 128, 1 << 30, 64),        # 0 modulo 2^64
    (16384, 64, 1 << 30, 64),
    (16384, 128, (1 << 30) - 63, 97),
    (8, 128, 1 << 30, 1 << 18),
])
def test_q4_create_refuses_bytes_past_64_bits(g, d, max_seq, owners):
    """A product that wraps would be allocated as what is left of it."""
    assert 1024 * g * owners * ((max_seq + 63) // 64 * 4 * 18 * d) >= 1 << 63
    with pytest.raises(mlkv.MLKVError) as e:
        mlkv.mlkv_q4_create(owners, g, d, list(range(owners)), g, 1024, max_seq)
    assert e.value.code == mlkv.MLKV_ERR_OOM


@pytest.mark.parametrize("g,d,max_seq,owners", [
    (16384, 128, 1 << 30, 32),          # 0 modulo 2^64
    (16384, 64, (1 << 31) - 1, 63),
    (8, 128, (1 << 31) - 1, 1100),
])
def test_cache_create_refuses_bytes_past_64_bits(g, d, max_seq, owners):
    assert 2 * 1024 * g * owners * max_seq * d * 2 >= 1 << 63
    with pytest.raises(mlkv.MLKVError) as e:
        mlkv.mlkv_cache_create(owners, g, d, list(range(owners)), g, 1024, max_seq)
    assert e.value.code == mlkv.MLKV_ERR_OOM


def _norm_rope_args(torch):
    b, s, h, g, d = 2, 3, 4, 2, 64
    bf16 = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)
    return dict(Q=bf16(b, s, h, d), K=bf16(b, s, g, d), V=bf16(b, s, g, d), q_gain=bf16(d), k_gain=bf16(d),
                cos=torch.zeros(8, 16), sin=torch.zeros(8, 16),
                positions=torch.zeros(b, s, dtype=torch.int32), Q_out=bf16(b, s, h, d),
                K_out=bf16(b, g, s, d), V_out=bf16(b, g, s, d))


@pytest.mark.parametrize("name,dtype", [
    *[(name, dtype) for name in ("Q", "K", "V", "q_gain", "k_gain", "Q_out", "K_out", "V_out")
      for dtype in ("float32", "float16", "int8")],
    ("cos", "int32"), ("sin", "int32"), ("positions", "float32"),
])
def test_norm_rope_binding_refuses_other_types(monkeypatch, name, dtype):
    """Their bytes would be read as bf16, or an output of one byte an element written past its end."""
    torch = pytest.importorskip("torch")
    calls = []

    class NoLibrary:   # nothing reaches the GPU
        def mlkv_qk_norm_rope_struct(self, args):
            calls.append(args)
            return 0

    monkeypatch.setattr(mlkv.mlkv, "lib", NoLibrary())
    args = _norm_rope_args(torch)
    mlkv.mlkv_qk_norm_rope(**args, stream=0)
    assert len(calls) == 1
    args[name] = args[name].to(getattr(torch, dtype))
    with pytest.raises(mlkv.MLKVError) as e:
        mlkv.mlkv_qk_norm_rope(**args, stream=0)
    assert e.value.code == mlkv.MLKV_ERR_INVALID_ARG and len(calls) == 1


def test_norm_rope_takes_one_token_in_place():
    """One token's heads keep their places whatever the stride to the next.  (Without a GPU the launch is
    what fails.)"""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the addresses are the host's")
    h, g, d = 4, 2, 64
    rows = torch.zeros((1, 1, h + 2 * g, d), dtype=torch.bfloat16)
    Q, K, V = rows[:, :, :h], rows[:, :, h:h + g], rows[:, :, h + g:]
    with pytest.raises(mlkv.MLKVError) as e:
        mlkv.mlkv_qk_norm_rope(Q, K, V, None, None, None, None, None, Q, K.view(1, g, 1, d),
                               V.view(1, g, 1, d), stream=0)
    assert e.value.code == mlkv.MLKV_ERR_CUDA

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

"""What the entry points for long caches refuse without a GPU: null handles, and tensors that the binding checks."""
import numpy as np
import pytest

import paper_2406_09297_gb300 as mlkv

torch = pytest.importorskip("torch")
BAD = mlkv.MLKV_ERR_INVALID_ARG


def test_null_handles():
    one = np.ones(4, dtype=np.int32).ctypes.data
    lib = mlkv.lib
    for rc in (lib.mlkv_decode_attention_prefix(None, 0, None, one, one, None, None, one, None),
               lib.mlkv_prefill_prefix(None, 0, None, one, one, None, None, None, None, one, 1, None),
               lib.mlkv_block_bounds(None, 0, None, one, None, None, None),
               lib.mlkv_select_blocks(None, 0, None, None, None, one, 1, 0, 0, None, None),
               lib.mlkv_decode_attention_blocks(None, 0, None, None, one, None, 1, None),
               lib.mlkv_decode_attention_weights(None, 0, None, None, one, None, None, None),
               lib.mlkv_evict(None, None, 0, None, None, one, one, 0, None, 1, None)):
        assert rc == BAD
        assert mlkv.mlkv_last_error()


def _cache(b=2, g=3, d=64, max_seq=130):
    """A handle that no call reaches: everything below is refused before."""
    c = mlkv.MLKVCache.__new__(mlkv.MLKVCache)
    c.l, c.h, c.d, c.owner, c.g, c.b, c.max_seq, c.handle = 2, 2 * g, d, [0, 0], g, b, max_seq, None
    return c


def _refused(call, good, changes):
    for change in changes:
        with pytest.raises(mlkv.MLKVError) as e:
            call(**dict(good, **change), stream=0)
        assert e.value.code == BAD, change


def test_binding_rejects_tensors():
    c = _cache()
    Q, out = torch.zeros(2, 6, 64).bfloat16(), torch.zeros(2, 6, 64).bfloat16()
    bounds, scales = torch.zeros(2, 3, 3, 2, 64, dtype=torch.int8), torch.zeros(2, 3, 3)
    _refused(c.block_bounds, dict(layer=0, seq_lens=[1, 1], bounds=bounds, scales=scales), [
        dict(bounds=bounds.float()), dict(bounds=bounds[:, :, :2]), dict(bounds=bounds.transpose(1, 2)),
        dict(scales=scales.bfloat16()), dict(scales=scales[:1]), dict(seq_lens=[1]), dict(first=[0, 0, 0]),
        dict(scales=torch.zeros(2, 3, 6)[:, :, ::2])])
    blocks = torch.zeros(2, 3, 5, dtype=torch.int32)
    _refused(c.select_blocks, dict(layer=0, Q=Q, bounds=bounds, scales=scales, seq_lens=[1, 1], blocks=blocks), [
        dict(blocks=blocks.long()), dict(blocks=blocks[:, :2]), dict(blocks=blocks[:, :, ::2]),
        dict(bounds=bounds.to(torch.uint8)), dict(scales=scales[:, :, :2]), dict(seq_lens=1)])
    _refused(c.decode_attention_blocks, dict(layer=0, Q=Q, out=out, seq_lens=[1, 1], blocks=blocks), [
        dict(blocks=blocks.short()), dict(blocks=blocks[:1]), dict(seq_lens=[[1, 1]])])
    w = torch.zeros(2, 3, 130)
    _refused(c.decode_attention_weights,
             dict(layer=0, Q=Q, out=out, seq_lens=[1, 1], weights_in=None, weights_out=w), [
                 dict(weights_out=w.double()), dict(weights_out=w[:, :, :129]), dict(weights_in=w.half()),
                 dict(weights_in=w[:, :1]), dict(weights_out=torch.zeros(3, 2, 130).transpose(0, 1))])
    kept = torch.zeros(2, 3, 9, dtype=torch.int32)
    _refused(c.evict, dict(layer=0, weights_in=w, weights_out=w, seq_lens=[9, 9], keep=[9, 9], recent=0, kept=kept), [
        dict(kept=kept.float()), dict(kept=kept[:1]), dict(weights_in=w.double()), dict(weights_out=w[:, :2]),
        dict(keep=[9]), dict(to=_cache(max_seq=20)), dict(seq_lens=[9, 9, 9])])
    _refused(c.decode_attention_prefix, dict(layer=0, prefix=_cache(b=1), prefix_of=[0, 0], prefix_lens=[1], Q=Q,
                                             out=out, seq_lens=[1, 1]), [
        dict(prefix_of=[0]), dict(prefix_lens=[1, 1]), dict(seq_lens=[1]), dict(prefix_of=[[0, 0]])])


def test_lists_are_read_as_whole_numbers():
    with pytest.raises((mlkv.MLKVError, TypeError, ValueError)):
        _cache().decode_attention_blocks(0, None, None, ["a", "b"], torch.zeros(2, 3, 5, dtype=torch.int32), stream=0)

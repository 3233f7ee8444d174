"""What the entry points around the decode step refuse before they touch a GPU."""
import ctypes
import os
import struct

import numpy as np
import pytest

import paper_2406_09297_gb300 as mlkv

NULL = None
BAD, UNSUPPORTED, MAP = mlkv.MLKV_ERR_INVALID_ARG, mlkv.MLKV_ERR_UNSUPPORTED, mlkv.MLKV_ERR_MAP


def _lens(*n):
    return np.asarray(n, dtype=np.int32)


@pytest.mark.parametrize("args,code", [
    ((3, 4, 64, [0, 2, 2], 2, 1, 16), MAP),           # owner after its layer
    ((3, 4, 64, [0, 0, 1], 2, 1, 16), MAP),           # owner not self-owned
    ((3, 6, 64, [0, 0, 0], 4, 1, 16), MAP),           # g does not divide h
    ((3, 4, 64, [0, 0, 0], 8, 1, 16), MAP),           # g > h
    ((3, 4, 96, [0, 0, 0], 2, 1, 16), UNSUPPORTED),   # head_dim
    ((2, 64, 64, [0, 0], 2, 1, 16), UNSUPPORTED),     # 32 query heads a KV head
    ((2, 4, 64, [0, 0], 2, 2000, 16), UNSUPPORTED),   # batch
    ((1, 4, 64, [0], 2, 1, (1 << 30) + 1), UNSUPPORTED),
    ((0, 4, 64, [], 2, 1, 16), BAD),
    ((2, 4, 64, [0, 0], 2, 0, 16), BAD),
    ((2, 4, 64, [0, 0], 2, 1, 0), BAD),
])
def test_q4_create_rejects(args, code):
    with pytest.raises(mlkv.MLKVError) as e:
        mlkv.mlkv_q4_create(*args)
    assert e.value.code == code and mlkv.mlkv_last_error()


def test_q4_create_without_a_place_for_the_handle():
    owner = (ctypes.c_int * 1)(0)
    assert mlkv.lib.mlkv_q4_create(NULL, 1, 4, 64, owner, 2, 1, 16) == BAD


def test_null_handles():
    lens = _lens(1).ctypes.data
    lib = mlkv.lib
    for rc in (lib.mlkv_q4_bytes(NULL), lib.mlkv_q4_append(NULL, 0, NULL, NULL, lens, NULL),
               lib.mlkv_q4_load_prefix(NULL, 0, NULL, NULL, 0, NULL),
               lib.mlkv_q4_read(NULL, 0, NULL, NULL, 0, 0, NULL),
               lib.mlkv_q4_decode_attention(NULL, 0, NULL, NULL, lens, 0, 0, NULL),
               lib.mlkv_q4_prefill(NULL, 0, NULL, NULL, NULL, NULL, lens, 1, 0, 0, NULL),
               lib.mlkv_q4_sync_status(NULL),
               lib.mlkv_decode_attention_window(NULL, 0, NULL, NULL, lens, 1, 0, NULL),
               lib.mlkv_prefill_window(NULL, 0, NULL, NULL, NULL, NULL, lens, 1, 1, 0, NULL)):
        assert rc == BAD
    assert lib.mlkv_q4_destroy(NULL) == mlkv.MLKV_OK


# Addresses that nothing ever reads: every call below is refused from its arguments alone.
PLACE = {name: 0x10000000 * (i + 1) for i, name in enumerate(
    ["Q", "K", "V", "q_gain", "k_gain", "cos", "sin", "positions", "Q_out", "K_out", "V_out"])}
# a fused projection of 2 * 3 tokens: 4 query heads, 2 KV heads of 64
GOOD = dict(PLACE, q_stride=512, k_stride=512, v_stride=512, n_pos=100, rot=32, interleaved=0,
            eps=1e-6, batch=2, s=3, h=4, g=2, d=64)
ORDER = ["Q", "K", "V", "q_stride", "k_stride", "v_stride", "q_gain", "k_gain", "cos", "sin", "n_pos",
         "rot", "interleaved", "positions", "eps", "batch", "s", "h", "g", "d", "Q_out", "K_out", "V_out"]


@pytest.mark.parametrize("change,code", [
    (dict(Q=NULL), BAD), (dict(Q_out=NULL), BAD),
    (dict(K=NULL), BAD), (dict(K_out=NULL), BAD), (dict(V=NULL), BAD), (dict(V_out=NULL), BAD),
    (dict(K=NULL, K_out=NULL), BAD),                                   # values without keys
    (dict(cos=NULL), BAD), (dict(sin=NULL), BAD), (dict(positions=NULL), BAD), (dict(n_pos=0), BAD),
    (dict(batch=0), BAD), (dict(s=0), BAD), (dict(h=0), BAD), (dict(g=0), BAD), (dict(s=-1), BAD),
    (dict(d=96), UNSUPPORTED), (dict(rot=24), UNSUPPORTED), (dict(rot=-16), BAD), (dict(rot=80), BAD),
    (dict(eps=-1e-6), BAD), (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD),
    (dict(q_stride=-8), BAD), (dict(k_stride=12), BAD), (dict(v_stride=4), BAD),
    (dict(q_stride=1 << 62), UNSUPPORTED), (dict(k_stride=1 << 58), UNSUPPORTED),
    (dict(batch=1 << 20, s=1 << 20), UNSUPPORTED), (dict(h=1 << 21), UNSUPPORTED),
    (dict(h=(1 << 31) - 1, g=(1 << 31) - 1), UNSUPPORTED),
    (dict(positions=PLACE["positions"] + 2), BAD),
    *[({name: PLACE[name] + 8}, BAD) for name in PLACE if name != "positions"],
    (dict(Q_out=PLACE["Q"]), BAD),                                     # rows of another stride
    (dict(K_out=PLACE["K"], k_stride=128), BAD),                       # heads that change places
    (dict(V_out=PLACE["Q"] + 1024), BAD),
    (dict(K_out=PLACE["Q_out"] + 2 * 6 * 4 * 64 - 16), BAD),           # the last row's end
    (dict(V_out=PLACE["K_out"]), BAD),
])
def test_qk_norm_rope_rejects(change, code):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    a = dict(GOOD, **change)
    assert mlkv.lib.mlkv_qk_norm_rope(*[a[k] for k in ORDER], NULL) == code
    assert mlkv.mlkv_last_error()


def test_qk_norm_rope_struct_rejects_the_same():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    assert mlkv.lib.mlkv_qk_norm_rope_struct(NULL) == BAD
    order = ["Q", "K", "V", "q_stride", "k_stride", "v_stride", "q_gain", "k_gain", "cos", "sin",
             "positions", "Q_out", "K_out", "V_out", "stream", "n_pos", "rot", "interleaved", "batch", "s",
             "h", "g", "d", "eps"]
    # every field at a value that only its own check refuses
    for change, code in ((dict(Q=0), BAD), (dict(Q_out=0), BAD), (dict(K=0), BAD), (dict(V_out=0), BAD),
                         (dict(K_out=0), BAD), (dict(V=0), BAD), (dict(q_stride=-8), BAD),
                         (dict(k_stride=4), BAD), (dict(v_stride=12), BAD), (dict(cos=0), BAD),
                         (dict(sin=0), BAD), (dict(positions=0), BAD), (dict(q_gain=8), BAD),
                         (dict(k_gain=8), BAD), (dict(n_pos=0), BAD), (dict(rot=24), UNSUPPORTED),
                         (dict(batch=0), BAD), (dict(s=0), BAD), (dict(h=0), BAD), (dict(g=0), BAD),
                         (dict(d=96), UNSUPPORTED), (dict(eps=-1.0), BAD)):
        a = dict(dict(GOOD, stream=0), **change)
        args = struct.pack("@3P3q9P8if", *[a[k] for k in order])
        assert mlkv.lib.mlkv_qk_norm_rope_struct(args) == code, change


def test_qk_norm_rope_binding_rejects_layouts():
    import torch

    def call(**change):
        b, s, h, g, d = 2, 3, 4, 2, 64
        a = dict(Q=torch.zeros(b, s, h, d).bfloat16(), K=torch.zeros(b, s, g, d).bfloat16(), V=None,
                 q_gain=None, k_gain=None, cos=torch.zeros(8, 16), sin=torch.zeros(8, 16),
                 positions=torch.zeros(b, s, dtype=torch.int32),
                 Q_out=torch.zeros(b, s, h, d).bfloat16(), K_out=torch.zeros(b, g, s, d).bfloat16(),
                 V_out=None)
        a.update(change)
        with pytest.raises(mlkv.MLKVError) as e:
            mlkv.mlkv_qk_norm_rope(**a, stream=0)
        assert e.value.code == BAD

    call(Q=torch.zeros(2, 4, 3, 64).bfloat16().transpose(1, 2))   # heads apart
    call(K=torch.zeros(2, 5, 2, 64).bfloat16()[:, :3])            # sequences further apart than tokens
    call(K=torch.zeros(2, 2, 2, 64).bfloat16())                   # fewer tokens
    call(positions=torch.zeros(2, 3, dtype=torch.int64))
    call(cos=torch.zeros(8, 16).double())
    call(sin=None)
    call(positions=torch.zeros(5, dtype=torch.int32))
    call(sin=torch.zeros(8, 15))
    call(q_gain=torch.ones(32).bfloat16())
    call(K=None)                                                  # K_out is left without its input
    call(K=None, K_out=None, V=torch.zeros(2, 3, 2, 64).bfloat16())
    call(K=None, K_out=None, V_out=torch.zeros(2, 2, 3, 64).bfloat16())
    call(Q_out=torch.zeros(2, 4, 3, 64).bfloat16().transpose(1, 2))
    call(K_out=torch.zeros(2, 2, 2, 64).bfloat16())


def test_header_and_binding_name_the_same_calls():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "mlkv.h")) as f:
        header = f.read()
    for name in mlkv.EXPORTED:
        assert f"{name}(" in header, name

"""The Python binding of the calls for long caches, with the library's functions replaced: what is refused never reaches
them, and what reaches them is what was given."""
import ctypes
import importlib

import numpy as np
import pytest

import paper_2406_09297_gb300 as package

torch = pytest.importorskip("torch")
binding = importlib.import_module("paper_2406_09297_gb300.mlkv")
BAD = package.MLKV_ERR_INVALID_ARG


class Library:
    """Stands for the library: keeps every call's arguments, host arrays as lists of whole numbers."""

    # places of the host arrays among a function's arguments, and what gives each one's length
    ARRAYS = {
        "mlkv_decode_attention_prefix": {3: "b", 4: "prefix_b", 7: "b"},
        "mlkv_prefill_prefix": {3: "b", 4: "prefix_b", 9: "b"},
        "mlkv_block_bounds": {2: "b", 3: "b"},
        "mlkv_select_blocks": {5: "b"},
        "mlkv_decode_attention_blocks": {4: "b"},
        "mlkv_decode_attention_weights": {4: "b"},
        "mlkv_evict": {5: "b", 6: "b"},
    }

    def __init__(self, b, prefix_b):
        self.n, self.calls = {"b": b, "prefix_b": prefix_b}, []

    def __getattr__(self, name):
        arrays = Library.ARRAYS[name]

        def call(*args):
            seen = list(args)
            for i, n in arrays.items():
                if args[i] is not None:
                    seen[i] = list((ctypes.c_int32 * self.n[n]).from_address(args[i]))
            self.calls.append((name, seen))
            return 0
        return call


def _cache(handle, b=2, g=3, d=64, max_seq=130):
    c = package.MLKVCache.__new__(package.MLKVCache)
    c.l, c.h, c.d, c.owner, c.g, c.b, c.max_seq, c.handle = 2, 2 * g, d, [0, 0], g, b, max_seq, handle
    c.close = lambda: None
    return c


@pytest.fixture
def lib(monkeypatch):
    stub = Library(2, 1)
    monkeypatch.setattr(binding, "lib", stub)
    return stub


CACHE, PREFIX = _cache(1001), _cache(1002, b=1)
Q, OUT = torch.zeros(2, 6, 64).bfloat16(), torch.zeros(2, 6, 64).bfloat16()
BOUNDS, SCALES = torch.zeros(2, 3, 3, 2, 64, dtype=torch.int8), torch.zeros(2, 3, 3)
BLOCKS, KEPT = torch.zeros(2, 3, 5, dtype=torch.int32), torch.zeros(2, 3, 9, dtype=torch.int32)
W, W2 = torch.zeros(2, 3, 130), torch.zeros(2, 3, 130)
PQ, POUT, K, V = (torch.zeros(2, 10, 6, 64).bfloat16(), torch.zeros(2, 10, 6, 64).bfloat16(),
                  torch.zeros(2, 3, 10, 64).bfloat16(), torch.zeros(2, 3, 10, 64).bfloat16())


def _at(t):
    return t.data_ptr()


# call, its arguments, what the library gets
GOOD = {
    "block_bounds": (dict(layer=0, seq_lens=[7, 130], bounds=BOUNDS, scales=SCALES, first=[1, 2]),
                     [1001, 0, [1, 2], [7, 130], _at(BOUNDS), _at(SCALES), 5]),
    "select_blocks": (dict(layer=1, Q=Q, bounds=BOUNDS, scales=SCALES, seq_lens=[7, 9], blocks=BLOCKS, n_first=2,
                           n_last=1),
                      [1001, 1, _at(Q), _at(BOUNDS), _at(SCALES), [7, 9], 5, 2, 1, _at(BLOCKS), 5]),
    "decode_attention_blocks": (dict(layer=1, Q=Q, out=OUT, seq_lens=[7, 9], blocks=BLOCKS),
                                [1001, 1, _at(Q), _at(OUT), [7, 9], _at(BLOCKS), 5, 5]),
    "decode_attention_weights": (dict(layer=1, Q=Q, out=OUT, seq_lens=[7, 9], weights_in=W, weights_out=W2),
                                 [1001, 1, _at(Q), _at(OUT), [7, 9], _at(W), _at(W2), 5]),
    "evict": (dict(layer=0, weights_in=W, weights_out=W2, seq_lens=[7, 9], keep=[3, 4], recent=2, kept=KEPT),
              [1001, 1001, 0, _at(W), _at(W2), [7, 9], [3, 4], 2, _at(KEPT), 9, 5]),
    "decode_attention_prefix": (dict(layer=1, prefix=PREFIX, prefix_of=[0, -1], prefix_lens=[6], Q=Q, out=OUT,
                                     seq_lens=[7, 9]),
                                [1001, 1, 1002, [0, -1], [6], _at(Q), _at(OUT), [7, 9], 5]),
    "prefill_prefix": (dict(layer=0, prefix=PREFIX, prefix_of=[0, -1], prefix_lens=[6], Q=PQ, K=K, V=V, out=POUT,
                            prompt_lens=[7, 9]),
                       [1001, 0, 1002, [0, -1], [6], _at(PQ), _at(K), _at(V), _at(POUT), [7, 9], 10, 5]),
}


@pytest.mark.parametrize("call", sorted(GOOD))
def test_arguments_reach_the_library(lib, call):
    kwargs, want = GOOD[call]
    getattr(CACHE, call)(**kwargs, stream=5)
    assert lib.calls == [("mlkv_" + call, want)]


@pytest.mark.parametrize("numbers", [(7, 9), np.array([7, 9]), np.array([7, 9], dtype=np.int32),
                                     np.array([7, 0, 9], dtype=np.int32)[::2], np.array([7.0, 9.0]),
                                     np.frombuffer(np.array([7, 9], dtype=np.int32).tobytes(), dtype=np.int32)])
def test_numbers_of_any_kind_reach_it_as_int32(lib, numbers):
    CACHE.decode_attention_blocks(1, Q, OUT, numbers, BLOCKS, stream=5)
    assert lib.calls[0][1][4] == [7, 9]


def test_numbers_that_are_none(lib):
    with pytest.raises(ValueError):
        CACHE.decode_attention_blocks(1, Q, OUT, ["a", "b"], BLOCKS, stream=5)
    assert not lib.calls


def test_absent_arguments(lib):
    CACHE.block_bounds(0, [7, 9], BOUNDS, SCALES, stream=5)
    CACHE.decode_attention_weights(1, Q, OUT, [7, 9], None, W, stream=5)
    assert lib.calls[0][1][2] is None and lib.calls[1][1][5] is None


BAD_CHANGES = {
    "block_bounds": [
        dict(bounds=BOUNDS.float()), dict(bounds=BOUNDS[:, :, :2]), dict(bounds=BOUNDS.transpose(1, 2)),
        dict(scales=SCALES.bfloat16()), dict(scales=SCALES[:1]), dict(seq_lens=[1]), dict(first=[0, 0, 0]),
        dict(scales=torch.zeros(2, 3, 6)[:, :, ::2])],
    "select_blocks": [
        dict(blocks=BLOCKS.long()), dict(blocks=BLOCKS[:, :2]), dict(blocks=torch.zeros(2, 3, 10).int()[:, :, ::2]),
        dict(bounds=BOUNDS.to(torch.uint8)), dict(scales=SCALES[:, :, :2]), dict(seq_lens=1)],
    "decode_attention_blocks": [dict(blocks=BLOCKS.short()), dict(blocks=BLOCKS[:1]), dict(seq_lens=[[1, 1]])],
    "decode_attention_weights": [
        dict(weights_out=W.double()), dict(weights_out=torch.zeros(2, 3, 129)), dict(weights_in=W.half()),
        dict(weights_in=W[:, :1]), dict(weights_out=torch.zeros(3, 2, 130).transpose(0, 1))],
    "evict": [
        dict(kept=KEPT.float()), dict(kept=KEPT[:1]), dict(weights_in=W.double()), dict(weights_out=W[:, :2]),
        dict(keep=[9]), dict(to=_cache(1003, max_seq=20)), dict(seq_lens=[9, 9, 9])],
    "decode_attention_prefix": [
        dict(prefix_of=[0]), dict(prefix_lens=[1, 1]), dict(seq_lens=[1]), dict(prefix_of=[[0, 0]])],
    "prefill_prefix": [dict(prefix_of=[0]), dict(prefix_lens=[1, 1]), dict(prompt_lens=[1])],
}


@pytest.mark.parametrize("call,i", [(c, i) for c in sorted(BAD_CHANGES) for i in range(len(BAD_CHANGES[c]))])
def test_refused_before_the_library(lib, call, i):
    kwargs = dict(GOOD[call][0], **BAD_CHANGES[call][i])
    with pytest.raises(package.MLKVError) as e:
        getattr(CACHE, call)(**kwargs, stream=5)
    assert e.value.code == BAD and "must" in str(e.value)
    assert not lib.calls


# Tensors that the kernels would read or write as they lie: another type, other sizes, gaps.
DECODE = [("Q", Q), ("out", OUT)]
PROMPT = [("Q", PQ), ("out", POUT), ("K", K), ("V", V)]
TENSORS = {"select_blocks": DECODE[:1], "decode_attention_blocks": DECODE, "decode_attention_weights": DECODE,
           "decode_attention_prefix": DECODE, "prefill_prefix": PROMPT}


def _others(name, t):
    yield dict([(name, t.float())])
    yield dict([(name, t.half())])
    yield dict([(name, t[..., :32])])
    yield dict([(name, t[:1])])
    yield dict([(name, torch.cat([t, t], 1)[:, ::2])])
    yield dict([(name, None)])


@pytest.mark.parametrize("call", sorted(TENSORS))
def test_queries_and_outputs_of_another_kind_are_refused(lib, call):
    for name, t in TENSORS[call]:
        for change in _others(name, t):
            with pytest.raises(package.MLKVError) as e:
                getattr(CACHE, call)(**dict(GOOD[call][0], **change), stream=5)
            assert e.value.code == BAD and name in str(e.value), (name, change)
    assert not lib.calls


def test_prompts_of_a_reading_layer_need_no_keys(lib):
    CACHE.prefill_prefix(**dict(GOOD["prefill_prefix"][0], layer=1, K=None, V=None), stream=5)
    assert lib.calls[0][1][6:8] == [None, None]


def test_layers_out_of_range_are_the_library_s_to_refuse(lib):
    for layer in (-1, 2):
        CACHE.prefill_prefix(**dict(GOOD["prefill_prefix"][0], layer=layer), stream=5)
    assert [c[1][1] for c in lib.calls] == [-1, 2]


# The functions of the library's names, on handles: those take sizes as they are given.
def _function(call):
    kwargs = dict(GOOD[call][0])
    for name in ("prefix",):
        if name in kwargs:
            kwargs[name] = kwargs[name].handle
    if call == "select_blocks":
        kwargs["n_select"] = 5
    if call == "decode_attention_blocks":
        kwargs["n_blocks"] = 5
    if call == "evict":
        kwargs.update(to=1001, k_max=9)
    if call == "prefill_prefix":
        kwargs["s_max"] = 10
    return getattr(package, "mlkv_" + call), kwargs


@pytest.mark.parametrize("call", sorted(GOOD))
def test_functions_on_handles(lib, call):
    fn, kwargs = _function(call)
    fn(1001, **kwargs, stream=5)
    assert lib.calls == [("mlkv_" + call, GOOD[call][1])]


@pytest.mark.parametrize("call", sorted(GOOD))
def test_functions_on_handles_refuse_other_types(lib, call):
    fn, kwargs = _function(call)
    tensors = [k for k, v in kwargs.items() if isinstance(v, torch.Tensor)]
    assert tensors
    for name in tensors:
        t = kwargs[name]
        for other in (t.to(torch.float64), torch.cat([t, t], 1)[:, ::2]):
            with pytest.raises(package.MLKVError) as e:
                fn(1001, **dict(kwargs, **{name: other}), stream=5)
            assert e.value.code == BAD and name in str(e.value)
    assert not lib.calls

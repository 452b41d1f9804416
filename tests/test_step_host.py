"""Rotary positions, block norms and logits rules on the host: what is refused,
descriptors and frequencies.  No GPU is needed."""

import ctypes
import math
import os
import subprocess

import pytest
import torch

import step_reference as ref
from paper_2606_14782_gb300 import bacon, build

A = 1 << 20  # an address that nobody follows
OK, EINVAL = bacon.BACON_OK, bacon.BACON_EINVAL


@pytest.fixture(scope="module")
def lib():
    build.build()
    return bacon.load()


def test_descriptor_layouts(tmp_path):
    mirrors = {"bacon_rows": bacon.Rows, "bacon_block": bacon.Block, "bacon_logits_rows": bacon.LogitsRows}
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "bacon.h"\nint main(void) {\n' + "".join(
        f'printf("{t} size %zu\\n", sizeof({t}));\n' + "".join(
            f'printf("{t} {n} %zu\\n", offsetof({t}, {n.rstrip("_")}));\n' for n, _ in cls._fields_)
        for t, cls in mirrors.items()) + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(build.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        t, field, at = line.split()
        cls = mirrors[t]
        assert int(at) == (ctypes.sizeof(cls) if field == "size" else getattr(cls, field).offset), line


def test_packed_descriptors_have_the_mirrors_layout():
    for cls, pack in ((bacon.Rows, bacon._pack_rows), (bacon.Block, bacon._pack_block),
                      (bacon.LogitsRows, bacon._pack_logits)):
        values = [i + 1 for i in range(len(cls._fields_))]
        raw = pack(*values)
        assert len(raw) <= ctypes.sizeof(cls)  # but for what lies behind the last field
        back = cls.from_buffer_copy(raw + bytes(ctypes.sizeof(cls) - len(raw)))
        assert [getattr(back, n) for n, _ in cls._fields_] == values


# -------------------------------------------------------------- frequencies

@pytest.mark.parametrize("dim", [2, 16, 24, 64, 128, 256])
@pytest.mark.parametrize("kw", [
    {}, dict(base=500000.0), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
    dict(scaling="rotations", factor=8.0, original=8192, low=1.0, high=4.0, base=500000.0),
    dict(scaling="dims", factor=16.0, original=4096), dict(scaling="dims", factor=2.0, original=64),
    dict(scaling="dims", factor=40.0, original=100000, base=1e6)])
def test_frequencies(lib, dim, kw):
    """pow, log and two products in 64 bits: 2^-45 of the value, log's part in the
    ramp (up to 2^10 pairs wide) 2^-40."""
    if kw.get("scaling") == "base" and dim == 2:
        with pytest.raises(bacon.BaconError):
            bacon.Rotary(dim, **kw)
        return
    got, want = bacon.Rotary(dim, **kw).frequencies, ref.frequencies(dim, **kw)
    assert len(got) == dim // 2
    for g, w in zip(got, want):
        assert abs(g - w) <= 2.0 ** -40 * w


def test_scaled_frequencies_are_what_they_say():
    plain = bacon.Rotary(64).frequencies
    assert plain[0] == 1.0 and math.isclose(plain[-1], 10000.0 ** (-62 / 64))
    assert all(math.isclose(a, b / 4) for a, b in
               zip(bacon.Rotary(64, scaling="linear", factor=4.0).frequencies, plain))
    ramp = bacon.Rotary(64, scaling="rotations", factor=8.0, original=4096, low=1.0, high=4.0).frequencies
    for a, b in zip(ramp, plain):
        turns = 4096 * b / (2 * math.pi)
        assert math.isclose(a, b) if turns >= 4 else math.isclose(a, b / 8) if turns <= 1 else b / 8 < a < b
    own = [0.5, 0.25]
    assert bacon.Rotary(8, 4, frequencies=own).frequencies == own


@pytest.mark.parametrize("args,kw", [
    ((0,), {}), ((7,), {}), ((258,), {}), ((64, 0), {}), ((64, 66), {}), ((64, 3), {}),
    ((64,), dict(base=1.0)), ((64,), dict(base=math.inf)), ((64,), dict(scaling="linear", factor=0.0)),
    ((64,), dict(scaling="dims", factor=2.0)), ((64,), dict(scaling="dims", factor=2.0, original=100, low=4, high=4)),
    ((64,), dict(scaling="base", factor=math.nan)), ((64,), dict(amplitude=math.inf)),
    ((64,), dict(frequencies=[math.nan] * 32)), ((64,), dict(frequencies=[1e9] * 32))])
def test_rotary_refuses(lib, args, kw):
    with pytest.raises((bacon.BaconError, ValueError)):
        bacon.Rotary(*args, **kw)


@pytest.mark.parametrize("kw", [dict(scaling="other"), dict(frequencies=[1.0]), dict(axes=[0]),
                                dict(axes=[3] * 32)])
def test_rotary_binding_refuses(kw):
    with pytest.raises(ValueError):
        bacon.Rotary(64, **kw)


# -------------------------------------------------------------------- calls

ROWS = dict(in_=A, out=A, weight=0, heads=4, in_request=0, in_token=512, in_head=128, out_request=0,
            out_token=512, out_head=128)


def rows(**change):
    return bacon._pack_rows(*{**ROWS, **change}.values())


def rotary_call(lib, handle=None, requests=1, tokens=3, q=None, k=None, dtype=0, weight=0, eps=1e-6,
                offset=0.0, transposed=0, positions=A):
    return lib.bacon_rotary_apply(handle, requests, tokens, q, k, dtype, weight, eps, offset, transposed,
                                  positions, None)


@pytest.mark.parametrize("change,word", [
    (dict(tokens=-1), "negative"), (dict(requests=-1), "negative"), (dict(dtype=3), "dtype"),
    (dict(q=rows(in_=0)), "null"), (dict(q=rows(out=0)), "null"), (dict(q=rows(out=A + 1)), "aligned"),
    (dict(q=rows(heads=-1)), "heads"), (dict(q=rows(out_head=127)), "overlap"),
    (dict(q=rows(out_token=0)), "overlap"), (dict(q=rows(out_token=511)), "overlap"),
    (dict(q=rows(in_token=-512)), "stride"), (dict(k=rows(out_head=-1)), "stride"),
    (dict(q=rows(weight=A), weight=1), "type"), (dict(q=rows(weight=A), transposed=1), "transposed"),
    (dict(q=rows(weight=A), eps=0.0), "eps"), (dict(q=rows(weight=A), eps=math.nan), "eps"),
    (dict(q=rows(weight=A), offset=math.inf), "offset"), (dict(q=rows(weight=A + 2), weight=2), "aligned"),
    (dict(q=rows(), positions=None), "positions"), (dict(q=rows(), tokens=1 << 30), "2^31"),
    (dict(q=rows(out_request=512), requests=2), "overlap")])
def test_rotary_calls_refused(lib, change, word):
    r = bacon.Rotary(128)
    change = dict(change)
    change.setdefault("q", rows())
    assert rotary_call(lib, r.handle, **change) == EINVAL
    assert word in lib.bacon_last_error().decode()
    assert rotary_call(lib, None, **change) == EINVAL


def test_rotary_of_nothing(lib):
    r = bacon.Rotary(128)
    assert rotary_call(lib, r.handle) == OK
    assert rotary_call(lib, r.handle, tokens=0, q=rows(in_=0, out=0), positions=None) == OK
    assert rotary_call(lib, r.handle, q=rows(heads=0, in_=0)) == OK


BLOCK = dict(tokens=3, width=64, dtype=0, residual_dtype=0, weight_dtype=0, post=0, pre=1, activation=0,
             scale=1.0, eps=1e-6, weight_offset=0.0, gate_channel=0, gate_token=0, y_token=64, x_token=64,
             sum_token=64, normed_token=64, y=A, x=A, gate=0, post_weight=0, post_bias=0, pre_weight=0,
             pre_bias=0, sum=A, normed=A)


@pytest.mark.parametrize("change,word", [
    (dict(tokens=-1), "tokens"), (dict(width=0), "width"), (dict(width=32769), "width"),
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(dtype=0, residual_dtype=1), "residual"),
    (dict(dtype=2, residual_dtype=0, weight_dtype=2), "residual"), (dict(weight_dtype=1), "weight"),
    (dict(post=3), "norm"), (dict(pre=-1), "norm"), (dict(activation=4), "activation"),
    (dict(scale=math.nan), "scale"), (dict(eps=0.0), "eps"), (dict(eps=math.inf), "eps"),
    (dict(weight_offset=math.inf), "offset"), (dict(sum=0, normed=0), "wanted"), (dict(pre=0), "pre"),
    (dict(y=0), "null"), (dict(y=A + 1), "aligned"), (dict(residual_dtype=2, x=A + 2), "aligned"),
    (dict(weight_dtype=2, pre_bias=A + 2), "aligned"), (dict(sum_token=63), "overlap"),
    (dict(normed_token=0), "overlap"), (dict(y_token=-64), "stride"), (dict(x_token=1 << 60), "stride")])
def test_norm_calls_refused(lib, change, word):
    assert lib.bacon_block_norm(bacon._pack_block(*{**BLOCK, **change}.values()), None) == EINVAL
    assert word in lib.bacon_last_error().decode()


def test_norm_of_nothing(lib):
    assert lib.bacon_block_norm(None, None) == EINVAL
    assert lib.bacon_block_norm(bacon._pack_block(*{**BLOCK, "tokens": 0, "y": 0}.values()), None) == OK


LOGITS = dict(rows=3, dtype=2, out_dtype=2, requests=3, capacity=10, biases=4, row_stride=100, out_stride=100,
              token_stride=10, mask_stride=4, logits=A, out=A, tokens=A, request=0, prompt=0, lengths=A,
              repetition=A, frequency=0, presence=0, temperature=0, bias_tokens=A, bias_values=A, mask=A,
              best=A, logprob=A, lse=A)


@pytest.fixture(scope="module")
def handle(tmp_path_factory):
    """A logits handle on a CUDA runtime of the host, and that library."""
    import fake_cuda
    lib = fake_cuda.library(str(tmp_path_factory.mktemp("fake")))
    h = ctypes.c_void_p()
    assert lib.bacon_logits_create(ctypes.byref(h), 100) == OK
    yield lib, h
    lib.bacon_logits_destroy(h)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(dtype=3), "dtype"), (dict(dtype=0, out_dtype=1), "dtype"),
    (dict(out=0, best=0, logprob=0, lse=0), "wanted"), (dict(biases=-1), "biases"),
    (dict(biases=2048), "biases"), (dict(bias_values=0), "null"), (dict(requests=0), "requests"),
    (dict(capacity=1 << 20), "capacity"), (dict(capacity=-1), "capacity"), (dict(token_stride=-1), "capacity"),
    (dict(lengths=0), "lengths"), (dict(logits=0), "null"),
    (dict(logits=A + 2), "aligned"), (dict(mask=A + 1), "aligned"), (dict(best=A + 2), "aligned"),
    (dict(row_stride=-1), "stride"), (dict(mask_stride=-1), "stride"), (dict(out_stride=99), "overlap"),
    (dict(row_stride=104), "in place"), (dict(dtype=0), "in place")])
def test_logits_calls_refused(handle, change, word):
    lib, h = handle
    assert lib.bacon_logits_process(h, bacon._pack_logits(*{**LOGITS, **change}.values()), None) == EINVAL
    assert word in lib.bacon_last_error().decode()
    assert lib.bacon_logits_process(None, bacon._pack_logits(*LOGITS.values()), None) == EINVAL


def test_logits_handles(handle):
    lib, h = handle
    assert lib.bacon_logits_process(h, None, None) == EINVAL
    assert lib.bacon_logits_sync(None, None) == EINVAL
    assert lib.bacon_logits_process(h, bacon._pack_logits(*{**LOGITS, "rows": 0, "logits": 0}.values()),
                                    None) == OK
    other = ctypes.c_void_p()
    for vocab in (0, -5, 458753):
        assert lib.bacon_logits_create(ctypes.byref(other), vocab) == EINVAL and not other.value
    lib.fake_fail_allocations(1)
    assert lib.bacon_logits_create(ctypes.byref(other), 100) == bacon.BACON_ENOMEM and not other.value
    assert lib.cudaPeekAtLastError() == 0
    assert lib.bacon_logits_sync(h, None) == OK


def test_rotated_store_refused(handle):
    from test_cache_host_order import create
    lib, _ = handle
    cache, r = create(lib), bacon.Rotary(64)
    other = bacon.Rotary(128)
    k = rows(out=0, heads=2, in_token=128, in_head=64)

    def call(rotary=r.handle, tokens=3, q=None, k=k, v=A, weight=0, positions=A, slots=A, v_token=128):
        return lib.bacon_cache_store_rotated(cache, rotary, tokens, q, k, v, v_token, 64, weight, 1e-6, 0.0,
                                             positions, slots, None)

    word = lib.bacon_last_error
    for change, said in ((dict(rotary=other.handle), "rotation"),
                         (dict(rotary=None), "null"), (dict(k=None), "null"), (dict(tokens=-1), "tokens"),
                         (dict(k=rows(heads=0)), "heads"), (dict(positions=None), "positions"),
                         (dict(slots=None), "null"), (dict(v=None), "v must"), (dict(v_token=12), "strides"),
                         (dict(k=rows(in_=A + 2, heads=2, in_token=128, in_head=64)), "k must"),
                         (dict(q=rows(out=0)), "null")):
        assert call(**change) == EINVAL
        assert said in word().decode(), change
    assert call(tokens=0) == OK
    lib.bacon_cache_destroy(cache)


# ------------------------------------------------------------------ binding

def cpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_host_tensors_are_refused():
    r = bacon.Rotary(64)
    with pytest.raises(ValueError):
        r.apply(cpu(2, 4, 64), cpu(2, 1, 64), cpu(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        r.apply(None, None, cpu(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        bacon.BlockNorm(64)(cpu(2, 64))
    with pytest.raises(ValueError):
        bacon.BlockNorm(64, pre_weight=cpu(64))
    for kw in (dict(pre="other"), dict(post="other"), dict(gate="other")):
        with pytest.raises(ValueError):
            bacon.BlockNorm(64, **kw)

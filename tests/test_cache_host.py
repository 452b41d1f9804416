"""The 8-bit cache's ABI on the host: refusals before the device is touched,
and the binding's mirror of the descriptor."""

import ctypes
import os
import subprocess

import pytest

from paper_2606_14782_gb300 import bacon, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return bacon.load()


def desc(**kw):
    d = dict(layers=2, kv_heads=2, q_heads=8, head_dim=64, page=16, pages=10, max_requests=3,
             max_blocks=4, format=0, dtype=0, k=1 << 20, v=2 << 20, k_scale=3 << 20,
             v_scale=4 << 20)
    d.update(kw)
    return bacon.CacheDesc(**d)


@pytest.mark.parametrize("change,word", [
    (dict(layers=0), "positive"), (dict(kv_heads=0), "positive"), (dict(q_heads=-8), "positive"),
    (dict(pages=0), "positive"), (dict(max_requests=0), "positive"),
    (dict(max_blocks=0), "positive"), (dict(q_heads=7), "multiple"),
    (dict(head_dim=96), "head_dim"), (dict(page=48), "page"), (dict(page=256), "page"),
    (dict(pages=1 << 27), "2^31"), (dict(max_blocks=1 << 27), "2^31"),
    (dict(layers=1 << 20, max_requests=1 << 12), "2^31"),
    (dict(format=2), "format"), (dict(dtype=-1), "dtype"),
    (dict(k=None), "pools"), (dict(v=(2 << 20) + 8), "pools"), (dict(v_scale=None), "pools"),
])
def test_create_refuses(lib, change, word):
    h = ctypes.c_void_p()
    assert lib.bacon_cache_create(ctypes.byref(h), ctypes.byref(desc(**change))) \
        == bacon.BACON_EINVAL
    assert word in lib.bacon_last_error().decode()
    assert not h.value


def test_null_arguments_are_refused(lib):
    E = bacon.BACON_EINVAL
    assert lib.bacon_cache_create(None, ctypes.byref(desc())) == E
    h = ctypes.c_void_p()
    assert lib.bacon_cache_create(ctypes.byref(h), None) == E
    assert lib.bacon_cache_plan(None, 1, None, None, 0, None, None, None, 0, None, None, None,
                                None) == E
    assert lib.bacon_cache_locate(None, 1, None, None, None, 0, None, None) == E
    assert lib.bacon_cache_release(None, 1, None, None, None, None, None, None) == E
    assert lib.bacon_cache_store(None, 1, 1, None, 0, 0, None, 0, 0, None, None) == E
    assert lib.bacon_cache_load(None, 1, None, None, None, None) == E
    assert lib.bacon_cache_attend(None, 1, 0, 1, None, 0, 0, None, None, None, 1, 0.0, None, None,
                                  None) == E
    assert lib.bacon_cache_sync(None, None) == E
    lib.bacon_cache_destroy(None)


def test_descriptor_layout(tmp_path):
    fields = [f for f, _ in bacon.CacheDesc._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "bacon.h"\n'
                   "int main(void) {\n"
                   '  printf("size %zu\\n", sizeof(bacon_cache_desc));\n'
                   + "".join(f'  printf("{f} %zu\\n", offsetof(bacon_cache_desc, {f}));\n'
                             for f in fields) + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = dict(line.split() for line in subprocess.run(
        [str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(bacon.CacheDesc)
    for f in fields:
        assert int(got[f]) == getattr(bacon.CacheDesc, f).offset, f

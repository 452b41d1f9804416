"""The axes of a rotation arrive as they are given, whatever holds them.  No GPU is needed."""

from array import array

import numpy as np
import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

AXES = [0, 2, 1, 0, 1, 2, 2, 0]


@pytest.mark.parametrize("axes", [AXES, tuple(AXES), bytes(AXES), array("i", AXES), np.array(AXES),
                                  np.array(AXES, np.uint8), np.array(AXES, np.float32), torch.tensor(AXES)],
                         ids=["list", "tuple", "bytes", "array", "int64", "uint8", "float32", "tensor"])
def test_axes(axes, monkeypatch):
    build.build()
    lib, seen = bacon.load(), []

    class Library:
        def __getattr__(self, name):
            call = getattr(lib, name)
            if name != "bacon_rotary_create":
                return call
            return lambda *args: seen.append(args[-1]) or call(*args)

    monkeypatch.setattr(bacon, "load", lambda: Library())
    rotary = bacon.Rotary(16, axes=axes)
    assert seen == [bytes(AXES)] and rotary.axes == 3

"""Arguments of the 8-bit cache's binding: what lies on the host or on another
device is refused before the library is called.  Stand-ins of tensors, streams
and the library; no GPU is needed."""

import contextlib

import pytest
import torch

from paper_2606_14782_gb300 import bacon

L, H, HQ, D, PAGES, PAGE, R, BLOCKS, T = 2, 2, 4, 64, 10, 16, 3, 4, 6
BF16, I32, F32, U8 = torch.bfloat16, torch.int32, torch.float32, torch.uint8


class Tensor:
    def __init__(self, shape, dtype, index=0):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index
        self.is_cuda = index >= 0
        self.device = torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def stride(self):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def record_stream(self, stream):
        pass


class Stream:
    def __init__(self, index=0):
        self.cuda_stream, self.device_index, self.device = 0x77, index, torch.device("cuda", index)
        self.stream_id = 1


class Library:
    """Every call succeeds; what was called, and on which device."""

    def __init__(self):
        self.calls, self.device = [], 0

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.device))
            return bacon.BACON_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()

    @contextlib.contextmanager
    def device(d):
        kept, lib.device = lib.device, torch.device(d).index
        yield
        lib.device = kept

    monkeypatch.setattr(bacon, "load", lambda: lib)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: lib.device)
    return lib


def pools(index=0, **other):
    kind = dict(k=((PAGES, PAGE, D), U8), v=((PAGES, PAGE, D), U8), k_scale=((PAGES,), F32),
                v_scale=((PAGES,), F32))
    return {n: Tensor(s, t, other.get(n, index)) for n, (s, t) in kind.items()}


def cache(**given):
    return bacon.Cache(L, H, HQ, D, PAGES, page=PAGE, max_requests=R, max_blocks=BLOCKS,
                       **(given or pools()))


UNITS, TABLE = (R, L, H), (R, L, H, BLOCKS)
CALLS = {
    "plan": dict(lengths=(UNITS, I32), added=(UNITS, I32), table=(TABLE, I32), ring=((PAGES,), I32),
                 state=((2,), I32), slots=((T,), I32), lengths_out=(UNITS, I32),
                 state_out=((2,), I32)),
    "locate": dict(count=(UNITS, I32), table=(TABLE, I32), first=(UNITS, I32), slots=((T,), I32)),
    "release": dict(done=((R,), I32), lengths=(UNITS, I32), table=(TABLE, I32), ring=((PAGES,), I32),
                    state=((2,), I32)),
    "shorten": dict(fewer=((R,), I32), lengths=(UNITS, I32), table=(TABLE, I32),
                    ring=((PAGES,), I32), state=((2,), I32)),
    "store": dict(k=((T, H, D), BF16), v=((T, H, D), BF16), slots=((T, H), I32)),
    "load": dict(slots=((T,), I32), k_out=((T, D), BF16), v_out=((T, D), BF16)),
    "attend": dict(q=((T, HQ, D), BF16), lengths=(UNITS, I32), table=(TABLE, I32),
                   starts=((R + 1,), I32), out=((T, HQ, D), BF16), lse=((T, HQ), F32)),
}
MORE = {"plan": dict(rows=T), "locate": dict(rows=T), "attend": dict(layer=1)}


def call(c, name, stream=None, **index):
    args = {n: Tensor(s, t, index.get(n, 0)) for n, (s, t) in CALLS[name].items()}
    getattr(c, name)(**args, **MORE.get(name, {}), stream=stream or Stream())


@pytest.mark.parametrize("name", CALLS)
def test_arguments_on_the_caches_device_are_taken(lib, name):
    c = cache()
    call(c, name)
    assert [n for n, _ in lib.calls] == ["bacon_cache_create", "bacon_cache_" + name]


@pytest.mark.parametrize("where", [-1, 1])  # the host, another device
@pytest.mark.parametrize("name,arg", [(n, a) for n in CALLS for a in CALLS[n]])
def test_arguments_elsewhere_are_refused(lib, name, arg, where):
    c = cache()
    with pytest.raises(ValueError):
        call(c, name, **{arg: where})
    assert [n for n, _ in lib.calls] == ["bacon_cache_create"]


@pytest.mark.parametrize("name", CALLS)
def test_another_devices_stream_is_refused(lib, name):
    c = cache()
    with pytest.raises(ValueError):
        call(c, name, stream=Stream(1))
    assert [n for n, _ in lib.calls] == ["bacon_cache_create"]


def test_the_handle_is_made_on_the_pools_device(lib):
    cache(**pools(index=1))
    assert lib.calls == [("bacon_cache_create", 1)] and lib.device == 0


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale"])
@pytest.mark.parametrize("where", [-1, 1])
def test_pools_apart_are_refused(lib, name, where):
    with pytest.raises(ValueError):
        cache(**pools(**{name: where}))
    assert lib.calls == []

"""Threads with handles of their own: what one call sets for a kernel must not take away
what another's launch needs."""

import ctypes
import threading

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

A = 1 << 20  # an address that nobody follows
# pairs whose calls run one kernel with different shared memory: rows of each call
VOCABS = [(262144, 131072, 1), (458752, 200000, 1), (140000, 120000, 64), (458752, 150000, 40)]


def together(*work):
    """Runs them on threads of their own; their results."""
    results, gate = [None] * len(work), threading.Barrier(len(work))

    def run(i):
        gate.wait()
        results[i] = work[i]()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return results


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    import fake_cuda
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


@pytest.mark.parametrize("one,other,rows", VOCABS)
def test_two_handles_on_two_threads(lib, one, other, rows):
    """On the host's runtime, which refuses a launch above what is set for its kernel."""
    def calls(vocab):
        handle = ctypes.c_void_p()
        assert lib.bacon_logits_create(ctypes.byref(handle), vocab) == bacon.BACON_OK
        raw = bacon._pack_logits(rows, 2, 2, rows, 10, 0, vocab, vocab, 10, 0, A, A, A, 0, 0, A, A, 0, 0, 0, 0, 0,
                                 0, A, A, A)

        # (the host's runtime gets to know the kernel here, before the threads)
        assert lib.bacon_logits_process(handle, raw, None) == bacon.BACON_OK

        def work():
            return {lib.bacon_logits_process(handle, raw, None) for _ in range(30000)}
        return work, handle

    made = [calls(v) for v in (one, other)]
    try:
        assert together(*(w for w, _ in made)) == [{bacon.BACON_OK}] * 2
    finally:
        for _, handle in made:
            lib.bacon_logits_destroy(handle)


@pytest.mark.gpu
@pytest.mark.parametrize("one,other,rows", VOCABS)
def test_two_handles_on_two_threads_of_a_gpu(one, other, rows):
    build.build()

    def calls(vocab, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(rows, vocab, generator=gen, device="cuda")
        said = torch.randint(0, vocab, (rows, 10), generator=gen, device="cuda", dtype=torch.int32)
        length = torch.full((rows,), 10, dtype=torch.int32, device="cuda")
        penalty = torch.full((rows,), 1.5, device="cuda")
        handle, stream = bacon.Logits(vocab), torch.cuda.Stream()

        def process():
            return handle.process(x, tokens=said, lengths=length, repetition=penalty, stream=stream)
        torch.cuda.synchronize()
        want = process()
        torch.cuda.synchronize()

        def work():
            for _ in range(300):
                got = process()
            stream.synchronize()
            return all(torch.equal(a, b) for a, b in zip(got, want))
        return work, handle

    made = [calls(v, i) for i, v in enumerate((one, other))]
    assert together(*(w for w, _ in made)) == [True, True]
    for _, handle in made:
        handle.sync()
        handle.close()

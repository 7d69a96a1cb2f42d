"""relation_sample from several host threads at once: every call launches with what its own rows need."""
import threading

import pytest
import torch

from paper_2608_20172_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_calls_of_different_sizes_at_once():
    """Vocabularies whose slices take different amounts of shared memory, 20000 calls of the C entry a
    thread (ctypes lets go of the interpreter's lock)."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    lib = binding.load()
    g = torch.Generator(device=DEV).manual_seed(0)
    jobs = []
    for V in (200, 30000, 100000, 131000, 900, 50257, 80000, 2000):
        x, u = torch.randn((1, V), generator=g, device=DEV), torch.rand(1, generator=g, device=DEV)
        want = binding.sample(x, u)
        jobs.append((x, u, want, tuple(torch.empty_like(t) for t in want), torch.cuda.Stream()))
    torch.cuda.synchronize()
    failed, begin = [], threading.Barrier(len(jobs))

    def work(x, u, want, out, stream):
        args = (x.data_ptr(), 1, x.shape[1], x.stride(0), binding.F32, u.data_ptr(), None, None, None,
                None, *(t.data_ptr() for t in out), None, stream.cuda_stream)
        begin.wait()
        for _ in range(20000):
            rc = lib.relation_sample(*args)
            if rc != binding.OK or failed:
                failed.append((x.shape[1], binding.status_string(rc)))
                return

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for _, _, want, out, _ in jobs:
        for a, b in zip(out, want):
            assert torch.equal(a, b)

"""The host's side of the MXFP4 and grouped calls: what the compiled calls allocate, and the context's state under several threads."""
import threading

import pytest
import torch

from paper_2605_26632_b200 import binding
from test_gpu_mxfp4 import rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pair():
    fast, general = binding.Lynx(0), binding.Lynx(0)
    assert fast._calls is binding.load_calls()
    general._calls = binding._GeneralPathOnly
    yield fast, general
    torch.cuda.synchronize()
    for c in (fast, general):
        assert c.last_error() == 0
        c.close()


def test_new_results_are_filled_in_the_deterministic_mode(pair):
    """torch.use_deterministic_algorithms fills new memory (NaN, or the largest integer): rows that a call does not write hold that."""
    M, N, K = 300, 264, 256
    X, W = rand((M, K), 1).cuda(), rand((N, K), 2).cuda()
    off = torch.tensor([10, 200], dtype=torch.int32, device="cuda")
    none = [*range(10), *range(200, M)]
    torch.use_deterministic_algorithms(True)
    try:
        assert torch.utils.deterministic.fill_uninitialized_memory
        for c in pair:
            wq, ws = c.quantize_mxfp4(W)
            for call, filled in ((lambda: c.grouped_linear(X, off, W[None]), lambda t: t.isnan()),
                                 (lambda: c.act_grouped_linear_mxfp4(X, off, wq[None], ws), lambda t: t.isnan()),
                                 (lambda: c.quantize_mxfp4(X, off)[0], lambda t: t == 255),
                                 (lambda: c.dequantize_mxfp4(*c.quantize_mxfp4(X, off), off), lambda t: t.isnan())):
                call()
                held = [torch.zeros(M, n, dtype=torch.uint8, device="cuda") for n in (K // 2, 2 * K, 2 * N)]  # what new memory would show
                del held
                t = call()
                assert filled(t[none]).all() and not filled(t[10:200]).all()
    finally:
        torch.use_deterministic_algorithms(False)


def test_launches_of_two_threads_are_all_counted(pair):
    """One context, two threads with a stream and tensors each, through the C ABI: calls as close to one another as they come.  (A plain
    counter lost 3 of 200000.)"""
    lx, calls = pair[0], 400000
    sets = []
    for i in range(2):
        X = rand((1, 32), 10 + i).cuda()
        sets.append((X, *lx.quantize_mxfp4(X), torch.cuda.Stream()))
    want = [s[1].clone() for s in sets]
    torch.cuda.synchronize()
    before, start, status = lx.launch_count(), threading.Barrier(2), []

    def work(X, codes, scales, stream):
        torch.cuda.set_device(0)
        f = lx._lib.lynx_quantize_mxfp4
        a = [t(v) for t, v in zip(f.argtypes, (lx._address, X.data_ptr(), 1, 32, 32, None, 1, codes.data_ptr(), scales.data_ptr(), stream.cuda_stream))]
        start.wait()
        status.append(sum(f(*a) for _ in range(calls)))

    threads = [threading.Thread(target=work, args=s) for s in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert status == [0, 0] and all(torch.equal(s[1], w) for s, w in zip(sets, want))
    assert lx.launch_count() - before == 2 * calls

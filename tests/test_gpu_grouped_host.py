"""The host's side of the MXFP4 and grouped calls."""
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

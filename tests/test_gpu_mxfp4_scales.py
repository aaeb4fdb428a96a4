"""What quantize_mxfp4 returns, scales and codes, against the definition in every way a program makes the call: the compiled calls and
the general path, two streams, two host threads, captured and replayed."""
import threading

import pytest
import torch

import mxfp4_reference as ref
from paper_2605_26632_b200 import binding
from test_gpu_mxfp4 import rand, u16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lx():
    ctx = binding.Lynx(0)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.last_error() == 0
    ctx.close()


OFFSETS = [[0, 20, 20, 151], [5, 5, 160, 160], [0, 1, 2, 3], [0, 33, 130, 170]]


class Quantised:
    """The three ways to cut rows into groups, on tensors of one's own."""

    def __init__(self, M=170, N=150, K=1184, E=3, seed=1):
        self.M, self.N, self.K, self.E = M, N, K, E
        self.X, self.W = rand((M, K), seed, dist="spread").cuda(), rand((E * N, K), seed + 1, dist="spread").cuda()
        self.off = torch.tensor(OFFSETS[0], dtype=torch.int32, device="cuda")
        self.define()

    def calls(self, lx):
        # (buffers made here: rows of no group are left as they were)
        new = lambda M, n, **kw: dict(codes=torch.full((M, self.K // 2), 0xAB, dtype=torch.uint8, device="cuda"),
                                      scales=torch.full((binding.mxfp4_scale_bytes(M, self.K, n, **kw),), 0xEE, dtype=torch.uint8, device="cuda"))
        return {
            "rows": lambda: lx.quantize_mxfp4(self.X),
            "rows into buffers": lambda: lx.quantize_mxfp4(self.X, **new(self.M, 1)),
            "equal groups": lambda: lx.quantize_mxfp4(self.W, groups=self.E),
            "by offsets": lambda: lx.quantize_mxfp4(self.X, self.off, **new(self.M, self.E, ragged=True)),
        }

    def define(self):
        self.x, self.w, self.offsets = ref.quantize(u16(self.X)), ref.quantize(u16(self.W)), self.off.tolist()

    def wrong(self, name, codes, scales):
        """What differs from the definition, '' if nothing does."""
        code, s = self.w if name == "equal groups" else self.x
        cut = dict(groups=self.E) if name == "equal groups" else dict(offsets=self.offsets) if name == "by offsets" else {}
        rows = slice(self.offsets[0], self.offsets[-1]) if name == "by offsets" else slice(0, len(code))
        c, sc = codes.cpu().numpy(), ref.scales_of(scales.cpu().numpy(), *code.shape, **cut)
        out = [] if (ref.unpack(c)[rows] == code[rows]).all() else ["codes"]
        out += [] if (sc[rows] == s[rows]).all() else ["scales"]
        out += [] if (c[:rows.start] == 0xAB).all() and (c[rows.stop:] == 0xAB).all() else ["rows of no group"]
        return ", ".join(out)


def test_a_wrong_scale_is_seen(lx):
    q = Quantised()
    for name, call in q.calls(lx).items():
        codes, scales = call()
        assert q.wrong(name, codes, scales) == ""
        # the byte of the last row that is in a group, its last block
        M = q.E * q.N if name == "equal groups" else q.M
        tile, row = ref.row_tiles(M, q.E if name == "equal groups" else 1, q.offsets if name == "by offsets" else None)[
            q.offsets[-1] - 1 if name == "by offsets" else M - 1]
        b = q.K // 32 - 1
        at = (tile * -(-q.K // 128) + b // 4) * 512 + (row % 32) * 16 + (row // 32) * 4 + b % 4
        host = scales.cpu()
        host[at] += 1
        assert q.wrong(name, codes, host) == "scales"


def test_compiled_calls_and_general_path(lx):
    general = binding.Lynx(0)
    general._calls = binding._GeneralPathOnly
    q = Quantised()
    for c in (lx, general):
        for name, call in q.calls(c).items():
            assert q.wrong(name, *call()) == "", name
    torch.cuda.synchronize()
    assert general.last_error() == 0
    general.close()


def test_two_streams(lx):
    q = Quantised()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got += [(n, f()) for n, f in q.calls(lx).items()]
    for s in streams:
        s.synchronize()
    for n, r in got:
        assert q.wrong(n, *r) == "", n


def test_two_host_threads(lx):
    sets, found = [Quantised(), Quantised(M=151, N=90, K=480, seed=5)], []
    torch.cuda.synchronize()

    def work(q):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = [(n, f()) for _ in range(8) for n, f in q.calls(lx).items()]
            torch.cuda.current_stream().synchronize()
        found.extend((n, w) for n, w in ((n, q.wrong(n, *r)) for n, r in got))

    threads = [threading.Thread(target=work, args=(q,)) for q in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(found) == 2 * 8 * 4 and not [f for f in found if f[1]]


def test_captured_and_replayed(lx):
    q = Quantised()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for f in q.calls(lx).values():
            f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = {n: f() for n, f in q.calls(lx).items()}
    for step, offsets in enumerate(OFFSETS):
        q.X.copy_(rand((q.M, q.K), 50 + step, dist="spread"))
        q.W.copy_(rand((q.E * q.N, q.K), 60 + step, dist="spread"))
        q.off.copy_(torch.tensor(offsets, dtype=torch.int32))
        q.define()
        graph.replay()
        torch.cuda.synchronize()
        for n, r in out.items():
            assert q.wrong(n, *r) == "", (step, n)

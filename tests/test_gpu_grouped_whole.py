"""Whole outputs of grouped and MXFP4 products where a CTA or a pair takes one item after the other, and where the list of offsets
decides how K is split; against 64-bit references on the same operand values, by test_gpu_mxfp4's bar."""
import functools
import os

import numpy as np
import pytest
import torch

import mxfp4_reference as ref
from test_gpu_mxfp4 import check, f64, rand, u16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def contexts():
    """The library's own choice of tiles, 256 x 256 on pairs, 128 x 64 on single CTAs."""
    from paper_2605_26632_b200 import binding

    made = []
    for cfg in (0, 1, 2):
        os.environ["LYNX_GROUPED_CFG"] = str(cfg)
        made.append(binding.Lynx(0))
        del os.environ["LYNX_GROUPED_CFG"]
    yield made
    torch.cuda.synchronize()
    for ctx in made:
        assert ctx.last_error() == 0
        ctx.close()


def offsets_of(sizes, first=0):
    return (first + np.concatenate([[0], np.cumsum(sizes)])).tolist()


# Nine row tiles of 256 in W.  A group of 4500 rows has 18 token tiles of 256 (71 of 64): one block of sixteen and a partial one,
# four whole blocks and one.  The others are of every width (192 twice, 128, 64, 256 three times, ...), empty and single rows among
# them; 5 and 9 rows at the ends are of no group.  In all 31 x 9 items of 256 x 256 for at most 74 pairs: three each and more.
RAGGED = [4500, 0, 1, 370, 192, 100, 64, 700, 300, 129, 33]
N = 2056


@functools.lru_cache(maxsize=2)
def operands(sizes, front, back, K, mx):
    E, M = len(sizes), front + sum(sizes) + back
    X, W = rand((M, K), 400 + K), rand((E * N, K), 401 + K, K ** -0.5)
    terms = dict(bias=rand((E, N), 402), row_scale=torch.rand(M, generator=torch.Generator().manual_seed(403)), residual=rand((M, N), 404))
    values = (lambda t: ref.values(*ref.quantize(u16(t)))) if mx else f64
    offsets = offsets_of(sizes, front)
    y, mag = ref.grouped(values(X), values(W).reshape(E, N, K), offsets, terms["row_scale"].double().numpy(), f64(terms["bias"]), f64(terms["residual"]))
    return X, W, terms, offsets, y, mag


def compare(Y, y, mag, K, terms, offsets):
    for a in range(offsets[0], offsets[-1], 1024):  # (in pieces: 64-bit copies of a whole output are large)
        r = slice(a, min(a + 1024, offsets[-1]))
        check(Y[r], y[r], mag[r], K, (np.abs(f64(terms["bias"])).max(), f64(terms["residual"][r])))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("K", [96, 1376])
def test_one_item_after_the_other(contexts, K, mx):
    """K = 96: one stage per item, every wait of an item is for the one before it; 1376: more stages than the ring has."""
    X, W, terms, offsets, y, mag = operands(tuple(RAGGED), 5, 9, K, mx)
    E, M = len(RAGGED), X.shape[0]
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    on = {k: v.cuda() for k, v in terms.items()}
    for lx in contexts:
        out = torch.full((M, N), 9.0, dtype=torch.bfloat16, device="cuda")
        if mx:
            wq, ws = lx.quantize_mxfp4(W.cuda(), groups=E)
            lx.act_grouped_linear_mxfp4(X.cuda(), off, wq.view(E, N, K // 2), ws, out=out, **on)
            xq, xs = lx.quantize_mxfp4(X.cuda(), off)
            again = lx.grouped_linear_mxfp4(xq, xs, off, wq.view(E, N, K // 2), ws, out=torch.full_like(out, 9.0), **on)
        else:
            lx.grouped_linear(X.cuda(), off, W.cuda().view(E, N, K), out=out, **on)
            again = lx.grouped_linear(X.cuda(), off, W.cuda().view(E, N, K), out=torch.full_like(out, 9.0), **on)
        assert torch.equal(again, out)
        compare(out, y, mag, K, terms, offsets)
        assert (out[:offsets[0]] == 9).all() and (out[offsets[-1]:] == 9).all()


@pytest.mark.parametrize("M,K", [(6500, 288), (7300, 1376)])
def test_one_item_after_the_other_without_offsets(contexts, M, K):
    """26 and 29 token tiles of 256 times nine of W."""
    X, W, terms, offsets, y, mag = operands((M,), 0, 0, K, True)
    on = dict(row_scale=terms["row_scale"].cuda(), residual=terms["residual"].cuda())
    for lx in contexts:
        wq, ws = lx.quantize_mxfp4(W.cuda())
        xq, xs = lx.quantize_mxfp4(X.cuda())
        Y = lx.linear_mxfp4(xq, xs, wq, ws, terms["bias"][0].cuda(), **on)
        compare(Y, y, mag, K, terms, offsets)
        assert torch.equal(lx.act_linear_mxfp4(X.cuda(), wq, ws, terms["bias"][0].cuda(), **on), Y)
        # the result over its own residual
        over = on["residual"].clone()
        lx.linear_mxfp4(xq, xs, wq, ws, terms["bias"][0].cuda(), on["row_scale"], over, out=over)
        assert torch.equal(over, Y)


# Clusters that split K, by offsets: rows of 12 stages and more (MXFP4 2880, bf16 720), up to four tiles per CTA.  The parts of a
# tile follow from the offsets: four where few tiles are left for a last round of 132 or 148 CTAs, two, one.
SPLITS = [  # (sizes, rows of no group at the ends, N)
    ([20, 0, 50, 10], 3, 136),                       # 6 tiles: in four
    ([64, 1, 0, 65, 128], 0, 1032),                  # 54 tiles: in two
    ([40, 70, 8, 130, 64, 1, 0, 3, 5], 2, 1032),     # 99 tiles: whole
    ([33, 64, 64, 60, 2, 1, 64, 64, 17], 0, 2056),   # 153 tiles: one round whole, what is left in four
    ([0, 0, 90], 7, 264),
]


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("case", range(len(SPLITS)))
def test_split_along_long_rows_by_offsets(contexts, case, mx):
    sizes, apart, N = SPLITS[case]
    K = 3232 if mx else 840
    E, M = len(sizes), sum(sizes) + 2 * apart
    offsets = offsets_of(sizes, apart)
    X, W = rand((M, K), 420 + case), rand((E * N, K), 421 + case, K ** -0.5)
    bias, res, scale = rand((E, N), 422), rand((M, N), 423), torch.rand(M, generator=torch.Generator().manual_seed(424))
    values = (lambda t: ref.values(*ref.quantize(u16(t)))) if mx else f64
    x, w = values(X), values(W).reshape(E, N, K)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    inside = slice(offsets[0], offsets[-1])
    for lx in (contexts[0], contexts[2]):
        for terms in (False, True):
            kw = dict(bias=bias.cuda(), row_scale=scale.cuda(), residual=res.cuda()) if terms else {}
            new = lambda: torch.full((M, N), 9.0, dtype=torch.bfloat16, device="cuda")
            if mx:
                wq, ws = lx.quantize_mxfp4(W.cuda(), groups=E)
                xq, xs = lx.quantize_mxfp4(X.cuda(), off)
                call = lambda: lx.grouped_linear_mxfp4(xq, xs, off, wq.view(E, N, K // 2), ws, out=new(), **kw)
                assert torch.equal(lx.act_grouped_linear_mxfp4(X.cuda(), off, wq.view(E, N, K // 2), ws, out=new(), **kw), call())
            else:
                call = lambda: lx.grouped_linear(X.cuda(), off, W.cuda().view(E, N, K), out=new(), **kw)
            Y = call()
            assert all(torch.equal(call(), Y) for _ in range(5))
            y, mag = ref.grouped(x, w, offsets, *((scale.double().numpy(), f64(bias), f64(res)) if terms else ()))
            check(Y[inside], y[inside], mag[inside], K, (np.abs(f64(bias)).max(), f64(res)[inside]) if terms else ())
            assert (Y[:offsets[0]] == 9).all() and (Y[offsets[-1]:] == 9).all()


@pytest.mark.parametrize("M", [1, 3, 16, 40, 70, 200])
def test_split_products_repeat_bit_for_bit(contexts, M):
    """Long rows and few tiles: the parts of K come from four CTAs in any order and are added in one."""
    K, N = 3840, 520
    X, W = rand((M, K), 440).cuda(), rand((N, K), 441, K ** -0.5).cuda()
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    for lx in (contexts[0], contexts[2]):
        wq, ws = lx.quantize_mxfp4(W)
        xq, xs = lx.quantize_mxfp4(X)
        for call in (lambda: lx.linear_mxfp4(xq, xs, wq, ws), lambda: lx.act_linear_mxfp4(X, wq, ws), lambda: lx.grouped_linear(X, off, W[None])):
            first = call()
            assert all(torch.equal(call(), first) for _ in range(30))


@pytest.mark.parametrize("M,K", [(1, 32), (77, 1056), (300, 1056), (900, 704)])
def test_tiles_of_either_width_give_the_same_bits(contexts, M, K):
    """Where nothing splits K (bf16 up to 704, MXFP4 up to 2816) it is added in ascending order in every tile."""
    N = 392
    X, W = rand((M, K), 450).cuda(), rand((N, K), 451, K ** -0.5).cuda()
    off = torch.tensor([0, M // 2, M], dtype=torch.int32, device="cuda")
    wq, ws = contexts[0].quantize_mxfp4(W)
    xq, xs = contexts[0].quantize_mxfp4(X)
    Y = [lx.linear_mxfp4(xq, xs, wq, ws) for lx in contexts]
    assert torch.equal(Y[0], Y[1]) and torch.equal(Y[1], Y[2])
    if K <= 704:
        Y = [lx.grouped_linear(X, off, torch.stack([W, W])) for lx in contexts]
        assert torch.equal(Y[0], Y[1]) and torch.equal(Y[1], Y[2])


@pytest.mark.parametrize("M,K", [(1, 3840), (4, 3840), (40, 3840), (150, 3840), (150, 320)])
def test_result_over_its_residual(contexts, M, K):
    """In place, where K is split and where it is not, in one launch and in two."""
    N = 392
    X, W, res = rand((M, K), 460).cuda(), rand((2 * N, K), 461, K ** -0.5).cuda(), rand((M, N), 462).cuda()
    off = torch.tensor([0, M // 2, M], dtype=torch.int32, device="cuda")
    for lx in contexts:
        wq, ws = lx.quantize_mxfp4(W, groups=2)
        one, one_s = lx.quantize_mxfp4(W[:N])
        for call in (lambda **kw: lx.act_linear_mxfp4(X, one, one_s, **kw), lambda **kw: lx.grouped_linear(X, off, W.view(2, N, K), **kw),
                     lambda **kw: lx.act_grouped_linear_mxfp4(X, off, wq.view(2, N, K // 2), ws, **kw)):
            over = res.clone()
            assert call(residual=over, out=over) is over
            assert torch.equal(over, call(residual=res))


@pytest.mark.parametrize("M,K", [(2, 3840), (150, 320), (150, 3840)])
def test_factor_of_a_row_is_for_the_product_only(contexts, M, K):
    """With a factor of 0 the fp32 sum of bias and residual is left, to the bit."""
    N = 264
    X, W, bias, res = rand((M, K), 470).cuda(), rand((2 * N, K), 471).cuda(), rand((2, N), 472).cuda(), rand((M, N), 473).cuda()
    off, zero = torch.tensor([0, M // 2, M], dtype=torch.int32, device="cuda"), torch.zeros(M, device="cuda")
    one = (bias[0].double() + res.double()).float().to(torch.bfloat16)
    two = (bias[(torch.arange(M, device="cuda") >= M // 2).long()].double() + res.double()).float().to(torch.bfloat16)
    for lx in contexts:
        wq, ws = lx.quantize_mxfp4(W, groups=2)
        q, s = lx.quantize_mxfp4(W[:N])
        assert torch.equal(lx.act_linear_mxfp4(X, q, s, bias[0], res, zero), one)
        assert torch.equal(lx.linear_mxfp4(*lx.quantize_mxfp4(X), q, s, bias[0], zero, res), one)
        assert torch.equal(lx.grouped_linear(X, off, W.view(2, N, K), bias, zero, res), two)
        assert torch.equal(lx.act_grouped_linear_mxfp4(X, off, wq.view(2, N, K // 2), ws, bias, zero, res), two)

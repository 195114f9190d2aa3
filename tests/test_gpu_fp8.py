"""Block quantisation and linear layers in e4m3 against plain statements in 64 bits."""
import pytest
import torch

import paper_2506_02780_gb300 as E
from weights_util import (BLOCK, F8, STEP, blocks, blocks_value, make_rows, make_weights, quant_blocks, quant_rows,
                          rows_value, sum_bound)

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def acts(seed, n, c, spread=True):
    x = torch.randn(n, c, generator=gen(seed), device=DEV)
    if spread:      # blocks of very different size, down to bf16's denormals
        x *= torch.exp2(torch.randint(-140, 100, (n, blocks(c)), generator=gen(seed + 1), device=DEV).float()
                        ).repeat_interleave(BLOCK, 1)[:, :c]
    return x.to(torch.bfloat16)


def same_codes(q, want):
    got = q.double()
    assert torch.equal(got, want), (got != want).sum()


@pytest.mark.parametrize("n,c", [(1, 16), (1, 128), (3, 144), (8, 496), (9, 512), (17, 528), (130, 3584), (33, 7184)])
@pytest.mark.parametrize("spread", [False, True])
def test_rows(n, c, spread):
    """Codes are those of the exact quotient; scales are rounded once."""
    x = acts(n * 10000 + c, n, c, spread)
    q, s = torch.empty(n, c, dtype=F8, device=DEV), torch.empty(blocks(c), n, device=DEV)
    E.ee_fp8_quantize(x, q, s)
    wq, ws = quant_rows(x.double())
    same_codes(q, wq)
    assert ((s.double() - ws).abs() <= ws * 2.0 ** -24).all()


def test_rows_on_borders():
    """Quotients that are borders between two codes go to the even one, from any maximum that divides so."""
    rows = []
    for m in range(128, 256):                       # the significand of a bf16 maximum
        for j in range(0, 256, 15):
            rows.append([float(m)] + [float(v) for v in range(j, j + 15)])
    x = torch.tensor(rows, device=DEV).to(torch.bfloat16)
    q, s = torch.empty(*x.shape, dtype=F8, device=DEV), torch.empty(1, len(rows), device=DEV)
    E.ee_fp8_quantize(x, q, s)
    same_codes(q, quant_rows(x.double())[0])


def test_rows_of_a_wider_array_and_none():
    wide = acts(5, 40, 1024, False)
    x = wide[:, 256:256 + 144]
    q, s = torch.empty(40, 144, dtype=F8, device=DEV), torch.empty(2, 40, device=DEV)
    E.ee_fp8_quantize(x, q, s)
    same_codes(q, quant_rows(x.double())[0])
    E.ee_fp8_quantize(x[:0], q[:0], s[:, :0])


def test_rows_extremes():
    """Zeros, the least block, the largest number, infinities and NaN, each in a block of its own."""
    x = torch.zeros(6, 256, device=DEV)
    x[1, 3], x[1, 200] = 2.0 ** -120, -(2.0 ** -100)
    x[2, 0], x[2, 130] = 3.3895313892515355e38, 1e-30
    x[3, 5], x[3, 6] = float("inf"), 1.0
    x[4, 250] = float("nan")
    x[5, :] = -0.0
    x = x.to(torch.bfloat16)
    q, s = torch.empty(6, 256, dtype=F8, device=DEV), torch.empty(2, 6, device=DEV)
    E.ee_fp8_quantize(x, q, s)
    v = rows_value(q, s)
    assert (v[0] == 0).all() and (v[5] == 0).all() and torch.isfinite(s[:, [0, 1, 2, 5]]).all()
    # the scale is 2^-100 / 448 rounded once to fp32, and the block's largest code 448
    assert abs(s[0, 0].item() * 448 - 2.0 ** -100) <= 2.0 ** -124 and q[1, 200].float() == -448
    assert torch.equal(q[2].double(), quant_rows(x[2:3].double())[0][0])
    assert v[3, :128].isnan().all() and (v[3, 128:] == 0).all()
    assert v[4, 128:].isnan().all() and (v[4, :128] == 0).all()


@pytest.mark.parametrize("n,c", [(1, 16), (5, 208), (12, 1024), (67, 3600)])
def test_gated(n, c):
    x = acts(n + c, n, 2 * c, False) * 3
    x[0, :4] = torch.tensor([-100.0, 100.0, -88.0, 0.0], device=DEV)
    q, s = torch.empty(n, c, dtype=F8, device=DEV), torch.empty(blocks(c), n, device=DEV)
    E.ee_fp8_quantize(x, q, s, gated=True)
    g, u = x.double().chunk(2, 1)
    h = g * torch.sigmoid(g) * u
    _, ws = quant_rows(h)
    # silu * up in fp32: exponent (error 2 + |g| 2^-23 / ln 2 steps, |g| <= 20 in effect), sum, quotient (2), product
    err = 40 * 2.0 ** -23
    assert ((s.double() - ws).abs() <= ws * (err + 2.0 ** -24)).all()
    # a code is within half a step (2^-4 relative, or half the least step 2^-9) of what it stands for
    v, sc = rows_value(q, s), ws.t().repeat_interleave(BLOCK, 1)[:, :c]
    assert ((v - h).abs() <= torch.maximum(h.abs() * 2.0 ** -4, sc * 2.0 ** -10) * (1 + 1e-4) + h.abs() * err).all()


@pytest.mark.parametrize("shape", [(1, 16), (128, 128), (129, 144), (100, 272), (3, 200, 400), (2, 2, 130, 512)])
def test_weights(shape):
    w = (torch.randn(shape, generator=gen(sum(shape)), device=DEV) * 0.02).to(torch.bfloat16)
    lead, (r, c) = shape[:-2], shape[-2:]
    q, s = torch.empty(shape, dtype=F8, device=DEV), torch.empty(*lead, blocks(r), blocks(c), device=DEV)
    E.ee_fp8_quantize_weights(w, q, s)
    wq, ws = quant_blocks(w.double())
    same_codes(q, wq)
    assert ((s.double() - ws).abs() <= ws * 2.0 ** -24).all()


# ---------------------------------------------------------------- linear layers

@pytest.fixture(scope="module")
def ws():
    return E.new_linear_workspace()


def reference(x, xs, w, wsc, bias):
    """(fp64 result, bound on the error before the last rounding)."""
    xv, wv = rows_value(x, xs), blocks_value(w, wsc)
    y = xv @ wv.t()
    err = (xv.abs() @ wv.abs().t()) * sum_bound(x.shape[1])
    if bias is not None:
        y = y + bias.double()
        err = err + y.abs() * 2.0 ** -24
    return y, err


def check_linear(out, x, xs, w, wsc, bias):
    y, err = reference(x, xs, w, wsc, bias)
    bad = (out.double() - y).abs() > (y.abs() + err) * STEP + err
    assert not bad.any(), (int(bad.sum()), float((out.double() - y).abs().max()))


LINEAR = [(10, 400, 37), (14, 3584, 1500), (12, 2064, 20000), (1, 16, 1), (1, 128, 8), (1, 3584, 3584), (2, 112, 100), (7, 256, 128), (8, 144, 129), (9, 272, 257),
          (16, 1040, 384), (33, 3584, 512), (63, 400, 1000), (64, 3584, 4608), (65, 384, 255), (127, 512, 131),
          (128, 896, 640), (129, 896, 640), (200, 2064, 20000), (300, 128, 40), (534, 1536, 3584), (700, 640, 9000),
          (1025, 272, 5121), (2048, 512, 4096)]


@pytest.mark.parametrize("n,K,N", LINEAR)
def test_linear(ws, n, K, N):
    g = gen(n * 7 + K + N)
    x, xs = make_rows(g, n, K)
    w, wsc = make_weights(g, N, K)
    bias = torch.randn(N, generator=g, device=DEV).to(torch.bfloat16) if (n + N) % 2 else None
    out = torch.full((n, N), 7.0, dtype=torch.bfloat16, device=DEV)
    E.ee_fp8_linear(x, xs, w, wsc, out, ws, bias=bias)
    check_linear(out, x, xs, w, wsc, bias)
    again = torch.empty_like(out)
    E.ee_fp8_linear(x, xs, w, wsc, again, ws, bias=bias)
    assert torch.equal(out, again)
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("n,K,N,wide,at", [(5, 256, 130, 200, 3), (64, 512, 128, 512, 128), (300, 256, 512, 1031, 8),
                                           (150, 384, 77, 77, 0)])
def test_linear_into_wider_rows(ws, n, K, N, wide, at):
    """Output rows at any alignment; what is beside them stays."""
    g = gen(n + K + N)
    x, xs = make_rows(g, n, K)
    w, wsc = make_weights(g, N, K)
    whole = torch.full((n, wide), 3.0, dtype=torch.bfloat16, device=DEV)
    E.ee_fp8_linear(x, xs, w, wsc, whole[:, at:at + N], ws)
    check_linear(whole[:, at:at + N], x, xs, w, wsc, None)
    rest = torch.cat([whole[:, :at], whole[:, at + N:]], 1)
    assert (rest == 3.0).all()


def test_linear_rows_are_their_own(ws):
    """A token's output depends on that token alone: NaN and infinities stay in their rows, and NaN
    weights in their columns."""
    g = gen(11)
    for n, N in [(40, 300), (300, 700), (8, 40000)]:
        x, xs = make_rows(g, n, 512)
        w, wsc = make_weights(g, N, 512)
        clean = torch.empty(n, N, dtype=torch.bfloat16, device=DEV)
        E.ee_fp8_linear(x, xs, w, wsc, clean, ws)
        x2, xs2, w2 = x.clone(), xs.clone(), w.clone()
        x2.view(torch.uint8)[3, 100] = 0x7f
        xs2[1, 5] = float("inf")
        w2.view(torch.uint8)[37, 200] = 0xff
        out = torch.empty_like(clean)
        E.ee_fp8_linear(x2, xs2, w2, wsc, out, ws)
        keep = torch.ones(n, N, dtype=torch.bool, device=DEV)
        keep[3], keep[5], keep[:, 37] = False, False, False
        assert out[3].isnan().all() and not out[5].isfinite().any() and out[:, 37].isnan().all()
        assert torch.equal(out[keep], clean[keep])


def test_linear_streams_and_graphs(ws):
    """Quantise and multiply on another stream and replayed from a graph, with new inputs between replays."""
    g = gen(4)
    n, K, N = 64, 1024, 2000
    w, wsc = make_weights(g, N, K)
    x = acts(3, n, K, False)
    q, s = torch.empty(n, K, dtype=F8, device=DEV), torch.empty(blocks(K), n, device=DEV)
    out = torch.empty(n, N, dtype=torch.bfloat16, device=DEV)

    def step():
        E.ee_fp8_quantize(x, q, s)
        E.ee_fp8_linear(q, s, w, wsc, out, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    check_linear(out, q, s, w, wsc, None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        step()
    for seed in (8, 9):
        x.copy_(acts(seed, n, K, False))
        graph.replay()
        want = quant_rows(x.double())[0]
        same_codes(q, want)
        check_linear(out, q, s, w, wsc, None)
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n,c", [(2500, 1040), (700, 4624), (4100, 16)])
def test_many_rows(n, c, gated):
    """Sizes that fill the GPU, with rows and columns that end inside a CTA's."""
    x = acts(n + c, n, 2 * c if gated else c, False)
    q, s = torch.empty(n, c, dtype=F8, device=DEV), torch.empty(blocks(c), n, device=DEV)
    E.ee_fp8_quantize(x, q, s, gated=gated)
    if not gated:
        wq, want = quant_rows(x.double())
        same_codes(q, wq)
        assert ((s.double() - want).abs() <= want * 2.0 ** -24).all()
        return
    g, u = x.double().chunk(2, 1)
    h = g * torch.sigmoid(g) * u
    _, want = quant_rows(h)
    err = 40 * 2.0 ** -23                               # (as in test_gated: |g| <= 20 here as well)
    assert ((s.double() - want).abs() <= want * (err + 2.0 ** -24)).all()
    v, sc = rows_value(q, s), want.t().repeat_interleave(BLOCK, 1)[:, :c]
    assert ((v - h).abs() <= torch.maximum(h.abs() * 2.0 ** -4, sc * 2.0 ** -10) * (1 + 1e-4) + h.abs() * err).all()

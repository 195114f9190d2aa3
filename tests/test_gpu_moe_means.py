"""Expert layers held to the mean error of one rounding (``check_given``), where the worst-case bound of a sum would let a
wrong result pass: the few-entry kernel at every depth of its weight rings, live tokens, wider rows, shared workspaces, graphs."""
import os
import re

import pytest
import torch

import paper_2506_02780_gb300 as E
import test_gpu_moe as M
from weights_util import blocks_value, quant_rows, rows_value

DEV = "cuda"
gpu = pytest.mark.gpu


def _few_constants():
    """The kernel's own numbers: what is asserted about depths below follows them."""
    csrc = os.path.join(os.path.dirname(E.__file__), "csrc")
    text = "".join(open(os.path.join(csrc, f)).read() for f in ("moe_few.cu", "moe.cuh", "few.cuh"))
    def value(name):
        return eval(re.search(rf"constexpr \w+ [^;]*\b{name} = ([0-9 *]+)[;,]", text).group(1))
    return {n: value(n) for n in ("kGroups", "kMaxDeep", "kMinDeep", "kMostSmem", "kFewWarps", "kFewEntries")}


def few_depth(T, H, I, k, fp8):
    """Stages of the few-entry kernel's rings, or 0 where the tiles take the call: rows of x, later of h, in shared memory
    with 64 bytes between them and a float for each block, and behind two rings of 16 rows of up to 8 blocks a stage."""
    c = _few_constants()
    if T * k > c["kFewEntries"]:
        return 0
    kb = [-(-n * (1 if fp8 else 2) // 128) for n in (H, I)]
    wide = max(-(-b // -(-b // c["kFewWarps"])) for b in kb)
    rows = max(T * (kb[0] * 132 + 64), T * k * (kb[1] * 132 + 64))
    room = c["kMostSmem"] - 128 - rows
    depth = room // (c["kGroups"] * 16 * 128 * wide) if room > 0 else 0
    return min(depth, c["kMaxDeep"]) if depth >= c["kMinDeep"] else 0


# T, H, I, E, k, 8-bit, depth: h in the way (long I) and x (long H), the last size that fits and the first that does not
DEPTHS = [(1, 3584, 2560, 8, 8, False, 5), (8, 3584, 2560, 12, 1, False, 4), (1, 272, 4688, 10, 8, False, 3),
          (2, 272, 6656, 9, 4, False, 3), (2, 272, 6672, 9, 4, False, 0), (8, 4704, 144, 5, 1, False, 3), (8, 6656, 144, 5, 1, False, 3),
          (8, 6672, 144, 5, 1, False, 0), (1, 37648, 272, 3, 1, False, 3), (1, 272, 53504, 2, 1, False, 3),
          (1, 272, 4368, 9, 8, True, 5), (8, 272, 6288, 5, 1, True, 4), (2, 272, 9360, 6, 4, True, 3), (1, 272, 13312, 8, 8, True, 3),
          (1, 272, 13328, 8, 8, True, 0), (4, 11664, 400, 6, 2, True, 4), (8, 9360, 272, 4, 1, True, 3), (8, 13312, 272, 4, 1, True, 3),
          (8, 13328, 272, 4, 1, True, 0), (1, 272, 43408, 2, 1, True, 4), (3, 528, 400, 16, 2, True, 6)]


@pytest.mark.parametrize("T,H,I,n_exp,k,fp8,depth", DEPTHS)
def test_depths_as_listed(T, H, I, n_exp, k, fp8, depth):
    assert few_depth(T, H, I, k, fp8) == depth


@gpu
@pytest.mark.parametrize("T,H,I,n_exp,k,fp8,depth", DEPTHS)
def test_every_depth(T, H, I, n_exp, k, fp8, depth):
    m = M.Layer(T, H, I, n_exp, k, fp8, seed=60)
    live = torch.tensor([T], dtype=torch.int32, device=DEV)
    for renorm, n in ((True, T), (False, T), (True, (T + 1) // 2)):
        live.fill_(n)
        m.clear()
        m.run(renorm, live)
        assert E.ee_read_errors(m.ws) == 0
        m.check(renorm, n)
        m.check_given(n)


@gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,H,I,n_exp,k", [(1, 64, 16384, 8, 8), (8, 16384, 64, 3, 1), (8, 32768, 64, 3, 1), (1, 64, 32768, 9, 8)])
def test_long_rows(T, H, I, n_exp, k, fp8):
    m = M.Layer(T, H, I, n_exp, k, fp8, seed=61)
    m.run(True)
    m.check_given()


@gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,n_exp,k,live", [(40, 8, 2, 1), (40, 8, 2, 17), (40, 8, 2, 40), (40, 8, 2, 99), (700, 8, 2, 513),
                                            (4, 24, 2, 1), (4, 24, 2, 3), (2, 130, 4, 1), (40, 24, 2, 17), (40, 130, 3, 16),
                                            (200, 130, 2, 37), (700, 130, 2, 513), (700, 24, 2, 1), (2500, 8, 2, 900)])
def test_live_tokens(T, n_exp, k, live, fp8):
    m = M.Layer(T, 272, 208, n_exp, k, fp8, seed=62 + live)
    n = min(T, live)
    m.x[n:] = float("nan")
    m.run(True, torch.tensor([live], dtype=torch.int32, device=DEV))
    assert E.ee_read_errors(m.ws) == 0
    m.check(True, n)
    m.check_given(n)


@gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_wider_rows(fp8):
    m = M.Layer(37, 400, 144, 8, 3, fp8, seed=63, wide=48)
    for at, wide in [(4, 412), (3, 407)]:
        m.out = torch.full((37, wide), 7.0, dtype=torch.bfloat16, device=DEV)[:, at:at + 400]
        m.run()
        m.check_given()


@gpu
def test_one_workspace():
    sizes = [(2500, 8, 2), (3, 24, 2), (64, 24, 4), (700, 24, 2), (1, 8, 8), (300, 130, 2), (16, 8, 2), (700, 130, 3)]
    layers = [M.Layer(T, 272, 80, n, k, i % 2 == 0, seed=64 + i) for i, (T, n, k) in enumerate(sizes)]
    ws = E.new_moe_workspace(2500, 272, 80, 130, 8)
    for n_of in (lambda T: T, lambda T: (T + 1) // 2, lambda T: T):
        for m in layers:
            m.ws = ws
            m.clear()
            m.run(True, torch.tensor([n_of(m.T)], dtype=torch.int32, device=DEV))
            m.check_given(n_of(m.T))
    assert E.ee_read_errors(ws) == 0


@gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,n_exp,k", [(48, 16, 4), (2, 16, 4)])
def test_graphs(T, n_exp, k, fp8):
    a, b = M.Layer(T, 512, 256, n_exp, k, fp8, seed=80), M.Layer(T, 512, 256, n_exp, k, fp8, seed=81)
    b.ws = a.ws
    live = torch.tensor([T], dtype=torch.int32, device=DEV)
    a.run(True, live)
    b.run(False, live)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(True, live)
        b.run(False, live)
    for n in (T, 1, (T + 1) // 2):
        a.x.copy_(torch.randn(T, 512, generator=M.gen(n), device=DEV))
        live.fill_(n)
        for m in (a, b):
            m.out.fill_(7.0), m.ids.fill_(-1), m.p.fill_(-2.0)
        graph.replay()
        for m, renorm in ((a, True), (b, False)):
            m.check(renorm, n)
            m.check_given(n)


# ---------------------------------------------------------------- the oracle itself (CPU)

def plain(m, renorm):
    """The layer in 32 bits: what a right kernel returns, up to the order of its sums."""
    x = m.x.float()
    logits = x @ m.router.float().t()
    order = logits.sort(dim=1, descending=True, stable=True).indices[:, :m.k].sort(1).values
    l = logits.gather(1, order)
    p = torch.exp(l - torch.logsumexp(l if renorm else logits, 1, keepdim=True))
    xv = rows_value(*[t.float() for t in quant_rows(x.double())]).float() if m.fp8 else x
    y = torch.zeros(m.T, m.H)
    I = m.I
    for e in range(m.E):
        tok, j = torch.nonzero(order == e, as_tuple=True)
        if not len(tok):
            continue
        w1, w2 = m.w1[e], m.w2[e]
        if m.fp8:
            w1 = torch.cat([blocks_value(w1[:I], m.s1[e, 0]), blocks_value(w1[I:], m.s1[e, 1])])
            w2 = blocks_value(w2, m.s2[e])
        g, u = (xv[tok] @ w1.float().t()).chunk(2, 1)
        h = M.silu(g) * u
        h = rows_value(*[t.float() for t in quant_rows(h.double())]).float() if m.fp8 else h.to(torch.bfloat16).float()
        y[tok] += (h @ w2.float().t()) * p[tok, j][:, None]
    return y, order.to(torch.int32), p


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,H,I,n_exp,k", [(1, 64, 16384, 8, 8), (8, 16384, 64, 3, 1), (40, 272, 208, 8, 2), (48, 512, 256, 16, 4),
                                           (1, 3584, 400, 8, 8), (2, 272, 6656, 4, 4), (8, 13312, 272, 4, 1), (37, 400, 144, 8, 3),
                                           (300, 272, 80, 30, 2), (2, 272, 80, 24, 2)])
def test_the_mean_tells_right_from_wrong(monkeypatch, T, H, I, n_exp, k, fp8):
    """check_given takes what 32 bits give and no result that is two percent off, has another sign or stands elsewhere."""
    monkeypatch.setattr(M, "DEV", "cpu")
    monkeypatch.setattr(E, "new_moe_workspace", lambda *a, **kw: None)
    m = M.Layer(T, H, I, n_exp, k, fp8, seed=90)
    y, m.ids, m.p = plain(m, True)
    m.out = y.to(torch.bfloat16)
    m.check_given()
    for wrong in (y * 0, -y, 0.98 * y, 1.02 * y, y.roll(1, 1), y.roll(1, 0) if T > 1 else -y):
        m.out = wrong.to(torch.bfloat16)
        with pytest.raises(AssertionError):
            m.check_given()

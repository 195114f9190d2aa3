"""Mixture-of-experts layers against a plain statement in 64 bits."""
import pytest
import torch

import paper_2506_02780_gb300 as E
from weights_util import (BLOCK, STEP, blocks, blocks_value, make_weights, quant_rows, rows_value, sum_bound)

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def silu(g):
    return g * torch.sigmoid(g)


class Layer:
    """Inputs of one layer, and its output in 64 bits with a bound on the error before the last rounding."""

    def __init__(self, T, H, I, n_exp, k, fp8, seed=0, wide=0):
        g = gen(seed * 1000003 + T * 31 + H + I + n_exp + k)
        self.T, self.H, self.I, self.E, self.k, self.fp8 = T, H, I, n_exp, k, fp8
        x = torch.randn(T, H + wide, generator=g, device=DEV).to(torch.bfloat16)
        self.x = x[:, wide // 2:wide // 2 + H]
        self.router = (torch.randn(n_exp, H, generator=g, device=DEV) * (4.0 / H ** 0.5)).to(torch.bfloat16)
        self.s1 = self.s2 = None
        if fp8:
            self.w1, self.s1 = make_weights(g, n_exp, 2, I, H)
            self.w1 = self.w1.view(n_exp, 2 * I, H)
            self.w2, self.s2 = make_weights(g, n_exp, H, I)
        else:
            self.w1 = (torch.randn(n_exp, 2 * I, H, generator=g, device=DEV) * 0.02).to(torch.bfloat16)
            self.w2 = (torch.randn(n_exp, H, I, generator=g, device=DEV) * 0.02).to(torch.bfloat16)
        self.ws = E.new_moe_workspace(T, H, I, n_exp, k)
        self.clear()

    def clear(self):
        self.out = torch.full((self.T, self.H), 7.0, dtype=torch.bfloat16, device=DEV)
        self.ids = torch.full((self.T, self.k), -1, dtype=torch.int32, device=DEV)
        self.p = torch.full((self.T, self.k), -2.0, device=DEV)

    def run(self, renorm=False, live=None):
        E.ee_moe_layer(self.x, self.router, self.w1, self.w2, self.k, self.out, self.ws, w1_scale=self.s1,
                       w2_scale=self.s2, renorm=renorm, live=live, ids=self.ids, probs=self.p)

    def check(self, renorm=False, live=None):
        n, k, I = self.T if live is None else live, self.k, self.I
        assert (self.out[n:] == 7.0).all() and (self.ids[n:] == -1).all() and (self.p[n:] == -2.0).all()
        if n == 0:
            return
        x = self.x[:n].double()
        logits = x @ self.router.double().t()
        # a logit's fp32 sum: at most H additions of products, an error of one step each
        lerr = (x.abs() @ self.router.double().abs().t()) * ((self.H + 16) * 2.0 ** -23)
        ids = self.ids[:n].long()
        assert (ids[:, 1:] > ids[:, :-1]).all() and (ids >= 0).all() and (ids < self.E).all()
        # the choice is right up to that error: no expert left out is clearly above one taken
        taken = torch.zeros(n, self.E, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
        low = torch.where(taken, logits + lerr, torch.inf).amin(1)
        high = torch.where(taken, -torch.inf, logits - lerr).amax(1)
        assert (high <= low).all()
        l, le = logits.gather(1, ids), lerr.amax(1, keepdim=True)
        den = torch.logsumexp(l if renorm else logits, 1, keepdim=True)
        p = torch.exp(l - den)
        # both logits, the exponential's argument (|l| 2^-24 below 2^-18) and value, the sum, the quotient
        perr = 2 * le + 2.0 ** -17 + (self.E + 8) * 2.0 ** -23
        assert ((self.p[:n].double() - p).abs() <= p * perr).all()
        y = torch.zeros(n, self.H, dtype=torch.float64, device=DEV)
        err = torch.zeros_like(y)
        xv = x
        if self.fp8:
            q, s = quant_rows(x)
            xv = rows_value(q, s.float())
        b1, b2 = sum_bound(self.H) + 2.0 ** -23, sum_bound(I) + 2.0 ** -23
        for e in range(self.E):
            tok, j = torch.nonzero(ids == e, as_tuple=True)
            if not len(tok):
                continue
            w1, w2 = self.w1[e], self.w2[e]
            if self.fp8:
                wg, wu = blocks_value(w1[:I], self.s1[e, 0]), blocks_value(w1[I:], self.s1[e, 1])
                w2 = blocks_value(w2, self.s2[e])
            else:
                wg, wu, w2 = w1[:I].double(), w1[I:].double(), w2.double()
            xe = xv[tok]
            g, u = xe @ wg.t(), xe @ wu.t()
            ge, ue = (xe.abs() @ wg.abs().t()) * b1, (xe.abs() @ wu.abs().t()) * b1
            h = silu(g) * u
            # |silu'| <= 1.1; silu * up itself in fp32: 40 steps of 2^-23 (|g| <= 20 in effect)
            he = 1.1 * ge * (u.abs() + ue) + silu(g).abs() * ue + h.abs() * 40 * 2.0 ** -23
            if self.fp8:
                a = torch.nn.functional.pad(h.abs() + he, (0, -I % BLOCK)).view(len(tok), -1, BLOCK).amax(-1)
                a = a.repeat_interleave(BLOCK, 1)[:, :I]
                # h and what the codes stand for: half a step of e4m3, 2^-4 relative or 2^-10 of the largest's scale
                he = he + torch.maximum((h.abs() + he) * 2.0 ** -4, a / 448 * 2.0 ** -10) * (1 + 2.0 ** -20)
            else:
                he = he + (h.abs() + he) * 2.0 ** -8
            ye = h @ w2.t()
            yerr = he @ w2.abs().t() + ((h.abs() + he) @ w2.abs().t()) * b2
            pe = p[tok, j][:, None]
            y[tok] += ye * pe
            err[tok] += yerr * pe + ye.abs() * pe * (perr[tok] + (k + 1) * 2.0 ** -24)
        bad = (self.out[:n].double() - y).abs() > (y.abs() + err) * STEP + err
        assert not bad.any(), (int(bad.sum()), float((self.out[:n].double() - y).abs().max()))

    def check_given(self, n=None):
        """Closer: the second product's error against the kernel's own rounding of h is not visible from outside,
        so the mean error, in which roundings to either side cancel, is held against a statement that rounds h
        as the kernel does.  A value of h next to a border between two codes may fall on either side: the
        share of such values is small, so the outputs' mean error is that of their own rounding."""
        n = self.T if n is None else n
        x = self.x[:n].double()
        xv = x
        if self.fp8:
            q, s = quant_rows(x)
            xv = rows_value(q, s.float())
        y = torch.zeros(n, self.H, dtype=torch.float64, device=DEV)
        ids, I = self.ids[:n].long(), self.I
        for e in range(self.E):
            tok, j = torch.nonzero(ids == e, as_tuple=True)
            if not len(tok):
                continue
            w1, w2 = self.w1[e], self.w2[e]
            if self.fp8:
                wg, wu = blocks_value(w1[:I], self.s1[e, 0]), blocks_value(w1[I:], self.s1[e, 1])
                w2 = blocks_value(w2, self.s2[e])
            else:
                wg, wu, w2 = w1[:I].double(), w1[I:].double(), w2.double()
            h = silu(xv[tok] @ wg.t()) * (xv[tok] @ wu.t())
            h = rows_value(*quant_rows(h)) if self.fp8 else h.to(torch.bfloat16).double()
            y[tok] += (h @ w2.t()) * self.p[tok, j].double()[:, None]
        # half a bf16 step of each value at most; half as much again for values of h on the other side of a border
        diff = (self.out[:n].double() - y).abs().sum()
        assert diff <= 1.5 * STEP * y.abs().sum(), (float(diff), float(y.abs().sum()))


# T, H, I, E, k
SIZES = [(1, 16, 16, 1, 1), (8, 528, 208, 16, 3), (3, 400, 2064, 5, 2), (8, 272, 1296, 24, 16), (8, 3584, 1280, 64, 6),
         (6, 640, 144, 200, 16), (65, 256, 128, 2, 2), (150, 272, 144, 5, 2), (180, 528, 400, 3, 1), (12, 400, 272, 30, 4), (9, 1040, 528, 256, 16), (15, 256, 2048, 6, 5), (16, 272, 16, 16, 16), (1, 528, 208, 8, 2), (1, 1024, 256, 64, 6), (2, 256, 128, 8, 8), (5, 272, 144, 9, 3),
         (16, 528, 208, 8, 2), (17, 640, 320, 60, 4), (33, 384, 112, 256, 16), (64, 1024, 384, 16, 4),
         (130, 512, 256, 4, 2), (200, 272, 80, 2, 1), (300, 400, 272, 1, 1), (576, 1536, 640, 64, 6),
         (1000, 256, 128, 130, 8), (4096, 144, 48, 3, 2), (4096, 16, 16, 256, 16)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,H,I,n_exp,k", SIZES)
def test_layer(T, H, I, n_exp, k, fp8):
    m = Layer(T, H, I, n_exp, k, fp8)
    renorm = (T + I // 16) % 2 == 0
    m.run(renorm)
    assert E.ee_read_errors(m.ws) == 0
    m.check(renorm)
    m.check_given()
    first = m.out.clone(), m.ids.clone(), m.p.clone()
    m.clear()
    m.run(renorm)
    assert torch.equal(first[0], m.out) and torch.equal(first[1], m.ids) and torch.equal(first[2], m.p)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,live", [(40, 0), (40, 1), (40, 17), (40, 40), (40, 99), (40, -3), (700, 513)])
def test_live_tokens(T, live, fp8):
    """Tokens behind the live ones change nothing and keep their rows, whatever they hold."""
    m = Layer(T, 272, 208, 8, 2, fp8, seed=live + 10)
    n = max(0, min(T, live))
    m.x[n:] = float("nan")
    m.run(True, torch.tensor([live], dtype=torch.int32, device=DEV))
    assert E.ee_read_errors(m.ws) == 0
    m.check(True, n)


@pytest.mark.parametrize("T,n_exp,k,live", [(4, 24, 2, 0), (4, 24, 2, 1), (4, 24, 2, 3), (2, 130, 4, 1), (40, 24, 2, 0),
                                            (40, 24, 2, 17), (40, 130, 3, 16), (200, 130, 2, 0), (200, 130, 2, 37),
                                            (700, 130, 2, 513), (700, 24, 2, 1), (2500, 8, 2, 900)])
def test_live_tokens_by_experts(T, n_exp, k, live):
    """The same where several CTAs share a token's experts, and for few entries."""
    m = Layer(T, 272, 80, n_exp, k, True, seed=live + 20)
    m.x[live:] = float("nan")
    m.run(True, torch.tensor([live], dtype=torch.int32, device=DEV))
    assert E.ee_read_errors(m.ws) == 0
    m.check(True, live)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,H,I,n_exp,k", [(1, 64, 16384, 8, 8), (8, 16384, 64, 3, 1), (8, 32768, 64, 3, 1), (1, 64, 32768, 9, 8)])
def test_few_entries_of_long_rows(T, H, I, n_exp, k, fp8):
    """Few entries whose rows do, or do not, fit in shared memory beside the weights' rings."""
    m = Layer(T, H, I, n_exp, k, fp8, seed=50)
    m.run()
    assert E.ee_read_errors(m.ws) == 0
    m.check()


def test_one_workspace_for_all_sizes():
    """Calls of any sizes after one another on one workspace: counts are left as the next call needs them."""
    sizes = [(2500, 8, 2), (3, 24, 2), (64, 24, 4), (700, 24, 2), (1, 8, 8), (300, 130, 2), (16, 8, 2), (700, 130, 3)]
    layers = [Layer(T, 272, 80, n, k, i % 2 == 0, seed=30 + i) for i, (T, n, k) in enumerate(sizes)]
    ws = E.new_moe_workspace(2500, 272, 80, 130, 8)
    for turn in range(3):
        for m in layers:
            m.ws = ws
            m.clear()
            m.run(True, torch.tensor([m.T if turn != 1 else m.T // 2], dtype=torch.int32, device=DEV))
            m.check(True, m.T if turn != 1 else m.T // 2)
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("T,n_exp", [(2, 12), (40, 12), (40, 200), (1000, 200)])
def test_equal_logits_in_any_share(T, n_exp):
    """Equal logits go to the lowest experts, a NaN logit is the last choice, wherever an expert's logit was summed."""
    m = Layer(T, 256, 32, n_exp, 3, False, seed=40)
    m.x.abs_()
    best = [1, 6, n_exp - 5, n_exp - 2]
    m.router[best] = m.router[1].abs() + 1.0
    m.run(True)
    assert (m.ids == torch.tensor(best[:3], dtype=torch.int32, device=DEV)).all()
    m.router[6] = float("nan")
    m.run(True)
    assert (m.ids == torch.tensor([1, n_exp - 5, n_exp - 2], dtype=torch.int32, device=DEV)).all()
    assert ((m.p - 1.0 / 3).abs() <= 2.0 ** -22).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_rows_of_wider_arrays(fp8):
    m = Layer(37, 400, 144, 8, 3, fp8, seed=3, wide=48)
    for at, wide in [(4, 412), (3, 407)]:
        whole = torch.full((37, wide), 7.0, dtype=torch.bfloat16, device=DEV)
        m.out = whole[:, at:at + 400]
        m.run()
        m.check()
        assert (whole[:, :at] == 7.0).all() and (whole[:, at + 400:] == 7.0).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_all_tokens_at_one_expert(fp8):
    """Several token tiles of one expert, and experts that nobody chose."""
    m = Layer(333, 256, 272, 16, 2, fp8, seed=5)
    m.router[3] = m.router[3].abs() + 0.5
    m.router[9] = m.router[9].abs() + 0.1
    m.x.abs_()
    m.run()
    assert (m.ids[:, 0] == 3).all() and (m.ids[:, 1] == 9).all()
    m.check()
    m.check_given()


def test_equal_logits_and_nan():
    """Equal logits go to the lowest experts; a NaN logit is the last choice."""
    m = Layer(9, 256, 64, 12, 3, False, seed=6)
    m.router[4:10] = m.router[4]
    m.x.abs_()
    m.router[4:10] = m.router[4:10].abs() + 1.0
    m.run(True)
    assert (m.ids == torch.tensor([4, 5, 6], dtype=torch.int32, device=DEV)).all()
    assert ((m.p - 1.0 / 3).abs() <= 2.0 ** -22).all()
    m.router[5] = float("nan")
    m.run(True)
    assert (m.ids == torch.tensor([4, 6, 7], dtype=torch.int32, device=DEV)).all()
    m.router[:] = float("nan")
    m.run(True)
    assert (m.ids == torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)).all() and m.p.isnan().all()
    assert m.out.isnan().all() and E.ee_read_errors(m.ws) == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_tokens_are_their_own(fp8):
    """A token with a NaN or an infinity is NaN; its neighbours are what they were."""
    m = Layer(70, 528, 208, 8, 2, fp8, seed=7)
    m.run()
    clean, ids = m.out.clone(), m.ids.clone()
    m.x[11, 100], m.x[40, 5] = float("nan"), float("inf")
    m.run()
    keep = torch.ones(70, dtype=torch.bool, device=DEV)
    keep[11] = keep[40] = False
    assert torch.equal(m.out[keep], clean[keep]) and torch.equal(m.ids[keep], ids[keep])
    assert m.out[11].isnan().all() and m.out[40].isnan().all()


@pytest.mark.parametrize("fp8", [False, True])
def test_streams_and_graphs(fp8):
    """Two layers on one workspace, on another stream and replayed from a graph with new inputs and live counts."""
    a, b = Layer(48, 512, 256, 16, 4, fp8, seed=8), Layer(48, 512, 256, 16, 4, fp8, seed=9)
    b.ws = a.ws
    live = torch.tensor([48], dtype=torch.int32, device=DEV)

    def step():
        a.run(True, live)
        b.run(False, live)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    a.check(True)
    b.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in (48, 5, 31):
        a.x.copy_(torch.randn(48, 512, generator=gen(n), device=DEV))
        live.fill_(n)
        for m in (a, b):
            m.out.fill_(7.0), m.ids.fill_(-1), m.p.fill_(-2.0)
        graph.replay()
        a.check(True, n)
        b.check(False, n)
    assert E.ee_read_errors(a.ws) == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_two_streams_at_once(fp8):
    """Calls with workspaces of their own on two streams, each many times, share the SMs."""
    ms = [Layer(96, 1024, 512, 32, 4, fp8, seed=s) for s in (1, 2)]
    want = []
    for m in ms:
        m.run()
        want.append(m.out.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ms]
    for _ in range(20):
        for m, s in zip(ms, streams):
            with torch.cuda.stream(s):
                m.run()
    torch.cuda.synchronize()
    for m, w in zip(ms, want):
        assert torch.equal(m.out, w) and E.ee_read_errors(m.ws) == 0


def test_a_pass_of_weight_products():
    """A target layer's products as they are used: quantise, project, run the experts on the result, and
    a gated linear pair beside them."""
    g = gen(12)
    T, H, I = 64, 512, 256
    m = Layer(T, H, I, 8, 2, True, seed=12)
    ws = E.new_linear_workspace()
    x = torch.randn(T, H, generator=g, device=DEV).to(torch.bfloat16)
    f8 = torch.float8_e4m3fn
    wraw = [(torch.randn(n, c, generator=g, device=DEV) * 0.05).to(torch.bfloat16) for n, c in
            [(H, H), (2 * I, H), (H, I)]]
    codes = [(torch.empty_like(w, dtype=f8), torch.empty(blocks(w.shape[0]), blocks(w.shape[1]), device=DEV)) for w in wraw]
    for w, (q, s) in zip(wraw, codes):
        E.ee_fp8_quantize_weights(w, q, s)
    q, s = torch.empty(T, H, dtype=f8, device=DEV), torch.empty(blocks(H), T, device=DEV)
    hq, hs = torch.empty(T, I, dtype=f8, device=DEV), torch.empty(blocks(I), T, device=DEV)
    gu, dense = (torch.empty(T, n, dtype=torch.bfloat16, device=DEV) for n in (2 * I, H))
    E.ee_fp8_quantize(x, q, s)
    E.ee_fp8_linear(q, s, *codes[0], m.x, ws)
    m.run(True)
    E.ee_fp8_quantize(m.x, q, s)
    E.ee_fp8_linear(q, s, *codes[1], gu, ws)
    E.ee_fp8_quantize(gu, hq, hs, gated=True)
    E.ee_fp8_linear(hq, hs, *codes[2], dense, ws)
    xv = rows_value(*quant_rows(x.double()))
    mid = xv @ blocks_value(*codes[0]).t()
    assert ((m.x.double() - mid).abs() <= mid.abs() * STEP + (xv.abs() @ blocks_value(*codes[0]).abs().t())
            * (sum_bound(H) + 2.0 ** -23) * (1 + STEP)).all()
    m.check(True)
    got = gu.double()
    hv = silu(got[:, :I]) * got[:, I:]
    want = rows_value(*quant_rows(hv)) @ blocks_value(*codes[2]).t()
    assert (dense.double() - want).abs().sum() <= 1.5 * STEP * want.abs().sum()
    assert E.ee_read_errors(ws) == 0 and E.ee_read_errors(m.ws) == 0

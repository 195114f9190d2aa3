"""A target layer's weight products as classes, and a whole layer with them: projections, attention over
the paged cache, experts, captured into a graph."""
import pytest
import torch

import paper_2506_02780_gb300 as E
from paper_2506_02780_gb300.layers import BlockLinear, Experts, quantize_weights
from paper_2506_02780_gb300.prompt import PromptIntake, rope_table
from weights_util import BLOCK, STEP, blocks_value, quant_rows, rows_value, sum_bound

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def linear_bound(x, lin, bias=None):
    """(64-bit value, bound) of a BlockLinear's output for bf16 rows x."""
    xv, w = rows_value(*[t.float() for t in quant_rows(x.double())]), blocks_value(lin.w, lin.w_scale)
    y, err = xv @ w.t(), (xv.abs() @ w.abs().t()) * (sum_bound(lin.K) + 2.0 ** -23)
    if bias is not None:
        y = y + bias.double()
    return y, (y.abs() + err) * STEP + err + y.abs() * 2.0 ** -23


@pytest.mark.parametrize("n", [0, 1, 8, 64, 200])
def test_block_linear(n):
    w, bias = rand(1, 700, 528, scale=0.03), rand(2, 700)
    lin = BlockLinear(w, bias, max_tokens=200)
    x = rand(3, n, 528)
    y = lin(x)
    assert y.shape == (n, 700)
    if n == 0:
        return
    want, bound = linear_bound(x, lin, bias)
    assert ((y.double() - want).abs() <= bound).all()
    same = BlockLinear(lin.w, bias, scale=lin.w_scale, max_tokens=200)(x)
    assert torch.equal(y, same) and lin.errors() == 0


def test_gated_feed_forward():
    """gate and up in one product, its gated halves quantised on the way to the down projection."""
    n, H, I = 77, 512, 400
    up, down = BlockLinear(rand(4, 2 * I, H, scale=0.05), max_tokens=n), BlockLinear(rand(5, H, I, scale=0.05), max_tokens=n)
    gu = up(rand(6, n, H))
    y = down(gu, gated=True)
    g, u = gu.double().chunk(2, 1)
    h = g * torch.sigmoid(g) * u
    want = rows_value(*quant_rows(h)) @ blocks_value(down.w, down.w_scale).t()
    # rounding of the output, half a bf16 step at most, and as much again for codes on the other side of a border
    assert (y.double() - want).abs().sum() <= 1.5 * STEP * want.abs().sum()


def test_refusals():
    lin = BlockLinear(rand(7, 64, 128), max_tokens=4)
    with pytest.raises(ValueError, match="at most"):
        lin(rand(8, 5, 128))
    with pytest.raises(ValueError, match="scale"):
        BlockLinear(lin.w, max_tokens=4)
    with pytest.raises(ValueError, match="scale"):
        BlockLinear(rand(7, 64, 128), scale=lin.w_scale, max_tokens=4)
    with pytest.raises(ValueError, match="w1"):
        Experts(rand(9, 4, 128), rand(10, 4, 64, 128), rand(11, 4, 128, 64), 2, max_tokens=4)


@pytest.mark.parametrize("quantize", [False, True])
def test_experts(quantize):
    """The class against the call, at token counts below its largest, on one workspace."""
    e = Experts(rand(12, 16, 256, scale=0.3), rand(13, 16, 2 * 144, 256, scale=0.05), rand(14, 16, 256, 144, scale=0.05), 3,
                quantize=quantize, max_tokens=90)
    for n in (90, 1, 2, 17, 0, 64, 90):
        x = rand(20 + n, n, 256)
        out = e(x).clone()
        if n == 0:
            continue
        ws = E.new_moe_workspace(n, 256, 144, 16, 3)
        want, ids = torch.empty_like(out), torch.empty(n, 3, dtype=torch.int32, device=DEV)
        E.ee_moe_layer(x, e.router, e.w1, e.w2, 3, want, ws, w1_scale=e.w1_scale, w2_scale=e.w2_scale, renorm=True, ids=ids)
        assert torch.equal(out, want) and torch.equal(e.ids, ids)
        assert ((e.probs.sum(1) - 1).abs() <= 4 * 2.0 ** -23).all()
    live = torch.tensor([5], dtype=torch.int32, device=DEV)
    kept = rand(30, 90, 256)
    out = e(rand(31, 90, 256), live=live, out=kept.clone())
    assert torch.equal(out[5:], kept[5:]) and e.errors() == 0


def test_a_layer_in_a_graph():
    """Fused q/k/v projection -> rotary positions and cache -> attention -> output projection -> experts, for
    the new tokens of four sequences, eager and replayed with other tokens."""
    n_q, n_kv, H, total = 4, 2, 512, 50
    qkv = BlockLinear(rand(40, (n_q + 2 * n_kv) * 128, H, scale=0.05), rand(41, (n_q + 2 * n_kv) * 128), max_tokens=total)
    o = BlockLinear(rand(42, H, n_q * 128, scale=0.05), max_tokens=total)
    moe = Experts(rand(43, 8, H, scale=0.2), rand(44, 8, 2 * 256, H, scale=0.05), rand(45, 8, H, 256, scale=0.05), 2, quantize=True,
                  max_tokens=total)
    kc, vc = (torch.zeros(1, 64, n_kv, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    new = torch.tensor([1, 20, 0, 29], dtype=torch.int32, device=DEV)

    def intake():
        return PromptIntake(B=4, n_q=n_q, k_cache=kc, v_cache=vc, rope=rope_table(256), max_pages=8, max_tokens=total)

    def layer(pi, x):
        h = qkv(x).view(total, n_q + 2 * n_kv, 128)
        a = pi.attend(0, h[:, :n_q], h[:, n_q:n_q + n_kv], h[:, n_q + n_kv:], whole=True)
        return moe(o(a.view(total, n_q * 128)))

    x = rand(50, total, H)
    pi = intake()
    pi.admit(new, total)
    eager = layer(pi, x).clone()
    assert torch.isfinite(eager.float()).all() and eager.float().std() > 0
    # the steps' own statements, each on what the kernels in front of it gave
    want, bound = linear_bound(x, qkv, qkv.bias)
    assert ((qkv._out[:total].double() - want).abs() <= bound).all()
    attended = pi._out[:total].view(total, -1)
    want, bound = linear_bound(attended, o)
    assert ((o._out[:total].double() - want).abs() <= bound).all()

    pi = intake()
    pi.admit(new, total)
    graph = torch.cuda.CUDAGraph()
    static = torch.zeros_like(x)
    with torch.cuda.graph(graph):
        out = layer(pi, static)
    for seed in (51, 50):
        static.copy_(rand(seed, total, H))
        graph.replay()
    assert torch.equal(out, eager)
    assert qkv.errors() == 0 and o.errors() == 0 and moe.errors() == 0 and pi.errors() == 0


def test_quantize_weights_of_experts():
    w = rand(60, 3, 2, 130, 272)
    q, s = quantize_weights(w)
    assert q.shape == w.shape and s.shape == (3, 2, 2, 3)
    v = blocks_value(q, s)
    top = s.double().repeat_interleave(BLOCK, 2)[:, :, :130].repeat_interleave(BLOCK, 3)[..., :272]
    assert ((v - w.double()).abs() <= torch.maximum(w.double().abs() * 2.0 ** -4, top * 2.0 ** -10) * (1 + 2.0 ** -20)).all()

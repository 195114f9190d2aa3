"""silu(gate) * up, wherever a kernel computes it, over the whole range of gates: its error does not grow with |gate|."""
import pytest
import torch

import paper_2506_02780_gb300 as E
from weights_util import F8, STEP, blocks, nearest_e4m3

pytestmark = pytest.mark.gpu
DEV = "cuda"

# half a step of fp32 (2^-24) each: e^(-|g|/2) 5 (exponential 4, its correction 1) and twice in the result, 1 + its square at
# most half of that and a rounding of its own (6), a reciprocal's 2, four products
SILU = 22 * 2.0 ** -24


def silu(g):
    return g * torch.sigmoid(g)


def test_every_gate():
    """All bf16 gates up to 120 in size, each in a block of its own: the block's scale is |silu(g) u| / 448 rounded once."""
    bits = torch.arange(1 << 16, device=DEV).to(torch.int32)
    g = (bits << 16).view(torch.float32)
    g = g[torch.isfinite(g) & (g.abs() <= 120) & (g.abs() >= 2.0 ** -20)]
    n = len(g)
    gen = torch.Generator(device=DEV).manual_seed(1)
    for power in (-20, 0, 40, 100):
        u = ((torch.rand(n, generator=gen, device=DEV) + 1) * 2.0 ** power).to(torch.bfloat16)
        u *= torch.where(torch.rand(n, generator=gen, device=DEV) < 0.5, -1, 1)
        x = torch.zeros(n, 32, dtype=torch.bfloat16, device=DEV)
        x[:, 3], x[:, 16 + 3] = g.to(torch.bfloat16), u
        q, s = torch.empty(n, 16, dtype=F8, device=DEV), torch.empty(1, n, device=DEV)
        E.ee_fp8_quantize(x, q, s, gated=True)
        h = silu(x[:, 3].double()) * u.double()
        want = h.abs().clamp(min=2.0 ** -100) / 448
        bad = (s[0].double() - want).abs() > want * (SILU + 2.0 ** -24)
        assert not bad.any(), (power, int(bad.sum()), g[bad][:5])
        big = h.abs() >= 2.0 ** -99
        assert torch.equal(q[big, 3].double(), 448 * torch.sign(h[big]))


@pytest.mark.parametrize("n,c,size", [(40, 400, 1.0), (40, 528, 4.0), (3000, 1040, 1.0), (64, 1024, 40.0)])
def test_codes_next_to_the_exact_ones(n, c, size):
    """A code differs from the exact quotient's only where that quotient is a border up to the arithmetic's error."""
    gen = torch.Generator(device=DEV).manual_seed(n + c)
    x = torch.randn(n, 2 * c, generator=gen, device=DEV)
    x[:, :c] *= size
    x = x.to(torch.bfloat16)
    q, s = torch.empty(n, c, dtype=F8, device=DEV), torch.empty(blocks(c), n, device=DEV)
    E.ee_fp8_quantize(x, q, s, gated=True)
    h = silu(x[:, :c].double()) * x[:, c:].double()
    a = torch.nn.functional.pad(h.abs(), (0, -c % 128)).view(n, -1, 128).amax(-1).clamp(min=2.0 ** -100)
    v = h * 448 / a.repeat_interleave(128, 1)[:, :c]
    # the value's and the maximum's error, the quotient's last rounding and what is left of its two parts
    err = 2 * SILU + 2.0 ** -23
    low, high = nearest_e4m3(v * (1 - err)), nearest_e4m3((v * (1 + err)).clamp(-448, 448))
    got = q.double()
    assert ((got == low) | (got == high)).all()


def test_gates_without_end():
    """Infinite gates are what the formula makes of them: inf u, and a NaN from -inf; finite ones of any size are numbers."""
    x = torch.zeros(6, 32, device=DEV)
    x[:, 16] = 2.0
    x[:, 0] = torch.tensor([float("inf"), float("-inf"), float("nan"), 1e38, -1e38, -300.0], device=DEV)
    q, s = torch.empty(6, 16, dtype=F8, device=DEV), torch.empty(1, 6, device=DEV)
    E.ee_fp8_quantize(x.to(torch.bfloat16), q, s, gated=True)
    assert s[0, 0].isinf() and q[:3].float().isnan().all() and not s[0, 1:3].isfinite().any()
    assert s[0, 3:].isfinite().all() and q[3, 0].float() == 448 and (q[4:].float() == 0).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 20, 40, 300])
@pytest.mark.parametrize("gate", [64, 72, 80, 88, 96, 104])
def test_experts_with_far_gates(T, gate, fp8):
    """Gates of -64 to -104 against an up of 2^100: what is left of them is not small, in any of the kernels."""
    H = I = 128
    x = torch.zeros(T, H, dtype=torch.bfloat16, device=DEV)
    x[:, 0] = 1.0
    router = torch.zeros(2, H, dtype=torch.bfloat16, device=DEV)
    router[1, 0] = 1.0
    w1, w2 = torch.zeros(2, 2, I, H, device=DEV), torch.zeros(2, H, I, device=DEV)
    s1 = s2 = None
    w2[1] = torch.eye(H, device=DEV)
    if fp8:       # codes of 4 gate and 256, scales of 1/4 and 2^92
        w1[1, 0, :, 0], w1[1, 1, :, 0] = -4.0 * gate, 256.0
        s1 = torch.tensor([0.25, 2.0 ** 92], device=DEV).repeat(2, 1).view(2, 2, 1, 1).contiguous()
        s2 = torch.ones(2, 1, 1, device=DEV)
    else:
        w1[1, 0, :, 0], w1[1, 1, :, 0] = -float(gate), 2.0 ** 100
    t = F8 if fp8 else torch.bfloat16
    w1, w2 = w1.view(2, 2 * I, H).to(t), w2.to(t)
    ws = E.new_moe_workspace(T, H, I, 2, 1)
    out = torch.full((T, H), 7.0, dtype=torch.bfloat16, device=DEV)
    E.ee_moe_layer(x, router, w1, w2, 1, out, ws, w1_scale=s1, w2_scale=s2, renorm=True)
    want = float(silu(torch.tensor(-float(gate), dtype=torch.float64))) * 2.0 ** 100
    # the gate is off by two roundings of x's scale and product, which e^g turns into 104 times as much; h is
    # rounded to bf16, or is its block's largest value; the output is rounded to bf16
    err = 2 * STEP + 104 * 2.0 ** -22 + 2 * SILU
    assert ((out.double() - want).abs() <= abs(want) * err).all(), (out[0, :4], want)
    assert E.ee_read_errors(ws) == 0

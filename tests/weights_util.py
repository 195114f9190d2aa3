"""Plain 64-bit statements of the weight products, and how far fp32 arithmetic may be from them."""
import torch

BLOCK = 128
STEP = 2.0 ** -8          # half a bf16 step, relative
F8 = torch.float8_e4m3fn


def blocks(n):
    return -(-n // BLOCK)


def nearest_e4m3(v):
    """fp64: the nearest e4m3 number to |v| <= 448, an even one where two are as near."""
    m = torch.frexp(v).mantissa                            # v / m is a power of two, exactly
    step = torch.where(v == 0, 0.0, v / m * 2.0 ** -4).clamp(min=2.0 ** -9)
    return (v / step).round() * step


def quant_rows(x):
    """fp64 rows -> (values of the codes [rows, cols], scales [blocks, rows]), both fp64."""
    n, c = x.shape
    b = torch.zeros(n, blocks(c) * BLOCK, dtype=torch.float64, device=x.device)
    b[:, :c] = x
    b = b.view(n, -1, BLOCK)
    a = b.abs().amax(-1).clamp(min=2.0 ** -100)
    q = nearest_e4m3(b * 448.0 / a[..., None]).view(n, -1)[:, :c]
    return q, (a / 448.0).t().contiguous()


def quant_blocks(w):
    """fp64 [..., rows, cols] -> (values of the codes, scales [..., row blocks, column blocks])."""
    *lead, r, c = w.shape
    b = torch.zeros(*lead, blocks(r) * BLOCK, blocks(c) * BLOCK, dtype=torch.float64, device=w.device)
    b[..., :r, :c] = w
    b = b.view(*lead, blocks(r), BLOCK, blocks(c), BLOCK)
    a = b.abs().amax((-3, -1), keepdim=True).clamp(min=2.0 ** -100)
    q = nearest_e4m3(b * 448.0 / a).view(*lead, blocks(r) * BLOCK, blocks(c) * BLOCK)[..., :r, :c]
    return q, (a / 448.0).squeeze(-1).squeeze(-2)


def rows_value(q, scale):
    return q.double() * scale.double().t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def blocks_value(q, scale):
    r, c = q.shape[-2:]
    s = scale.double().repeat_interleave(BLOCK, -2)[..., :r, :].repeat_interleave(BLOCK, -1)[..., :c]
    return q.double() * s


def make_rows(gen, n, c):
    """Codes and scales of random activations (by the definition, on the generator's device)."""
    x = torch.randn(n, c, generator=gen, device=gen.device, dtype=torch.float64)
    q, s = quant_rows(x)
    return q.float().to(F8), s.float()


def make_weights(gen, *shape):
    w = torch.randn(shape, generator=gen, device=gen.device, dtype=torch.float64)
    w *= torch.rand(*shape[:-1], 1, generator=gen, device=gen.device, dtype=torch.float64) * 0.04
    q, s = quant_blocks(w)
    return q.float().to(F8), s.float()


def sum_bound(K):
    """Error of an fp32 sum of K products, blocks of 128 scaled and added, relative to the sum of
    magnitudes: at most 127 additions within a block, a scale product, a fused add for each
    block and one for a split's join each (8 at most), an error of one step (2^-23, which also covers truncation) each."""
    return (127 + 1 + blocks(K) + 8) * 2.0 ** -23

"""Inputs and 64-bit references of the prompt-intake tests, and the error bounds
they compare with.

Bounds (u = 2^-24 the fp32 unit roundoff, b = 2^-8 bf16's; written before the
kernels were first run):
  - attention output: rounding it to bf16 costs b |o|; rounding each probability
    to bf16 for the product with V costs at most b A with A = sum_j p_j |v_j| / l;
    fp32 scores and sums are far finer (2^-13 A covers them for scores of a few
    tens and 2^16 keys): |got - o| <= b |o| + (b + 2^-13) A, with 1 % for the
    product of the two roundings;
  - log-sum-exp: a score's 128 exact products are summed in fp32, 128 u sum|q k|
    scale; n exponentials, n u; exponent and logarithm, a few u of their size:
    u (130 max_j sum|q k| scale + n + 8 (1 + |lse|));
  - rotary: two fp32 products and a sum, 4 u (|a| + |b|), and the rounding b |x|.
"""
import math

import torch

D = 128
U, BF = 2.0 ** -24, 2.0 ** -8


def pages(n):
    return -(-n // 16)


def randn(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(torch.bfloat16)


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return off


def packed_qkv(gen, total, n_q, n_kv, fused):
    if fused:
        qkv = randn(gen, total, n_q + 2 * n_kv + 1, D)     # (a token's row is wider than its heads)
        qkv[:, :n_q] *= 1.4
        return qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:n_q + 2 * n_kv]
    return randn(gen, total, n_q, D, std=1.4), randn(gen, total, n_kv, D), randn(gen, total, n_kv, D)


def make_cache(gen, lens, ctxs, n_kv, extra=5, num_pages=None, first_page=0):
    """Cache pages in random order with random contents everywhere, and the table."""
    need = [pages(n + c) for n, c in zip(lens, ctxs)]
    num_pages = num_pages or sum(need) + extra
    perm = torch.randperm(num_pages - first_page, generator=torch.Generator().manual_seed(7)) + first_page
    table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n].to(torch.int32)
        at += n
    k, v = randn(gen, num_pages, n_kv, 16, D), randn(gen, num_pages, n_kv, 16, D)
    return k, v, table.cuda()


def cache_rows(cache, table, s, n):
    """Positions 0 .. n - 1 of sequence s: [n, n_kv, D]."""
    pg = table[s, :pages(n)].long()
    return cache[pg].transpose(1, 2).reshape(-1, cache.shape[1], D)[:n]


def ref_rows(q, K, V, ctx, scale, seen=None):
    """One sequence in 64 bits: q [T, n_q, D], K, V [ctx + T, n_kv, D] -> out, A, lse and
    the lse bound.  seen: optional [keys] mask of keys that exist."""
    T, n_q, _ = q.shape
    if T == 0:
        return (torch.empty_like(q),) * 2 + (torch.empty(0, n_q, device=q.device),) * 2
    n_kv = K.shape[1]
    g = n_q // n_kv
    q, K, V = q.double(), K.double(), V.double()
    out, A = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(T, n_q, dtype=torch.float64, device=q.device)
    tol = torch.empty_like(lse)
    last = ctx + torch.arange(T, device=q.device)
    mask = torch.arange(K.shape[0], device=q.device)[None, :] > last[:, None]
    if seen is not None:
        mask = mask | ~seen[None, :]
    for h in range(n_q):
        x = q[:, h] @ K[:, h // g].T * scale
        x = x.masked_fill(mask, -math.inf)
        z = torch.logsumexp(x, -1)
        p = torch.exp(x - z[:, None]).masked_fill(mask, 0.0)
        out[:, h] = p @ V[:, h // g]
        A[:, h] = p @ V[:, h // g].abs()
        lse[:, h] = z
        big = (q[:, h].abs() @ K[:, h // g].abs().T * scale).masked_fill(mask, 0.0).amax(-1)
        tol[:, h] = U * (130 * big + K.shape[0] + 8 * (1 + z.abs()))
    return out, A, lse, tol


def assert_attn(out, lse, ref, what=""):
    o, A, z, tol = ref
    err = (out.double() - o).abs()
    bound = 1.01 * (BF * o.abs() + (BF + 2.0 ** -13) * A)
    worst = (err - bound).max().item() if err.numel() else 0.0
    assert not torch.isnan(out).any(), f"{what}: NaN in the output"
    assert worst <= 0, f"{what}: output {err.max().item():.3e}, past its bound by {worst:.3e}"
    if lse is not None and z.numel():
        e = (lse.double() - z).abs()
        assert ((e <= tol) | (lse.double() == z)).all(), f"{what}: lse off by {e.max().item():.3e}"

"""ee_prompt_attn and ee_chunk_attn over batches of hundreds and thousands of sequences, most
of them without new tokens; head groups that do not divide a row tile in the paged form; a
prompt of 9,001 tokens against 64 bits."""
import math

import pytest
import torch

import prompt_util as P

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1.0 / math.sqrt(D)


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2506_02780_gb300 as E
    from paper_2506_02780_gb300 import build
    build.build_lib()
    E.lib()
    return E


@pytest.fixture(scope="module")
def ws(E):
    return E.new_prompt_workspace()


def chunk(E, ws, q, kc, vc, table, ctxs, lens):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    z = torch.full(q.shape[:2], float("nan"), device="cuda")
    E.ee_chunk_attn(q, kc, vc, table, P.i32(ctxs), P.i32(P.offsets(lens)), SCALE, out, ws, lse=z)
    return out, z


def check(out, z, q, kc, vc, table, ctxs, lens):
    off = P.offsets(lens)
    for s, n in enumerate(lens):
        if n:
            r = slice(off[s], off[s + 1])
            K, V = (P.cache_rows(c, table, s, ctxs[s] + n) for c in (kc, vc))
            P.assert_attn(out[r], z[r], P.ref_rows(q[r], K, V, ctxs[s], SCALE), f"sequence {s}")


def spread(B, busy):
    """B sequences without new tokens but those of {index from the end or start: (new, ctx)}."""
    lens, ctxs = [0] * B, [(37 * s) % 50 for s in range(B)]
    for s, (n, c) in busy.items():
        lens[s], ctxs[s] = n, c
    return lens, ctxs


@pytest.mark.parametrize("n_q,n_kv", [(28, 4), (8, 8)])
@pytest.mark.parametrize("B,busy", [
    (66, {33: (300, 0)}), (385, {384: (1, 900)}), (385, {0: (1, 3000), 384: (1, 0)}), (512, {100: (100, 3000)}),
    (700, {3: (500, 700), 350: (1, 5000), 699: (33, 100)}), (4096, {0: (2, 60), 2000: (1200, 50), 4095: (1, 2000)}),
    (1000, {}), (769, {s: (1, 100 + s) for s in range(0, 769, 7)}), (5000, {4999: (130, 1)})])
def test_idle_sequences(E, ws, n_q, n_kv, B, busy):
    """A few sequences with tokens among many without; and the same calls without those."""
    gen = torch.Generator("cuda").manual_seed(B)
    lens, ctxs = spread(B, busy)
    table = torch.full((B, max([P.pages(n + c) for n, c in zip(lens, ctxs)])), -1, dtype=torch.int32)
    some = sorted(busy)
    need = [P.pages(sum(busy[s])) for s in some]
    num_pages = sum(need) + 3
    perm = torch.randperm(num_pages, generator=torch.Generator().manual_seed(B)).to(torch.int32)
    at = 0
    for s, n in zip(some, need):
        table[s, :n] = perm[at:at + n]
        at += n
    table = table.cuda()
    kc, vc = P.randn(gen, num_pages, n_kv, 16, D), P.randn(gen, num_pages, n_kv, 16, D)
    q = P.randn(gen, sum(lens), n_q, D, std=1.4)
    out, z = chunk(E, ws, q, kc, vc, table, ctxs, lens)
    check(out, z, q, kc, vc, table, ctxs, lens)
    again, za = chunk(E, ws, q, kc, vc, table, ctxs, lens)
    assert torch.equal(out, again) and torch.equal(z, za)
    if some:
        idx = torch.tensor(some, device="cuda")
        alone = [[x[s] for s in some] for x in (ctxs, lens)]
        few, zf = chunk(E, ws, q, kc, vc, table[idx].contiguous(), *alone)
        check(few, zf, q, kc, vc, table[idx], *alone)
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("B", [385, 900, 3000])
def test_many_packed_prompts(E, ws, B):
    """Hundreds of prompts of none to dozens of tokens, one of thousands among them."""
    gen = torch.Generator("cuda").manual_seed(B)
    rs = torch.Generator().manual_seed(B)
    lens = [int(x) if x < 40 else 0 for x in torch.randint(0, 60, (B,), generator=rs)]
    lens[B // 3] = 2500
    total = sum(lens)
    q, k, v = P.packed_qkv(gen, total, 8, 2, fused=True)
    out = torch.full((total, 8, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    z = torch.full((total, 8), float("nan"), device="cuda")
    E.ee_prompt_attn(q, k, v, P.i32(P.offsets(lens)), SCALE, out, ws, lse=z)
    off = P.offsets(lens)
    for s in {B // 3, 0, 1, B - 1, B - 2} | set(range(0, B, 29)):
        r = slice(off[s], off[s + 1])
        P.assert_attn(out[r], z[r], P.ref_rows(q[r], k[r], v[r], 0, SCALE), f"sequence {s}")
    assert not torch.isnan(out).any() and not torch.isnan(z).any()
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("n_q,n_kv", [(128, 1), (66, 2), (100, 1), (43, 1)])
@pytest.mark.parametrize("lens,ctxs", [([1, 1], [4096, 7]), ([3, 0, 130], [500, 5, 61]),
                                       ([1] * 20, [53 * i for i in range(20)])])
def test_wide_groups_over_the_cache(E, ws, n_q, n_kv, lens, ctxs):
    gen = torch.Generator("cuda").manual_seed(n_q)
    q = P.randn(gen, sum(lens), n_q, D, std=1.4)
    kc, vc, table = P.make_cache(gen, lens, ctxs, n_kv)
    out, z = chunk(E, ws, q, kc, vc, table, ctxs, lens)
    check(out, z, q, kc, vc, table, ctxs, lens)
    assert E.ee_read_errors(ws) == 0


def test_a_prompt_of_nine_thousand(E, ws):
    n = 9001
    q, k, v = P.packed_qkv(torch.Generator("cuda").manual_seed(9), n, 4, 2, fused=False)
    out = torch.empty_like(q)
    z = torch.empty(n, 4, device="cuda")
    E.ee_prompt_attn(q, k, v, P.i32([0, n]), SCALE, out, ws, lse=z)
    P.assert_attn(out, z, P.ref_rows(q, k, v, 0, SCALE))
    assert E.ee_read_errors(ws) == 0

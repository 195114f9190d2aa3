"""PromptIntake: prompts taken whole, in chunks and token by token into the paged
cache, each layer's attention against 64 bits over the rows the sequences were given,
and the verification step's chain attention on what it leaves."""
import math

import pytest
import torch

import prompt_util as P

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1.0 / math.sqrt(D)
DEVERR_PAGE = 0x04


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2506_02780_gb300 as E
    from paper_2506_02780_gb300 import build
    build.build_lib()
    E.lib()
    return E


def make(B, n_q, n_kv, L=2, num_pages=128, max_pages=40, max_tokens=1024, fill=float("nan"), **kw):
    from paper_2506_02780_gb300.prompt import PromptIntake, rope_table
    kc = torch.full((L, num_pages, n_kv, 16, D), fill, dtype=torch.bfloat16, device="cuda")
    free = torch.randperm(num_pages, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    return PromptIntake(B=B, n_q=n_q, k_cache=kc, v_cache=kc.clone(), rope=rope_table(2048), max_pages=max_pages,
                        max_tokens=max_tokens, free_pages=free, **kw)


def take(pi, gen, lens, whole, kept):
    """One pass of `lens` new tokens through both layers, each checked."""
    before = [len(r) for r in kept]
    off = P.offsets(lens)
    pi.admit(P.i32(lens), off[-1])
    for s, n in enumerate(lens):
        kept[s].extend([None] * n)
    got = []
    for layer in range(pi.L):
        q, k, v = P.packed_qkv(gen, off[-1], pi.n_q, pi.n_kv, fused=True)
        lse = torch.full((off[-1], pi.n_q), float("nan"), device="cuda")
        out = pi.attend(layer, q, k, v, whole=whole, lse=lse)
        for s, n in enumerate(lens):
            rows = slice(off[s], off[s + 1])
            K = P.cache_rows(pi.k_cache[layer], pi.block_table, s, before[s] + n)
            V = P.cache_rows(pi.v_cache[layer], pi.block_table, s, before[s] + n)
            assert torch.equal(V[before[s]:], v[rows])          # the new rows stand at their positions
            P.assert_attn(out[rows], lse[rows], P.ref_rows(pi.q_rot[rows], K, V, before[s], SCALE),
                          f"layer {layer} sequence {s}")
        got.append(out.clone())
    assert pi.errors() == 0
    assert pi.ctx_len.tolist() == [len(r) for r in kept] and pi.ctx_before.tolist() == before
    return got


@pytest.mark.parametrize("n_q,n_kv", [(8, 2), (28, 4), (6, 1), (5, 5)])
def test_whole_then_chunks_then_tokens(E, n_q, n_kv):
    gen = torch.Generator("cuda").manual_seed(n_q)
    pi = make(4, n_q, n_kv, reserve=20)
    kept = [[] for _ in range(4)]
    take(pi, gen, [37, 300, 1, 129], True, kept)
    take(pi, gen, [1, 64, 0, 250], False, kept)
    for _ in range(3):
        take(pi, gen, [1, 1, 1, 1], False, kept)
    # every sequence holds the pages its tokens and the reserve need, none of them twice
    held = pi.held.tolist()
    assert held == [P.pages(len(r) + 20) for r in kept]
    used = [p for s in range(4) for p in pi.block_table[s, :held[s]].tolist()]
    assert len(set(used)) == len(used) and min(used) >= 0
    assert sorted(used + pi.free_pages[:pi.free_cnt.item()].tolist()) == list(range(128))


def test_chunks_give_what_whole_prompts_give(E):
    """The same rows through ee_prompt_attn and, in two parts, through ee_chunk_attn."""
    n_q, n_kv, lens = 28, 4, [150, 33, 400]
    off = P.offsets(lens)
    q, k, v = P.packed_qkv(torch.Generator("cuda").manual_seed(5), off[-1], n_q, n_kv, fused=True)
    a = make(3, n_q, n_kv, L=1)
    a.admit(P.i32(lens), off[-1])
    want = a.attend(0, q, k, v, whole=True)
    refs = [P.ref_rows(a.q_rot[off[s]:off[s + 1]], P.cache_rows(a.k_cache[0], a.block_table, s, n),
                       P.cache_rows(a.v_cache[0], a.block_table, s, n), 0, SCALE) for s, n in enumerate(lens)]
    b = make(3, n_q, n_kv, L=1)
    for part in ([(0, 100), (0, 33), (0, 17)], [(100, 150), (33, 33), (17, 400)]):
        idx = torch.cat([torch.arange(off[s] + lo, off[s] + hi) for s, (lo, hi) in enumerate(part)]).cuda()
        n = P.i32([hi - lo for lo, hi in part])
        b.admit(n, idx.numel())
        out = b.attend(0, q[idx], k[idx], v[idx])
        at = 0
        for s, (lo, hi) in enumerate(part):
            P.assert_attn(out[at:at + hi - lo], None, tuple(x[lo:hi] for x in refs[s]), f"sequence {s} from {lo}")
            P.assert_attn(want[off[s] + lo:off[s] + hi], None, tuple(x[lo:hi] for x in refs[s]), f"sequence {s}")
            at += hi - lo
    assert a.errors() == 0 and b.errors() == 0


def test_verification_reads_what_intake_left(E):
    """Chain attention (linear drafts verified in place) over the intake's cache, table and
    lengths gives what the chunk's attention gives."""
    n_q, n_kv = 28, 4
    gen = torch.Generator("cuda").manual_seed(9)
    pi = make(3, n_q, n_kv, fill=3.0)
    kept = [[] for _ in range(3)]
    take(pi, gen, [100, 7, 333], True, kept)
    draft = [40, 3, 60]
    off = P.offsets(draft)
    got = take(pi, gen, draft, False, kept)
    out = torch.empty(off[-1], n_q, D, device="cuda")
    ws = E.new_workspace(3, off[-1], n_q, 512)
    E.ee_chain_verify_attn(pi.q_rot, pi.k_cache[1], pi.v_cache[1], pi.block_table, pi.ctx_before, 512, pi.tok_off,
                           max(draft), SCALE, out, ws)
    assert E.ee_read_errors(ws) == 0
    for s, n in enumerate(draft):
        rows, ctx = slice(off[s], off[s + 1]), len(kept[s]) - n
        K, V = (P.cache_rows(c[1], pi.block_table, s, ctx + n) for c in (pi.k_cache, pi.v_cache))
        ref = P.ref_rows(pi.q_rot[rows], K, V, ctx, SCALE)
        P.assert_attn(out[rows], None, ref, f"chain, sequence {s}")
        P.assert_attn(got[1][rows], None, ref, f"chunk, sequence {s}")


def test_captured_decode(E):
    """Two decoding steps in one graph, replayed: lengths, pages and cache rows advance."""
    n_q, n_kv, B = 8, 2, 5
    pi = make(B, n_q, n_kv, L=1)
    kept = [[] for _ in range(B)]
    gen = torch.Generator("cuda").manual_seed(1)
    lens = [15, 16, 1, 64, 30]
    take(pi, gen, lens, True, kept)
    q, k, v = P.packed_qkv(gen, B, n_q, n_kv, fused=True)
    ones = P.i32([1] * B)

    def steps():
        for _ in range(2):
            pi.admit(ones, B)
            pi.attend(0, q, k, v)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        steps()
    for _ in range(9):
        g.replay()
    torch.cuda.synchronize()
    assert pi.errors() == 0
    assert pi.ctx_len.tolist() == [n + 20 for n in lens]
    out = pi._out[:B]
    for s in range(B):
        n = lens[s] + 20
        K, V = (P.cache_rows(c[0], pi.block_table, s, n) for c in (pi.k_cache, pi.v_cache))
        P.assert_attn(out[s:s + 1], None, P.ref_rows(pi.q_rot[s:s + 1], K, V, n - 1, SCALE), f"sequence {s}")


def test_nothing_new(E):
    """A pass without tokens between two with: lengths and cache stay, the output is empty."""
    pi = make(2, 8, 2, L=1)
    kept = [[], []]
    gen = torch.Generator("cuda").manual_seed(2)
    take(pi, gen, [5, 40], True, kept)
    table, cache = pi.block_table.clone(), pi.k_cache.clone()
    q, k, v = P.packed_qkv(gen, 0, 8, 2, fused=True)
    pi.admit(P.i32([0, 0]), 0)
    assert pi.attend(0, q, k, v).shape == (0, 8, D)
    assert pi.ctx_len.tolist() == [5, 40] == pi.ctx_before.tolist() and torch.equal(pi.block_table, table)
    assert torch.equal(pi.k_cache.view(torch.int16), cache.view(torch.int16)) and pi.errors() == 0
    take(pi, gen, [1, 2], False, kept)


def test_no_room(E):
    """More pages than are free: the error word says so, nothing is written, lengths stay."""
    pi = make(2, 8, 2, L=1, num_pages=4)
    pi.admit(P.i32([40, 40]), 80)
    assert pi.errors() == DEVERR_PAGE
    assert pi.ctx_len.tolist() == [0, 0] and pi.free_cnt.item() == 4 and (pi.slot == -1).all()
    with pytest.raises(ValueError):
        pi.admit(P.i32([1, 1]), 5000)

"""PromptIntake beside the steps that verify over its cache: sequences whose tokens
EditSession or VerifyStep committed get new ones after them, at their own positions."""
import math

import pytest
import torch

import prompt_util as P

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1.0 / math.sqrt(D)
L, N_Q, N_KV, VOCAB, H = 2, 8, 2, 512, 256


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2506_02780_gb300 as E
    from paper_2506_02780_gb300 import build
    build.build_lib()
    E.lib()
    return E


def intake(B, reserve, num_pages=200, max_pages=24, max_tokens=512):
    from paper_2506_02780_gb300.prompt import PromptIntake, rope_table
    kc = torch.full((L, num_pages, N_KV, 16, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    free = torch.randperm(num_pages, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    return PromptIntake(B=B, n_q=N_Q, k_cache=kc, v_cache=kc.clone(), rope=rope_table(1024), max_pages=max_pages,
                        max_tokens=max_tokens, free_pages=free, reserve=reserve)


def rows(pi, lens):
    """K and V of every layer's first lens[s] positions of every sequence."""
    return [[P.cache_rows(c[layer], pi.block_table, s, n) for s, n in enumerate(lens)]
            for c in (pi.k_cache, pi.v_cache) for layer in range(L)]


def same(a, b):
    return all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for u, w in zip(a, b) for x, y in zip(u, w))


def take(pi, gen, lens, before, whole=False):
    """New tokens in both layers: what the cache held stays, the new rows follow, and the
    attention is that over all of them."""
    held = rows(pi, before)
    off = P.offsets(lens)
    pi.admit(P.i32(lens), off[-1])
    assert pi.ctx_before.tolist() == before
    for layer in range(L):
        q, k, v = P.packed_qkv(gen, off[-1], N_Q, N_KV, fused=True)
        out = pi.attend(layer, q, k, v, whole=whole)
        for s, n in enumerate(lens):
            r = slice(off[s], off[s + 1])
            K = P.cache_rows(pi.k_cache[layer], pi.block_table, s, before[s] + n)
            V = P.cache_rows(pi.v_cache[layer], pi.block_table, s, before[s] + n)
            assert torch.equal(V[before[s]:], v[r])
            P.assert_attn(out[r], None, P.ref_rows(pi.q_rot[r], K, V, before[s], SCALE), f"layer {layer}, sequence {s}")
    assert same(rows(pi, before), held)
    now = [b + n for b, n in zip(before, lens)]
    assert pi.errors() == 0 and pi.ctx_len.tolist() == now
    assert pi.held.tolist() == [P.pages(n + pi.reserve) if n else 0 for n in now]
    used = [p for s in range(pi.B) for p in pi.block_table[s, :pi.held[s].item()].tolist()]
    assert len(set(used)) == len(used)
    assert sorted(used + pi.free_pages[:pi.free_cnt.item()].tolist()) == list(range(pi.num_pages))
    return now


def session(pi, lens, gen):
    """An edit session over the intake's cache whose target's choices are random."""
    from paper_2506_02780_gb300.session import EditSession
    B = pi.B
    codes = [torch.randint(0, VOCAB, (100,), generator=gen, device="cuda").tolist() for _ in range(B)]
    lm_w = P.randn(gen, VOCAB, H, std=0.02)

    def forward(ss):
        ss.q.copy_(P.randn(gen, *ss.q.shape))
        ss.k_tree.copy_(P.randn(gen, *ss.k_tree.shape))
        ss.v_tree.copy_(P.randn(gen, *ss.v_tree.shape))
        ss.hidden.copy_((lm_w[ss.draft_tok.long().roll(-1)].float() * 200.0).bfloat16())   # the next node's token

    return EditSession(orig_tokens=P.i32([t for c in codes for t in c]),
                       orig_off=torch.arange(B + 1, dtype=torch.int64, device="cuda") * 100,
                       committed=[c[:20] for c in codes], ctx_len=pi.ctx_len, k_cache=pi.k_cache, v_cache=pi.v_cache,
                       block_table=pi.block_table, lm_w=lm_w, n_q=N_Q, chain_len=6, n_branches=1, gen_len=0,
                       target_forward=forward)


def test_new_tokens_follow_what_a_session_committed(E):
    gen = torch.Generator("cuda").manual_seed(1)
    pi = intake(3, reserve=7 * 4)
    now = take(pi, gen, [37, 130, 1], [0, 0, 0], whole=True)
    for part in ([20, 1, 0], [0, 3, 33]):
        ss = session(pi, now, gen)
        for _ in range(4):
            ss.step()
        assert E.ee_read_errors(ss.ws) == 0
        committed = ss.ctx_len.tolist()
        assert all(c >= n + 4 for c, n in zip(committed, now))
        pi.commit(ss.ctx_len)
        now = take(pi, gen, part, committed)
    # without new tokens, what was committed still gets its reserve
    ss = session(pi, now, gen)
    for _ in range(4):
        ss.step()
    pi.commit(ss.ctx_len)
    take(pi, gen, [0, 0, 0], ss.ctx_len.tolist())
    assert E.ee_read_errors(ss.ws) == 0


@pytest.mark.parametrize("chain", [False, True])
def test_new_tokens_follow_what_a_step_committed_in_place(E, chain):
    """VerifyStep with its drafts' K/V in the cache: it takes the intake's own block table
    (which has columns for them), and its ctx_out are the lengths that intake goes on from."""
    from paper_2506_02780_gb300.step import VerifyStep
    gen = torch.Generator("cuda").manual_seed(2)
    B, T = 3, 9
    pi = intake(B, reserve=T)
    now = take(pi, gen, [48, 7, 100], [0, 0, 0], whole=True)
    for _ in range(2):
        lm_w = P.randn(gen, VOCAB, H, std=0.02)
        draft = torch.randint(0, VOCAB, (B * T,), generator=gen, device="cuda", dtype=torch.int32)
        hidden = (lm_w[draft.long().roll(-1)].float() * 200.0).bfloat16()
        hidden[4] = hidden[3]                       # the first sequence's draft ends here
        step = VerifyStep(orig_tokens=P.i32(list(range(90))), orig_off=torch.arange(B + 1, device="cuda") * 30,
                          tail=P.i32([[1, 2, 3, 4]] * B), cursor=P.i32([0] * B),
                          parent=P.i32([i - 1 for i in range(T)] * B), node_off=P.i32([T * s for s in range(B + 1)]),
                          draft_tok=draft, ctx_len=pi.ctx_len, block_table=pi.block_table,
                          q=P.randn(gen, L, B * T, N_Q, D), k_tree=P.randn(gen, L, B * T, N_KV, D),
                          v_tree=P.randn(gen, L, B * T, N_KV, D), k_cache=pi.k_cache, v_cache=pi.v_cache,
                          hidden=hidden, lm_w=lm_w, max_ctx=max(now), max_T=T, inplace_kv=True, chain=chain)
        assert step.inp["block_table"] is pi.block_table
        step.run()
        assert E.ee_read_errors(step.ws) == 0
        committed = step.ctx_out.tolist()
        assert all(c > n for c, n in zip(committed, now)) and max(c - n for c, n in zip(committed, now)) > 2
        pi.commit(step.ctx_out)
        now = take(pi, gen, [5, 30, 0], committed)


def test_commit_refuses_other_lengths(E):
    pi = intake(3, reserve=0)
    for bad, error in ((P.i32([1, 2]), ValueError), (torch.zeros(3, device="cuda"), TypeError),
                       (torch.zeros(3, dtype=torch.int32), ValueError)):
        with pytest.raises(error):
            pi.commit(bad)


def test_committed_lengths_past_the_pages_are_reported(E):
    """A length that the sequence's pages do not hold: no tokens for it, and the error word."""
    gen = torch.Generator("cuda").manual_seed(4)
    pi = intake(2, reserve=0)
    take(pi, gen, [20, 20], [0, 0], whole=True)
    pi.commit(P.i32([33, 20]))
    pi.admit(P.i32([1, 1]), 1)
    assert pi.errors() == 0x08
    assert pi.ctx_len.tolist() == [33, 21] and pi.held.tolist() == [2, 2]


@pytest.mark.parametrize("seed", range(4))
def test_released_pages_serve_other_sequences(E, seed):
    """Sequences come, grow, end and are replaced: a released one has no pages or tokens, the
    others keep theirs, and no page is lost or held twice (``take`` looks)."""
    rs = torch.Generator().manual_seed(seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    B = 6
    pi = intake(B, reserve=5, num_pages=60, max_pages=10)
    now = [0] * B
    for i in range(12):
        lens = [0 if n > 100 else int(torch.randint(0, 40, (1,), generator=rs)) for n in now]
        now = take(pi, gen, lens, now)
        done = torch.rand(B, generator=rs) < 0.3 if i % 3 else torch.zeros(B, dtype=torch.bool)
        if i == 7:
            done[:] = True
        kept, table, free = rows(pi, now), pi.block_table.clone(), pi.free_pages[:pi.free_cnt.item()].clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        pi.release(done.cuda(), stream=side)
        torch.cuda.current_stream().wait_stream(side)
        back = [p for s in range(B) if done[s] and now[s] for p in table[s, :P.pages(now[s] + 5)].tolist()]
        assert pi.free_pages[:pi.free_cnt.item()].tolist() == free.tolist() + back
        for s in range(B):
            if done[s]:
                now[s] = 0
                assert (pi.block_table[s] == -1).all()
            else:
                assert torch.equal(pi.block_table[s], table[s])
        left = [[k if n else k[:0] for k, n in zip(r, now)] for r in kept]
        assert same(rows(pi, now), left) and pi.ctx_len.tolist() == now
    assert pi.errors() == 0


def test_release_refuses_other_masks(E):
    pi = intake(3, reserve=0)
    for bad, error in ((torch.zeros(2, dtype=torch.bool, device="cuda"), ValueError), (P.i32([0, 1, 2]), TypeError),
                       (torch.zeros(3, dtype=torch.bool), ValueError)):
        with pytest.raises(error):
            pi.release(bad)


def test_release_in_a_graph(E):
    """A pass that admits, releases and admits again, captured and replayed."""
    pi = intake(4, reserve=0, num_pages=40, max_pages=8, max_tokens=64)
    new, done = P.i32([20, 5, 0, 7]), torch.tensor([True, False, False, True], device="cuda")

    def passes():
        pi.admit(new, 32)
        pi.release(done)
        pi.admit(new, 32)
        pi.release(done)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        passes()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        passes()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert pi.errors() == 0 and pi.ctx_len.tolist() == [0, 40, 0, 0] and pi.held.tolist() == [0, 3, 0, 0]
    used = pi.block_table[1, :3].tolist() + pi.free_pages[:pi.free_cnt.item()].tolist()
    assert sorted(used) == list(range(40))

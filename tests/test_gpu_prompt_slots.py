"""ee_prompt_slots against a loop over sequences and tokens, and ee_rope_append
against the rotation in 64 bits."""
import numpy as np
import pytest
import torch

import prompt_util as P

pytestmark = pytest.mark.gpu
D = 128
CTX, PAGE = 0x08, 0x04


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


def loop(ctx, new, held, table, free, cnt, reserve):
    """The definition, one token and one page at a time."""
    table = table.copy()
    off, pos, slot, held_out, left = [0], [], [], [], cnt
    for s in range(len(ctx)):
        have = held[s]
        while ctx[s] + new[s] > 0 and have * 16 < ctx[s] + new[s] + reserve:
            left -= 1
            table[s, have] = free[left]
            have += 1
        held_out.append(have)
        for p in range(ctx[s], ctx[s] + new[s]):
            pos.append(p)
            slot.append(table[s, p // 16] * 16 + p % 16)
        off.append(off[-1] + new[s])
    return off, pos, slot, table, [c + n for c, n in zip(ctx, new)], held_out, left


def call(E, ws, ctx, new, held, table, free, cnt, num_pages, reserve, total=None):
    B = len(ctx)
    total = sum(new) if total is None else total
    full = lambda n: torch.full((n,), -9, dtype=torch.int32, device="cuda")  # noqa: E731
    o = dict(tok_off=full(B + 1), pos=full(total), slot=full(total), ctx_out=full(B), held_out=full(B), free_out=full(1))
    t = P.i32(table)
    E.ee_prompt_slots(P.i32(ctx), P.i32(new), P.i32(held), t, P.i32(free), P.i32([cnt]), num_pages, reserve, o["tok_off"],
                      o["pos"], o["slot"], o["ctx_out"], o["held_out"], o["free_out"], ws)
    bits = E.ee_read_errors(ws)
    return {k: v.cpu().numpy() for k, v in o.items()}, t.cpu().numpy(), bits


def case(B, new_hi, ctx_hi, reserve, seed, more_held=0):
    rs = np.random.RandomState(seed)
    new = rs.randint(0, new_hi + 1, B)
    ctx = rs.randint(0, ctx_hi + 1, B)
    held = -(-ctx // 16) + (rs.randint(0, more_held + 1, B) if more_held else 0)
    want = (new + ctx + reserve + 15) // 16
    cols = int(max(want.max(), held.max())) + 1
    n = int(held.sum() + want.sum()) + 3
    ids = rs.permutation(n)
    table = np.full((B, cols), -1, dtype=np.int64)
    at = 0
    for s in range(B):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
    return [int(x) for x in ctx], [int(x) for x in new], [int(x) for x in held], table, ids[at:], n


@pytest.mark.parametrize("B,new_hi,ctx_hi,reserve,more", [
    (1, 1, 0, 0, 0), (1, 1, 16, 0, 0), (3, 0, 40, 5, 0), (8, 1, 1000, 0, 0), (33, 70, 100, 128, 3), (513, 20, 60, 1, 0),
    (4096, 3, 33, 0, 1), (2, 5000, 17, 16, 0), (700, 900, 10, 0, 0)])
def test_slots(E, ws, B, new_hi, ctx_hi, reserve, more):
    ctx, new, held, table, free, n = case(B, new_hi, ctx_hi, reserve, B + new_hi, more)
    got, t, bits = call(E, ws, ctx, new, held, table, free, len(free), n, reserve)
    off, pos, slot, tr, co, ho, left = loop(ctx, new, held, table, free, len(free), reserve)
    assert bits == 0
    np.testing.assert_array_equal(got["tok_off"], off)
    np.testing.assert_array_equal(got["pos"], pos)
    np.testing.assert_array_equal(got["slot"], slot)
    np.testing.assert_array_equal(got["ctx_out"], co)
    np.testing.assert_array_equal(got["held_out"], ho)
    assert got["free_out"][0] == left
    np.testing.assert_array_equal(t, tr)


def test_free_list_is_taken_from_its_end_by_count(E, ws):
    """Only the first *free_cnt entries are free."""
    ctx, new, held, table, free, n = case(5, 40, 20, 0, 3)
    got, t, bits = call(E, ws, ctx, new, held, table, np.concatenate([free, [10 ** 6] * 7]), len(free), n, 0)
    assert bits == 0
    np.testing.assert_array_equal(got["slot"], loop(ctx, new, held, table, free, len(free), 0)[2])


def test_exhausted_free_list_changes_nothing(E, ws):
    ctx, new, held, table, free, n = case(6, 60, 20, 0, 4)
    need = sum(max(-(-(c + m) // 16) - h, 0) for c, m, h in zip(ctx, new, held))
    got, t, bits = call(E, ws, ctx, new, held, table, free, need - 1, n, 0)
    assert bits == PAGE
    np.testing.assert_array_equal(t, table)
    np.testing.assert_array_equal(got["ctx_out"], ctx)
    np.testing.assert_array_equal(got["held_out"], held)
    assert got["free_out"][0] == need - 1 and (got["slot"] == -1).all()
    got, t, bits = call(E, ws, ctx, new, held, table, free, need, n, 0)
    assert bits == 0 and got["free_out"][0] == 0
    np.testing.assert_array_equal(got["slot"], loop(ctx, new, held, table, free, need, 0)[2])


@pytest.mark.parametrize("field,value", [("ctx", -1), ("new", -5), ("held", -1), ("held", 10 ** 6), ("ctx", 33),
                                         ("new", 10 ** 9)])
def test_a_bad_sequence_gets_nothing(E, ws, field, value):
    ctx, new, held = [3, 20, 0], [5, 9, 30], [1, 2, 0]
    table = np.full((3, 8), -1)
    table[0, 0], table[1, :2] = 4, (7, 2)
    free = np.array([0, 1, 3, 5, 6])
    good, _, bits = call(E, ws, ctx, [5, 0, 30], held, table, free, 5, 8, 0)
    assert bits == 0
    dict(ctx=ctx, new=new, held=held)[field][1] = value
    got, t, bits = call(E, ws, ctx, new, held, table, free, 5, 8, 0, total=35)
    assert bits == CTX
    for k in ("pos", "slot", "tok_off", "free_out"):
        np.testing.assert_array_equal(got[k], good[k])
    assert got["ctx_out"][1] == ctx[1] and got["held_out"][1] == held[1]


@pytest.mark.parametrize("total", [0, 10, 50])
def test_a_wrong_total_is_reported(E, ws, total):
    ctx, new, held = [0, 4], [30, 5], [0, 1]
    table = np.full((2, 4), -1)
    table[1, 0] = 3
    free = np.array([0, 1, 2])
    got, _, bits = call(E, ws, ctx, new, held, table, free, 3, 4, 0, total=total)
    _, pos, slot, _, _, _, _ = loop(ctx, new, held, table, free, 3, 0)
    assert bits == CTX
    n = min(total, 35)
    np.testing.assert_array_equal(got["pos"][:n], pos[:n])
    np.testing.assert_array_equal(got["slot"][:n], slot[:n])
    assert (got["pos"][n:] == -1).all() and (got["slot"][n:] == -1).all()


def test_a_page_outside_the_cache_is_reported(E, ws):
    table = np.full((2, 4), -1)
    got, _, bits = call(E, ws, [0, 0], [20, 3], [0, 0], table, np.array([2, 99, 1]), 3, 4, 0)
    assert bits == PAGE
    want = [16 + i for i in range(16)] + [-1] * 4 + [32 + i for i in range(3)]
    np.testing.assert_array_equal(got["slot"], want)


# ---------------------------------------------------------------- rotary positions and the cache write

def rotated(x, rope, pos):
    a, b = x[..., :64].double(), x[..., 64:].double()
    c, s = rope.double()[pos.long()][:, None, :64], rope.double()[pos.long()][:, None, 64:]
    y = torch.cat([a * c - b * s, b * c + a * s], -1)
    size = torch.cat([a.abs() + b.abs()] * 2, -1)
    return y, P.BF * y.abs() + 4 * P.U * size


def rope_table(n_pos, base=1e6):
    inv = base ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    ang = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def near(got, ref):
    y, tol = ref
    assert ((got.double() - y).abs() <= tol).all()


@pytest.mark.parametrize("n_q,n_kv", [(8, 2), (28, 4), (56, 8), (1, 1), (3, 3)])
@pytest.mark.parametrize("total", [1, 2, 31, 300])
@pytest.mark.parametrize("fused,keep_k", [(False, False), (True, True)])
def test_rope_append(E, ws, n_q, n_kv, total, fused, keep_k):
    gen = torch.Generator(device="cuda").manual_seed(total)
    q, k, v = P.packed_qkv(gen, total, n_q, n_kv, fused)
    rope = rope_table(5000)
    pos = torch.randint(0, 5000, (total,), generator=gen, device="cuda", dtype=torch.int32)
    num_pages = P.pages(total) + 3
    slot = torch.randperm(num_pages * 16, generator=gen, device="cuda")[:total].to(torch.int32)
    if total > 2:
        slot[1] = -1                     # a padding token: turned, not stored
    kc, vc = P.randn(gen, num_pages, n_kv, 16, D), P.randn(gen, num_pages, n_kv, 16, D)
    k0, v0 = kc.clone(), vc.clone()
    qo = torch.full((total, n_q, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ko = torch.full((total, n_kv, D), float("nan"), dtype=torch.bfloat16, device="cuda") if keep_k else None
    E.ee_rope_append(q, k, v, rope, pos, slot, qo, kc, vc, ws, k_out=ko)
    assert E.ee_read_errors(ws) == 0
    near(qo, rotated(q, rope, pos))
    if keep_k:
        near(ko, rotated(k, rope, pos))
    live = slot >= 0
    page, row = slot[live].long() // 16, slot[live].long() % 16
    y, tol = rotated(k, rope, pos)
    near(kc[page, :, row], (y[live], tol[live]))
    assert torch.equal(vc[page, :, row], v[live])
    kc[page, :, row] = k0[page, :, row]
    vc[page, :, row] = v0[page, :, row]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)      # nothing else was written


def test_rope_in_place(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = P.packed_qkv(gen, 77, 28, 4, True)
    rope, pos = rope_table(100), P.i32(list(range(77)))
    q0, k0, v0 = q.clone(), k.clone(), v.clone()
    kc = torch.zeros(5, 4, 16, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    E.ee_rope_append(q, k, v, rope, pos, pos, q, kc, vc, ws, k_out=k)
    near(q, rotated(q0, rope, pos))
    near(k, rotated(k0, rope, pos))
    assert torch.equal(v, v0)
    assert torch.equal(kc.transpose(1, 2).reshape(-1, 4, D)[:77], k)
    assert torch.equal(vc.transpose(1, 2).reshape(-1, 4, D)[:77], v)


def test_rope_bad_positions_and_slots(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = P.packed_qkv(gen, 6, 8, 2, False)
    rope = rope_table(50)
    kc = torch.zeros(2, 2, 16, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    qo = torch.full_like(q, 7.0)
    E.ee_rope_append(q, k, v, rope, P.i32([0, 49, 50, 3, 4, 5]), P.i32([0, 1, 2, 32, 3, 4]), qo, kc, vc, ws)
    assert E.ee_read_errors(ws) == CTX | PAGE
    E.ee_workspace_init(ws)
    E.ee_rope_append(q, k, v, rope, P.i32([-1, 1, 2, 3, 4, 5]), P.i32([0, -2, 5, 6, 7, 8]), qo[:], kc, vc, ws)
    assert E.ee_read_errors(ws) == CTX | PAGE
    E.ee_workspace_init(ws)
    qo = torch.full_like(q, 7.0)
    kc.zero_()
    E.ee_rope_append(q, k, v, rope, P.i32([0, 49, 50, 3, 4, 5]), P.i32([0, 1, 2, 32, 3, 4]), qo, kc, vc, ws)
    assert (qo[2] == 7.0).all() and (kc[0, :, 2] == 0).all()          # position 50 of 50: skipped
    assert not (qo[3] == 7.0).any() and (kc[1] == 0).all()            # slot 32 of 32: turned, not stored
    near(qo[3:4], rotated(q[3:4], rope, P.i32([3])))
    E.ee_read_errors(ws)
    E.ee_workspace_init(ws)


def test_rope_cache_past_four_gib(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(3)
    n_kv, num_pages = 8, 140_000
    kc = torch.empty(num_pages, n_kv, 16, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    q, k, v = P.packed_qkv(gen, 9, 8, n_kv, False)
    rope, pos = rope_table(9), P.i32(list(range(9)))
    slot = P.i32([num_pages * 16 - 9 + i for i in range(9)])
    E.ee_rope_append(q, k, v, rope, pos, slot, q.clone(), kc, vc, ws)
    near(kc[-1, :, -9:].transpose(0, 1), rotated(k, rope, pos))
    assert torch.equal(vc[-1, :, -9:].transpose(0, 1), v)
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("B,new_hi,ctx_hi", [(1, 9, 40), (70, 1, 100), (300, 37, 90)])
def test_slots_at_any_alignment(E, ws, shift, B, new_hi, ctx_hi):
    """pos and slot need four-byte alignment only; what lies around them stays."""
    ctx, new, held, table, free, n = case(B, new_hi, ctx_hi, 7, B + shift)
    new[-1] += 1
    off, pos, slot, tab, ctx_out, held_out, left = loop(ctx, new, held, table, free, len(free), 7)
    total = off[-1]
    full = lambda k: torch.full((k,), -9, dtype=torch.int32, device="cuda")  # noqa: E731
    wide = [full(total + 8) for _ in range(2)]
    p, s = (w[shift:shift + total] for w in wide)
    t, o, c, h, f = P.i32(table), full(B + 1), full(B), full(B), full(1)
    E.ee_prompt_slots(P.i32(ctx), P.i32(new), P.i32(held), t, P.i32(free), P.i32([len(free)]), n, 7, o, p, s, c, h, f, ws)
    assert E.ee_read_errors(ws) == 0
    assert p.tolist() == pos and s.tolist() == slot and o.tolist() == off and f.item() == left
    assert (t.cpu().numpy() == tab).all() and c.tolist() == ctx_out and h.tolist() == held_out
    for w in wide:
        assert (w[:shift] == -9).all() and (w[shift + total:] == -9).all()


def test_tables_and_lengths_are_read_as_just_written(E, ws):
    """Slots, then attention over the table that they wrote, then slots of the other
    sequences into the same table, with nothing in between: each call reads what the one
    before it wrote, although it may have started earlier."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, n_q, n_kv, num_pages, cols = 24, 8, 2, 400, 8
    kc, vc = P.randn(gen, num_pages, n_kv, 16, D), P.randn(gen, num_pages, n_kv, 16, D)
    lens = [100 - s for s in range(B)]
    q = P.randn(gen, B, n_q, D)
    table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    zero, ones, off = P.i32([0] * B), P.i32([1] * B), P.i32(list(range(B + 1)))
    ctx0, free = P.i32([n - 1 for n in lens]), []
    perm = torch.randperm(num_pages, generator=torch.Generator().manual_seed(5)).to(torch.int32).cuda()
    need = sum(P.pages(n) for n in lens)
    free = [perm[:need].contiguous(), perm[-need:].contiguous()]
    cnt, new = P.i32([need]), P.i32(lens)
    total = sum(lens)
    o = dict(tok_off=P.i32([0] * (B + 1)), pos=P.i32([0] * total), slot=P.i32([0] * total), ctx=P.i32([0] * B),
             held=P.i32([0] * B), left=P.i32([0]))
    o2 = dict(pos=P.i32([0] * B), slot=P.i32([0] * B), ctx=P.i32([0] * B), held=P.i32([0] * B), left=P.i32([0]),
              off=P.i32([0] * (B + 1)))
    got = [(torch.empty_like(q), torch.empty_like(o2["slot"])) for _ in range(40)]
    scale = 128 ** -0.5

    def once(i, out):
        # all pages anew, from the one list or the other; then what they hold is attended to
        E.ee_prompt_slots(zero, new, zero, table, free[i % 2], cnt, num_pages, 0, o["tok_off"], o["pos"], o["slot"],
                          o["ctx"], o["held"], o["left"], ws)
        E.ee_chunk_attn(q, kc, vc, table, ctx0, off, scale, out, ws)
        # one more token each, from the lengths that the first call wrote
        E.ee_prompt_slots(o["ctx"], ones, o["held"], table, perm, P_ALL, num_pages, 0, o2["off"], o2["pos"],
                          o2["slot"], o2["ctx"], o2["held"], o2["left"], ws)

    P_ALL = P.i32([num_pages])
    want = []
    for i in range(2):
        out = torch.empty_like(q)
        once(i, out)
        torch.cuda.synchronize()
        for s in range(B):
            K, V = P.cache_rows(kc, table, s, lens[s]), P.cache_rows(vc, table, s, lens[s])
            P.assert_attn(out[s:s + 1], None, P.ref_rows(q[s:s + 1], K, V, lens[s] - 1, scale), f"sequence {s}")
        assert o2["pos"].tolist() == lens
        want.append((out, o2["slot"].clone()))
    for i, (out, slot) in enumerate(got):
        once(i, out)
        slot.copy_(o2["slot"])
    for i, (out, slot) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(slot, want[i % 2][1]), f"pass {i}"
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("total", [0, 1, 10, 30, 33, 35, 50])
def test_lengths_count_the_tokens_that_got_a_slot(E, ws, total):
    """More new tokens than were packed: those past `total` are dropped, and the lengths do
    not claim them (positions that nobody would ever write).  Pages go by the lengths asked for."""
    ctx, new, held = [0, 4, 7], [30, 5, 0], [0, 1, 1]
    table = np.full((3, 4), -1)
    table[1, 0], table[2, 0] = 3, 4
    free = np.array([0, 1, 2])
    got, t, bits = call(E, ws, ctx, new, held, table, free, 3, 5, 0, total=total)
    off, _, _, tr, _, ho, left = loop(ctx, new, held, table, free, 3, 0)
    assert bits == (0 if total == 35 else CTX)
    placed = np.diff(np.minimum(off, total))
    np.testing.assert_array_equal(got["tok_off"], np.minimum(off, total))
    np.testing.assert_array_equal(got["ctx_out"], ctx + placed)
    np.testing.assert_array_equal(got["held_out"], ho)
    np.testing.assert_array_equal(t, tr)
    assert got["free_out"][0] == left and (got["slot"] >= 0).sum() == placed.sum()


@pytest.mark.parametrize("reserve", [0, 1, 20, 64, 65, 5000, 1 << 30])
def test_reserve_ends_where_the_table_ends(E, ws, reserve):
    """Room for what may follow is given as far as the table's columns go: it refuses no
    tokens that fit, nor a sequence without new ones, and an empty sequence gets none."""
    cols = 4
    ctx, new, held = [50, 60, 0, 33, 64, 0, 1], [10, 0, 0, 31, 0, 64, 1], [4, 4, 0, 3, 4, 0, 1]
    table, at = np.full((7, cols), -1), 0
    for s, h in enumerate(held):
        table[s, :h] = np.arange(at, at + h)
        at += h
    free = np.arange(at, at + 30)
    want = [max(-(-min(c + n + reserve, 16 * cols) // 16) - h, 0) if c + n else 0 for c, n, h in zip(ctx, new, held)]
    tab, left = table.copy(), len(free)
    for s, n in enumerate(want):
        for j in range(n):
            left -= 1
            tab[s, held[s] + j] = free[left]
    got, t, bits = call(E, ws, ctx, new, held, table, free, len(free), at + 30, reserve)
    assert bits == 0
    np.testing.assert_array_equal(t, tab)
    np.testing.assert_array_equal(got["held_out"], np.add(held, want))
    np.testing.assert_array_equal(got["ctx_out"], np.add(ctx, new))
    pos = [c + i for c, n in zip(ctx, new) for i in range(n)]
    slot = [tab[s, p // 16] * 16 + p % 16 for s, (c, n) in enumerate(zip(ctx, new)) for p in range(c, c + n)]
    np.testing.assert_array_equal(got["pos"], pos)
    np.testing.assert_array_equal(got["slot"], slot)
    assert got["free_out"][0] == left
    new[1] = 5                          # 65 positions do not fit, whatever the reserve
    got, _, bits = call(E, ws, ctx, new, held, table, free, len(free), at + 30, reserve, total=sum(new) - 5)
    assert bits == CTX and got["ctx_out"][1] == 60 and got["held_out"][1] == 4
    np.testing.assert_array_equal(got["slot"], slot)

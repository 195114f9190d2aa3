"""Units of ee_prompt_attn and ee_chunk_attn that are split among CTAs: pieces joined by
the last of a few, by the last of many, and by all of a cooperative launch; maxima that
differ from piece to piece, pieces without a key, the same bits every time."""
import math

import pytest
import torch

import prompt_util as P

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1.0 / math.sqrt(D)
PAGE_ERR = 0x04


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


# heads, new tokens, cached ones
CASES = [
    ((28, 4), [1], [5000]),                             # few long units: all CTAs join
    ((28, 4), [70], [8000]),                            # the same, two row tiles and an odd unit
    ((6, 1), [1, 0, 3], [20000, 0, 2500]),
    ((28, 4), [1], [1500]),                             # few short units: the last of many joins
    ((7, 1), [1], [1800]),
    ((16, 16), [1, 2, 1, 1], [12000, 30, 0, 7000]),     # many units, some in many pieces
    ((56, 8), [1] * 8, [15000, 100, 40, 900, 17, 3, 0, 2000]),
    ((28, 4), [40] * 16, [200 * i for i in range(16)]),  # units of two or three pieces
    ((8, 2), [260, 1, 33], [6000, 9000, 100]),
]


def inputs(heads, lens, ctxs, climb):
    n_q, n_kv = heads
    gen = torch.Generator("cuda").manual_seed(len(lens) + n_q)
    kc, vc, table = P.make_cache(gen, lens, ctxs, n_kv)
    q = P.randn(gen, sum(lens), n_q, D, std=1.4)
    if climb:      # keys grow (or shrink) with their position: every piece has its own maximum
        for s, (n, c) in enumerate(zip(lens, ctxs)):
            for j, pg in enumerate(table[s, :P.pages(n + c)].tolist()):
                x = j / max(P.pages(n + c) - 1, 1)
                kc[pg] *= 0.2 + 3.0 * (x if climb > 0 else 1.0 - x)
    return q, kc, vc, table


def run(E, ws, q, kc, vc, table, lens, ctxs):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    z = torch.full(q.shape[:2], float("nan"), device="cuda")
    E.ee_chunk_attn(q, kc, vc, table, P.i32(ctxs), P.i32(P.offsets(lens)), SCALE, out, ws, lse=z)
    return out, z


def check(out, z, q, kc, vc, table, lens, ctxs, seen=None):
    off = P.offsets(lens)
    for s, (n, c) in enumerate(zip(lens, ctxs)):
        rows = slice(off[s], off[s + 1])
        K, V = P.cache_rows(kc, table.clamp(min=0), s, c + n), P.cache_rows(vc, table.clamp(min=0), s, c + n)
        ref = P.ref_rows(q[rows], K, V, c, SCALE, None if seen is None else seen[s])
        P.assert_attn(out[rows], z[rows], ref, f"sequence {s}")


@pytest.mark.parametrize("climb", [0, 1, -1])
@pytest.mark.parametrize("heads,lens,ctxs", CASES)
def test_joined_pieces(E, ws, heads, lens, ctxs, climb):
    q, kc, vc, table = inputs(heads, lens, ctxs, climb)
    out, z = run(E, ws, q, kc, vc, table, lens, ctxs)
    check(out, z, q, kc, vc, table, lens, ctxs)
    for _ in range(4):
        again, za = run(E, ws, q, kc, vc, table, lens, ctxs)
        assert torch.equal(out, again) and torch.equal(z, za)
    assert E.ee_read_errors(ws) == 0


def test_the_same_bits_whoever_joins(E, ws):
    """Units in many pieces that the last CTA to arrive joins: which one that is, and whether
    it has a second unit to join, differs from run to run; the sum's order must not."""
    heads, lens, ctxs = (56, 8), [1, 1, 0, 3, 1, 1, 1], [2442, 3623, 6356, 0, 0, 2641, 0]
    q, kc, vc, table = inputs(heads, lens, ctxs, 0)
    out, z = run(E, ws, q, kc, vc, table, lens, ctxs)
    check(out, z, q, kc, vc, table, lens, ctxs)
    for _ in range(100):
        again, za = run(E, ws, q, kc, vc, table, lens, ctxs)
        assert torch.equal(out, again) and torch.equal(z, za)


@pytest.mark.parametrize("heads,lens,ctxs", [CASES[1], CASES[3], CASES[5], CASES[7]])
def test_a_join_reads_this_calls_partials(E, ws, heads, lens, ctxs):
    """Two sets of inputs in turn, one workspace, nothing waited for in between: a piece that
    was read before its writer was done would still hold the other set's partial."""
    sets = [inputs(heads, lens, ctxs, climb) for climb in (1, -1)]
    want = [run(E, ws, *x, lens, ctxs) for x in sets]
    for x, (out, z) in zip(sets, want):
        check(out, z, *x, lens, ctxs)
    ctx, off = P.i32(ctxs), P.i32(P.offsets(lens))
    got = [(torch.empty_like(want[i % 2][0]), torch.empty_like(want[i % 2][1])) for i in range(60)]
    for i, (out, z) in enumerate(got):
        q, kc, vc, table = sets[i % 2]
        E.ee_chunk_attn(q, kc, vc, table, ctx, off, SCALE, out, ws, lse=z)
    for i, (out, z) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(z, want[i % 2][1]), f"call {i}"
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("heads,lens,ctxs", [CASES[0], CASES[1], CASES[3], CASES[6], CASES[8]])
@pytest.mark.parametrize("part", ["first half", "second half", "all"])
def test_pieces_without_a_key(E, ws, heads, lens, ctxs, part):
    """Missing pages take a stretch of the first sequence's keys, and with it whole pieces."""
    q, kc, vc, table = inputs(heads, lens, ctxs, 0)
    n = P.pages(lens[0] + ctxs[0])
    lo, hi = {"first half": (0, n // 2), "second half": (n // 2, n), "all": (0, n)}[part]
    table[0, lo:hi] = -1
    seen = [None] * len(lens)
    seen[0] = torch.ones(lens[0] + ctxs[0], dtype=torch.bool, device="cuda")
    seen[0][16 * lo:16 * hi] = False
    out, z = run(E, ws, q, kc, vc, table, lens, ctxs)
    assert E.ee_read_errors(ws) == PAGE_ERR
    E.ee_workspace_init(ws)
    if part == "all":
        first = slice(0, lens[0])
        assert (out[first] == 0).all() and (z[first] == -math.inf).all()
        out, z = out[lens[0]:], z[lens[0]:]
        check(out, z, q[lens[0]:], kc, vc, table[1:], lens[1:], ctxs[1:])
    else:
        check(out, z, q, kc, vc, table, lens, ctxs, seen)


@pytest.mark.parametrize("n_q,n_kv,lens", [(7, 1, [1700]), (28, 4, [300]), (128, 1, [90, 1, 200]), (8, 8, [5000, 1])])
def test_joined_prompts(E, ws, n_q, n_kv, lens):
    total = sum(lens)
    q, k, v = P.packed_qkv(torch.Generator("cuda").manual_seed(total), total, n_q, n_kv, fused=False)
    k = k * torch.linspace(0.2, 2.5, total, device="cuda").to(torch.bfloat16)[:, None, None]
    off = P.offsets(lens)
    got = []
    for _ in range(3):
        out = torch.full((total, n_q, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        z = torch.full((total, n_q), float("nan"), device="cuda")
        E.ee_prompt_attn(q, k, v, P.i32(off), SCALE, out, ws, lse=z)
        got.append((out, z))
    for s in range(len(lens)):
        r = slice(off[s], off[s + 1])
        P.assert_attn(out[r], z[r], P.ref_rows(q[r], k[r], v[r], 0, SCALE), f"sequence {s}")
    assert all(torch.equal(a, out) and torch.equal(b, z) for a, b in got)
    assert E.ee_read_errors(ws) == 0


def test_cooperative_launch_in_a_graph(E, ws):
    """A call that every CTA waits in, captured beside one that none does."""
    a, b = CASES[0], CASES[7]
    ia, ib = inputs(*a, 1), inputs(*b, 0)
    bufs = []
    for (heads, lens, ctxs), (q, kc, vc, table) in ((a, ia), (b, ib)):
        bufs.append((q, kc, vc, table, P.i32(ctxs), P.i32(P.offsets(lens)), SCALE,
                     torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda"), ws))

    def calls():
        for x in bufs:
            E.ee_chunk_attn(*x)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    want = [x[7].clone() for x in bufs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for x in bufs:
        x[7].zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x[7], w) for x, w in zip(bufs, want))
    assert E.ee_read_errors(ws) == 0


# split units of several rows: joined by all, by the last of a few, of many
EDGE = [((28, 4), [70], [8000]), ((28, 4), [40] * 16, [200 * i for i in range(16)]),
        ((8, 2), [260, 1, 33], [6000, 9000, 100]), ((7, 1), [90], [1800])]


def gapped(heads, lens, ctxs, high):
    """Inputs whose scores differ by 360 between a sequence's context and its new tokens:
    `high` says which of the two carries the row's weight."""
    q, kc, vc, table = inputs(heads, lens, ctxs, 0)
    q[:] = 4.0
    for s, (n, c) in enumerate(zip(lens, ctxs)):
        for p in range(c + n):
            kc[table[s, p // 16], :, p % 16] = 4.0 if (p < c) == (high == "context") else -4.0
    return q, kc, vc, table


@pytest.mark.parametrize("heads,lens,ctxs", EDGE)
@pytest.mark.parametrize("high", ["context", "new"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_seen_value_shows_whatever_its_weight(E, ws, heads, lens, ctxs, high, bad):
    """A non-finite value among the new tokens of a sequence whose unit is split: the queries
    from it on show it, also where its weight is below 2^-500 beside another piece's, and
    whichever piece joins; the others do not.  As it is in the value's own unit (it is kept
    from the product with V there, and added); in a later unit, all of whose queries see it,
    it meets its weight, and 0 times an infinity is a NaN."""
    q, kc, vc, table = gapped(heads, lens, ctxs, high)
    s = len(lens) - 1 if len(lens) > 3 else 0
    at, g = min(30, lens[s] // 2), heads[0] // heads[1]
    clean, zc = run(E, ws, q, kc, vc, table, lens, ctxs)
    p = ctxs[s] + at
    vc[table[s, p // 16], 0, p % 16, 77] = bad
    row0 = sum(lens[:s])
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[row0 + at:row0 + lens[s], :g, 77] = True
    unit = 2 * (128 // g)              # tokens of two row tiles of g heads each
    for i in range(40):
        out, z = run(E, ws, q, kc, vc, table, lens, ctxs)
        assert torch.equal(z, zc) and torch.equal(out[~hit], clean[~hit])
        if i == 0:
            first = out
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))
        assert not torch.isfinite(out[hit]).any()
        own = out[row0 + at:row0 + min(unit, lens[s]), :g, 77]
        assert torch.isnan(own).all() if math.isnan(bad) else (own == bad).all()
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("heads,lens,ctxs", EDGE)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_value_of_the_context_shows_whatever_its_weight(E, ws, heads, lens, ctxs, bad):
    """The same of a value that every query sees: nowhere finite (0 times it is NaN)."""
    q, kc, vc, table = gapped(heads, lens, ctxs, "new")
    s = len(lens) - 1 if len(lens) > 3 else 0
    g = heads[0] // heads[1]
    clean, zc = run(E, ws, q, kc, vc, table, lens, ctxs)
    vc[table[s, 0], 0, 3, 5] = bad
    rows = slice(sum(lens[:s]), sum(lens[:s + 1]))
    first = None
    for _ in range(40):
        out, z = run(E, ws, q, kc, vc, table, lens, ctxs)
        first = out.clone() if first is None else first
        assert torch.equal(z, zc) and not torch.isfinite(out[rows, :g, 5]).any()
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))
        out[rows, :g, 5] = clean[rows, :g, 5]
        assert torch.equal(out, clean)


def test_a_seen_value_shows_in_a_split_prompt(E, ws):
    """The same over packed K/V: one prompt whose last rows hold all the weight."""
    n_q, n_kv, n = 7, 1, 1700
    q, k, v = P.packed_qkv(torch.Generator("cuda").manual_seed(3), n, n_q, n_kv, fused=False)
    q[:] = 4.0
    k[:] = torch.where(torch.arange(n, device="cuda") % 640 < 320, -4.0, 4.0).to(torch.bfloat16)[:, None, None]
    off = P.i32([0, n])
    got = {}
    for at in (None, 1, 200, 1601):
        x = v.clone()
        if at is not None:
            x[at, 0, 8] = float("inf")
        for i in range(20):
            out = torch.empty_like(q)
            E.ee_prompt_attn(q, k, x, off, SCALE, out, ws)
            if i == 0:
                got[at] = out
            assert torch.equal(out.view(torch.int16), got[at].view(torch.int16))
        if at is not None:
            assert not torch.isfinite(out[at:, :, 8]).any()
            out[at:, :, 8] = got[None][at:, :, 8]
            assert torch.equal(out, got[None])

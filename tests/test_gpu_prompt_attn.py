"""ee_prompt_attn and ee_chunk_attn against plain attention in 64 bits: head layouts,
lengths from none to thousands, strides, keys that no query may see, missing pages,
caches past 4 GiB, streams."""
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


def run_prompt(E, ws, q, k, v, lens, scale=SCALE, lse=True, stream=None):
    total, n_q, _ = q.shape
    out = torch.full((total, n_q, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    z = torch.full((total, n_q), float("nan"), device="cuda") if lse else None
    E.ee_prompt_attn(q, k, v, P.i32(P.offsets(lens)), scale, out, ws, lse=z, stream=stream)
    return out, z


def run_chunk(E, ws, q, kc, vc, table, ctxs, lens, scale=SCALE):
    total, n_q, _ = q.shape
    out = torch.full((total, n_q, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    z = torch.full((total, n_q), float("nan"), device="cuda")
    E.ee_chunk_attn(q, kc, vc, table, P.i32(ctxs), P.i32(P.offsets(lens)), scale, out, ws, lse=z)
    return out, z


HEADS = [(8, 2), (28, 4), (5, 5), (6, 1), (128, 1), (66, 2)]
LENS = [[1], [37], [0, 5, 0], [127, 128, 129], [1, 2, 300, 0, 1000], [511, 18, 36, 37]]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("n_q,n_kv", HEADS)
@pytest.mark.parametrize("lens", LENS)
def test_prompt_attn(E, ws, n_q, n_kv, lens, fused):
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = P.packed_qkv(gen, sum(lens), n_q, n_kv, fused)
    out, z = run_prompt(E, ws, q, k, v, lens)
    off = P.offsets(lens)
    for s in range(len(lens)):
        a, b = off[s], off[s + 1]
        P.assert_attn(out[a:b], z[a:b], P.ref_rows(q[a:b], k[a:b], v[a:b], 0, SCALE), f"sequence {s}")
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("n_q,n_kv,lens", [(28, 4, [3001]), (56, 8, [1025, 2047]), (4, 4, [4097]), (2, 1, [6001])])
def test_long_prompts(E, ws, n_q, n_kv, lens):
    """Work divided between CTAs inside a row block, and many row blocks a CTA."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = P.packed_qkv(gen, sum(lens), n_q, n_kv, True)
    out, z = run_prompt(E, ws, q, k, v, lens)
    again, _ = run_prompt(E, ws, q, k, v, lens, lse=False)
    assert torch.equal(out, again)                     # the same bits every time, with and without lse
    off = P.offsets(lens)
    for s in range(len(lens)):
        a, b = off[s], off[s + 1]
        P.assert_attn(out[a:b], z[a:b], P.ref_rows(q[a:b], k[a:b], v[a:b], 0, SCALE), f"sequence {s}")
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("scale,std", [(1.0, 1.0), (SCALE, 6.0), (1e-4, 1.0)])
def test_scores_large_and_small(E, ws, scale, std):
    """Scores of hundreds (the running maximum moves) and of nearly nothing."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    lens = [700]
    q, k, v = P.packed_qkv(gen, 700, 8, 2, False)
    q = (q.float() * std).to(torch.bfloat16)
    out, z = run_prompt(E, ws, q, k, v, lens, scale=scale)
    P.assert_attn(out, z, P.ref_rows(q, k, v, 0, scale))


def test_rising_maximum(E, ws):
    """Every later key scores higher: the accumulator is rescaled again and again."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    n = 900
    q, k, v = P.packed_qkv(gen, n, 4, 1, False)
    q[:] = 1.0
    k[:] = (torch.arange(n, device="cuda") / 64).to(torch.bfloat16)[:, None, None]
    out, z = run_prompt(E, ws, q, k, v, [n])
    P.assert_attn(out, z, P.ref_rows(q, k, v, 0, SCALE))


@pytest.mark.parametrize("n_q,n_kv", [(8, 2), (28, 4), (3, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 5, 130, 299])
def test_values_reach_only_the_queries_that_see_them(E, ws, n_q, n_kv, bad, at):
    """A non-finite value of token `at`: earlier queries and other sequences are
    untouched, later ones show it in that dimension alone."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    lens = [200, 300, 50]
    q, k, v = P.packed_qkv(gen, sum(lens), n_q, n_kv, True)
    clean, zc = run_prompt(E, ws, q, k, v, lens)
    v = v.clone()
    v[200 + at, 0, 9] = bad
    out, z = run_prompt(E, ws, q, k, v, lens)
    g = n_q // n_kv
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[200 + at:500, :g, 9] = True
    assert torch.equal(z, zc)
    assert torch.equal(out[~hit], clean[~hit])
    if math.isnan(bad):
        assert torch.isnan(out[hit]).all()
    else:
        assert (out[hit] == bad).all()
    assert E.ee_read_errors(ws) == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_keys_reach_only_the_queries_that_see_them(E, ws, bad):
    gen = torch.Generator(device="cuda").manual_seed(6)
    lens = [150, 260]
    q, k, v = P.packed_qkv(gen, sum(lens), 8, 2, False)
    clean, zc = run_prompt(E, ws, q, k, v, lens)
    k[150 + 77, 1] = bad
    out, z = run_prompt(E, ws, q, k, v, lens)
    assert torch.equal(out[:227], clean[:227]) and torch.equal(z[:227], zc[:227])
    assert torch.equal(out[:, :4], clean[:, :4])
    assert torch.isnan(out[227:, 4:]).all()


def test_query_of_nan_stays_in_its_row(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(7)
    q, k, v = P.packed_qkv(gen, 333, 28, 4, False)
    clean, _ = run_prompt(E, ws, q, k, v, [333])
    q[100, 3] = float("nan")
    out, _ = run_prompt(E, ws, q, k, v, [333])
    keep = torch.ones(333, 28, dtype=torch.bool, device="cuda")
    keep[100, 3] = False
    assert torch.equal(out[keep], clean[keep]) and torch.isnan(out[100, 3]).all()


def test_tokens_outside_every_sequence_are_not_written(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(8)
    q, k, v = P.packed_qkv(gen, 90, 8, 2, False)
    out = torch.full((90, 8, D), 3.0, dtype=torch.bfloat16, device="cuda")
    E.ee_prompt_attn(q, k, v, P.i32([10, 40, 40, 70]), SCALE, out, ws)
    assert (out[:10] == 3.0).all() and (out[70:] == 3.0).all()
    for a, b in ((10, 40), (40, 70)):
        P.assert_attn(out[a:b], None, P.ref_rows(q[a:b], k[a:b], v[a:b], 0, SCALE))


@pytest.mark.parametrize("off", [[40, 64, 30, 40], [-1, 30, 30, 64], [0, 30, 40, 65]])
def test_bad_offsets_are_reported(E, ws, off):
    """A sequence whose offsets decrease or leave the tokens is skipped, the others are computed."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = P.packed_qkv(gen, 64, 8, 2, False)
    out = torch.full((64, 8, D), 3.0, dtype=torch.bfloat16, device="cuda")
    E.ee_prompt_attn(q, k, v, P.i32(off), SCALE, out, ws)
    assert E.ee_read_errors(ws) == 0x02
    E.ee_workspace_init(ws)
    good = [(a, b) for a, b in zip(off, off[1:]) if 0 <= a <= b <= 64]
    for a, b in good:
        P.assert_attn(out[a:b], None, P.ref_rows(q[a:b], k[a:b], v[a:b], 0, SCALE))


CHUNKS = [([1], [0]), ([1], [4096]), ([1, 1, 1], [15, 16, 17]), ([1] * 40, [97 * i for i in range(40)]),
          ([5, 0, 40], [1000, 33, 127]), ([300], [1]), ([129, 1, 256], [0, 5000, 128]), ([1], [30000])]


@pytest.mark.parametrize("n_q,n_kv", HEADS[:4])
@pytest.mark.parametrize("lens,ctxs", CHUNKS)
def test_chunk_attn(E, ws, n_q, n_kv, lens, ctxs):
    gen = torch.Generator(device="cuda").manual_seed(10)
    q = P.packed_qkv(gen, sum(lens), n_q, n_kv, True)[0]
    kc, vc, table = P.make_cache(gen, lens, ctxs, n_kv)
    out, z = run_chunk(E, ws, q, kc, vc, table, ctxs, lens)
    off = P.offsets(lens)
    for s in range(len(lens)):
        a, b = off[s], off[s + 1]
        n = ctxs[s] + lens[s]
        P.assert_attn(out[a:b], z[a:b], P.ref_rows(q[a:b], P.cache_rows(kc, table, s, n),
                                                   P.cache_rows(vc, table, s, n), ctxs[s], SCALE), f"sequence {s}")
    assert E.ee_read_errors(ws) == 0


def test_chunk_longer_than_a_chain(E, ws):
    """2,500 new tokens after 700 cached ones: past the limit of the linear drafts."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    q = P.randn(gen, 2500, 8, D)
    kc, vc, table = P.make_cache(gen, [2500], [700], 2)
    out, z = run_chunk(E, ws, q, kc, vc, table, [700], [2500])
    P.assert_attn(out, z, P.ref_rows(q, P.cache_rows(kc, table, 0, 3200), P.cache_rows(vc, table, 0, 3200), 700, SCALE))


def test_chunk_of_a_whole_prompt_equals_prompt_attn(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(12)
    lens = [77, 400]
    q = P.randn(gen, 477, 28, D)
    kc, vc, table = P.make_cache(gen, lens, [0, 0], 4)
    k = torch.cat([P.cache_rows(kc, table, s, n) for s, n in enumerate(lens)])
    v = torch.cat([P.cache_rows(vc, table, s, n) for s, n in enumerate(lens)])
    a, za = run_chunk(E, ws, q, kc, vc, table, [0, 0], lens)
    b, zb = run_prompt(E, ws, q, k, v, lens)
    assert torch.equal(a, b) and torch.equal(za, zb)


@pytest.mark.parametrize("lens,ctxs", [([1, 1], [37, 500]), ([20, 140], [3, 61])])
def test_stale_rows_past_the_end_are_never_seen(E, ws, lens, ctxs):
    """Pages of other sequences and rows past a sequence's end hold NaN and infinities."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    q = P.randn(gen, sum(lens), 28, D)
    kc, vc, table = P.make_cache(gen, lens, ctxs, 4)
    clean, zc = run_chunk(E, ws, q, kc, vc, table, ctxs, lens)
    live = torch.zeros(kc.shape[0], 16, dtype=torch.bool, device="cuda")
    for s in range(len(lens)):
        for t in range(lens[s] + ctxs[s]):
            live[table[s, t // 16].item(), t % 16] = True
    dead = ~live[:, None, :].expand(-1, 4, -1)
    kc[dead] = float("nan")
    vc[dead] = float("inf")
    out, z = run_chunk(E, ws, q, kc, vc, table, ctxs, lens)
    assert torch.equal(out, clean) and torch.equal(z, zc)


def test_missing_pages(E, ws):
    """Keys of missing pages are skipped and reported; a query without any key gets
    zeros and minus infinity."""
    gen = torch.Generator(device="cuda").manual_seed(14)
    lens, ctxs = [3, 1, 40], [100, 20, 300]
    q = P.randn(gen, sum(lens), 28, D)
    kc, vc, table = P.make_cache(gen, lens, ctxs, 4)
    full = table.clone()
    table[0, 2] = -1
    table[1, :] = -1
    table[2, 5] = kc.shape[0]          # past the cache
    out, z = run_chunk(E, ws, q, kc, vc, table, ctxs, lens)
    assert E.ee_read_errors(ws) == 0x04
    E.ee_workspace_init(ws)
    for s, gone in ((0, 2), (2, 5)):
        a, b, n = sum(lens[:s]), sum(lens[:s + 1]), lens[s] + ctxs[s]
        seen = torch.ones(n, dtype=torch.bool, device="cuda")
        seen[16 * gone:16 * gone + 16] = False
        P.assert_attn(out[a:b], z[a:b], P.ref_rows(q[a:b], P.cache_rows(kc, full, s, n), P.cache_rows(vc, full, s, n),
                                                   ctxs[s], SCALE, seen), f"sequence {s}")
    assert (out[3] == 0).all() and (z[3] == -math.inf).all()


@pytest.mark.parametrize("ctx", [-3, 16 * 7, 2 ** 31 - 1])
def test_bad_context_is_skipped_and_reported(E, ws, ctx):
    """A negative context, or more positions than the table has pages for."""
    gen = torch.Generator(device="cuda").manual_seed(15)
    q = P.randn(gen, 2, 8, D)
    kc, vc, table = P.make_cache(gen, [1, 1], [64, 80], 2)
    assert table.shape[1] == 7
    out, z = run_chunk(E, ws, q, kc, vc, table, [ctx, 64], [1, 1])
    assert E.ee_read_errors(ws) == 0x08
    E.ee_workspace_init(ws)
    assert torch.isnan(out[0]).all() and torch.isnan(z[0]).all()
    P.assert_attn(out[1:], z[1:], P.ref_rows(q[1:], P.cache_rows(kc, table, 1, 65), P.cache_rows(vc, table, 1, 65), 64,
                                             SCALE))


def test_cache_past_four_gib(E, ws):
    """A layer's cache of 4.6 GB: rows past 2^32 bytes."""
    gen = torch.Generator(device="cuda").manual_seed(17)
    n_kv, num_pages = 8, 140_000
    kc = torch.empty(num_pages, n_kv, 16, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    n = 333
    table = torch.arange(num_pages - P.pages(n), num_pages, device="cuda", dtype=torch.int32)[None, :].contiguous()
    kc[-P.pages(n):] = P.randn(gen, P.pages(n), n_kv, 16, D)
    vc[-P.pages(n):] = P.randn(gen, P.pages(n), n_kv, 16, D)
    q = P.randn(gen, 3, 16, D)
    out, z = run_chunk(E, ws, q, kc, vc, table, [330], [3])
    P.assert_attn(out, z, P.ref_rows(q, P.cache_rows(kc, table, 0, n), P.cache_rows(vc, table, 0, n), 330, SCALE))


def test_other_stream_and_the_verification_workspace(E):
    """Work enqueued on a stream of its own, with a workspace that the verification
    entry points use in between."""
    gen = torch.Generator(device="cuda").manual_seed(18)
    w = E.new_workspace(8, 64, 28, 4096)
    assert w.numel() >= E.ee_prompt_workspace_size()
    lens = [900, 1300]
    q, k, v = P.packed_qkv(gen, sum(lens), 28, 4, True)
    kc, vc, table = P.make_cache(gen, [64], [4000], 4)
    off, ctx = P.i32([0, 64]), P.i32([4000])
    tree = torch.empty(64, 28, D, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(3):
        with torch.cuda.stream(side):
            got.append(run_prompt(E, w, q, k, v, lens, stream=side)[0])
            E.ee_chain_verify_attn(q[:64].contiguous(), kc, vc, table, ctx, 4000, off, 64, SCALE, tree, w, stream=side)
            got.append(tree.clone())
    side.synchronize()
    assert E.ee_read_errors(w) == 0
    assert torch.equal(got[0], got[2]) and torch.equal(got[2], got[4])
    assert torch.equal(got[1], got[3]) and torch.equal(got[3], got[5])
    P.assert_attn(got[0][:900], None, P.ref_rows(q[:900], k[:900], v[:900], 0, SCALE))


def test_captured_in_a_graph(E, ws):
    gen = torch.Generator(device="cuda").manual_seed(19)
    q, k, v = P.packed_qkv(gen, 500, 28, 4, False)
    off = P.i32([0, 200, 500])
    out = torch.empty(500, 28, D, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        E.ee_prompt_attn(q, k, v, off, SCALE, out, ws, stream=side)
        side.synchronize()
        want = out.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for _ in range(3):
                E.ee_prompt_attn(q, k, v, off, SCALE, out, ws, stream=side)
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)

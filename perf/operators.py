"""Performance cases of prompt intake: how a prompt's tokens get into the paged cache that the verification step reads.

A server that takes new requests beside its edit sessions gives every new token a
position and a cache slot (``slots``), rotates queries and keys and writes K/V into
the slots, each layer (``rope``), and attends: a whole prompt over its own packed K/V
(``prompt``), or a chunk of new tokens -- a part of a long prompt, or one token each of
many sequences -- over what the paged cache holds (``chunk``).

Values: keys and values N(0, 1), queries N(0, 1.4^2), which gives scores of standard
deviation 1.4 (a peaked but not degenerate softmax); the rotary table is that of base
1e6.  Lengths come from the case alone (``sizes`` seeds them, uniform in their
logarithm), their order over the batch and all values from the seed.  Cache pages are
handed out in random order and every page, also past a sequence's end, holds stale
values.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
PAGE = 16
DEV = "cuda"

# attention heads of the configurations' models, and two generic ones (no groups; one shared K/V head)
TINY = dict(n_q=8, n_kv=2)
M7 = dict(n_q=28, n_kv=4)
M33 = dict(n_q=56, n_kv=8)
MHA = dict(n_q=16, n_kv=16)
MQA = dict(n_q=6, n_kv=1)


def listed():
    return [
        # eight running sequences get room for one more token each: launch latency is all
        dict(name="slots-step", op="slots", B=8, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=16384, reserve=0,
             max_pages=2048, sizes=1),
        # a full queue admitted at once: prompts of one to 2048 tokens, some with a cached prefix, room for a draft tree
        dict(name="slots-admit", op="slots", B=1024, new_lo=1, new_hi=2048, ctx_lo=0, ctx_hi=4096, reserve=128,
             max_pages=512, sizes=2),
        # one decoding step of eight sequences
        dict(M7, name="rope-step", op="rope", total=8, n_pos=32768, fused=True, packed=False),
        # a prompt of odd length, from the fused projection's output, rotated K also kept packed
        dict(M7, name="rope-fill", op="rope", total=8191, n_pos=32768, fused=True, packed=True),
        # the smallest whole prompt
        dict(TINY, name="prompt-tiny", op="prompt", B=1, t_lo=37, t_hi=37, fused=False, sizes=1),
        # sixteen prompts of different lengths packed into one pass
        dict(M7, name="prompt-packed", op="prompt", B=16, t_lo=33, t_hi=4097, fused=True, sizes=3),
        # two long prompts, 33B-shaped
        dict(M33, name="prompt-33b", op="prompt", B=2, t_lo=4001, t_hi=6000, fused=True, sizes=4),
        # one whole repository file set as the prompt: 16,384 tokens
        dict(M7, name="prompt-long", op="prompt", B=1, t_lo=16384, t_hi=16384, fused=False, sizes=1),
        # plain decoding of one session
        dict(M7, name="chunk-one", op="chunk", B=1, t_lo=1, t_hi=1, ctx_lo=4096, ctx_hi=4096, sizes=1),
        # plain decoding of a large batch of different contexts
        dict(M7, name="chunk-decode", op="chunk", B=64, t_lo=1, t_hi=1, ctx_lo=1024, ctx_hi=16384, sizes=5),
        # chunks of prompts beside single tokens of running sequences
        dict(M7, name="chunk-mixed", op="chunk", B=12, t_lo=1, t_hi=1025, ctx_lo=0, ctx_hi=8191, sizes=6),
        # the last chunk of a 32,768-token prompt, 33B-shaped
        dict(M33, name="chunk-33b", op="chunk", B=1, t_lo=2048, t_hi=2048, ctx_lo=30720, ctx_hi=30720, sizes=1),
    ]


def _logi(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["slots", "rope", "prompt", "prompt", "prompt", "chunk", "chunk", "chunk"])
    shape = rng.choice([TINY, M7, M7, M33, M33, MHA, MQA])
    sizes = rng.randrange(1, 1 << 20)
    if op == "slots":
        B = _logi(rng, 1, 1024)
        hi = _logi(rng, 1, 2048)
        return dict(op=op, B=B, new_lo=rng.randrange(0, 2) if hi > 1 else 1, new_hi=hi, ctx_lo=rng.randrange(0, 100),
                    ctx_hi=_logi(rng, 100, 4096), reserve=rng.choice([0, 0, 16, 128]), max_pages=512, sizes=sizes)
    if op == "rope":
        total = _logi(rng, 1, 8191 * (M7["n_q"] + 2 * M7["n_kv"]) // (shape["n_q"] + 2 * shape["n_kv"]))
        return dict(shape, op=op, total=total, n_pos=32768, fused=rng.random() < 0.7, packed=rng.random() < 0.5)
    if op == "prompt":
        t = _logi(rng, 1, 8192)
        # no more scores than the longest prompt's: 16384 x 16384 x 28
        most = 16384 * 16384 * 28 // (shape["n_q"] * t * t)
        B = max(1, min(_logi(rng, 1, 64), most))
        return dict(shape, op=op, B=B, t_lo=rng.randrange(1, t + 1), t_hi=t, fused=rng.random() < 0.5, sizes=sizes)
    ctx = _logi(rng, 16, 32768)
    # no more cached keys than the large batch's, no more scores than the 33B-shaped chunk's
    B = max(1, min(_logi(rng, 1, 64), 64 * 16384 * 4 // ((ctx + 1) * shape["n_kv"])))
    most = 2048 * 32768 * 56 // (shape["n_q"] * B * (ctx + 2048))
    t = 1 if rng.random() < 0.3 else _logi(rng, 1, max(1, min(4096, most)))
    return dict(shape, op=op, B=B, t_lo=1 if rng.random() < 0.5 else t, t_hi=t, ctx_lo=rng.randrange(0, ctx + 1),
                ctx_hi=ctx, sizes=sizes)


# ---------------------------------------------------------------- sizes (from the case alone)

def _spread(rs, lo, hi, n):
    """n whole numbers of [lo, hi], uniform in log(1 + x), the first of them hi."""
    x = np.floor(np.exp(rs.uniform(math.log(1 + lo), math.log(2 + hi), n)) - 1).astype(np.int64)
    x = np.clip(x, lo, hi)
    x[0] = hi
    return x


def _lengths(case):
    """Per sequence (new tokens, cached tokens), before the seed orders them."""
    rs = np.random.RandomState(case["sizes"])
    t = _spread(rs, case.get("new_lo", case.get("t_lo")), case.get("new_hi", case.get("t_hi")), case["B"])
    ctx = _spread(rs, case["ctx_lo"], case["ctx_hi"], case["B"]) if "ctx_hi" in case else np.zeros_like(t)
    return t, ctx


def _pages(n):
    return -(-n // PAGE)


def work(case):
    op = case["op"]
    if op == "slots":
        t, ctx = _lengths(case)
        held = _pages(ctx)
        new_pages = int((np.maximum(_pages(t + ctx + case["reserve"]), held) - held).sum())
        touched = int((_pages(ctx + t) - ctx // PAGE).sum())      # table entries the tokens fall on
        # lengths and pages held in, offsets, lengths and pages held out; new pages read and entered; two words a token
        return {"bytes": 4.0 * (6 * case["B"] + 2 * new_pages + touched + 2 * int(t.sum())), "flops": 0.0}
    if op == "rope":
        n, h = case["total"], case["n_q"] + 2 * case["n_kv"]
        rows = 2 * h + (case["n_kv"] if case["packed"] else 0)    # each head read and written once, packed K once more
        table = min(n, case["n_pos"]) * D * 4
        turned = n * (case["n_q"] + case["n_kv"]) * (D // 2)
        return {"bytes": float(n * rows * D * 2 + n * 8 + table), "flops": 6.0 * turned}
    t, ctx = (x.astype(np.float64) for x in _lengths(case))
    scores = float((t * ctx + t * (t + 1) / 2).sum()) * case["n_q"]
    keys = float((t + ctx).sum())
    n = float(t.sum())
    table = 4.0 * float(_pages((t + ctx).astype(np.int64)).sum()) if op == "chunk" else 0.0
    rows = 2 * keys * case["n_kv"] + 2 * n * case["n_q"]
    return {"bytes": 2 * D * rows + 4 * n * case["n_q"] + table + 8 * case["B"], "flops": 4 * D * scores}


# ---------------------------------------------------------------- inputs

def _randn(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(torch.bfloat16)


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).to(DEV)


def _table(rs, n_pages_of, max_pages, num_pages):
    """A block table that gives sequence s its first n_pages_of[s] pages, in random order, and the pages left over."""
    ids = rs.permutation(num_pages)
    table = np.full((len(n_pages_of), max_pages), -1, dtype=np.int64)
    at = 0
    for s, n in enumerate(n_pages_of):
        table[s, :n] = ids[at:at + n]
        at += int(n)
    return table, ids[at:]


def _qkv(gen, case, total):
    """Queries, keys and values of `total` packed tokens: views of one projection's output, or tensors of their own."""
    n_q, n_kv = case["n_q"], case["n_kv"]
    if case.get("fused"):
        qkv = _randn(gen, total, n_q + 2 * n_kv, D)
        qkv[:, :n_q] *= 1.4
        return qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    return _randn(gen, total, n_q, D, std=1.4), _randn(gen, total, n_kv, D), _randn(gen, total, n_kv, D)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    op = case["op"]
    s = {"case": case}
    if op == "rope":
        n, n_pos = case["total"], case["n_pos"]
        s["q"], s["k"], s["v"] = _qkv(gen, case, n)
        first = rs.randint(0, n_pos - n + 1)
        s["pos"] = _i32(first + np.arange(n))
        num_pages = _pages(n) + 8
        table, _ = _table(rs, [_pages(n)], _pages(n), num_pages)
        s["slot"] = _i32(table[0][np.arange(n) // PAGE] * PAGE + np.arange(n) % PAGE)
        inv = 1e6 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) / (D // 2))
        ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * inv
        s["rope"] = torch.cat([ang.cos(), ang.sin()], 1).float()
        s["k_cache"] = _randn(gen, num_pages, case["n_kv"], PAGE, D)
        s["v_cache"] = _randn(gen, num_pages, case["n_kv"], PAGE, D)
        s["q_out"] = torch.empty(n, case["n_q"], D, dtype=torch.bfloat16, device=DEV)
        s["k_out"] = torch.empty(n, case["n_kv"], D, dtype=torch.bfloat16, device=DEV) if case["packed"] else None
    else:
        t, ctx = _lengths(case)
        order = rs.permutation(case["B"])
        t, ctx = t[order], ctx[order]
        total = int(t.sum())
        s["total"], s["t_max"], s["max_ctx"] = total, int(t.max()), int(ctx.max())
        s["tok_off"] = _i32(np.concatenate([[0], np.cumsum(t)]))
        if op == "slots":
            num_pages = int(_pages(t + ctx + case["reserve"]).sum()) + 64
            table, free = _table(rs, _pages(ctx), case["max_pages"], num_pages)
            s["ctx_len"], s["new_len"], s["held"] = _i32(ctx), _i32(t), _i32(_pages(ctx))
            s["block_table"], s["free_pages"], s["free_cnt"] = _i32(table), _i32(free), _i32([len(free)])
            s["num_pages"] = num_pages
            s["pos"], s["slot"] = _i32(np.zeros(total)), _i32(np.zeros(total))
            s["ctx_out"], s["held_out"], s["free_out"] = _i32(np.zeros(case["B"])), _i32(np.zeros(case["B"])), _i32([0])
        elif op == "prompt":
            s["q"], s["k"], s["v"] = _qkv(gen, case, total)
        else:
            s["q"] = _randn(gen, total, case["n_q"], D, std=1.4)
            need = _pages(t + ctx)
            num_pages = int(need.sum()) + 64
            table, _ = _table(rs, need, int(need.max()) + 2, num_pages)
            s["block_table"], s["ctx_len"] = _i32(table), _i32(ctx)
            s["k_cache"] = _randn(gen, num_pages, case["n_kv"], PAGE, D)
            s["v_cache"] = _randn(gen, num_pages, case["n_kv"], PAGE, D)
        if op != "slots":
            s["scale"] = 1.0 / math.sqrt(D)
            s["out"] = torch.empty(total, case["n_q"], D, dtype=torch.bfloat16, device=DEV)
            s["lse"] = torch.empty(total, case["n_q"], dtype=torch.float32, device=DEV)
    if own:
        import paper_2506_02780_gb300 as E
        s["E"] = E
        s["ws"] = E.new_prompt_workspace(device=DEV)
    return s


# ---------------------------------------------------------------- one pass

def _run_own(s):
    E, op = s["E"], s["case"]["op"]
    if op == "slots":
        E.ee_prompt_slots(s["ctx_len"], s["new_len"], s["held"], s["block_table"], s["free_pages"], s["free_cnt"],
                          s["num_pages"], s["case"]["reserve"], s["tok_off"], s["pos"], s["slot"], s["ctx_out"],
                          s["held_out"], s["free_out"], s["ws"])
        return {k: s[k] for k in ("tok_off", "pos", "slot", "block_table", "ctx_out", "held_out", "free_out")}
    if op == "rope":
        E.ee_rope_append(s["q"], s["k"], s["v"], s["rope"], s["pos"], s["slot"], s["q_out"], s["k_cache"], s["v_cache"],
                         s["ws"], k_out=s["k_out"])
        return {k: s[k] for k in ("q_out", "k_out", "k_cache", "v_cache")}
    if op == "prompt":
        E.ee_prompt_attn(s["q"], s["k"], s["v"], s["tok_off"], s["scale"], s["out"], s["ws"], lse=s["lse"])
    else:
        E.ee_chunk_attn(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["ctx_len"], s["tok_off"], s["scale"],
                        s["out"], s["ws"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_slots(s):
    case, ctx, new, held = s["case"], s["ctx_len"].long(), s["new_len"].long(), s["held"].long()
    B, total = case["B"], s["total"]
    end = torch.cumsum(new, 0)
    off = torch.cat([end.new_zeros(1), end])
    need = torch.clamp((ctx + new + case["reserve"] + PAGE - 1) // PAGE, min=0)
    need = torch.maximum(torch.where(ctx + new > 0, need, torch.zeros_like(need)), held)
    given = torch.cumsum(need - held, 0)
    col = torch.arange(case["max_pages"], device=DEV)[None, :]
    fresh = (col >= held[:, None]) & (col < need[:, None])
    at = s["free_cnt"].long() - 1 - ((given - (need - held))[:, None] + col - held[:, None])
    page = s["free_pages"].long()[at.clamp(0, s["free_pages"].numel() - 1)]
    table = torch.where(fresh, page, s["block_table"].long())
    i = torch.arange(total, device=DEV)
    seq = torch.searchsorted(end, i, right=True)
    pos = ctx[seq] + i - off[seq]
    slot = table[seq, pos // PAGE] * PAGE + pos % PAGE
    out = dict(tok_off=off, pos=pos, slot=slot, block_table=table, ctx_out=ctx + new, held_out=need,
               free_out=s["free_cnt"].long() - given[B - 1:])
    return {k: v.to(torch.int32) for k, v in out.items()}


def _plain_rope(s):
    cs = s["rope"][s["pos"].long()][:, None, :]
    cos, sin = cs[..., :D // 2], cs[..., D // 2:]

    def turn(x):
        a, b = x[..., :D // 2].float(), x[..., D // 2:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)

    q, k = turn(s["q"]), turn(s["k"])
    page, row = s["slot"].long() // PAGE, s["slot"].long() % PAGE
    s["k_cache"][page, :, row] = k
    s["v_cache"][page, :, row] = s["v"]
    return dict(q_out=q, k_out=k if s["case"]["packed"] else None, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_attn(s):
    """Every sequence padded to the longest: scores, softmax and products over [B, n_kv, group, T, keys]."""
    case, off = s["case"], s["tok_off"].long()
    B, T, n_q, n_kv = case["B"], s["t_max"], case["n_q"], case["n_kv"]
    n = off[1:] - off[:-1]
    i = torch.arange(T, device=DEV)
    tok = (off[:-1, None] + i).clamp(max=s["total"] - 1)
    real = i[None, :] < n[:, None]
    q = s["q"][tok].float().view(B, T, n_kv, n_q // n_kv, D).permute(0, 2, 3, 1, 4)
    if case["op"] == "prompt":
        ctx = torch.zeros_like(n)
        j = i
        k, v = s["k"][tok].float(), s["v"][tok].float()
    else:
        ctx = s["ctx_len"].long()
        j = torch.arange(s["max_ctx"] + T, device=DEV).clamp(max=s["block_table"].shape[1] * PAGE - 1)
        page, row = s["block_table"].long().clamp(min=0)[:, j // PAGE], (j % PAGE)[None, :].expand(B, -1)
        k, v = s["k_cache"][page, :, row].float(), s["v_cache"][page, :, row].float()
    k, v = k.permute(0, 2, 3, 1), v.permute(0, 2, 1, 3)
    L = k.shape[-1]
    x = torch.matmul(q.reshape(B, n_kv, -1, D), k).view(B, n_kv, -1, T, L).mul_(s["scale"])
    x.masked_fill_((j[None, None, :] > (ctx[:, None] + i)[:, :, None])[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, n_kv, -1, L), v).view(B, n_kv, -1, T, D) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(B, T, n_q, D)[real].to(torch.bfloat16)
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, T, n_q)[real]
    return {"out": o, "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    return {"slots": _plain_slots, "rope": _plain_rope}.get(state["case"]["op"], _plain_attn)(state)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    def slots(s):
        case = s["case"]
        ctx, new, held = (s[k].cpu().numpy().astype(np.int64) for k in ("ctx_len", "new_len", "held"))
        table, free = s["block_table"].cpu().numpy().copy(), s["free_pages"].cpu().numpy()
        left = int(s["free_cnt"].item())
        off, pos, slot, held_out = [0], [], [], []
        for b in range(case["B"]):
            have = int(held[b])
            while ctx[b] + new[b] > 0 and have * PAGE < ctx[b] + new[b] + case["reserve"]:
                left -= 1
                table[b, have] = free[left]
                have += 1
            held_out.append(have)
            p = np.arange(ctx[b], ctx[b] + new[b])
            pos.append(p)
            slot.append(table[b, p // PAGE].astype(np.int64) * PAGE + p % PAGE)
            off.append(off[-1] + int(new[b]))
        out = dict(tok_off=np.array(off), pos=np.concatenate(pos), slot=np.concatenate(slot), block_table=table,
                   ctx_out=ctx + new, held_out=np.array(held_out), free_out=np.array([left]))
        return {k: _i32(v) for k, v in out.items()}

    def rope(s):
        at = torch.stack([s["rope"][:, :D // 2], s["rope"][:, D // 2:]], -1).double()
        at = torch.view_as_complex(at)[s["pos"].long()]

        def turn(x):
            z = torch.complex(x[..., :D // 2].double(), x[..., D // 2:].double()) * at[:, None, :]
            return torch.cat([z.real, z.imag], -1)

        q, k, v = turn(s["q"]), turn(s["k"]), s["v"].double()
        caches = []
        for cache, rows in ((s["k_cache"], k), (s["v_cache"], v)):
            flat = cache.double().transpose(1, 2).reshape(-1, *rows.shape[1:])
            flat[s["slot"].long()] = rows
            caches.append(flat.view(-1, PAGE, *rows.shape[1:]).transpose(1, 2).contiguous())
        return dict(q_out=q, k_out=k if s["case"]["packed"] else None, k_cache=caches[0], v_cache=caches[1])

    def attention(s):
        case, off = s["case"], s["tok_off"].tolist()
        n_q, n_kv, g = case["n_q"], case["n_kv"], case["n_q"] // case["n_kv"]
        out = torch.zeros(s["total"], n_q, D, dtype=torch.float64, device=DEV)
        lse = torch.zeros(s["total"], n_q, dtype=torch.float64, device=DEV)
        for b in range(case["B"]):
            lo, hi = off[b], off[b + 1]
            if hi == lo:
                continue
            if case["op"] == "prompt":
                ctx, K, V = 0, s["k"][lo:hi], s["v"][lo:hi]
            else:
                ctx = int(s["ctx_len"][b])
                pages = s["block_table"][b, :_pages(ctx + hi - lo)].long()
                K, V = (s[c][pages].transpose(1, 2).reshape(-1, n_kv, D) for c in ("k_cache", "v_cache"))
            for h in range(n_kv):
                kd, vd = K[:, h].double(), V[:, h].double()
                for r in range(lo, hi, 2048):
                    e = min(hi, r + 2048)
                    seen = ctx + e - lo
                    a = torch.einsum("thd,kd->htk", s["q"][r:e, h * g:(h + 1) * g].double(), kd[:seen]) * s["scale"]
                    last = torch.arange(ctx + r - lo, ctx + e - lo, device=DEV)
                    a.masked_fill_(torch.arange(seen, device=DEV)[None, :] > last[:, None], -math.inf)
                    z = torch.logsumexp(a, -1)
                    lse[r:e, h * g:(h + 1) * g] = z.T
                    out[r:e, h * g:(h + 1) * g] = torch.einsum("htk,kd->thd", torch.exp(a - z[..., None]), vd[:seen])
        return {"out": out, "lse": lse}

    state = prepare(case, seed)
    return {"slots": slots, "rope": rope}.get(case["op"], attention)(state)

"""Performance cases of a pass's weight products: what a target model does between the attention and the LM head.

Weights in 8-bit floating point (e4m3) carry one scale for each 128 x 128 block, activations
one for each token and 128 columns.  ``quant`` makes both from bf16, activations also from a
gated unit's two halves; ``linear`` multiplies them; ``moe`` is a whole mixture-of-experts
layer (router, choice, gated experts, weighted sum) for the few tokens of a verification
pass, on such weights or on bf16 ones.

Values: activations N(0, 1) with some channels ten times as large, as residual streams
have them; weights N(0, 0.02^2) with rows of different norms.  A token of ``moe`` leans towards
top_k experts whose router rows it contains (five standard deviations of the other
logits); experts are of unequal popularity (1 / (rank + 5)).  Which experts the tokens lean towards comes
from the case alone (``sizes`` seeds them), the experts' order and all values from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 128
TOP = 448.0               # largest e4m3 number
LEAST = 2.0 ** -100       # a block's maximum counts as at least this
DEV = "cuda"
E4M3 = torch.float8_e4m3fn

H7, H33 = 3584, 7168      # hidden sizes of the configurations' models
QKV7 = (28 + 2 * 4) * 128


def listed():
    return [
        # the activations of one draft tree, in front of a projection
        dict(name="quant-tree", op="quant", kind="rows", rows=64, cols=H7),
        # a prompt's gate and up halves on the way to the down projection: the layer's widest array
        dict(name="quant-gated", op="quant", kind="gated", rows=8191, cols=4 * H7),
        # a layer's gate and up weights as they are loaded
        dict(name="quant-weights", op="quant", kind="weights", rows=8 * H7, cols=H7),
        # the attention's output projection for one token of plain decoding
        dict(name="linear-one", op="linear", n=1, K=H7, N=H7, bias=False),
        # the fused query, key and value projection of one draft tree
        dict(name="linear-tree", op="linear", n=64, K=H7, N=QKV7, bias=True),
        # its gate and up projection: a stream of weights
        dict(name="linear-up", op="linear", n=64, K=H7, N=8 * H7, bias=False),
        # the down projection of eight sequences' trees, a ragged number of nodes
        dict(name="linear-batched", op="linear", n=534, K=4 * H7, N=H7, bias=False),
        # a prompt of odd length through the gate and up projection: tensor-bound
        dict(name="linear-fill", op="linear", n=8191, K=H7, N=8 * H7, bias=False),
        # a small layer with sizes that end inside blocks and tiles
        dict(name="moe-tiny", op="moe", T=16, live=16, H=528, I=208, E=8, k=2, fp8=False, renorm=True, sizes=1),
        # plain decoding of one token: the chosen experts' weights and latency
        dict(name="moe-one", op="moe", T=1, live=1, H=H7, I=1280, E=64, k=6, fp8=True, renorm=False, sizes=2),
        # one draft tree: nearly every expert has a few tokens
        dict(name="moe-tree", op="moe", T=64, live=64, H=H7, I=1280, E=64, k=6, fp8=True, renorm=True, sizes=3),
        # eight sequences' trees in a batch padded to 576, on bf16 weights
        dict(name="moe-batched", op="moe", T=576, live=534, H=H7, I=1280, E=64, k=6, fp8=False, renorm=False, sizes=4),
    ]


def _logi(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _log16(rng, lo, hi):
    """A multiple of 16 of [lo, hi], uniform in its logarithm."""
    return max(lo, _logi(rng, lo, hi) // 16 * 16)


def draw(rng):
    op = rng.choice(["quant", "linear", "linear", "linear", "moe", "moe", "moe"])
    if op == "quant":
        kind = rng.choice(["rows", "gated", "weights"])
        cols = rng.choice([_log16(rng, 16, 4 * H33), H7, H33])
        return dict(op=op, kind=kind, rows=_logi(rng, 1, min(16384, 8191 * 4 * H7 // cols)), cols=cols)
    if op == "linear":
        n = rng.choice([_logi(rng, 1, 128), _logi(rng, 1, 8191)])
        K = rng.choice([_log16(rng, 128, 4 * H33), H7, H33])
        # no more multiplications than the prompt's, no more weights than four times its
        most = min(8191 * H7 * 8 * H7 // (n * K), 4 * 8 * H7 * H7 // K)
        return dict(op=op, n=n, K=K, N=_logi(rng, 8, max(8, min(8 * H33, most))), bias=rng.random() < 0.4)
    T = rng.choice([_logi(rng, 1, 128), _logi(rng, 1, 2048)])
    E = rng.choice([8, 16, 60, 64, 128, 160])
    k = rng.choice([1, 2, 4, 6, 8])
    H = rng.choice([_log16(rng, 256, H7), 2048, H7])
    fp8 = rng.random() < 0.6
    # no more bytes of weights than the batch's, no more multiplications than twice its
    most = min(64 * 1280 * H7 * (2 if fp8 else 1) // (E * H), 2 * 534 * 6 * 1280 * H7 // (T * k * H))
    I = _log16(rng, 64, max(64, min(2560, most)))
    live = T if rng.random() < 0.7 else rng.randrange(1, T + 1)
    return dict(op=op, T=T, live=live, H=H, I=I, E=E, k=k, fp8=fp8, renorm=rng.random() < 0.5,
                sizes=rng.randrange(1, 1 << 20))


# ---------------------------------------------------------------- sizes (from the case alone)

def _blocks(n):
    return -(-n // BLOCK)


def _leanings(case):
    """[live, k] ranks of popularity of the experts that each token leans towards, none twice."""
    rs = np.random.RandomState(case["sizes"])
    E, k = case["E"], case["k"]
    # the k largest of log(popularity) + Gumbel noise: a draw without replacement
    key = -np.log(np.arange(E) + 5.0) + rs.gumbel(size=(case["live"], E))
    return np.argsort(-key, axis=1)[:, :k]


def work(case):
    op = case["op"]
    if op == "quant":
        n, c = case["rows"], case["cols"]
        scales = _blocks(n) * _blocks(c) if case["kind"] == "weights" else n * _blocks(c)
        return {"bytes": float(n * c * (5 if case["kind"] == "gated" else 3) + 4 * scales), "flops": 0.0}
    if op == "linear":
        n, K, N = case["n"], case["K"], case["N"]
        scales = _blocks(K) * (n + _blocks(N))
        return {"bytes": float(n * K + N * K + 4 * scales + 2 * n * N + 2 * N * case["bias"]), "flops": 2.0 * n * N * K}
    T, H, I, E, k = case["live"], case["H"], case["I"], case["E"], case["k"]
    active = len(np.unique(_leanings(case)))
    each = 3 * I * H + 4 * (3 * _blocks(I) * _blocks(H)) if case["fp8"] else 6 * I * H
    return {"bytes": float(active * each + 2 * E * H + 4 * T * H + 8 * T * k),
            "flops": 2.0 * T * E * H + 6.0 * T * k * I * H}


# ---------------------------------------------------------------- inputs

def _acts(gen, n, cols):
    x = torch.randn(n, cols, generator=gen, device=DEV)
    loud = torch.rand(cols, generator=gen, device=DEV) < 0.02
    return (x * torch.where(loud, 10.0, 1.0)).to(torch.bfloat16)


def _weights(gen, *shape):
    w = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    rows = torch.empty(*shape[:-1], 1, device=DEV, dtype=torch.bfloat16).uniform_(0.01, 0.03, generator=gen)
    return w.mul_(rows)


def _row_scales(x):
    """x fp32 [rows, cols] in blocks of 128 columns: (e4m3 values, scales [blocks, rows])."""
    n, c = x.shape
    b = torch.zeros(n, _blocks(c) * BLOCK, device=DEV, dtype=torch.float32)
    b[:, :c] = x
    b = b.view(n, -1, BLOCK)
    a = b.abs().amax(-1).clamp(min=LEAST)
    q = (b * TOP / a[..., None]).to(E4M3)           # 448 x is exact for bf16, so no quotient crosses a border
    return q.view(n, -1)[:, :c].contiguous(), (a / TOP).t().contiguous()


def _block_scales(w):
    """w bf16 [..., rows, cols] in blocks of 128 x 128: (e4m3 values, scales [..., row blocks, column blocks])."""
    r, c = w.shape[-2:]
    b = torch.nn.functional.pad(w, (0, -c % BLOCK, 0, -r % BLOCK)) if c % BLOCK or r % BLOCK else w
    b = b.reshape(*w.shape[:-2], _blocks(r), BLOCK, _blocks(c), BLOCK).float()
    a = b.abs().amax((-3, -1), keepdim=True).clamp(min=LEAST)
    q = (b * TOP / a).to(E4M3).view(*w.shape[:-2], _blocks(r) * BLOCK, _blocks(c) * BLOCK)[..., :r, :c]
    return q.contiguous(), (a / TOP).squeeze(-1).squeeze(-2)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op == "quant":
        n, c, kind = case["rows"], case["cols"], case["kind"]
        s["x"] = _weights(gen, n, c) if kind == "weights" else _acts(gen, n, 2 * c if kind == "gated" else c)
        s["q"] = torch.empty(n, c, dtype=E4M3, device=DEV)
        s["scale"] = torch.empty(*((_blocks(n), _blocks(c)) if kind == "weights" else (_blocks(c), n)), device=DEV)
    elif op == "linear":
        n, K, N = case["n"], case["K"], case["N"]
        s["x"], s["xs"] = _row_scales(_acts(gen, n, K).float())
        s["w"], s["ws"] = _block_scales(_weights(gen, N, K))
        s["bias"] = torch.randn(N, generator=gen, device=DEV).to(torch.bfloat16) if case["bias"] else None
        s["out"] = torch.empty(n, N, dtype=torch.bfloat16, device=DEV)
    else:
        T, live, H, I, E, k = (case[x] for x in ("T", "live", "H", "I", "E", "k"))
        s["router"] = (torch.randn(E, H, generator=gen, device=DEV) * 0.02).to(torch.bfloat16)
        w1, w2 = _weights(gen, E, 2, I, H), _weights(gen, E, H, I)
        s["s1"], s["s2"] = None, None
        if case["fp8"]:
            (w1, s["s1"]), (w2, s["s2"]) = _block_scales(w1), _block_scales(w2)
        s["w1"], s["w2"] = w1.view(E, 2 * I, H), w2
        expert = np.random.RandomState(seed % (1 << 32)).permutation(E)[_leanings(case)]
        lean = torch.zeros(T, E, device=DEV)
        lean[:live].scatter_(1, torch.as_tensor(expert, device=DEV), 5.0 * 0.02 * math.sqrt(H) / (0.02 * 0.02 * H))
        s["x"] = (torch.randn(T, H, generator=gen, device=DEV) + lean @ s["router"].float()).to(torch.bfloat16)
        s["live"] = torch.tensor([live], dtype=torch.int32, device=DEV) if live < T else None
        s["out"] = torch.randn(T, H, generator=gen, device=DEV).to(torch.bfloat16)
        s["ids"] = torch.full((T, k), -1, dtype=torch.int32, device=DEV)
        s["p"] = torch.zeros(T, k, device=DEV)
    if own:
        import paper_2506_02780_gb300 as E_
        s["E"] = E_
        if op == "linear":
            s["work"] = E_.new_linear_workspace(device=DEV)
        elif op == "moe":
            s["work"] = E_.new_moe_workspace(T, H, I, E, k, device=DEV)
    return s


# ---------------------------------------------------------------- one pass

def _run_own(s):
    E, case = s["E"], s["case"]
    if case["op"] == "quant":
        if case["kind"] == "weights":
            E.ee_fp8_quantize_weights(s["x"], s["q"], s["scale"])
        else:
            E.ee_fp8_quantize(s["x"], s["q"], s["scale"], gated=case["kind"] == "gated")
        return {"q": s["q"], "scale": s["scale"]}
    if case["op"] == "linear":
        E.ee_fp8_linear(s["x"], s["xs"], s["w"], s["ws"], s["out"], s["work"], bias=s["bias"])
        return {"out": s["out"]}
    E.ee_moe_layer(s["x"], s["router"], s["w1"], s["w2"], case["k"], s["out"], s["work"], w1_scale=s["s1"],
                   w2_scale=s["s2"], renorm=case["renorm"], live=s["live"], ids=s["ids"], probs=s["p"])
    return {"out": s["out"], "ids": s["ids"], "p": s["p"]}


def _silu_times(x):
    """silu of the first half of the columns times the second, fp32."""
    g, u = x.float().chunk(2, -1)
    return g / (1.0 + torch.exp(-g)) * u


def _plain_quant(s):
    if s["case"]["kind"] == "weights":
        q, scale = _block_scales(s["x"])
    else:
        q, scale = _row_scales(_silu_times(s["x"]) if s["case"]["kind"] == "gated" else s["x"].float())
    return {"q": q, "scale": scale}


def _rows_value(q, scale):
    """What quantised rows stand for, fp32."""
    return q.float() * scale.t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _blocks_value(q, scale):
    """What quantised weights [..., rows, cols] stand for, fp32."""
    r, c = q.shape[-2:]
    v = q.float()
    if r % BLOCK or c % BLOCK:
        return v * scale.repeat_interleave(BLOCK, -2)[..., :r, :].repeat_interleave(BLOCK, -1)[..., :c]
    return v.view(*q.shape[:-2], r // BLOCK, BLOCK, c // BLOCK, BLOCK).mul_(scale[..., :, None, :, None]).view(q.shape)


def _plain_linear(s):
    y = _rows_value(s["x"], s["xs"]) @ _blocks_value(s["w"], s["ws"]).t()
    if s["bias"] is not None:
        y += s["bias"].float()
    return {"out": y.to(torch.bfloat16)}


def _plain_moe(s):
    """The chosen experts' tokens padded to the busiest expert's: two batched products over the experts in use."""
    case, k, I = s["case"], s["case"]["k"], s["case"]["I"]
    x = s["x"][:case["live"]]
    T, H = x.shape
    logits = x.double() @ s["router"].double().t()          # 64 bits: the choice is next to a border
    ids = logits.sort(dim=1, descending=True, stable=True).indices[:, :k].sort(1).values
    e = torch.exp(logits - logits.amax(1, keepdim=True)).float()
    chosen = e.gather(1, ids)
    p = chosen / (chosen if case["renorm"] else e).sum(1, keepdim=True)
    order = ids.reshape(-1).argsort(stable=True)
    counts = torch.bincount(ids.reshape(-1), minlength=case["E"])
    active = counts.nonzero().squeeze(1)
    n = counts[active]
    group = torch.repeat_interleave(torch.arange(len(active), device=DEV), n)
    rank = torch.arange(T * k, device=DEV) - (n.cumsum(0) - n)[group]
    if case["fp8"]:
        x = _rows_value(*_row_scales(x.float()))
        w1 = _blocks_value(s["w1"].view(torch.uint8)[active].view(E4M3).view(-1, 2, I, H), s["s1"][active])
        w1, w2 = w1.view(-1, 2 * I, H), _blocks_value(s["w2"].view(torch.uint8)[active].view(E4M3), s["s2"][active])
    else:
        x, w1, w2 = x.float(), s["w1"][active].float(), s["w2"][active].float()
    padded = torch.zeros(len(active), int(n.max()), H, device=DEV)
    padded[group, rank] = x[order // k]
    h = _silu_times(torch.bmm(padded, w1.transpose(1, 2)))
    if case["fp8"]:
        h = _rows_value(*_row_scales(h.view(-1, I))).view(h.shape)
    else:
        h = h.to(torch.bfloat16).float()
    y = torch.bmm(h, w2.transpose(1, 2))[group, rank]
    mine = torch.empty_like(y)
    mine[order] = y
    s["out"][:T] = (mine.view(T, k, H) * p[..., None]).sum(1).to(torch.bfloat16)
    s["ids"][:T] = ids.to(torch.int32)
    s["p"][:T] = p
    return {"out": s["out"], "ids": s["ids"], "p": s["p"]}


def run(state):
    if own:
        return _run_own(state)
    return {"quant": _plain_quant, "linear": _plain_linear, "moe": _plain_moe}[state["case"]["op"]](state)


# ---------------------------------------------------------------- the definition in 64 bits

def _nearest_e4m3(v):
    """The nearest multiple of the step at |v|, an even one where two are as near: 4 significant bits, no step below 2^-9."""
    m = torch.frexp(v).mantissa                            # v / m is a power of two, exactly
    step = torch.where(v == 0, 0.0, v / m * 2.0 ** -4).clamp(min=2.0 ** -9)
    return (v / step).round() * step


def exact(case, seed):
    def cut(x, dim):
        return [x.narrow(dim, at, min(BLOCK, x.shape[dim] - at)) for at in range(0, x.shape[dim], BLOCK)]

    def quant_rows(x):
        """(the values of the codes, scales [blocks, rows]) of fp64 rows."""
        vals, scales = [], []
        for b in cut(x, 1):
            a = torch.maximum(b.abs().amax(1), b.new_tensor(LEAST))
            vals.append(_nearest_e4m3(b * TOP / a[:, None]))
            scales.append(a / TOP)
        return torch.cat(vals, 1), torch.stack(scales)

    def of_rows(v, scales):
        return torch.cat([b * f.double()[:, None] for b, f in zip(cut(v, 1), scales)], 1)

    def of_blocks(w, scales):
        fine = scales.double().repeat_interleave(BLOCK, 0)[:w.shape[0]]
        return torch.cat([b * fine[:, i:i + 1] for i, b in enumerate(cut(w.double(), 1))], 1)

    def gate(x):
        half = x.shape[1] // 2
        return x[:, :half] * torch.sigmoid(x[:, :half]) * x[:, half:]

    def quant(s):
        if case["kind"] == "weights":
            vals, scales = [], []
            for strip in cut(s["x"], 0):
                b = [(t, torch.maximum(t.abs().amax(), t.new_tensor(LEAST))) for t in cut(strip.double(), 1)]
                vals.append(torch.cat([_nearest_e4m3(t * TOP / a) for t, a in b], 1))
                scales.append(torch.stack([a / TOP for _, a in b]))
            return {"q": torch.cat(vals), "scale": torch.stack(scales)}
        vals, scales = [], []
        for at in range(0, case["rows"], 2048):
            x = s["x"][at:at + 2048].double()
            v, f = quant_rows(gate(x) if case["kind"] == "gated" else x)
            vals.append(v)
            scales.append(f)
        return {"q": torch.cat(vals), "scale": torch.cat(scales, 1)}

    def linear(s):
        x, out = of_rows(s["x"].double(), s["xs"]), []
        for at in range(0, case["N"], 8192):              # a multiple of the blocks' rows
            w = of_blocks(s["w"][at:at + 8192], s["ws"][at // BLOCK:(at + 8192) // BLOCK])
            out.append(x @ w.t() + (s["bias"][at:at + 8192].double() if case["bias"] else 0.0))
        return {"out": torch.cat(out, 1)}

    def moe(s):
        T, k, I, fp8 = case["live"], case["k"], case["I"], case["fp8"]
        x = s["x"][:T].double()
        logits = x @ s["router"].double().t()
        out, ids, p = s["out"].double(), s["ids"].clone(), s["p"].double()
        choice = torch.from_numpy(np.sort(np.argsort(-logits.cpu().numpy(), axis=1, kind="stable")[:, :k], axis=1)).to(DEV)
        ids[:T] = choice.to(torch.int32)
        l = logits.gather(1, choice)
        p[:T] = torch.exp(l - torch.logsumexp(l if case["renorm"] else logits, 1, keepdim=True))
        out[:T] = 0
        v = of_rows(*quant_rows(x)) if fp8 else x
        for e in range(case["E"]):
            tok, j = torch.nonzero(choice == e, as_tuple=True)
            if len(tok) == 0:
                continue
            w1, w2 = s["w1"][e], s["w2"][e]
            if fp8:
                g, u, w2 = of_blocks(w1[:I], s["s1"][e, 0]), of_blocks(w1[I:], s["s1"][e, 1]), of_blocks(w2, s["s2"][e])
            else:
                g, u, w2 = w1[:I].double(), w1[I:].double(), w2.double()
            h = gate(torch.cat([v[tok] @ g.t(), v[tok] @ u.t()], 1))
            h = of_rows(*quant_rows(h)) if fp8 else h.to(torch.bfloat16).double()
            out[tok] += (h @ w2.t()) * p[tok, j][:, None]
        return {"out": out, "ids": ids, "p": p}

    return {"quant": quant, "linear": linear, "moe": moe}[case["op"]](prepare(case, seed))

"""Refusals of the prompt-intake entry points before any launch (CPU only): the C ABI
on pointers that are never dereferenced, and the binding on wrong tensors."""
import ctypes
import os
import types

import pytest
import torch

FAKE = ctypes.c_void_p(0x10000)
OTHER = ctypes.c_void_p(0x20000)
ODD = ctypes.c_void_p(0x10008)
BIG = 1 << 30
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 5


@pytest.fixture(scope="module")
def L():
    import paper_2506_02780_gb300 as E
    from paper_2506_02780_gb300 import build
    if not os.path.exists(E.LIB_PATH):
        try:
            build.build_lib()
        except RuntimeError as e:   # no nvcc on this machine
            pytest.skip(str(e))
    return E.lib()


def with_(args, names, **over):
    a = dict(args)
    assert set(over) <= set(names), over
    a.update(over)
    return [a[n] for n in names]


SLOT_NAMES = ("ctx_len new_len held B total reserve block_table max_pages free_pages n_free free_cnt num_pages tok_off "
              "pos slot ctx_out held_out free_out ws ws_bytes stream").split()
SLOT = dict(ctx_len=FAKE, new_len=FAKE, held=FAKE, B=2, total=10, reserve=0, block_table=FAKE, max_pages=4,
            free_pages=FAKE, n_free=9, free_cnt=FAKE, num_pages=9, tok_off=FAKE, pos=FAKE, slot=FAKE, ctx_out=OTHER,
            held_out=OTHER, free_out=OTHER, ws=FAKE, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("over,want", [
    (dict(B=0), INVALID), (dict(total=-1), INVALID), (dict(reserve=-1), INVALID), (dict(max_pages=0), INVALID),
    (dict(n_free=-1), INVALID), (dict(num_pages=0), INVALID), (dict(B=4097), UNSUPPORTED),
    (dict(max_pages=1 << 27), UNSUPPORTED), (dict(num_pages=1 << 27), UNSUPPORTED),
    (dict(total=(1 << 30) + 1), UNSUPPORTED), (dict(reserve=(1 << 30) + 1), UNSUPPORTED),
    (dict(ctx_out=FAKE), INVALID), (dict(held_out=FAKE), INVALID), (dict(free_out=FAKE), INVALID),
    (dict(ws=ctypes.c_void_p(0x10010)), INVALID), (dict(ws_bytes=100), WORKSPACE)]
    + [({n: None}, INVALID) for n in SLOT_NAMES if isinstance(SLOT[n], ctypes.c_void_p)])
def test_slots_refuse(L, over, want):
    assert L.ee_prompt_slots(*with_(SLOT, SLOT_NAMES, **over)) == want


ROPE_NAMES = ("q q_stride k k_stride v v_stride rope n_pos pos slot total n_q n_kv head_dim q_out q_out_stride k_out "
              "k_out_stride k_cache v_cache num_pages ws ws_bytes stream").split()
ROPE = dict(q=FAKE, q_stride=1536, k=FAKE, k_stride=1536, v=FAKE, v_stride=1536, rope=FAKE, n_pos=10, pos=FAKE,
            slot=FAKE, total=5, n_q=8, n_kv=2, head_dim=128, q_out=FAKE, q_out_stride=1024, k_out=None, k_out_stride=0,
            k_cache=FAKE, v_cache=FAKE, num_pages=3, ws=FAKE, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("over,want", [
    (dict(total=-1), INVALID), (dict(n_q=0), INVALID), (dict(n_kv=0), INVALID), (dict(n_pos=0), INVALID),
    (dict(num_pages=0), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(num_pages=1 << 27), UNSUPPORTED),
    (dict(q_stride=1023), INVALID), (dict(q_stride=1016), INVALID), (dict(k_stride=248), INVALID),
    (dict(v_stride=260), INVALID), (dict(q_out_stride=0), INVALID), (dict(k_out=FAKE), INVALID), (dict(q=ODD), INVALID),
    (dict(k=ODD), INVALID), (dict(v=ODD), INVALID), (dict(rope=ODD), INVALID), (dict(q_out=ODD), INVALID),
    (dict(k_cache=ODD), INVALID), (dict(v_cache=ODD), INVALID), (dict(k_out=ODD, k_out_stride=256), INVALID),
    (dict(ws_bytes=100), WORKSPACE), (dict(total=0, q=None), OK)]
    + [({n: None}, INVALID) for n in ROPE_NAMES if isinstance(ROPE[n], ctypes.c_void_p)])
def test_rope_refuses(L, over, want):
    assert L.ee_rope_append(*with_(ROPE, ROPE_NAMES, **over)) == want


PROMPT_NAMES = ("q q_stride k k_stride v v_stride tok_off B total n_q n_kv head_dim scale out lse ws ws_bytes "
                "stream").split()
PROMPT = dict(q=FAKE, q_stride=1024, k=FAKE, k_stride=256, v=FAKE, v_stride=256, tok_off=FAKE, B=2, total=9, n_q=8,
              n_kv=2, head_dim=128, scale=0.1, out=FAKE, lse=None, ws=FAKE, ws_bytes=BIG, stream=None)
SHARED = [
    (dict(B=-1), INVALID), (dict(total=-1), INVALID), (dict(n_q=0), INVALID), (dict(n_kv=0), INVALID),
    (dict(head_dim=64), UNSUPPORTED), (dict(n_q=9), UNSUPPORTED), (dict(n_q=258), UNSUPPORTED),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(q_stride=1020), INVALID), (dict(q_stride=512), INVALID),
    (dict(q=ODD), INVALID), (dict(out=ODD), INVALID), (dict(ws=ctypes.c_void_p(0x10010)), INVALID),
    (dict(ws_bytes=1 << 20), WORKSPACE), (dict(B=0, q=None), OK), (dict(total=0, q=None), OK)]


@pytest.mark.parametrize("over,want", SHARED + [(dict(k_stride=128), INVALID), (dict(v_stride=252), INVALID),
                                                (dict(k=ODD), INVALID), (dict(v=ODD), INVALID)]
                         + [({n: None}, INVALID) for n in PROMPT_NAMES if isinstance(PROMPT[n], ctypes.c_void_p)])
def test_prompt_attn_refuses(L, over, want):
    assert L.ee_prompt_attn(*with_(PROMPT, PROMPT_NAMES, **over)) == want


CHUNK_NAMES = ("q q_stride k_cache v_cache num_pages block_table max_pages ctx_len tok_off B total n_q "
               "n_kv head_dim scale out lse ws ws_bytes stream").split()
CHUNK = dict(q=FAKE, q_stride=1024, k_cache=FAKE, v_cache=FAKE, num_pages=20, block_table=FAKE, max_pages=4,
             ctx_len=FAKE, tok_off=FAKE, B=2, total=9, n_q=8, n_kv=2, head_dim=128, scale=0.1,
             out=FAKE, lse=None, ws=FAKE, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("over,want", SHARED + [
    (dict(num_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(num_pages=1 << 26), UNSUPPORTED),
    (dict(k_cache=ODD), INVALID), (dict(v_cache=ODD), INVALID)]
    + [({n: None}, INVALID) for n in CHUNK_NAMES if isinstance(CHUNK[n], ctypes.c_void_p)])
def test_chunk_attn_refuses(L, over, want):
    assert L.ee_chunk_attn(*with_(CHUNK, CHUNK_NAMES, **over)) == want


def test_workspace_size(L):
    """Four partial slots a CTA (two pieces of two row blocks each) on 152 SMs, after the
    part that the verification entry points keep before their slots."""
    slot = 128 * 128 * 4 + 128 * 8 + 256
    assert L.ee_prompt_workspace_size() == L.ee_workspace_size(1, 1, 1, 128, 0) + 4 * 152 * slot


def test_binding_refuses_wrong_tensors():
    import paper_2506_02780_gb300 as E
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    kv = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    off = torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(16, dtype=torch.uint8)
    out = torch.zeros_like(q)
    cache = torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16)
    table = torch.zeros(1, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        E.ee_prompt_attn(q, kv, kv, off, 0.1, out, ws)
    with pytest.raises(TypeError, match="tok_off"):
        E.ee_prompt_attn(q, kv, kv, off.long(), 0.1, out, ws)
    with pytest.raises(TypeError, match="out"):
        E.ee_prompt_attn(q, kv, kv, off, 0.1, out.float(), ws)
    with pytest.raises(ValueError, match="k and v"):
        E.ee_prompt_attn(q, kv[:3], kv, off, 0.1, out, ws)
    with pytest.raises(ValueError, match="out"):
        E.ee_prompt_attn(q, kv, kv, off, 0.1, out[:3], ws)
    with pytest.raises(ValueError, match="lse"):
        E.ee_prompt_attn(q, kv, kv, off, 0.1, out, ws, lse=torch.zeros(4, 2))
    with pytest.raises(ValueError, match="fit together"):
        E.ee_chunk_attn(q, cache, cache[:2], table, off[:1], off, 0.1, out, ws)
    with pytest.raises(TypeError, match="block_table"):
        E.ee_chunk_attn(q, cache, cache, table.long(), off[:1], off, 0.1, out, ws)
    with pytest.raises(ValueError, match="fit together"):
        E.ee_rope_append(q, kv, kv, torch.zeros(5, 64), off, off, out, cache, cache, ws)
    with pytest.raises(ValueError, match="entries"):
        E.ee_prompt_slots(off, off, off, table, off, off[:1], 3, 0, off, off, off, off, off, off[:1], ws)


class OnDevice(torch.Tensor):
    """A host tensor that says it is a CUDA tensor: the binding's checks, without a GPU."""
    is_cuda = property(lambda self: True)


NULL = types.SimpleNamespace(cuda_stream=0)


def calls(E, ws, kind):
    """Each prompt-intake call with a workspace of this kind; `kind` makes its other tensors."""
    def t(*shape, dtype=torch.bfloat16):
        return kind(torch.zeros(shape, dtype=dtype))

    def i(*shape):
        return t(*shape, dtype=torch.int32)
    q, kv, cache = t(4, 8, 128), t(4, 2, 128), t(3, 2, 16, 128)
    return {
        "slots": lambda: E.ee_prompt_slots(i(1), i(1), i(1), i(1, 3), i(3), i(1), 3, 0, i(2), i(4), i(4), i(1), i(1),
                                           i(1), ws, stream=NULL),
        "rope": lambda: E.ee_rope_append(q, kv, kv, t(5, 128, dtype=torch.float32), i(4), i(4), t(4, 8, 128), cache,
                                         cache, ws, stream=NULL),
        "prompt": lambda: E.ee_prompt_attn(q, kv, kv, i(2), 0.1, t(4, 8, 128), ws, stream=NULL),
        "chunk": lambda: E.ee_chunk_attn(q, cache, cache, i(1, 3), i(1), i(2), 0.1, t(4, 8, 128), ws, stream=NULL),
    }


class Library:
    """Stands for libee: notes the calls that reach it."""
    def __init__(self):
        self.reached = []

    def __getattr__(self, name):
        return lambda *a: self.reached.append(name) or 0


@pytest.mark.parametrize("call", ["slots", "rope", "prompt", "chunk"])
@pytest.mark.parametrize("ws,error", [("host", ValueError), ("strided", ValueError), ("good", None)])
def test_binding_looks_at_the_workspace(monkeypatch, call, ws, error):
    """A workspace in host memory or with gaps never reaches the library."""
    import paper_2506_02780_gb300 as E
    on = lambda x: x.as_subclass(OnDevice)  # noqa: E731
    u8 = torch.zeros(2048, dtype=torch.uint8)
    w = {"host": u8, "strided": on(u8[::2]), "good": on(u8)}[ws]
    L = Library()
    monkeypatch.setattr(E, "lib", lambda: L)
    go = calls(E, w, on)[call]
    if error is None:
        go()
        assert len(L.reached) == 1
    else:
        with pytest.raises(error, match="libee takes"):
            go()
        assert not L.reached


@pytest.mark.parametrize("max_pages,total", [((1 << 27) - 1, 9), ((1 << 27) - 255, 9), (4, (1 << 30) + 1)])
def test_chunk_positions_past_int32_are_refused(L, max_pages, total):
    """Positions are int32, and the kernel's tile arithmetic rounds them up: a table that
    reaches to within 4096 of 2^31 is refused, and so are more tokens than memory holds."""
    over = dict(max_pages=max_pages, total=total)
    assert L.ee_chunk_attn(*with_(CHUNK, CHUNK_NAMES, **over)) == UNSUPPORTED


def test_prompt_positions_past_int32_are_refused(L):
    assert L.ee_prompt_attn(*with_(PROMPT, PROMPT_NAMES, total=2 ** 31 - 1)) == UNSUPPORTED

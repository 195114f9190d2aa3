"""Refusals of the weight products' entry points before any launch (CPU only): the C ABI
on pointers that are never dereferenced, and the binding on wrong tensors."""
import ctypes
import os

import pytest
import torch

from test_prompt_abi import BIG, FAKE, INVALID, ODD, OK, OTHER, UNSUPPORTED, WORKSPACE, with_

UNALIGNED_WS = ctypes.c_void_p(0x10010)
ODD_FLOAT = ctypes.c_void_p(0x10002)
ODD_HALF = ctypes.c_void_p(0x10001)


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


def nulls(args, names, optional=()):
    return [({n: None}, INVALID) for n in names if isinstance(args[n], ctypes.c_void_p) and n not in optional]


QUANT_NAMES = "x x_stride rows cols gated q scale stream".split()
QUANT = dict(x=FAKE, x_stride=512, rows=3, cols=256, gated=0, q=OTHER, scale=OTHER, stream=None)


@pytest.mark.parametrize("over,want", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=250), UNSUPPORTED), (dict(cols=(1 << 24) + 16), UNSUPPORTED),
    (dict(rows=(1 << 30) + 1), UNSUPPORTED), (dict(x_stride=248), INVALID), (dict(x_stride=260), INVALID),
    (dict(gated=1, x_stride=504), INVALID), (dict(x=ODD), INVALID), (dict(q=ODD), INVALID), (dict(scale=ODD_FLOAT), INVALID),
    (dict(rows=0, x=None), OK)] + nulls(QUANT, QUANT_NAMES))
def test_quantize_refuses(L, over, want):
    assert L.ee_fp8_quantize(*with_(QUANT, QUANT_NAMES, **over)) == want


QW_NAMES = "w batch rows cols q scale stream".split()
QW = dict(w=FAKE, batch=2, rows=3, cols=256, q=OTHER, scale=OTHER, stream=None)


@pytest.mark.parametrize("over,want", [
    (dict(batch=-1), INVALID), (dict(rows=0), INVALID), (dict(cols=0), INVALID), (dict(cols=8), UNSUPPORTED),
    (dict(batch=1 << 20, rows=1 << 20, cols=1 << 16), UNSUPPORTED), (dict(w=ODD), INVALID), (dict(q=ODD), INVALID),
    (dict(scale=ODD_FLOAT), INVALID), (dict(batch=0, w=None), OK)] + nulls(QW, QW_NAMES))
def test_quantize_weights_refuses(L, over, want):
    assert L.ee_fp8_quantize_weights(*with_(QW, QW_NAMES, **over)) == want


LIN_NAMES = "x x_scale w w_scale bias n K N out out_stride ws ws_bytes stream".split()
LIN = dict(x=FAKE, x_scale=FAKE, w=FAKE, w_scale=FAKE, bias=FAKE, n=20, K=256, N=100, out=OTHER, out_stride=100, ws=FAKE,
           ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("over,want", [
    (dict(n=-1), INVALID), (dict(K=0), INVALID), (dict(N=0), INVALID), (dict(K=200), UNSUPPORTED),
    (dict(K=(1 << 24) + 16), UNSUPPORTED), (dict(N=(1 << 24) + 1), UNSUPPORTED), (dict(n=(1 << 24) + 1), UNSUPPORTED),
    (dict(out_stride=99), INVALID), (dict(x=ODD), INVALID), (dict(w=ODD), INVALID), (dict(x_scale=ODD_FLOAT), INVALID),
    (dict(w_scale=ODD_FLOAT), INVALID), (dict(bias=ODD_HALF), INVALID), (dict(out=ODD_HALF), INVALID),
    (dict(ws=UNALIGNED_WS), INVALID), (dict(ws_bytes=100), WORKSPACE), (dict(n=0, x=None), OK)]
    + nulls(LIN, LIN_NAMES, ("bias",)))
def test_linear_refuses(L, over, want):
    assert L.ee_fp8_linear(*with_(LIN, LIN_NAMES, **over)) == want


MOE_NAMES = ("x x_stride router w1 w1_scale w2 w2_scale T H I E k renorm live out out_stride ids probs ws ws_bytes "
             "stream").split()
MOE = dict(x=FAKE, x_stride=256, router=FAKE, w1=FAKE, w1_scale=FAKE, w2=FAKE, w2_scale=FAKE, T=20, H=256, I=128, E=8, k=2,
           renorm=0, live=FAKE, out=OTHER, out_stride=256, ids=FAKE, probs=FAKE, ws=FAKE, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(I=0), INVALID), (dict(E=0), INVALID), (dict(k=0), INVALID),
    (dict(k=9), INVALID), (dict(H=250), UNSUPPORTED), (dict(I=120), UNSUPPORTED), (dict(E=257), UNSUPPORTED),
    (dict(E=32, k=17), UNSUPPORTED), (dict(T=4097), UNSUPPORTED), (dict(H=(1 << 16) + 16), UNSUPPORTED),
    (dict(I=(1 << 16) + 16), UNSUPPORTED), (dict(x_stride=248), INVALID), (dict(x_stride=260), INVALID),
    (dict(out_stride=255), INVALID), (dict(x=ODD), INVALID), (dict(router=ODD), INVALID), (dict(w1=ODD), INVALID),
    (dict(w2=ODD), INVALID), (dict(w1_scale=ODD_FLOAT), INVALID), (dict(w2_scale=ODD_FLOAT), INVALID),
    (dict(w1_scale=None), INVALID), (dict(w2_scale=None), INVALID), (dict(out=ODD_HALF), INVALID),
    (dict(live=ODD_FLOAT), INVALID), (dict(ids=ODD_FLOAT), INVALID), (dict(probs=ODD_FLOAT), INVALID),
    (dict(ws=UNALIGNED_WS), INVALID), (dict(ws_bytes=1 << 12), WORKSPACE), (dict(T=0, x=None), OK)]
    + nulls(MOE, MOE_NAMES, ("w1_scale", "w2_scale", "live", "ids", "probs")))
def test_moe_refuses(L, over, want):
    assert L.ee_moe_layer(*with_(MOE, MOE_NAMES, **over)) == want


def test_workspace_sizes(L):
    """Monotonic in every size, so that a workspace of the largest serves them all; zero for sizes that do not exist."""
    base = (64, 512, 256, 16, 4)
    for i in range(5):
        more = list(base)
        more[i] *= 2
        assert L.ee_moe_workspace_size(*more) >= L.ee_moe_workspace_size(*base) > 0
    assert L.ee_moe_workspace_size(-1, 512, 256, 16, 4) == 0 and L.ee_moe_workspace_size(64, 512, 256, 16, 0) == 0
    assert L.ee_linear_workspace_size() > 0
    # no 32-bit product on the way
    assert L.ee_moe_workspace_size(4096, 1 << 16, 1 << 16, 256, 16) > 4 * 4096 * 16 * (1 << 16)


@pytest.mark.parametrize("sizes", [(4097, 512, 256, 16, 4), (64, (1 << 16) + 16, 256, 16, 4), (64, 512, (1 << 16) + 16, 16, 4),
                                   (64, 512, 256, 257, 4), (64, 512, 256, 32, 17), (2**31 - 1,) * 5])
def test_no_workspace_for_sizes_out_of_range(L, sizes):
    """... whose layer is refused, too: nobody finds out at the first call."""
    assert L.ee_moe_workspace_size(*sizes) == 0


# ---------------------------------------------------------------- the binding

def t(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype)


F8, F32, I32 = torch.float8_e4m3fn, torch.float32, torch.int32


def test_binding_refuses_wrong_shapes_and_types(L):
    import paper_2506_02780_gb300 as E
    with pytest.raises(ValueError, match="fit"):
        E.ee_fp8_quantize(t(4, 128), t(4, 256, dtype=F8), t(2, 4, dtype=F32))
    with pytest.raises(ValueError, match="fit"):
        E.ee_fp8_quantize(t(4, 256), t(4, 256, dtype=F8), t(4, 2, dtype=F32))
    with pytest.raises(ValueError, match="fit"):
        E.ee_fp8_quantize(t(4, 256), t(4, 256, dtype=F8), t(2, 4, dtype=F32), gated=True)
    with pytest.raises(TypeError):
        E.ee_fp8_quantize(t(4, 256, dtype=F32), t(4, 256, dtype=F8), t(2, 4, dtype=F32))
    with pytest.raises(ValueError, match="CUDA"):
        E.ee_fp8_quantize(t(4, 256), t(4, 256, dtype=F8), t(2, 4, dtype=F32))
    with pytest.raises(ValueError, match="fit"):
        E.ee_fp8_quantize_weights(t(2, 130, 256), t(2, 130, 256, dtype=F8), t(2, 1, 2, dtype=F32))
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    lin = dict(x=t(4, 256, dtype=F8), x_scale=t(2, 4, dtype=F32), w=t(130, 256, dtype=F8), w_scale=t(2, 2, dtype=F32),
               out=t(4, 130), ws=ws)
    for bad in (dict(x_scale=t(4, 2, dtype=F32)), dict(w_scale=t(1, 2, dtype=F32)), dict(out=t(4, 128)),
                dict(w=t(130, 128, dtype=F8)), dict(bias=t(128))):
        with pytest.raises(ValueError, match="fit"):
            E.ee_fp8_linear(**dict(lin, **bad))
    for bad in (dict(x=t(4, 256)), dict(out=t(4, 130, dtype=F32)), dict(w_scale=t(2, 2))):
        with pytest.raises((TypeError, ValueError)):
            E.ee_fp8_linear(**dict(lin, **bad))
    moe = dict(x=t(4, 256), router=t(8, 256), w1=t(8, 256, 256), w2=t(8, 256, 128), k=2, out=t(4, 256), ws=ws)
    for bad in (dict(router=t(7, 256)), dict(w1=t(8, 128, 256)), dict(out=t(3, 256)), dict(ids=t(4, 3, dtype=I32)),
                dict(probs=t(2, 4, dtype=F32)), dict(live=t(2, dtype=I32)),
                dict(w1_scale=t(8, 2, 1, 2, dtype=F32), w2_scale=t(8, 1, 2, dtype=F32))):
        with pytest.raises(ValueError, match="fit"):
            E.ee_moe_layer(**dict(moe, **bad))
    with pytest.raises(ValueError, match="together"):
        E.ee_moe_layer(**moe, w1_scale=t(8, 2, 1, 2, dtype=F32))
    with pytest.raises(TypeError):
        E.ee_moe_layer(**dict(moe, x=t(4, 256, dtype=F32)))
    with pytest.raises(ValueError, match="CUDA"):
        E.ee_moe_layer(**moe)


def test_rows_of_a_strided_array_must_be_contiguous(L):
    import paper_2506_02780_gb300 as E
    with pytest.raises(ValueError):
        E.ee_fp8_quantize(t(256, 4).t(), t(4, 256, dtype=F8), t(2, 4, dtype=F32))

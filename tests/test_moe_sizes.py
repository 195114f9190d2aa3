"""Sizes that ee_moe_layer refuses are refused where its workspace and its class are made (CPU only)."""
import pytest
import torch

import paper_2506_02780_gb300 as E
from paper_2506_02780_gb300.layers import Experts
from test_prompt_abi import INVALID, OK, UNSUPPORTED, WORKSPACE, with_
from test_weights_abi import L, MOE, MOE_NAMES  # noqa: F401  (L: the fixture)


@pytest.mark.parametrize("T", [-1, 0, 1, 4096, 4097])
@pytest.mark.parametrize("H,I", [(256, 128), (250, 128), (256, 120), (0, 128), (256, 0), (1 << 16, 16), ((1 << 16) + 16, 16),
                                 (16, 1 << 16), (16, (1 << 16) + 16)])
@pytest.mark.parametrize("n_exp,k", [(8, 2), (8, 8), (8, 9), (4, 8), (256, 16), (256, 17), (257, 2), (0, 1), (8, 0)])
def test_a_workspace_exactly_where_a_layer(L, T, H, I, n_exp, k):  # noqa: F811
    """A size of 0 and a refused layer go together (one with a workspace too small is refused for that alone)."""
    status = L.ee_moe_layer(*with_(MOE, MOE_NAMES, T=T, H=H, I=I, E=n_exp, k=k, x_stride=1 << 17, out_stride=1 << 17, ws_bytes=256))
    size = L.ee_moe_workspace_size(T, H, I, n_exp, k)
    assert status in ((INVALID, UNSUPPORTED) if size == 0 else (OK,) if T == 0 else (WORKSPACE,))


@pytest.mark.parametrize("n_exp,H,I,k,tokens", [(4, 256, 128, 8, 16), (4, 256, 120, 2, 16), (4, 250, 128, 2, 16), (4, 256, 128, 2, 5000),
                                                (4, 256, 128, 17, 16), (4, 256, 128, 0, 16)])
@pytest.mark.parametrize("quantize", [False, True])
def test_experts_refuse_at_construction(L, n_exp, H, I, k, tokens, quantize):  # noqa: F811
    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="unsupported sizes"):
        Experts(zeros(n_exp, H), zeros(n_exp, 2 * I, H), zeros(n_exp, H, I), k, quantize=quantize, max_tokens=tokens)
    with pytest.raises(ValueError, match="unsupported sizes"):
        E.new_moe_workspace(tokens, H, I, n_exp, k, device="cpu")


def test_experts_refuse_another_router(L):  # noqa: F811
    with pytest.raises(ValueError, match="router"):
        Experts(torch.zeros(5, 256), torch.zeros(4, 256, 256), torch.zeros(4, 256, 128), 2, max_tokens=4)

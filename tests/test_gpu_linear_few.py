"""Linear layers of a few tokens on both sides of the weights' size from which they go by tiles."""
import pytest
import torch

import paper_2506_02780_gb300 as E
from test_gpu_fp8 import check_linear, gen
from weights_util import make_rows, make_weights

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("K,N", [(8192, 8191), (8192, 8192), (8192, 8200), (8208, 8300), (2064, 40000), (65536, 1030), (16384, 2048),
                                 (16384, 2049)])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16])
def test_few_tokens_on_large_weights(n, K, N):
    g = gen(n + K + N)
    x, xs = make_rows(g, n, K)
    w, wsc = make_weights(g, N, K)
    bias = torch.randn(N, generator=g, device=DEV).to(torch.bfloat16) if n % 2 else None
    ws = E.new_linear_workspace()
    whole = torch.full((n + 1, N + 3), 3.0, dtype=torch.bfloat16, device=DEV)
    out = whole[:n, 1:1 + N]
    E.ee_fp8_linear(x, xs, w, wsc, out, ws, bias=bias)
    assert E.ee_read_errors(ws) == 0
    check_linear(out, x, xs, w, wsc, bias)
    assert (whole[n] == 3.0).all() and (whole[:, 0] == 3.0).all() and (whole[:, 1 + N:] == 3.0).all()
    again = torch.empty(n, N, dtype=torch.bfloat16, device=DEV)
    E.ee_fp8_linear(x, xs, w, wsc, again, ws, bias=bias)
    assert torch.equal(out, again)


@pytest.mark.parametrize("n,K,N", [(20, 16, 300), (64, 48, 5000), (200, 16, 257), (3, 16, 1 << 22), (8, 112, 600007)])
def test_rows_shorter_than_a_block_by_tiles(n, K, N):
    g = gen(n + K + N)
    x, xs = make_rows(g, n, K)
    w, wsc = make_weights(g, N, K)
    ws = E.new_linear_workspace()
    out = torch.empty(n, N, dtype=torch.bfloat16, device=DEV)
    E.ee_fp8_linear(x, xs, w, wsc, out, ws)
    assert E.ee_read_errors(ws) == 0
    check_linear(out, x, xs, w, wsc, None)

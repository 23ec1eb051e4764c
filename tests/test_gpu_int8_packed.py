"""8-bit logits of operands that are copied to rows of whole 16 bytes first: rows of more than one pass of the copy (1,024 bytes), in every
size of tile, either matrix copied alone, with bytes around the rows that are no part of them.  Tolerances are those of test_gpu_int8.py."""
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding
from test_gpu_int8 import DEV, check, operands

pytestmark = pytest.mark.gpu

# rows x vocabulary of tiles of 64 x 128, 128 x 128, 256 x 128 and 256 x 256
TILES = [(65, 900), (100, 3000), (300, 2000), (160, 20000), (700, 12000)]


@pytest.mark.parametrize("h_pad,w_pad,offset", [(0, 0, 0), (0, 0, 1), (7, 0, 0), (0, 3, 15), (1, 1, 0)])
@pytest.mark.parametrize("T,V", TILES)
@pytest.mark.parametrize("D", [1023, 1025, 2047, 4095])
def test_rows_of_several_passes(T, V, D, h_pad, w_pad, offset):
    g = torch.Generator(device=DEV).manual_seed(T + V + D)
    check(*operands(T, V, D, g, h_pad, w_pad, offset), bias=torch.randn(V, device=DEV, generator=g).to(torch.bfloat16), cap=30.0 * (D % 2))


@pytest.mark.parametrize("h_pad,w_pad", [(5, 0), (0, 9), (16, 8), (8, 16)])
@pytest.mark.parametrize("T,V", TILES)
def test_one_matrix_alone(T, V, h_pad, w_pad):
    D = 1040
    g = torch.Generator(device=DEV).manual_seed(T + V)
    need = npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, D, hidden_stride=D + h_pad, weight_stride=D + w_pad)
    assert need == sum(-(-n * D // 256) * 256 for n, pad in ((T, h_pad), (V, w_pad)) if pad % 16)
    check(*operands(T, V, D, g, h_pad, w_pad), workspace=torch.empty(need, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("D", [1, 15, 16, 17, 1024, 1039, 65521])
def test_ends_of_rows(D):
    """Ones, so that a byte of the copy that is wrong changes a sum; the matrices end with their memory."""
    T, V = 70, 500
    h, w = torch.ones((T, D), dtype=torch.int8, device=DEV), torch.ones((V, D + 1), dtype=torch.int8, device=DEV)[:, 1:]
    w[:, :1] = -7 if D > 1 else 1
    out = torch.empty((T, V), dtype=torch.bfloat16, device=DEV)
    npd.npd_head_logits_int8(h, torch.ones(T, device=DEV), w, torch.ones(V, device=DEV), logits_out=out)
    assert torch.equal(out, torch.full_like(out, D - 8 if D > 1 else 1))


@pytest.mark.parametrize("T", [40, 70, 300])
def test_rows_laid_out_with_zeros_are_read_as_they_are(T):
    """What npd_quantize_rows' documentation says: rows of the next multiple of 16, zeros behind the width, need no copy and have the same
    logits.  Rows that only begin there are copied."""
    V, D, S = 1200, 1000, 1008
    g = torch.Generator(device=DEV).manual_seed(T)
    rows, scales = [], []
    for n in (T, V):
        whole, scale = torch.zeros((n, S), dtype=torch.int8, device=DEV), torch.empty(n, device=DEV)
        npd.npd_quantize_rows(torch.randn((n, D), device=DEV, generator=g).to(torch.bfloat16), q_out=whole[:, :D], scale_out=scale)
        assert not bool(whole[:, D:].any())
        rows.append(whole)
        scales.append(scale)
    assert npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, S) == 0
    copied = npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, D, hidden_stride=S, weight_stride=S)
    assert copied == (0 if T <= 64 else -(-T * S // 256) * 256 + -(-V * S // 256) * 256)
    a, b = torch.empty((2, T, V), dtype=torch.bfloat16, device=DEV)
    npd.npd_head_logits_int8(rows[0], scales[0], rows[1], scales[1], logits_out=a, workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
    npd.npd_head_logits_int8(rows[0][:, :D], scales[0], rows[1][:, :D], scales[1], logits_out=b)
    assert torch.equal(a, b)

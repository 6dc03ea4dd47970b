"""One row out of a buffer whose pitch is no multiple of 16 bytes: a single row has no leading dimension, only its own alignment."""
import numpy as np
import pytest
import torch

from helpers import to_dev_bf16
from test_gpu_paged import Attention, cuda, rd, status_clean  # noqa: F401

pytestmark = pytest.mark.gpu


def odd_row(width, fill=None):
    """Row 0 of a [3, width + 3] buffer."""
    t = torch.zeros((3, width + 3), dtype=torch.bfloat16, device="cuda")[:1, :width]
    if fill is not None:
        t.copy_(fill)
    return t


def test_one_row_of_an_odd_pitch(rd):  # noqa: F811
    w = rd.rudder_pack_weights(torch.randn((64, 256), device="cuda"), None, rd.W4A8_INT, 64)
    x = torch.randn((1, 256), device="cuda").to(torch.bfloat16)
    assert torch.equal(rd.rudder_linear_a16(w, odd_row(256, x), None, odd_row(64)), rd.rudder_linear_a16(w, x))
    D, heads = 64, 2
    x = torch.randn((1, 3 * heads * D), device="cuda").to(torch.bfloat16)
    outs = []
    for make in (lambda n: torch.zeros((1, n), dtype=torch.bfloat16, device="cuda"), odd_row):
        X, Q, K = make(x.shape[1]), make(heads * D), make(heads * D)
        X.copy_(x)
        rd.rudder_qk_norm_rope(rd.QkArgs(X, heads, heads, D, None, None, 1e-6, None, None, rd.ROPE_HALF, None, Q, K=K))
        outs.append((Q.clone(), K.clone()))
    assert all(torch.equal(a, b) and a.abs().sum().item() > 0 for a, b in zip(*outs))
    a = Attention(rd, [77], [1], heads, heads, D, 16, "bf16")
    want, _ = a.run(False)
    Q, O = odd_row(heads * D, to_dev_bf16(a.qb)), odd_row(heads * D)
    rd.rudder_attention_paged(rd.AttentionArgs(Q, heads, a.cache, cuda(a.table), cuda(np.array(a.lens, np.int32)), a.scale, O))
    assert np.array_equal(O.float().cpu().numpy().astype(np.float64).reshape(want.shape), want)
    status_clean(rd)

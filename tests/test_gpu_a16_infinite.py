"""Infinite and undefined activations in rudder_linear_a16: what the definition gives for their row, nothing for the others."""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np, to_dev_bf16
from oracle import glue, paged
from test_gpu_paged import A16, cuda, rd, status_clean  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,N", [(1, 256, 64), (6, 768, 128), (16, 4608, 64)])
@pytest.mark.parametrize("scheme,group", A16)
def test_infinite_activations(rd, scheme, group, M, K, N):  # noqa: F811
    rng = np.random.default_rng(K)
    W = torch.from_numpy((rng.standard_normal((N, K)) * 0.02).astype(np.float32)).cuda()
    w = rd.rudder_pack_weights(W, None, rd.SCHEMES[scheme], group or K)
    ex = {k: v.cpu() for k, v in rd.rudder_weight_export(w).items()}
    scales = ex["scales"].view(torch.float8_e4m3fn).float().numpy() if scheme == "nvfp4" else ex["scales"].float().numpy()
    ts = float(ex["tensor_scale"]) if scheme == "nvfp4" else None
    bias = rng.standard_normal(N).astype(np.float32)
    xb = glue.f32_to_bf16(rng.standard_normal((M, K)).astype(np.float32))
    clean = bf16_to_np(rd.rudder_linear_a16(w, to_dev_bf16(xb), cuda(bias)))
    hit = M // 2
    for bad in ([(5, np.inf)], [(K - 1, -np.inf)], [(3, np.inf), (K // 2, np.inf)], [(3, np.inf), (K - 2, -np.inf)], [(7, np.nan)]):
        x = glue.bf16_to_f32(xb).astype(np.float64)
        for channel, value in bad:
            x[hit, channel] = value
        y = bf16_to_np(rd.rudder_linear_a16(w, to_dev_bf16(glue.f32_to_bf16(x.astype(np.float32))), cuda(bias)))
        with np.errstate(invalid="ignore"):
            want, _ = paged.linear_a16(x[hit:hit + 1], ex["codes"].numpy(), scales, ex["dinv"].numpy(), bias, ts)
        got = glue.bf16_to_f32(y[hit])
        # infinity times a weight of zero is undefined, like infinities of both signs: everything else is infinite
        assert not np.isfinite(want[0]).any() and np.array_equal(got.astype(np.float64), want[0], equal_nan=True), (scheme, bad)
        assert np.array_equal(np.delete(y, hit, 0), np.delete(clean, hit, 0))
    status_clean(rd)

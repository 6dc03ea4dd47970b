"""rudder_lora at the ends of the numbers' range, on the GPU: infinite weights, inner sums beside the largest number."""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np
from oracle import glue
from test_gpu_paged import U, rd, status_clean  # noqa: F401  (rd: the fixture)
from test_gpu_shared import i32

pytestmark = pytest.mark.gpu


def bf(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)


def f64(t):
    return glue.bf16_to_f32(bf16_to_np(t.contiguous())).astype(np.float64)


def definition(x, a, b, ranks, scales, rows, base):
    """In 64 bits, as IEEE arithmetic has it: 0 x infinity and infinity - infinity are not numbers."""
    y = f64(base)
    x, a, b = f64(x), f64(a), f64(b)
    with np.errstate(invalid="ignore", over="ignore"):
        for m, i in enumerate(rows):
            if i >= 0 and ranks[i] > 0:
                r = ranks[i]
                h = (a[i, :r] * x[m][None]).sum(1)
                y[m] += float(scales[i]) * (b[i, :, :r] * h[None]).sum(1)
    return y


@pytest.mark.parametrize("M,K,N,R", [(1, 64, 64, 8), (4, 128, 200, 24), (33, 64, 1000, 40), (100, 64, 264, 16), (300, 128, 136, 64), (150, 64, 520, 256)])
@pytest.mark.parametrize("in_place", [False, True])
def test_infinite_weights(rd, M, K, N, R, in_place):
    """Weights of the second product that are infinite or no numbers, beside inner sums that bf16 holds exactly (whole numbers), that it rounds up and that it rounds down, and
    sums of zero: what the definition gives, and every other channel as without them."""
    rng = np.random.default_rng(M + R)
    n = 3
    x, a, b = bf(rng.integers(-3, 4, (M, K))), bf(rng.integers(-2, 3, (n, R, K))), bf(rng.standard_normal((n, N, R)))
    x[M // 2:] = bf(rng.standard_normal((M - M // 2, K)))          # inner sums of 24 bits
    if M > 3:
        x[0] = 0                                                   # inner sums of zero
    ranks, scales = [R, max(1, R - 3), 1], np.array([0.5, -2.0, 1.5], np.float32)
    rows = rng.integers(-1, n, M).astype(np.int32)
    rows[-1], rows[0] = 1, max(0, rows[0])
    clean = b.clone()
    special = [(0, 0, float("inf")), (1, 0, -float("inf")), (N // 2, R - 1, float("inf")), (N // 2 + 1, 0, float("nan")), (N - 1, R // 2, -float("inf")), (N - 1, 0, float("inf"))]
    for col, r, value in special:
        b[:, col, r] = value
    base = bf(rng.standard_normal((M, N)))
    X, A, B, C, ranks_d, scales_d, rows_d = x.cuda(), a.cuda(), b.cuda(), clean.cuda(), i32(ranks), torch.from_numpy(scales).cuda(), i32(rows)

    def run(weights):
        Y = base.cuda() if in_place else torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        rd.rudder_lora(rd.LoraArgs(X, A, weights, ranks_d, scales_d, rows_d, Y if in_place else base.cuda(), Y))
        return f64(Y)

    without, got = run(C), run(B)
    want = definition(x, a, b, ranks, scales, rows, base)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[~odd], without[~odd])
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    assert odd.any() and np.isinf(want).any() and np.isnan(want).any()
    status_clean(rd)


@pytest.mark.parametrize("M", [2, 100])
def test_infinite_weights_of_another_step_of_columns(rd, M):
    """The same where a CTA goes over many columns."""
    N, R, K = 16392, 40, 64
    rng = np.random.default_rng(M)
    x, a, b = bf(rng.integers(-3, 4, (M, K))), bf(rng.integers(1, 3, (1, R, K))), bf(rng.standard_normal((1, N, R)))
    x[:, 0] = 200
    cols = np.arange(5, N, 777)
    b[0, cols, 33] = float("inf")
    base = bf(rng.standard_normal((M, N)))
    Y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    rd.rudder_lora(rd.LoraArgs(x.cuda(), a.cuda(), b.cuda(), i32([R]), torch.ones(1, device="cuda"), i32(np.zeros(M)), base.cuda(), Y))
    got = f64(Y)
    h = f64(a)[0] @ f64(x).T
    assert (h[33] != 0).all()
    assert (got[:, cols] == np.where(h[33] > 0, np.inf, -np.inf)[:, None]).all()
    rest = np.setdiff1d(np.arange(N), cols)
    assert np.isfinite(got[:, rest]).all()
    status_clean(rd)


@pytest.mark.parametrize("M", [3, 90])
def test_inner_sums_beside_the_largest_number(rd, M):
    """An inner sum between the largest bf16 number and 2^128 is a number, not infinity.  Bound as in the other tests: 2^-8 |y| + s (2^-16 + (K + 2 R + 16) 2u)."""
    K, N, R = 64, 72, 8
    x, a, b = np.zeros((M, K), np.float32), np.zeros((1, R, K), np.float32), np.zeros((1, N, R), np.float32)
    x[:, 0], x[:, 1] = 2.0 ** 64, 2.0 ** 60
    a[0, 0, 0] = 2.0 ** 63 * (2 - 2.0 ** -7)                        # 2^127 (2 - 2^-7), and 0.75 2^120 on top: 2^127 (2 - 2^-9), which bf16 rounds to 2^128
    a[0, 0, 1] = 0.75 * 2.0 ** 60
    a[0, 1] = -a[0, 0]
    rng = np.random.default_rng(M)
    b[0, :, 0] = bf(rng.standard_normal(N) * 2.0 ** -120).float().numpy()
    b[0, :, 1] = bf(rng.standard_normal(N) * 2.0 ** -120).float().numpy()
    h = 2.0 ** 127 * (2 - 2.0 ** -9)
    want, s = h * (b[0, :, 0].astype(np.float64) - b[0, :, 1]), h * (np.abs(b[0, :, 0].astype(np.float64)) + np.abs(b[0, :, 1]))
    Y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    rd.rudder_lora(rd.LoraArgs(bf(x).cuda(), bf(a).cuda(), bf(b).cuda(), i32([2]), torch.ones(1, device="cuda"), i32(np.zeros(M)), None, Y))
    got = f64(Y)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + s * (2.0 ** -16 + (K + 2 * R + 16) * 2 * U)).all()
    status_clean(rd)

"""rudder_lora where a CTA goes over many steps of columns and of ranks, on the GPU, against 64 bits: rings that wrap around, base fetched steps ahead of what is written
over it, columns that end inside a step.  Bound as in test_gpu_shared.py: 2^-8 |y| + s (2^-16 + (K + 2 R + 16) 2u)."""
import numpy as np
import pytest

from test_gpu_paged import U, rd, status_clean  # noqa: F401  (rd: the fixture)
from test_gpu_shared import Lora

pytestmark = pytest.mark.gpu


def check(a, y):
    """Lora.check, an adapter at a time."""
    x, wa, wb, base = (h.astype(np.float64) for h in a.host)
    for i in np.unique(a.adapters):
        m = a.adapters == i
        r = 0 if i < 0 else int(a.ranks[i])
        if r == 0:
            assert np.array_equal(y[m], base[m]), i
            continue
        h, s = float(a.scales[i]), abs(float(a.scales[i]))
        want = base[m] + h * ((x[m] @ wa[i, :r].T) @ wb[i, :, :r].T)
        mag = np.abs(base[m]) + s * ((np.abs(x[m]) @ np.abs(wa[i, :r]).T) @ np.abs(wb[i, :, :r]).T)
        bound = 2.0 ** -8 * np.abs(want) + mag * (2.0 ** -16 + (a.K + 2 * a.R + 16) * 2 * U)
        assert np.isfinite(y[m]).all() and (np.abs(y[m] - want) <= bound + 1e-38).all(), (i, r, (np.abs(y[m] - want) / bound).max())


# (148 SMs: steps of columns of a CTA)
@pytest.mark.parametrize("M,K,N,R,ranks,run", [
    (64, 64, 10248, 40, [0, 1, 33, 40], 1),                        # 5, rows as they lie; the last CTA's steps end behind N
    (64, 72, 6152, 256, [256, 1, 33, 0, 130, 255], 1),             # 3 or 4
    (16, 64, 40968, 64, [64, 33, 1], 1),                           # 5
    (50, 64, 8264, 32, [32], 1),
    (2000, 64, 4104, 40, [0, 1, 33, 40], 3),                       # 5, sorted
    (2000, 72, 8200, 256, [256, 33, 1, 0], 500),                   # 9, up to eight steps of ranks
    (1000, 64, 16392, 24, [24, 7, 0, 1, 9], 7), (65, 64, 65544, 32, [32, 31], 1)])
@pytest.mark.parametrize("base", ["none", "same", "other"])
def test_many_steps_of_columns(rd, M, K, N, R, ranks, run, base):
    rng = np.random.default_rng(M + N)
    n = len(ranks)
    rows = np.repeat(rng.integers(-1, n, -(-M // run)), run)[:M]
    a = Lora(rd, M, K, N, R, n, rows, ranks, seed=N, base=base, pads=(8, 0, 16))
    tail = a.buf[:, N:].clone()
    y = a.run()
    check(a, y)
    assert (a.buf[:, N:] == tail).all().item()
    if base != "same":
        assert np.array_equal(y, a.run())
    status_clean(rd)

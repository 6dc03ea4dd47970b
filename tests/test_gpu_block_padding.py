"""rudder_block_cached on a batch that is padded request by request: rows with a negative position inside a request's range."""
import numpy as np
import pytest
import torch

from test_gpu_paged_chain import Step, rd  # noqa: F401

pytestmark = pytest.mark.gpu


class Padded(Step):
    """`width` rows for each request, `new` of them real: first (then padding) or last (padding in front)."""

    def __init__(self, rd, old, new, width, front, **kw):  # noqa: F811
        B = len(old)
        super().__init__(rd, old, new, pad=B * width - sum(new), **kw)
        rd.rudder_page_tables(self.tables)
        pos, slots = self.pos.clone(), self.slots.clone()
        self.pos.fill_(-1), self.slots.fill_(-1)
        at = 0
        for b, n in enumerate(new):
            to = b * width + (width - n if front else 0)
            self.pos[to:to + n], self.slots[to:to + n] = pos[at:at + n], slots[at:at + n]
            at += n
        self.starts, self.max_q = None, width

    def one_by_one(self, step):
        """The public calls with the attention output and lse of the padding cleared in between."""
        rd, M, L = self.rd, self.M, self.layers  # noqa: F811
        seg, pad = L[0].seg, self.pos < 0
        y0 = rd.rudder_linear(L[0].w, rd.rudder_rmsnorm(self.X, self.norm1, 1e-6), seg, step, L[0].tab, L[0].bias)
        q = torch.zeros((M, self.heads * self.D), dtype=torch.bfloat16, device="cuda")
        o, lse = torch.zeros_like(q), torch.full((M, self.heads), 9.0, device="cuda")
        rd.rudder_qk_norm_rope(rd.QkArgs(y0, self.heads, self.kv, self.D, self.qw, self.kw, 1e-6, self.cos, self.sin, rd.ROPE_HALF, self.pos, q, cache=self.cache, slots=self.slots))
        rd.rudder_attention_paged(rd.AttentionArgs(q, self.heads, self.cache, self.table, self.lens, self.scale, o, q_starts=self.starts, max_q=self.max_q, causal=self.causal, lse=lse))
        o[pad], lse[pad] = 0, float("-inf")
        y1 = rd.rudder_linear(L[1].w, o, seg, step, L[1].tab, L[1].bias)
        h = rd.rudder_add(self.X, y1)
        y2 = rd.rudder_linear(L[2].w, rd.rudder_rmsnorm(h, self.norm2, 1e-6), seg, step, L[2].tab, L[2].bias)
        y3 = rd.rudder_linear(L[3].w, rd.rudder_gelu(y2), seg, step, L[3].tab, L[3].bias)
        return [y0, y1, y2, y3], lse, rd.rudder_add(h, y3)

    def fused(self, state, step, stream=None):                      # (the tables are those of the constructor)
        ys, bargs, lse, qk, at, ws, out = state
        self.rd.rudder_block_cached(bargs, self.norm1, self.norm2, 1e-6, out, qk, at, self.M, self.layers[0].seg, step, ws, stream=stream)


@pytest.mark.parametrize("kw", [dict(old=[40, 0, 7, 130], new=[5, 3, 0, 9], width=9, front=False), dict(old=[700, 3], new=[16, 1], width=40, front=True, causal=True, D=128, fmt="e4m3"),
                                dict(old=[31, 64, 2000], new=[1, 2, 2], width=2, front=True, causal=True, heads=8, kv=1), dict(old=[90], new=[1], width=64, front=False, kv=4)])
def test_padding_inside_a_request(rd, kw):  # noqa: F811
    s = Padded(rd, **kw)
    ys, lse, out = s.one_by_one(1)                                  # (both paths append the same keys and values)
    state = s.fresh()
    for _ in range(2):
        s.fused(state, 1)
        torch.cuda.synchronize()
        pad = s.pos < 0
        assert pad.any().item() and torch.isneginf(state[2][pad]).all().item() and torch.isfinite(state[2][~pad]).all().item()
        assert all(torch.equal(a, b) for a, b in zip(state[0], ys))
        assert torch.equal(state[2], lse) and torch.equal(state[6], out)
    last, where = rd.rudder_device_status()
    assert last == 0, (last, where)


def test_padding_behind_the_requests_keeps_its_lse(rd):  # noqa: F811
    """Rows outside every request: zeros for the O projection, lse left as it was."""
    s = Step(rd, [31, 64], [1, 3], pad=3)
    state = s.fresh()
    s.fused(state, 1)
    torch.cuda.synchronize()
    assert (s.pos[-3:] == -1).all().item() and (state[2][-3:] == 9.0).all().item() and torch.isfinite(state[2][:-3]).all().item()
    ys = s.one_by_one(1)[0]
    assert torch.equal(state[0][1], ys[1])

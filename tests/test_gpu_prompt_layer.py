"""Output projection and whole layers of packed prompts at a prompt's number of rows, against fp64."""
from __future__ import annotations

import pytest
import torch

from paper_2607_27269_gb300 import abi
from tests.test_gpu_prompt import R8, Layer, cu_of, i32, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("total", [1, 17, 129, 1000, 4097])
@pytest.mark.parametrize("H,d,hidden", [(14, 64, 896), (24, 128, 520)])
def test_output_projection(H, d, hidden, total):
    """out = W_O o in fp32 sums and one rounding: a sum of K products is off by K 2^-24 of their magnitudes at most."""
    gen = torch.Generator(device="cuda").manual_seed(total)
    o = torch.randn(total, H, d, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(hidden, H * d, generator=gen, device="cuda") * (H * d) ** -0.5).bfloat16()
    out = torch.full((total + 1, hidden), 7.0, dtype=torch.bfloat16, device="cuda")
    abi.gqa_prompt_out_proj(abi.GqaDims(H, 2, d, 1.0), o, w, out)
    assert abi.check_status() == abi.MLA_OK
    a, b = o.double().view(total, -1), w.double()
    want, size = a @ b.T, a.abs() @ b.abs().T
    assert ((out[:total].double() - want).abs() <= R8 * want.abs() + H * d * 2.0 ** -24 * size).all()
    assert (out[total] == 7).all()


@pytest.mark.parametrize("H,G,d,hidden", [(14, 2, 64, 896), (8, 8, 64, 512), (12, 4, 128, 1024)])
def test_layer_from_hidden_at_prompt_lengths(H, G, d, hidden):
    """Ragged prompts, then a chunk behind them: attention over the entries that the layer itself cached, and W_O.  The
    weights' and o's roundings to bf16 enter with sum p|v| and |o| through |W_O|."""
    n = [300, 1, 513, 70]
    total = sum(n)
    kv = [m + 40 for m in n]
    L = Layer(H, G, d, kv, True, seed=41, capacity=640)
    h = L.normal(total + 160, hidden)
    w_q, w_k, w_v = (L.normal(x * d, hidden, std=hidden ** -0.5) for x in (H, G, G))
    w_o = L.normal(hidden, H * d, std=(H * d) ** -0.5)
    step = abi.GqaPrompt(L.dims, L.cache, 4, total, 640)
    chunks = [(h[:total], n, [0] * 4, n), (h[total:], [40] * 4, n, kv)]
    for x, new, start, now in chunks:
        out = step.from_hidden(x, w_q, w_k, w_v, w_o, cu_of(new), i32(start), i32(now))
        assert abi.check_status() == abi.MLA_OK
        L.kv = now
        q = step._proj[0][:sum(new)]  # (rotated in place)
        o, _, av, _ = reference(L, q, new)
        w = w_o.double()
        want = o.reshape(sum(new), -1) @ w.T
        moved = (R8 + 2.0 ** -12) * (av + o.abs()) + 1e-6
        size = (o.abs() + moved).reshape(sum(new), -1) @ w.abs().T
        bar = moved.reshape(sum(new), -1) @ w.abs().T + R8 * (want.abs() + size * R8) + H * d * 2.0 ** -24 * size
        assert ((out.double() - want).abs() <= bar).all()
        # the caches hold the projections: values are a product and one rounding
        t0 = 0
        for b, m in enumerate(new):
            v = x[t0:t0 + m].double() @ w_v.double().T
            most = x[t0:t0 + m].double().abs() @ w_v.double().abs().T
            for g in range(G):
                got = L.v[L.at(b, g, m, start[b])].double()
                cols = slice(g * d, (g + 1) * d)
                assert ((got - v[:, cols]).abs() <= R8 * v[:, cols].abs() + hidden * 2.0 ** -24 * most[:, cols]).all()
            t0 += m

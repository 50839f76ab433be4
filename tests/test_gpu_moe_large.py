"""The mixture-of-experts operators and AdamW where offsets pass 32 bits: what lies behind 2^32 elements against the same rows in a
small call (or the linear layer of one expert).  Codes are the same; sums of a product may be ordered otherwise."""
import pytest
import torch

import paper_2507_16099_amd as fp8

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
ROW = fp8.Recipe(gran=fp8.FP8_ROW)


def _normal(shape, scale=1.0):
    t = torch.empty(shape, dtype=BF16, device="cuda")
    return t.normal_(0, scale)


def _near(got, want):
    """bf16 of two fp32 sums of the same products: a rounding each, and the sums' own error, far below it, where terms cancel."""
    got, want = got.float(), want.float()
    assert torch.isfinite(got).all()
    assert ((got - want).norm() / want.norm()).item() < 2 ** -7
    assert ((got - want).abs() <= 2 ** -7 * want.abs() + 2 ** -10 * want.abs().max()).all()


@pytest.fixture(autouse=True)
def _free():
    torch.manual_seed(7)
    yield
    torch.cuda.empty_cache()


def test_weights_behind_32_bits():
    E, K, N = 40, 8192, 14336      # 4.7e9 weights
    w = _normal((E, N, K), 0.02)
    sizes = torch.tensor([3, 0] * 18 + [0, 1, 2, 70])
    M = int(sizes.sum())
    offsets = torch.cat([torch.zeros(1), sizes.cumsum(0)]).int().cuda()
    x, dy = _normal((M, K)), _normal((M, N), 1e-3)
    last = slice(M - 70, M)
    y = fp8.fp8_grouped_linear_fwd(x, w, offsets, ROW)
    _near(y[last], fp8.fp8_linear_fwd(x[last], w[-1], ROW))
    dx, dw = fp8.fp8_grouped_linear_bwd(dy, x, w, offsets, ROW)
    # (the linear layer's backward takes rows in sixteens: ten rows of zeros more)
    pad = torch.zeros((10, 1), dtype=BF16, device="cuda")
    want_dx, want_dw = fp8.fp8_linear_bwd(torch.cat([dy[last], pad.expand(-1, N)]), torch.cat([x[last], pad.expand(-1, K)]), w[-1], ROW)
    _near(dx[last], want_dx[:70])
    _near(dw[-1], want_dw)
    assert not dw[1].any()
    del dw, dx, want_dw
    wq, sw = fp8.fp8_quantize(w.view(E * N, K), fp8.FP8_ROW, ROW.fmt_w)
    y2 = fp8.fp8_grouped_linear_fwd_prequantized(x, wq.view(E, N, K), ROW.fmt_w, sw.view(E, N), offsets)
    _near(y2[last], y[last])
    # one token, the last expert
    one = torch.tensor([0] * E + [1], dtype=torch.int32, device="cuda")
    y3 = fp8.fp8_grouped_linear_fwd_prequantized(x[-1:], wq.view(E, N, K), ROW.fmt_w, sw.view(E, N), one)
    _near(y3, y[-1:])


def test_rows_behind_32_bits():
    E, K, N = 3, 256, 8192
    sizes = [300_000, 7, 250_000]      # 4.5e9 elements of dY
    M = sum(sizes)
    offsets = torch.tensor([0, 300_000, 300_007, M], dtype=torch.int32, device="cuda")
    x, w, dy = _normal((M, K)), _normal((E, N, K), 0.05), _normal((M, N), 1e-3)
    y = fp8.fp8_grouped_linear_fwd(x, w, offsets, ROW)
    end = slice(M - 500, M)
    _near(y[end], fp8.fp8_linear_fwd(x[end], w[2], ROW))
    _near(y[300_000:300_007], fp8.fp8_linear_fwd(x[300_000:300_007], w[1], ROW))
    del y
    dx, dw = fp8.fp8_grouped_linear_bwd(dy, x, w, offsets, ROW)
    last = slice(300_007, M)
    want_dx, want_dw = fp8.fp8_linear_bwd(dy[last], x[last], w[2], ROW)
    _near(dx[last], want_dx)
    _near(dw[2], want_dw)
    # the last two groups by themselves
    dx2, dw2 = fp8.fp8_grouped_linear_bwd(dy[300_000:], x[300_000:], w[1:], offsets[1:] - 300_000, ROW)
    _near(dx[300_000:], dx2)
    _near(dw[1:], dw2)


def test_combination_behind_32_bits():
    T, k, D = 300_000, 2, 8192
    gates, _, _, row_token, slot_row = fp8.fp8_moe_route(torch.randn((T, 8), device="cuda"), k)
    y, dout = _normal((T * k, D)), _normal((T, D))
    out = fp8.fp8_moe_combine(y, gates, slot_row)
    tail = slice(T - 64, T)
    rows = slot_row[tail].long()
    terms = y[rows].float() * gates[tail, :, None]
    assert ((out[tail].float() - terms.sum(1)).abs() <= 2 ** -8 * terms.sum(1).abs() + 2 ** -22 * terms.abs().sum(1)).all()
    dy, dgates = fp8.fp8_moe_combine_bwd(dout, y, gates, slot_row, row_token)
    want = gates[tail, :, None] * dout[tail, None].float()
    assert ((dy[rows].float() - want).abs() <= (2 ** -8 + 2 ** -23) * want.abs()).all()
    products = y[rows].double() * dout[tail, None].double()
    assert ((dgates[tail].double() - products.sum(2)).abs() <= (D + 1) * 2 ** -24 * products.abs().sum(2)).all()


def test_logits_behind_32_bits():
    T, E, k = (1 << 23) + 1000, 512, 2      # 4.3e9 logits
    logits = _normal((T, E))
    gates, experts, offsets, row_token, slot_row = fp8.fp8_moe_route(logits, k)
    tail = slice(T - 500, T)
    small = fp8.fp8_moe_route(logits[tail], k)
    assert torch.equal(experts[tail], small[1]) and torch.equal(gates[tail], small[0])
    assert torch.equal(row_token[slot_row[tail].long()], torch.arange(T - 500, T, device="cuda", dtype=torch.int32)[:, None].expand(-1, k))
    counts = torch.bincount(experts.flatten().long(), minlength=E)
    assert torch.equal(offsets.long(), torch.cat([torch.zeros(1, device="cuda", dtype=torch.long), counts.cumsum(0)]))
    dgates = torch.randn((T, k), device="cuda")
    d = fp8.fp8_moe_route_bwd(dgates, logits, gates, experts)
    want = fp8.fp8_moe_route_bwd(dgates[tail].contiguous(), logits[tail], gates[tail].contiguous(), experts[tail].contiguous())
    assert torch.equal(d[tail].view(torch.int16), want.view(torch.int16))


def test_adamw_behind_32_bits():
    n = (1 << 32) + 256 * 5 + 3
    tail = n - (256 * 5 + 3)
    p, g = _normal((n,)), _normal((n,), 1e-3)
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    sm, sv = (torch.ones(-(-n // 256), device="cuda") for _ in range(2))
    parts = [t[tail:].clone() for t in (p, g, m, v)] + [s[tail // 256:].clone() for s in (sm, sv)]
    head = p[:4096].clone()
    for tensors, step in ((fp8.fp8_adamw_tensors([p], [g], [m], [v], [sm], [sv]), 1),
                          (fp8.fp8_adamw_tensors(*[[t] for t in parts]), 1)):
        fp8.fp8_adamw_step(tensors, 1e-3, step)
    for big, small in zip((p, g, m, v), parts):
        assert torch.equal(big[tail:].view(torch.uint8), small.view(torch.uint8))
    assert torch.equal(sm[tail // 256:], parts[4]) and torch.equal(sv[tail // 256:], parts[5])
    assert not torch.equal(p[:4096], head)

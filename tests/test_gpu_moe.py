"""Router, grouped linear layers and combination of a mixture of experts against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref
from tests.gpu_util import knobs

pytestmark = pytest.mark.gpu

import paper_2507_16099_amd as fp8  # noqa: E402

BF16 = torch.bfloat16


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _logits(T, E, dtype, seed, masked=0.2, empty=0.1):
    g = _gen(seed)
    x = torch.randn((T, E), generator=g) * 2
    x = torch.where(torch.rand((T, E), generator=g) < 0.3, (x * 2).round() / 2, x)      # ties
    x = x.masked_fill(torch.rand((T, E), generator=g) < masked, -float("inf"))
    return x.masked_fill(torch.rand((T, 1), generator=g) < empty, -float("inf")).to(dtype)


ROUTES = [(1, 1, 1), (1, 8, 2), (3, 2, 2), (16, 64, 6), (17, 33, 16), (64, 16, 16), (65, 16, 4), (200, 17, 3), (257, 128, 8), (700, 130, 1),
          (1000, 256, 8), (333, 512, 5), (2049, 65, 6)]


@pytest.mark.parametrize("dtype", [BF16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("renorm", [False, True], ids=["all", "renorm"])
@pytest.mark.parametrize("T,E,k", ROUTES)
def test_route(T, E, k, renorm, dtype):
    x = _logits(T, E, dtype, T * 1000 + E)
    want = ref.route(x, k, renorm)
    wide = torch.full((T, E + 3), 9.0, dtype=dtype)      # rows further apart than they are long
    wide[:, :E] = x
    flags = fp8.FP8_ROUTE_RENORM if renorm else 0
    dgates = torch.randn((T, k), generator=_gen(5)).cuda()
    dg = dgates.cpu().double().numpy()
    full = ref.route_bwd(x, dg, want["gates"], want["experts"], renorm)
    for logits in (x.cuda(), wide.cuda()[:, :E]):
        gates, experts, offsets, row_token, slot_row = fp8.fp8_moe_route(logits, k, flags)
        for name, got in (("experts", experts), ("offsets", offsets), ("row_token", row_token), ("slot_row", slot_row)):
            assert np.array_equal(got.cpu().numpy(), want[name]), name
        # exponents: the difference's rounding (at most 20 here) and the function's own few; E terms in the sum, a division
        got = gates.cpu().double().numpy()
        assert (np.abs(got - want["gates"]) <= (20 + 8 + E) * 2.0 ** -24 * want["gates"]).all()
        d = fp8.fp8_moe_route_bwd(dgates, logits, gates, experts, flags)
        size = np.abs(dg).sum(1, keepdims=True) + 1e-30      # no entry's terms are larger
        step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
        assert (np.abs(d.cpu().double().numpy() - full) <= step * np.abs(full) + (3 * (28 + E) + k + 4) * 2.0 ** -24 * size).all()


def test_route_gradient_against_differences():
    """The gates' change with each logit, from the 64-bit definition, where the choice does not change."""
    T, E, k = 4, 9, 3
    x = torch.randn((T, E), generator=_gen(3), dtype=torch.float64)
    dg = torch.randn((T, k), generator=_gen(4), dtype=torch.float64)
    for renorm in (False, True):
        flags = fp8.FP8_ROUTE_RENORM if renorm else 0
        xs = x.float()
        gates, experts, *_ = fp8.fp8_moe_route(xs.cuda(), k, flags)
        d = fp8.fp8_moe_route_bwd(dg.float().cuda(), xs.cuda(), gates, experts, flags).cpu().double()
        h = 1e-5
        for e in range(E):
            up, down = xs.double(), xs.double()
            up, down = up.clone(), down.clone()
            up[:, e] += h
            down[:, e] -= h
            a, b = ref.route(up, k, renorm), ref.route(down, k, renorm)
            assert (a["experts"] == b["experts"]).all()
            slope = ((a["gates"] - b["gates"]) * dg.numpy()).sum(1) / (2 * h)
            assert np.abs(d[:, e].numpy() - slope).max() < 1e-5      # fp32 results; the difference's own error is h^2


def test_route_nan_and_infinity_choose_no_row_out_of_range():
    x = torch.randn((70, 24), generator=_gen(9))
    x[3, 5], x[7] = float("nan"), float("nan")
    x[11, 2] = float("inf")
    gates, experts, offsets, row_token, slot_row = (t.cpu() for t in fp8.fp8_moe_route(x.cuda(), 4))
    assert (experts[7] == -1).all() and (slot_row[7] == -1).all() and (gates[7] == 0).all()
    assert 5 not in experts[3].tolist() and experts[11, 0] == 2
    assert offsets[-1] == 69 * 4 and (row_token[:69 * 4] >= 0).all() and (row_token[69 * 4:] == -1).all()


def test_route_of_no_tokens():
    out = fp8.fp8_moe_route(torch.empty((0, 6), device="cuda", dtype=BF16), 2)
    assert out[2].tolist() == [0] * 7 and out[0].shape == (0, 2)


# ---- combination ----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("T,k,D,pad", [(1, 1, 8, 0), (5, 3, 24, 8), (33, 6, 520, 0), (64, 2, 1032, 16), (20, 16, 2048, 0), (9, 5, 4104, 0), (7, 2, 9000, 8)])
def test_combine(T, k, D, pad):
    g = _gen(T * 100 + D)
    routed = ref.route(torch.randn((T, 2 * k), generator=g).masked_fill(torch.rand((T, 2 * k), generator=g) < 0.6, -float("inf")), k, True)
    slot_row, row_token = torch.from_numpy(routed["slot_row"]).int(), torch.from_numpy(routed["row_token"]).int()
    gates = torch.rand((T, k), generator=g)
    M = T * k
    y = torch.full((M, D + pad), 1e30).to(BF16)
    y[:, :D] = torch.randn((M, D), generator=g).to(BF16)
    y[row_token < 0] = float("nan")      # rows of no token are not read
    dout = torch.randn((T, D), generator=g).to(BF16)
    yd, gd, sd, rd = y.cuda()[:, :D], gates.cuda(), slot_row.cuda(), row_token.cuda()
    rows = torch.where(slot_row >= 0, slot_row, 0).long()
    taken = torch.where((slot_row >= 0)[..., None], y[:, :D].double()[rows], 0.0)
    for with_gates in (True, False):
        terms = taken * (gates.double()[..., None] if with_gates else 1.0)
        want, size = terms.sum(1), terms.abs().sum(1)
        out = fp8.fp8_moe_combine(yd, gd if with_gates else None, sd).cpu().double()
        assert ((out - want).abs() <= 2.0 ** -8 * want.abs() + (2 * k + 1) * 2.0 ** -24 * size).all()
    dy, dgates = fp8.fp8_moe_combine_bwd(dout.cuda(), yd, gd, sd, rd)
    want = (taken * dout.double()[:, None]).sum(2)
    size = (taken * dout.double()[:, None]).abs().sum(2)
    assert ((dgates.cpu().double() - want).abs() <= (D + 1) * 2.0 ** -24 * size).all()
    want = torch.zeros((M, D), dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            if slot_row[t, j] >= 0:
                want[slot_row[t, j]] = gates[t, j].double() * dout[t].double()
    assert ((dy.cpu().double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all()
    only, none = fp8.fp8_moe_combine_bwd(dout.cuda(), yd, gd, sd, rd, need_dgates=False)
    assert none is None and torch.equal(only.view(torch.int16), dy.view(torch.int16))
    none, only = fp8.fp8_moe_combine_bwd(dout.cuda(), yd, gd, sd, None, need_dy=False)
    assert none is None and torch.equal(only, dgates)


def test_combine_leaves_out_rows_that_do_not_exist():
    y = torch.randn((4, 16), generator=_gen(1)).to(BF16).cuda()
    slots = torch.tensor([[0, 4], [-7, 3], [1 << 30, -1]], dtype=torch.int32).cuda()
    out = fp8.fp8_moe_combine(y, None, slots)
    assert torch.equal(out[0], y[0]) and torch.equal(out[1], y[3]) and (out[2] == 0).all()


# ---- grouped linear -------------------------------------------------------------------------------------------------


def _case(sizes, T, K, N, seed, tail=0):
    g = _gen(seed)
    M = sum(sizes) + tail
    offsets = torch.tensor([0, *np.cumsum(sizes)], dtype=torch.int32)
    row_token = torch.randint(0, T, (M,), generator=g, dtype=torch.int32)
    row_token[M - tail:] = -1
    x = torch.randn((T, K), generator=g).to(BF16)
    w = (torch.randn((len(sizes), N, K), generator=g) * 0.02 * torch.rand((len(sizes), N, 1), generator=g)).to(BF16)
    dy = (torch.randn((M, N), generator=g) * 1e-3).to(BF16)
    if tail:
        dy[M - tail:] = float("nan")      # rows of no expert: not used
    return offsets, row_token, x, w, dy


# (group sizes, tokens, K, N, rows behind the last group)
GROUPS = [
    ([1], 1, 16, 16, 0),
    ([0, 1, 0], 1, 32, 48, 0),
    ([0, 0], 3, 64, 64, 5),
    ([3, 0, 17, 1, 0, 40], 30, 144, 80, 2),
    ([128, 1, 127, 129], 200, 256, 272, 0),
    ([700], 512, 512, 384, 9),
    ([0, 300, 5, 0, 0, 260, 64, 63], 90, 640, 144, 100),
    ([2] * 70 + [0] * 3 + [9], 100, 128, 96, 1),
    ([511, 1, 513], 1000, 1040, 528, 0),
    ([90, 1200], 600, 784, 1040, 3),
    ([0, 5, 0, 1, 0, 2] * 52, 200, 64, 112, 7),      # more groups than are looked up at a time
    ([3000, 1], 1500, 80, 160, 0),                   # a group that does not stay in registers
    ([20] * 40, 300, 96, 272, 0),
    ([700, 0, 1500, 3], 400, 48, 4112, 5),           # long groups with long rows of the gradient
    ([1, 1400], 100, 32, 8208, 0),
    ([690], 64, 16, 16400, 2),
    ([1, 0, 3] * 170 + [5, 2], 100, 48, 80, 4),      # as many groups as there can be
]
RECIPES = {"row": {}, "pow2": {"flags": 1}, "swapped": {"fmt_x": 1, "fmt_w": 1, "fmt_dy": 0}}


@pytest.mark.parametrize("recipe", RECIPES)
@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_grouped_linear(case, recipe):
    sizes, T, K, N, tail = GROUPS[case]
    r = fp8.Recipe(gran=fp8.FP8_ROW, **RECIPES[recipe])
    fmt = {0: ref.E4M3, 1: ref.E5M2}
    pow2 = bool(r.flags & fp8.FP8_POW2_SCALE)
    offsets, row_token, x, w, dy = _case(sizes, T, K, N, 77 + case, tail)
    od, rd, xd, wd, dyd = offsets.cuda(), row_token.cuda(), x.cuda(), w.cuda(), dy.cuda()
    xr = ref.rows_of(x, row_token)
    want, size = ref.grouped_fwd(xr, w, offsets, fmt[r.fmt_x], fmt[r.fmt_w], pow2)
    y = fp8.fp8_grouped_linear_fwd(xd, wd, od, r, row_token=rd)
    ref.assert_product(y.cpu(), want, size)
    # the same with the weights quantized beforehand: the same codes, and the same bits where the sums have the same order
    E = len(sizes)
    wq, sw = fp8.fp8_quantize(wd.view(E * N, K), fp8.FP8_ROW, r.fmt_w, r.flags)
    y2 = fp8.fp8_grouped_linear_fwd_prequantized(xd, wq.view(E, N, K), r.fmt_w, sw.view(E, N), od, r.fmt_x, r.flags, row_token=rd)
    ref.assert_product(y2.cpu(), want, size)
    # rows given as they are: the same bits
    y3 = fp8.fp8_grouped_linear_fwd(xr.cuda(), wd, od, r)
    assert torch.equal(y.view(torch.int16), y3.view(torch.int16))
    (want_dx, size_dx), (want_dw, size_dw) = ref.grouped_bwd(dy, xr, w, offsets, fmt[r.fmt_dy], fmt[r.fmt_x], fmt[r.fmt_w], pow2)
    dx, dw = fp8.fp8_grouped_linear_bwd(dyd, xd, wd, od, r, row_token=rd)
    ref.assert_product(dx.cpu(), want_dx, size_dx)
    ref.assert_product(dw.cpu(), want_dw, size_dw)
    only, none = fp8.fp8_grouped_linear_bwd(dyd, xd, wd, od, r, row_token=rd, need_dw=False)
    assert none is None and torch.equal(only.view(torch.int16), dx.view(torch.int16))
    none, only = fp8.fp8_grouped_linear_bwd(dyd, xd, wd, od, r, row_token=rd, need_dx=False)
    assert none is None and torch.equal(only.view(torch.int16), dw.view(torch.int16))


# few rows per expert: a row, tiles of sixteen and more, runs that cross from expert to expert, none at all, long and odd rows
FEW = [([1], 1, 16, 16, 0), ([0, 1, 0, 1], 1, 4096, 4096, 0), ([2, 0, 0, 0], 2, 1040, 24, 0), ([16, 17, 0, 5, 1, 33], 40, 528, 200, 3),
       ([0] * 200 + [1] * 50 + [7, 0], 33, 256, 8, 4), ([6] * 64, 64, 2048, 112, 0), ([3, 1, 0, 12], 9, 9008, 40, 0), ([1, 2], 3, 16384, 24, 0),
       ([0, 0, 0], 2, 64, 32, 6), ([9, 15, 1], 25, 16400, 32, 0), ([1] * 31 + [0, 40], 9, 144, 600, 2)]


@pytest.mark.parametrize("recipe", RECIPES)
@pytest.mark.parametrize("case", range(len(FEW)))
def test_few_rows_against_quantized_weights(case, recipe):
    sizes, T, K, N, tail = FEW[case]
    r = fp8.Recipe(gran=fp8.FP8_ROW, **RECIPES[recipe])
    fmt = {0: ref.E4M3, 1: ref.E5M2}
    offsets, row_token, x, w, _ = _case(sizes, T, K, N, 177 + case, tail)
    if row_token.numel() > 3:
        row_token[2] = T + 5      # a token that is none: a row of zeros
    E, xr = len(sizes), ref.rows_of(x, row_token)
    want, size = ref.grouped_fwd(xr, w, offsets, fmt[r.fmt_x], fmt[r.fmt_w], bool(r.flags))
    wd = torch.zeros((E, N, K + 16), dtype=torch.bfloat16, device="cuda")      # rows of codes further apart than they are long
    wd[:, :, :K] = w.cuda()
    wq = torch.full((E * N, K + 16), 0x7F, dtype=torch.uint8, device="cuda")
    _, sw = fp8.fp8_quantize(wd.view(E * N, K + 16)[:, :K], fp8.FP8_ROW, r.fmt_w, r.flags, out=wq[:, :K])
    y = torch.full((len(row_token), N), float("nan"), dtype=BF16, device="cuda")
    fp8.fp8_grouped_linear_fwd_prequantized(x.cuda(), wq.view(E, N, K + 16)[:, :, :K], r.fmt_w, sw.view(E, N), offsets.cuda(), r.fmt_x, r.flags,
                                            row_token=row_token.cuda(), y=y)
    ref.assert_product(y.cpu(), want, size)
    # every form that takes such a call: quantization inside the product, tiles of every size, persistent workgroups
    for switches in ({"SKINNY_DMA": 2}, *({"SKINNY_DMA": 0, "GEMM_RING": 1 + f} for f in range(6)),
                     {"SKINNY_DMA": 0, "GEMM_STREAM": 8}):
        with knobs(**switches):
            other = torch.full_like(y, float("nan"))
            fp8.fp8_grouped_linear_fwd_prequantized(x.cuda(), wq.view(E, N, K + 16)[:, :, :K], r.fmt_w, sw.view(E, N), offsets.cuda(), r.fmt_x,
                                                    r.flags, row_token=row_token.cuda(), y=other)
            ref.assert_product(other.cpu(), want, size)
    if not tail and case % 2:      # the rows as they are
        y2 = fp8.fp8_grouped_linear_fwd_prequantized(xr.cuda(), wq.view(E, N, K + 16)[:, :, :K], r.fmt_w, sw.view(E, N), offsets.cuda(), r.fmt_x, r.flags)
        assert torch.equal(y.view(torch.int16), y2.view(torch.int16))


@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_every_form_of_the_products(case):
    """Tiles of every size, and few persistent workgroups that walk many tiles: the same results within the sums' bounds."""
    sizes, T, K, N, tail = GROUPS[case]
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    offsets, row_token, x, w, dy = _case(sizes, T, K, N, 300 + case, tail)
    xr = ref.rows_of(x, row_token)
    want, size = ref.grouped_fwd(xr, w, offsets, ref.E4M3, ref.E4M3, False)
    (want_dx, size_dx), (want_dw, size_dw) = ref.grouped_bwd(dy, xr, w, offsets, ref.E5M2, ref.E4M3, ref.E4M3, False)
    args = (x.cuda(), w.cuda(), offsets.cuda(), r)
    for switches in (*({"GEMM_RING": 1 + f} for f in range(6)), {"GEMM_RING": 5, "GEMM_STREAM": 8}, {"GEMM_RING": 6, "GEMM_STREAM": 8},
                     {"GEMM_RING": 3, "GEMM_STREAM": 8}, {"GEMM_RING": 4, "GEMM_STREAM": 0}):
        with knobs(**switches):
            y = fp8.fp8_grouped_linear_fwd(*args, row_token=row_token.cuda())
            dx, dw = fp8.fp8_grouped_linear_bwd(dy.cuda(), *args, row_token=row_token.cuda())
            ref.assert_product(y.cpu(), want, size)
            ref.assert_product(dx.cpu(), want_dx, size_dx)
            ref.assert_product(dw.cpu(), want_dw, size_dw)


@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_every_way_to_the_operands_gives_the_same_codes(case):
    """Strips, maxima and cast, rows and maxima from one read: the operands of a product are the same, so is what comes out."""
    sizes, T, K, N, tail = GROUPS[case]
    offsets, row_token, x, w, dy = _case(sizes, T, K, N, 500 + case, tail)
    for r in (fp8.Recipe(gran=fp8.FP8_ROW), fp8.Recipe(gran=fp8.FP8_ROW, fmt_x=1, fmt_w=1, fmt_dy=0, flags=1)):
        outs = []
        for strips in (-1, 0, 2):
            with knobs(STRIPS=strips):
                outs.append(fp8.fp8_grouped_linear_bwd(dy.cuda(), x.cuda(), w.cuda(), offsets.cuda(), r, row_token=row_token.cuda()))
        for dx, dw in outs[1:]:
            assert torch.equal(dx.view(torch.int16), outs[0][0].view(torch.int16)) and torch.equal(dw.view(torch.int16), outs[0][1].view(torch.int16))


@pytest.mark.parametrize("offsets", [[0, 50, 20, 90, 200, -5], [0, -3, -4, 1 << 30, 7, 100], [7, 7, 7, 7, 7, 7], [0, 2147483647, -2147483648, 60, 40, 100]])
def test_wrong_offsets_stay_in_bounds(offsets):
    """Cut to a rising sequence within the rows: the same as with what is left of them."""
    M, E, K, N = 100, 5, 256, 144
    _, row_token, x, w, dy = _case([M, 0, 0, 0, 0], 60, K, N, 8)
    cut = np.maximum.accumulate(np.clip([0, *offsets[1:]], 0, M))
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    row_token[::9] = torch.tensor([-1, 60, 1 << 30, -(1 << 31)], dtype=torch.int32).repeat(9)[:row_token[::9].numel()]      # tokens that are none: zeros
    outs = []
    for o in (offsets, cut):
        od = torch.tensor(np.array(o), dtype=torch.int32).cuda()
        y = fp8.fp8_grouped_linear_fwd(x.cuda(), w.cuda(), od, r, row_token=row_token.cuda())
        outs.append((y, *fp8.fp8_grouped_linear_bwd(dy.cuda(), x.cuda(), w.cuda(), od, r, row_token=row_token.cuda())))
    for a, b in zip(*outs):
        assert torch.isfinite(a.float()).all() and torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_grouped_linear_equals_the_linear_layer_of_a_lone_group():
    """One expert with all rows: the codes are those of the linear layer, the sums may differ in their order."""
    M, K, N = 300, 512, 256
    _, _, x, w, dy = _case([M], M, K, N, 4)
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    od = torch.tensor([0, M], dtype=torch.int32).cuda()
    y = fp8.fp8_grouped_linear_fwd(x.cuda(), w.cuda(), od, r).double()
    one = fp8.fp8_linear_fwd(x.cuda(), w[0].cuda(), r).double()
    assert ((y - one).norm() / one.norm()).item() < 1e-3
    dx, dw = fp8.fp8_grouped_linear_bwd(dy.cuda(), x.cuda(), w.cuda(), od, r)
    dx1, dw1 = fp8.fp8_linear_bwd(dy.cuda(), x.cuda(), w[0].cuda(), r)
    assert ((dx.double() - dx1.double()).norm() / dx1.double().norm()).item() < 1e-3
    assert ((dw[0].double() - dw1.double()).norm() / dw1.double().norm()).item() < 1e-3


def test_zero_and_tiny_rows():
    """Rows and columns of zeros, and of values below the scale's clamp, give zeros and what is left of them, no NaN."""
    M, K, N = 40, 128, 64
    offsets, row_token, x, w, dy = _case([25, 15], M, K, N, 6)
    x[3] = 0
    x[:, 7] = 0
    x[4] = 1e-20
    w[0, 5] = 0
    w[1, :, 9] = 0
    dy[:, 11] = 0
    dy[2] = 0
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    xr = ref.rows_of(x, row_token)
    y = fp8.fp8_grouped_linear_fwd(x.cuda(), w.cuda(), offsets.cuda(), r, row_token=row_token.cuda())
    ref.assert_product(y.cpu(), *ref.grouped_fwd(xr, w, offsets, ref.E4M3, ref.E4M3, False))
    dx, dw = fp8.fp8_grouped_linear_bwd(dy.cuda(), x.cuda(), w.cuda(), offsets.cuda(), r, row_token=row_token.cuda())
    a, b = ref.grouped_bwd(dy, xr, w, offsets, ref.E5M2, ref.E4M3, ref.E4M3, False)
    ref.assert_product(dx.cpu(), *a)
    ref.assert_product(dw.cpu(), *b)


def test_no_rows():
    E, K, N = 3, 64, 32
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    w = torch.ones((E, N, K), dtype=BF16, device="cuda")
    x, dy, o = torch.empty((0, K), dtype=BF16, device="cuda"), torch.empty((0, N), dtype=BF16, device="cuda"), torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    assert fp8.fp8_grouped_linear_fwd(x, w, o, r).shape == (0, N)
    dx, dw = fp8.fp8_grouped_linear_bwd(dy, x, w, o, r)
    assert dx.shape == (0, K) and (dw == 0).all()


def test_on_another_stream():
    offsets, row_token, x, w, dy = _case([60, 0, 200, 11], 150, 256, 512, 12, tail=4)
    args = [t.cuda() for t in (x, w, offsets)]
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    want = fp8.fp8_grouped_linear_fwd(*args, r, row_token=row_token.cuda())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = fp8.fp8_grouped_linear_fwd(*args, r, row_token=row_token.cuda())
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def _layer(x, wr, w1, w2, dout, k, r, out):
    """Forward and backward of a layer: router, two linear layers per expert, combination."""
    logits = x.float() @ wr.float().T
    gates, experts, offsets, row_token, slot_row = fp8.fp8_moe_route(logits, k, fp8.FP8_ROUTE_RENORM)
    h = fp8.fp8_grouped_linear_fwd(x, w1, offsets, r, row_token=row_token)
    y = fp8.fp8_grouped_linear_fwd(h, w2, offsets, r)
    o = fp8.fp8_moe_combine(y, gates, slot_row)
    dy, dgates = fp8.fp8_moe_combine_bwd(dout, y, gates, slot_row, row_token)
    dh, dw2 = fp8.fp8_grouped_linear_bwd(dy, h, w2, offsets, r)
    dxr, dw1 = fp8.fp8_grouped_linear_bwd(dh, x, w1, offsets, r, row_token=row_token)
    dx = fp8.fp8_moe_combine(dxr, None, slot_row)
    dlogits = fp8.fp8_moe_route_bwd(dgates, logits, gates, experts, fp8.FP8_ROUTE_RENORM)
    for to, t in zip(out, (o, dx, dw1, dw2, dlogits)):
        to.copy_(t)


def test_layer_replays_from_a_graph():
    """A whole layer, recorded; replays with other inputs, eager work in between, give the eager results bit for bit."""
    T, E, k, K, H = 300, 6, 2, 256, 320
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    g = _gen(2)
    rand = lambda *s: torch.randn(s, generator=g).to(BF16).cuda()      # noqa: E731
    sets = [(rand(T, K), rand(E, K), rand(E, H, K), rand(E, K, H), rand(T, K)) for _ in range(3)]
    held = [torch.empty_like(t) for t in sets[0]]
    outs = [torch.empty((T, K), dtype=BF16, device="cuda"), torch.empty((T, K), dtype=BF16, device="cuda"), torch.empty((E, H, K), dtype=BF16, device="cuda"),
            torch.empty((E, K, H), dtype=BF16, device="cuda"), torch.empty((T, E), dtype=torch.float32, device="cuda")]
    for h, t in zip(held, sets[0]):
        h.copy_(t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(*held, k, r, outs)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _layer(*held, k, r, outs)
    for n in (1, 2, 0, 1):
        for h, t in zip(held, sets[n]):
            h.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        _layer(*sets[n], k, r, outs)
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b), n


def test_empty_sums_are_zero():
    offsets, row_token = torch.tensor([0, 2, 5], dtype=torch.int32).cuda(), torch.zeros(5, dtype=torch.int32).cuda()
    r = fp8.Recipe(gran=fp8.FP8_ROW)
    bf16 = dict(dtype=BF16, device="cuda")
    y = torch.full((5, 24), 7.0, **bf16)
    fp8.fp8_grouped_linear_fwd(torch.empty((1, 0), **bf16), torch.empty((2, 24, 0), **bf16), offsets, r, row_token=row_token, y=y)
    assert (y == 0).all()
    dx = torch.full((5, 48), 7.0, **bf16)
    fp8.fp8_grouped_linear_bwd(torch.empty((5, 0), **bf16), torch.randn((1, 48), **bf16), torch.empty((2, 0, 48), **bf16), offsets, r,
                               row_token=row_token, dx=dx, need_dw=False)
    assert (dx == 0).all()
    # no rows at all: zeros for the weights
    none, dw = fp8.fp8_grouped_linear_bwd(torch.empty((0, 32), **bf16), torch.empty((0, 48), **bf16), torch.randn((2, 32, 48), **bf16),
                                          torch.zeros(3, dtype=torch.int32, device="cuda"), r, dw=torch.full((2, 32, 48), 7.0, **bf16), need_dx=False)
    assert (dw == 0).all()

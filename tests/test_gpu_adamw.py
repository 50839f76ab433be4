"""The AdamW step against the formula in 64 bits."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref

pytestmark = pytest.mark.gpu

import paper_2507_16099_amd as fp8  # noqa: E402

HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
SIZES = [1, 7, 8, 255, 256, 257, 511, 0, 4096, 8191, 8192, 8193, 70001]


def _make(sizes, p_type, g_type, seed, moments=True):
    g = torch.Generator().manual_seed(seed)
    ps = [(torch.randn(n, generator=g) * 0.05).to(p_type) for n in sizes]
    gs = [(torch.randn(n, generator=g) * torch.rand(n, generator=g) * 1e-2).to(g_type) for n in sizes]
    ms = [torch.randn(n, generator=g) * 1e-3 if moments else torch.zeros(n) for n in sizes]
    rs = [torch.rand(n, generator=g) * 1e-2 if moments else torch.zeros(n) for n in sizes]
    for x in (gs, ms, rs):      # unused rows
        for t in x:
            t[256:512] = 0
    return ps, gs, ms, rs


def _quantize(x, root):
    """Blocks of 256 -> (codes, scales) by the definition."""
    n = x.numel()
    b = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
    s = (448.0 / b.abs().amax(1).double().clamp(min=1e-12)).float()
    s = (s.view(torch.int32) & -0x800000).view(torch.float32)
    y = b * s[:, None]
    if root:
        y = torch.where(b > 0, y.clamp(min=2.0 ** -9), y)
    return y.to(ref.E4M3).view(torch.uint8).view(-1)[:n].clone(), s


def _values(q, s):
    return q.view(ref.E4M3).double() / s.double().repeat_interleave(256)[:q.numel()]


@pytest.mark.parametrize("g_type", [torch.bfloat16, torch.float32], ids=["g16", "g32"])
@pytest.mark.parametrize("p_type", [torch.bfloat16, torch.float32], ids=["p16", "p32"])
@pytest.mark.parametrize("scaled", [False, True])
def test_moments_in_32_bits(p_type, g_type, scaled):
    ps, gs, ms, rs = _make(SIZES, p_type, g_type, 1)
    vs = [r * r for r in rs]
    c = torch.tensor([0.37]) if scaled else None
    dev = [[t.cuda() for t in ts] for ts in (ps, gs, ms, vs)]
    fp8.fp8_adamw_step(fp8.fp8_adamw_tensors(*dev), step=7, grad_scale=None if c is None else c.cuda(), **HYPER)
    for i in range(len(SIZES)):
        want = ref.adamw(*(t[i].double() for t in (ps, gs, ms, vs)), step=7, c=1.0 if c is None else float(c), **HYPER)
        half = 2.0 ** -8 if p_type == torch.bfloat16 else 0.0
        for got, (value, off), step in zip((dev[0][i], dev[2][i], dev[3][i]), want, (half, 0.0, 0.0)):
            assert ((got.cpu().double() - value).abs() <= off + step * (value.abs() + off)).all()


@pytest.mark.parametrize("g_type", [torch.bfloat16, torch.float32], ids=["g16", "g32"])
@pytest.mark.parametrize("p_type", [torch.bfloat16, torch.float32], ids=["p16", "p32"])
@pytest.mark.parametrize("moments", [True, False], ids=["later", "first"])
def test_moments_in_8_bits(p_type, g_type, moments):
    ps, gs, ms, rs = _make(SIZES, p_type, g_type, 2, moments)
    mq, vq = [_quantize(m, False) for m in ms], [_quantize(r, True) for r in rs]
    c = torch.tensor([1.5])
    dev = [[t.cuda() for t in ts] for ts in (ps, gs, [q for q, _ in mq], [q for q, _ in vq], [s for _, s in mq], [s for _, s in vq])]
    step = 7 if moments else 1
    fp8.fp8_adamw_step(fp8.fp8_adamw_tensors(*dev), step=step, grad_scale=c.cuda(), **HYPER)
    for i, n in enumerate(SIZES):
        m0, r0 = _values(*mq[i]), _values(*vq[i])
        (p1, off_p), (m1, off_m), (v1, off_v) = ref.adamw(ps[i].double(), gs[i].double(), m0, r0 * r0, step=step, c=1.5, **HYPER)
        half = 2.0 ** -8 if p_type == torch.bfloat16 else 0.0
        assert ((dev[0][i].cpu().double() - p1).abs() <= off_p + half * (p1.abs() + off_p)).all()
        r1 = v1.sqrt()
        for q, s, value, off, root in ((dev[2][i], dev[4][i], m1, off_m, False), (dev[3][i], dev[5][i], r1, 5 * 2.0 ** -24 * r1, True)):
            q, s = q.cpu(), s.cpu()
            if n == 0:
                continue
            padded = torch.nn.functional.pad(value, (0, -n % 256)).view(-1, 256).abs().amax(1)
            # power-of-two scales that bring the block's largest into (224, 448]; the roundings in front of it count too
            assert (torch.frexp(s)[0] == 0.5).all()
            largest = padded * s.double()
            busy = padded > 1e-12
            assert (largest[busy] <= 448 * (1 + 2.0 ** -20)).all() and (largest[busy] > 224 * (1 - 2.0 ** -20)).all()
            assert (s[~busy] == 2.0 ** 48).all()
            got, scale = _values(q, s), s.double().repeat_interleave(256)[:n]
            # half a step: 2^-4 of the value, among the smallest codes half of 2^-9; a root's smallest code may be a whole step off
            bound = off + 2.0 ** -4 * (value.abs() + off) + (2.0 ** -9 if root else 2.0 ** -10) / scale
            assert ((got - value).abs() <= bound).all()
            if root:
                assert ((q != 0) == (value > 0)).all()


def test_roots_do_not_vanish():
    """An element far below the largest of its block keeps a root, so that its next update stays bounded."""
    n = 256
    p, g = torch.zeros(n), torch.full((n,), 1e-9)
    g[0] = 1.0
    dev = [[p.cuda()], [g.cuda()], [torch.zeros(n, dtype=torch.uint8).cuda()], [torch.zeros(n, dtype=torch.uint8).cuda()],
           [torch.ones(1).cuda()], [torch.ones(1).cuda()]]
    tensors = fp8.fp8_adamw_tensors(*dev)
    for step in range(1, 6):
        fp8.fp8_adamw_step(tensors, step=step, **HYPER)
        assert dev[0][0].abs().max() <= step * HYPER["lr"] * 1.5
    assert (dev[3][0] != 0).all()


def test_scales_that_were_never_written():
    """Codes of zero with scales of zero (cleared memory): a first step like any other."""
    n = 300
    z = lambda k, d: torch.zeros(k, dtype=d, device="cuda")      # noqa: E731
    g = torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda()
    runs = []
    for s in (0.0, 1.0):
        p = z(n, torch.float32)
        t = [[p], [g], [z(n, torch.uint8)], [z(n, torch.uint8)], [z(2, torch.float32) + s], [z(2, torch.float32) + s]]
        fp8.fp8_adamw_step(fp8.fp8_adamw_tensors(*t), step=1, **HYPER)
        runs.append(p)
    assert torch.isfinite(runs[0]).all() and torch.equal(*runs)


def test_more_tensors_than_a_launch_holds():
    sizes = [97 * (i % 5) + i for i in range(150)]
    ps, gs, ms, rs = _make(sizes, torch.float32, torch.bfloat16, 3)
    dev = [[t.cuda() for t in ts] for ts in (ps, gs, ms, [r * r for r in rs])]
    fp8.fp8_adamw_step(fp8.fp8_adamw_tensors(*dev), step=2, **HYPER)
    for i in range(len(sizes)):
        (value, off), *_ = ref.adamw(ps[i].double(), gs[i].double(), ms[i].double(), (rs[i] * rs[i]).double(), step=2, c=1.0, **HYPER)
        assert ((dev[0][i].cpu().double() - value).abs() <= off).all()


def test_nothing_outside_the_tensors_is_written():
    n = 1000
    base = [torch.full((n + 512,), 3.0).to(t).cuda() for t in (torch.bfloat16, torch.bfloat16)]
    codes = [torch.full((n + 512,), 77, dtype=torch.uint8).cuda() for _ in range(2)]
    scales = [torch.full((8,), 4.0).cuda() for _ in range(2)]
    t = [[base[0][:n]], [base[1][:n]], [codes[0][:n]], [codes[1][:n]], [scales[0][:4]], [scales[1][:4]]]
    fp8.fp8_adamw_step(fp8.fp8_adamw_tensors(*t), step=3, **HYPER)
    assert (base[0][n:] == 3).all() and all((c[n:] == 77).all() for c in codes) and all((s[4:] == 4).all() for s in scales)

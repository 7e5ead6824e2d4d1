"""AdamW over many tensors against the formula in 64 bits, and its 8-bit moments against the rounding rule."""
import math

import numpy as np
import pytest
import torch

from paper_2508_05370_amd import ops

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)


def _normal(seed, n, scale=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, generator=g) * scale).to(dtype).cuda()


def _step64(p, g, m, v, step, decay, h=HYPER):
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    p = p * (1 - h["lr"] * decay) - h["lr"] / (1 - h["beta1"] ** step) * m / (torch.sqrt(v / (1 - h["beta2"] ** step)) + h["eps"])
    return p, m, v


SIZES = [[1], [7, 0, 129, 128], [2048, 2047, 2049], [5000, 3, 70000], [64] * 100 + [3000]]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("p_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16, torch.float32])
def test_moments_in_32_bits(sizes, p_dtype, g_dtype, copy):
    p = [_normal(i, n, dtype=p_dtype) for i, n in enumerate(sizes)]
    g = [_normal(100 + i, n, dtype=g_dtype) for i, n in enumerate(sizes)]
    m = [_normal(200 + i, n, 0.1) for i, n in enumerate(sizes)]
    v = [_normal(300 + i, n).square() for i, n in enumerate(sizes)]
    decays = [0.1 * (i % 2) for i in range(len(sizes))]
    copies = [torch.zeros(n, dtype=copy, device="cuda") for n in sizes] if copy else None
    scale = torch.tensor([0.5], device="cuda")
    want = [_step64(a.double(), 0.5 * b.double(), c.double(), d.double(), 3, w) for a, b, c, d, w in zip(p, g, m, v, decays)]
    ops.adamw(p, g, m, v, copies=copies, step=3, weight_decay=decays, grad_scale=scale, **HYPER)
    ulp = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
    for i, (wp, wm, wv) in enumerate(want):
        # sums of two products, each rounded: a few units of the larger term
        assert ((m[i].double() - wm).abs() <= 2.0 ** -22 * (wm.abs() + 1)).all()
        assert ((v[i].double() - wv).abs() <= 2.0 ** -22 * wv.abs()).all()
        # the update is at most about lr * 10 here
        assert ((p[i].double() - wp).abs() <= ulp[p_dtype] * wp.abs() + 2.0 ** -20 * 0.1).all()
        if copy:
            assert torch.equal(copies[i], p[i].to(copy))


def _mix(x):
    x = np.asarray(x, np.uint64)
    m = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x9E3779B9)) & m
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x85A308D3)) & m
    return x ^ (x >> np.uint64(16))


def _noise(seed, step, first, n):
    key = _mix(_mix(_mix(seed & 0xFFFFFFFF) ^ np.uint64(seed >> 32)) ^ np.uint64(step))
    at = np.arange(first, first + n, dtype=np.uint64)
    bits = _mix(_mix(key ^ (at >> np.uint64(32))) ^ (at & np.uint64(0xFFFFFFFF)))
    return (bits & np.uint64(0xFFFF)).astype(np.float64) / 65536, (bits >> np.uint64(16)).astype(np.float64) / 65536


def _round_up_or_down(x, u, keep):
    """Codes (values) and scales of float32 x by the rule, in numpy."""
    n = x.size
    full = np.zeros(-(-n // 128) * 128, np.float32)
    full[:n] = x
    amax = np.maximum(np.abs(full.reshape(-1, 128)).max(1), np.float32(2.0 ** -110)).astype(np.float32)
    t = (full.reshape(-1, 128) * (np.float32(448) / amax)[:, None]).reshape(-1)[:n].astype(np.float64)
    _, e = np.frexp(t)
    q = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    c = np.minimum(np.floor(np.abs(t) / q + u) * q, 448)
    if keep:
        c = np.where((t > 0) & (c == 0), 2.0 ** -9, c)
    return np.copysign(c, t), (amax / np.float32(448)).astype(np.float32)


def _eight(x):
    """Codes and scales of a float32 vector, rounded to nearest (for a start)."""
    q, s = ops.quantize(x[None])
    return q[0, :x.numel()].clone(), s[:, 0].clone()


@pytest.mark.parametrize("sizes", [[1], [128, 129], [2048, 2047, 2049, 5], [5000, 3, 70000], [64] * 100 + [3000]], ids=str)
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16])
def test_moments_in_8_bits(sizes, g_dtype):
    f32 = np.float32
    p = [_normal(i, n) for i, n in enumerate(sizes)]
    g = [_normal(100 + i, n, dtype=g_dtype) for i, n in enumerate(sizes)]
    g[0][: sizes[0] // 2] *= 1e-4
    m, ms = zip(*[_eight(_normal(200 + i, n, 0.1)) for i, n in enumerate(sizes)])
    v, vs = zip(*[_eight(_normal(300 + i, n).abs()) for i, n in enumerate(sizes)])
    m, ms, v, vs = list(m), list(ms), list(v), list(vs)
    seed, first, want = (5 << 32) + 77, 0, []
    for i, n in enumerate(sizes):
        s = np.repeat(ms[i].cpu().numpy(), 128)[:n], np.repeat(vs[i].cpu().numpy(), 128)[:n]
        mm, rr = m[i].float().cpu().numpy() * s[0], v[i].float().cpu().numpy() * s[1]
        gg = g[i].float().cpu().numpy()
        # each operation rounded to 32 bits, as the operator says of the moments
        mm = f32(0.9) * mm + f32(1 - 0.9) * gg
        vv = f32(0.95) * (rr * rr) + (f32(1 - 0.95) * gg) * gg
        lo, hi = _noise(seed, 4, first, n)
        want.append((_round_up_or_down(mm, lo, False), _round_up_or_down(np.sqrt(vv), hi, True), mm.copy(), vv.copy()))
        first += -(-n // 128) * 128
    before = [x.double().clone() for x in p]
    ops.adamw(p, g, m, v, exp_avg_scales=ms, exp_avg_sq_scales=vs, step=4, weight_decay=0.1, seed=seed, **HYPER)
    for i in range(len(sizes)):
        for codes, scales, (wc, ws) in ((m[i], ms[i], want[i][0]), (v[i], vs[i], want[i][1])):
            assert np.array_equal(scales.cpu().numpy(), ws)
            assert np.array_equal(codes.float().cpu().numpy().astype(np.float64), wc)
        mm, vv = (torch.from_numpy(x).double().cuda() for x in want[i][2:])
        wp = before[i] * (1 - HYPER["lr"] * 0.1) - HYPER["lr"] / (1 - 0.9 ** 4) * mm / (torch.sqrt(vv / (1 - 0.95 ** 4)) + HYPER["eps"])
        assert ((p[i].double() - wp).abs() <= 2.0 ** -22 * wp.abs() + 2.0 ** -20 * 0.1).all()


def test_rounding_is_unbiased_and_follows_the_moments():
    """A constant gradient: the stored moments' mean goes where the exact ones go, although a step is far below a code's spacing."""
    n, steps = 1 << 16, 200
    g0 = 0.5 + torch.rand(n, generator=torch.Generator().manual_seed(1)).cuda()
    h = dict(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
    p = [torch.zeros(n, device="cuda")]
    m, ms = _eight(torch.zeros(n, device="cuda"))
    v, vs = _eight(torch.full((n,), 3.0, device="cuda"))
    for t in range(1, steps + 1):
        ops.adamw(p, [g0], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs], step=t, seed=9, **h)
    got_m = m.float() * ms.repeat_interleave(128)
    got_r = v.float() * vs.repeat_interleave(128)
    want_m = g0 * (1 - 0.9 ** steps)
    want_v = 9.0 * 0.999 ** steps + g0.square() * (1 - 0.999 ** steps)
    # noise of one rounding is below 2^-4 of a value; m remembers about 5 roundings, sqrt(v) all 200 of them: a random walk of
    # 2^-4 / sqrt(12) * sqrt(200) = 0.26 for one element, its mean over 65536 elements 0.001; squares add half of 0.26^2
    assert abs(float((got_m / want_m).mean()) - 1) < 0.003
    assert abs(float((got_r / want_v.sqrt()).mean()) - 1) < 0.05
    assert float((got_m / want_m - 1).abs().max()) < 0.5


def test_skip_scale_and_not_finite_gradients():
    def fresh():
        return [_normal(1, 300)], [_normal(2, 300)], [_normal(3, 300)], [_normal(4, 300).square()]
    p, g, m, v = fresh()
    skip = torch.ones(1, dtype=torch.int32, device="cuda")
    ops.adamw(p, g, m, v, step=1, skip=skip, **HYPER)
    for a, b in zip((p, g, m, v), fresh()):
        assert torch.equal(a[0], b[0])
    skip.zero_()
    ops.adamw(p, g, m, v, step=1, skip=skip, **HYPER)
    assert not torch.equal(p[0], fresh()[0][0])
    # in 8 bits an element that is not finite spoils its block of 128 at most
    p, g, _, _ = fresh()
    m, ms = _eight(_normal(3, 300))
    v, vs = _eight(_normal(4, 300).abs())
    g[0][5] = float("inf")
    g[0][140] = float("nan")
    ops.adamw(p, g, [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs], step=1, **HYPER)
    got = m.float() * ms.repeat_interleave(128)[:300]
    assert torch.isnan(got[5]) and torch.isnan(got[140]) and torch.isfinite(got[256:]).all()
    bad = ~torch.isfinite(p[0])
    assert bad.sum() == 2 and bad[5] and bad[140]


def test_misaligned_views():
    """Tensors that start anywhere in a buffer give what aligned ones do, and nothing beside them is written."""
    n = 5000
    for bits in (32, 8):
        outs = []
        for off in (0, 1, 3):
            p, g = _normal(1, n + 8)[off:off + n], _normal(2, n + 8, dtype=torch.bfloat16)
            p.copy_(_normal(11, n))
            g = g[off:off + n].copy_(_normal(12, n, dtype=torch.bfloat16))
            copy = torch.zeros(n + 8, dtype=torch.bfloat16, device="cuda")
            kw = dict(step=2, seed=3, copies=[copy[off:off + n]], **HYPER)
            if bits == 32:
                m, v = torch.zeros(n + 8, device="cuda"), torch.zeros(n + 8, device="cuda")
                ops.adamw([p], [g], [m[off:off + n]], [v[off:off + n]], **kw)
                scales = ()
            else:
                m, v = (torch.zeros(n + 8, dtype=torch.uint8, device="cuda") for _ in range(2))
                ms, vs = torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda")
                ops.adamw([p], [g], [m[off:off + n].view(ops.E4M3)], [v[off:off + n].view(ops.E4M3)], exp_avg_scales=[ms],
                          exp_avg_sq_scales=[vs], **kw)
                scales = (ms, vs)
            for b in (m, v, copy):
                assert (b[:off] == 0).all() and (b[off + n:] == 0).all()
            outs.append((p.clone(), m[off:off + n].clone(), v[off:off + n].clone(), copy[off:off + n].clone()) + scales)
        for other in outs[1:]:
            for a, b in zip(outs[0], other):
                assert torch.equal(a, b)


def test_graph_replay():
    p, g = [_normal(1, 3000)], [_normal(2, 3000)]
    m, v = [torch.zeros(3000, device="cuda")], [torch.zeros(3000, device="cuda")]
    q, gq, mq, vq = [p[0].clone()], g, [m[0].clone()], [v[0].clone()]
    ops.adamw([p[0].clone()], g, [m[0].clone()], [v[0].clone()], step=1, **HYPER)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.adamw(p, g, m, v, step=1, **HYPER)
    for _ in range(4):
        graph.replay()
        ops.adamw(q, gq, mq, vq, step=1, **HYPER)
        torch.cuda.synchronize()
        assert torch.equal(p[0], q[0]) and torch.equal(v[0], vq[0])
        assert math.isfinite(float(p[0].sum()))


def test_places_past_32_bits():
    """The last blocks of a tensor of more than 2^32 elements: their places, their scales and their rounding's counter."""
    n, tail = (1 << 32) + 256, 256
    first = n - tail
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(ops.E4M3) for _ in range(2))
    ms, vs = (torch.zeros(n // 128, device="cuda") for _ in range(2))
    p[first:] = _normal(1, tail, dtype=torch.bfloat16)
    g[first:] = _normal(2, tail, dtype=torch.bfloat16)
    before = p[first:].double()
    ops.adamw([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs], step=1, weight_decay=0.0, seed=11, **HYPER)
    f32 = np.float32
    gg = g[first:].float().cpu().numpy()
    mm, vv = f32(1 - 0.9) * gg, (f32(1 - 0.95) * gg) * gg
    lo, hi = _noise(11, 1, first, tail)
    for codes, scales, (wc, ws) in ((m, ms, _round_up_or_down(mm, lo, False)), (v, vs, _round_up_or_down(np.sqrt(vv), hi, True))):
        assert np.array_equal(scales[-2:].cpu().numpy(), ws)
        assert np.array_equal(codes[first:].float().cpu().numpy().astype(np.float64), wc)
        assert int(codes.view(torch.uint8)[:first].amax()) == 0
    want = _step64(before, g[first:].double(), 0.0, 0.0, 1, 0.0)[0]
    assert ((p[first:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * 0.1).all()
    assert float(p[:first].abs().amax()) == 0.0


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -130, 1e-30, 1e-20])
def test_small_gradients_and_small_eps(bits, eps):
    """Second moments below the smallest normal number, and denominators near it: the first step moves a parameter by
    lr g / (|g| + eps), and by nothing where g is zero (unless that is 0 / 0)."""
    n = 128
    g = torch.cat([torch.logspace(-23, -12, n - 1), torch.zeros(1)]).cuda()
    p, moments = [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda") for _ in range(2)]
    scales = None
    if bits == 8:
        (moments[0], ms), (moments[1], vs) = _eight(moments[0]), _eight(moments[1])
        scales = dict(exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
    ops.adamw(p, [g], moments[:1], moments[1:], step=1, weight_decay=0.0, lr=1e-2, beta1=0.5, beta2=0.75, eps=eps, **(scales or {}))
    d, v = g.double(), 0.25 * g.double().square()
    want = -1e-2 * d / (d + eps)
    if eps == 0.0:
        assert torch.isnan(p[0][-1])
        want[-1] = p[0][-1] = 0.0
    # v is a whole number of 2^-149 here: the root's error is that of v, half a spacing of 0.25 g^2 (after g * 0.25's own rounding)
    loss = (2.0 ** -149 / v.clamp_min(2.0 ** -300)).clamp_max(1e30) + 2.0 ** -20
    sure = v > 2.0 ** -146
    assert ((p[0].double() - want).abs() <= 1e-2 * loss)[sure].all()
    assert (p[0][:-1] <= 0).all() and p[0][-1] == 0.0
    if eps:
        # where v is zero the quotient is m / eps, however v is rounded an update of at most lr g / eps
        assert (p[0].double().abs() <= 1e-2 * d / eps * 1.001 + 1e-30).all()


def test_more_chunks_than_a_launch_takes():
    """A launch counts its threads in 32 bits, which is 2^24 - 1 chunks of 2048 elements: the rest goes into another.  The boundary
    lies inside a tensor of three chunks here; what fills the first launch is one tensor many times over, which a step with both
    betas and the rate zero leaves as it is after the first time (m = g, v = g^2)."""
    n, chunk, limit = 1 << 30, 2048, (1 << 24) - 1
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, device="cuda") for _ in range(2))
    g[-1] = 3.0
    full, rest = limit * chunk // n, limit % (n // chunk) - 1       # the last chunk of the first launch is left for the small tensor
    sizes = [n] * full + [rest * chunk, 3 * chunk - 5, 700]
    small = [(_normal(i, k, dtype=torch.bfloat16), _normal(9 + i, k, dtype=torch.bfloat16), _normal(20 + i, k), _normal(30 + i, k).square())
             for i, k in enumerate(sizes[-2:])]
    want = [g64[1].double() for g64 in small]
    lists = [[big] * full + [big[:rest * chunk]] + [s[i] for s in small] for i, big in enumerate((p, g, m, v))]
    ops.adamw(*lists, step=1, lr=0.0, beta1=0.0, beta2=0.0, eps=1e-8)
    for (_, gs, ms, vs), w in zip(small, want):
        assert torch.equal(ms.double(), w) and torch.equal(vs, gs.float().square())
    assert float(m[-1]) == 3.0 and float(v[-1]) == 9.0 and float(p.abs().amax()) == 0.0 and int(m.count_nonzero()) == 1

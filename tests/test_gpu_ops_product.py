"""The 8-bit block form and its products against plain implementations: the codes and scales exactly, the products against
64-bit sums of the same codes."""
import numpy as np
import pytest
import torch

from paper_2508_05370_amd import ops
import ops_abi

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
# unit of the last place of each output type, for a result rounded once
ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -22}


def _normal(seed, *shape, scale=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def _e4m3(t):
    """Nearest e4m3 value of float32 numbers below 464, ties to even."""
    t = t.astype(np.float64)
    _, e = np.frexp(t)
    q = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(t / q) * q


def _plain_blocks(x, block_rows):
    """Codes (as values, padded) and scales of a float32 numpy matrix."""
    r, c = x.shape
    kb, nb = -(-c // 128), -(-r // block_rows)
    codes, scales = np.zeros((r, kb * 128)), np.zeros((kb, nb), np.float32)
    for b in range(kb):
        for i in range(nb):
            part = x[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128]
            a = np.float32(max(np.abs(part).max(), 2.0 ** -110))
            f = np.float32(448) / a
            codes[i * block_rows:(i + 1) * block_rows, b * 128:b * 128 + part.shape[1]] = _e4m3(part * f)
            scales[b, i] = a / np.float32(448)
    return codes, scales


@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (3, 127), (17, 520), (130, 257), (256, 384)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_exact(shape, dtype, block_rows):
    x = _normal(1, *shape, dtype=dtype)
    x[0, 0] = 300.0                     # a loud element
    x[-1] = 0.0                         # a row of zeros
    q, s, qt, st = ops.quantize(x, block_rows, transposed=True)
    xn = x.float().cpu().numpy()
    for codes, scales, plain in ((q, s, xn), (qt, st, np.ascontiguousarray(xn.T))):
        want, want_s = _plain_blocks(plain, block_rows)
        assert np.array_equal(codes.float().cpu().numpy(), want)
        assert np.array_equal(scales.cpu().numpy(), want_s)
    only = ops.quantize(x, block_rows)
    assert torch.equal(only[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(only[1], s)
    only = ops.quantize(x, block_rows, rows=False, transposed=True)
    assert torch.equal(only[0].view(torch.uint8), qt.view(torch.uint8)) and torch.equal(only[1], st)


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 0), (3, 5)])
def test_quantize_strides_and_alignment(offset, pad):
    buf = _normal(2, 40 * 400, dtype=torch.bfloat16)
    x = buf[offset:].as_strided((33, 264), (264 + pad, 1))
    q, s, qt, st = ops.quantize(x, transposed=True)
    want, want_s = _plain_blocks(x.float().cpu().numpy(), 1)
    assert np.array_equal(q.float().cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), want_s)
    want, want_s = _plain_blocks(np.ascontiguousarray(x.float().cpu().numpy().T), 1)
    assert np.array_equal(qt.float().cpu().numpy(), want) and np.array_equal(st.cpu().numpy(), want_s)


def test_quantize_extremes():
    """Tiny blocks keep a usable scale; an infinity makes its block NaN, a NaN itself; other blocks stay."""
    x = torch.zeros(4, 256, device="cuda")
    x[0, :128] = 1e-38
    x[1, 5] = float("inf")
    x[2, 7] = float("nan")
    x[2, 8] = 2.0
    x[3] = 3e38
    q, s = ops.quantize(x)
    v = ops.dequantize(q, s, 256)
    # the scale is that of 2^-110, codes are 2^-9 apart
    assert float((v[0] - x[0]).abs().max()) <= 2.0 ** -10 * 2.0 ** -110 / 448
    assert torch.isnan(v[1, :128]).all() and (v[1, 128:] == 0).all()
    assert torch.isnan(v[2, 7]) and v[2, 8] == 2.0 and torch.isnan(v[2]).sum() == 1
    assert torch.allclose(v[3], x[3], rtol=2.0 ** -20)


def _product64(a, sa, b, sb, k):
    """The product in 64 bits, and a bound of what the matrix cores may lose: they align the products of a group of codes to
    the largest of them, of which 13 bits are certain; 128 products to a block."""
    av, bv = ops.dequantize(a, sa, k).double().cpu(), ops.dequantize(b, sb, k).double().cpu()
    loss = torch.zeros(av.shape[0], bv.shape[0], dtype=torch.float64)
    for c in range(0, k, 128):
        loss += av[:, c:c + 128].abs().amax(1)[:, None] * bv[:, c:c + 128].abs().amax(1)[None] * 128 * 2.0 ** -13
    return av @ bv.t(), loss


def _blocks(seed, r, k, block_rows, scale=1.0):
    return ops.quantize(_normal(seed, r, k, scale=scale), block_rows)


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 300, 1000), (2, 64, 256), (4, 130, 384), (5, 3, 129), (16, 128, 4096), (17, 100, 2050),
          (33, 48, 896), (64, 257, 512), (65, 96, 640), (128, 128, 128), (200, 16, 130), (257, 255, 640), (300, 513, 1000)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("ba,bb", [(1, 128), (1, 1), (128, 128), (128, 1)])
def test_matmul(m, n, k, ba, bb):
    a, sa = _blocks(m, m, k, ba)
    b, sb = _blocks(n + 7, n, k, bb)
    want, loss = _product64(a, sa, b, sb, k)
    for dtype in DTYPES:
        got = ops.matmul(a, sa, b, sb, k, dtype)
        assert got.dtype == dtype and tuple(got.shape) == (m, n)
        d = (got.double().cpu() - want).abs()
        assert (d <= loss + want.abs() * ULP[dtype]).all()
    # over the whole matrix the losses do not add up: a thousandth of the codes' own rounding
    if m * n >= 256:
        assert float((got.double().cpu() - want).norm() / want.norm()) < 6e-5


# few rows of A and of B with a long k, which is split: parts of unequal length, a last block that is not whole
SPLIT = [(1, 1000, 14400), (1, 30, 40000), (4, 515, 16385), (9, 77, 8200), (16, 1021, 13000), (33, 2048, 6001), (64, 258, 4097)]


@pytest.mark.parametrize("m,n,k", SPLIT)
@pytest.mark.parametrize("ba,bb", [(1, 128), (128, 1)])
def test_few_rows_split(m, n, k, ba, bb):
    assert ops_abi.lib().sim_op_matmul_workspace(m, n, k) >= 2 * m * n * 4      # the case is one that is split
    a, sa = _blocks(m, m, k, ba)
    b, sb = _blocks(n + 7, n, k, bb)
    want, loss = _product64(a, sa, b, sb, k)
    for dtype in DTYPES:
        buf = _normal(8, 1 + m * (n + 3), dtype=dtype)
        out = buf[1:].as_strided((m, n), (n + 3, 1))
        before, kept = out.double().cpu().clone(), buf.clone()
        got = ops.matmul(a, sa, b, sb, k, dtype)
        assert ((got.double().cpu() - want).abs() <= loss + want.abs() * ULP[dtype]).all()
        ops.matmul(a, sa, b, sb, k, out=out, accumulate=True)
        assert ((out.double().cpu() - (want + before)).abs() <= loss + (want.abs() + before.abs()) * 2 * ULP[dtype]).all()
        kept[1:].as_strided((m, n), (n + 3, 1)).copy_(out)
        assert torch.equal(kept, buf)          # nothing beside the matrix is written
        assert torch.equal(got, ops.matmul(a, sa, b, sb, k, dtype))


@pytest.mark.parametrize("tokens", [1, 2, 4, 7, 16, 40])
@pytest.mark.parametrize("n,k,bb", [(1000, 14400, 128), (259, 20001, 1)])
def test_linear_is_its_parts_when_split(tokens, n, k, bb):
    """Whoever brings the activations to 8 bits, the result is the same to the bit."""
    w, ws = _blocks(3, n, k, bb, 0.02)
    for dtype in DTYPES:
        for offset in (0, 1):
            x = _normal(tokens, offset + tokens * k, dtype=dtype)[offset:].view(tokens, k)
            q, s = ops.quantize(x)
            assert torch.equal(ops.linear(x, w, ws), ops.matmul(q, s, w, ws, k, dtype))


@pytest.mark.parametrize("m,n,k", [(2048, 2100, 512), (4100, 1800, 300)])
def test_matmul_many_tiles(m, n, k):
    """Enough tiles for the largest tile size, with ragged edges."""
    a, sa = _blocks(3, m, k, 1)
    for bb in (1, 128):
        b, sb = _blocks(4, n, k, bb)
        got = ops.matmul(a, sa, b, sb, k, torch.float32).double()
        want = ops.dequantize(a, sa, k).double() @ ops.dequantize(b, sb, k).double().t()
        assert float((got - want).norm() / want.norm()) < 6e-5
        assert float((got - want).abs().max()) < 1e-3 * float(want.abs().max())


@pytest.mark.parametrize("m,n,k", [(3, 17, 200), (70, 130, 1024), (257, 300, 256)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_matmul_accumulate_and_strides(m, n, k, dtype):
    a, sa = _blocks(5, m, k, 1)
    b, sb = _blocks(6, n, k, 128)
    want, loss = _product64(a, sa, b, sb, k)
    for offset, ld in ((0, n + 5), (1, n + 3), (4, (n + 7) // 4 * 4)):
        buf = _normal(8, offset + m * ld, dtype=dtype)
        out = buf[offset:].as_strided((m, n), (ld, 1))
        before, kept = out.double().cpu().clone(), buf.clone()
        ops.matmul(a, sa, b, sb, k, out=out, accumulate=True)
        d = (out.double().cpu() - (want + before)).abs()
        assert (d <= loss + (want.abs() + before.abs()) * 2 * ULP[dtype]).all()
        kept[offset:].as_strided((m, n), (ld, 1)).copy_(out)
        assert torch.equal(kept, buf)          # nothing beside the matrix is written


def test_matmul_empty():
    a, sa = _blocks(1, 4, 128, 1)
    b, sb = _blocks(2, 3, 128, 1)
    assert ops.matmul(a[:0], sa[:, :0], b, sb, 128).shape == (0, 3)
    e = torch.empty((4, 0), dtype=ops.E4M3, device="cuda")
    es = torch.empty((0, 4), device="cuda")
    f, fs = torch.empty((3, 0), dtype=ops.E4M3, device="cuda"), torch.empty((0, 3), device="cuda")
    out = torch.full((4, 3), 5.0, device="cuda")
    ops.matmul(e, es, f, fs, 0, out=out, accumulate=True)
    assert (out == 5.0).all()
    ops.matmul(e, es, f, fs, 0, out=out)
    assert (out == 0.0).all()
    assert ops.quantize(torch.empty((0, 5), device="cuda"))[0].shape == (0, 128)


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 33, 47, 64, 65, 128, 130])
@pytest.mark.parametrize("n,k", [(48, 128), (130, 1000), (768, 768), (260, 8200)])
def test_linear(tokens, n, k):
    for dtype in DTYPES:
        x = _normal(tokens, tokens, k, dtype=dtype)
        x[:, 0] *= 50
        w, ws = ops.quantize(_normal(n, n, k, scale=0.02), 128)
        y = ops.linear(x, w, ws)
        q, s = ops.quantize(x)
        want, loss = _product64(q, s, w, ws, k)
        assert y.dtype == dtype
        assert ((y.double().cpu() - want).abs() <= loss + want.abs() * ULP[dtype]).all()


@pytest.mark.parametrize("tokens", [1, 3, 40])
def test_linear_rowwise_weight_scales_and_views(tokens):
    n, k = 100, 300
    buf = _normal(1, tokens * (k + 3) + 1, dtype=torch.bfloat16)
    x = buf[1:].as_strided((tokens, k), (k + 3, 1))
    w, ws = ops.quantize(_normal(2, n, k), 1)
    out = torch.zeros(tokens, n + 1, dtype=torch.bfloat16, device="cuda")
    ops.linear(x, w, ws, out=out[:, :n])
    q, s = ops.quantize(x)
    want, loss = _product64(q, s, w, ws, k)
    assert ((out[:, :n].double().cpu() - want).abs() <= loss + want.abs() * ULP[torch.bfloat16]).all()
    assert (out[:, n] == 0).all()


def test_nan_and_infinity_stay_in_their_rows():
    for tokens in (1, 4, 20, 200):
        x = _normal(1, tokens, 256)
        w, ws = ops.quantize(_normal(2, 96, 256), 128)
        clean = ops.linear(x, w, ws)
        x[0, 3] = float("nan")
        y = ops.linear(x, w, ws)
        assert torch.isnan(y[0]).all() and torch.equal(y[1:], clean[1:])
        x[0, 3] = float("inf")
        y = ops.linear(x, w, ws)
        assert torch.isnan(y[0]).all() and torch.equal(y[1:], clean[1:])


@pytest.mark.parametrize("t,k,n", [(5, 130, 70), (128, 256, 128), (300, 200, 515)])
def test_linear_gradients(t, k, n):
    """Against the formulas in 64 bits on the block forms' values."""
    x, w, dy = (_normal(i, *s, dtype=torch.bfloat16) for i, s in enumerate(((t, k), (n, k), (t, n))))
    y, saved = ops.linear_forward(x, w)
    dx, dw = ops.linear_backward(dy, saved)
    assert dw.dtype == torch.bfloat16
    acc = torch.ones(n, k, device="cuda")
    ops.linear_backward(dy, saved, dw=acc)
    for got, (a, sa), (b, sb), kk in ((y, ops.quantize(x), ops.quantize(w, 128), k),
                                      (dx, ops.quantize(dy), ops.quantize(w, 128, rows=False, transposed=True), n),
                                      (dw, ops.quantize(dy, rows=False, transposed=True),
                                       ops.quantize(x, rows=False, transposed=True), t)):
        want, loss = _product64(a, sa, b, sb, kk)
        assert ((got.double().cpu() - want).abs() <= loss + want.abs() * ULP[torch.bfloat16]).all()
    assert ((acc.double().cpu() - 1 - want).abs() <= loss + (1 + want.abs()) * ULP[torch.float32]).all()


def test_linear_gradients_against_differences():
    """On small whole numbers, with 14 the largest of every block (448 / 14 is a power of two), the 8-bit form is exact and the
    loss sum(dy * y) is bilinear: a difference of one in an element gives its derivative exactly."""
    t, k, n = 6, 140, 9
    g = torch.Generator().manual_seed(1)

    def whole(r, c):
        v = torch.randint(-7, 8, (r, c), generator=g).float()
        v[:, ::128] = 14.0
        v[0] = 14.0
        v[:, c - 1] = 14.0
        return v.cuda()
    x, w, dy = whole(t, k), whole(n, k), whole(t, n)
    y, saved = ops.linear_forward(x, w)
    dx, dw = ops.linear_backward(dy, saved)

    def loss(x, w):
        return float((ops.linear_forward(x, w)[0].double() * dy.double()).sum())
    base = loss(x, w)
    for i, j in ((1, 1), (3, 77), (5, 130)):
        x2 = x.clone()
        x2[i, j] += 1.0
        assert loss(x2, w) - base == float(dx[i, j])
    for i, j in ((1, 1), (4, 100), (8, 138)):
        w2 = w.clone()
        w2[i, j] += 1.0
        assert loss(x, w2) - base == float(dw[i, j])


def test_offsets_past_32_bits():
    """Codes, activations and outputs further than 2^31 elements into their tensors."""
    n, k = 70000, 32768
    codes = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
    codes[-40:] = torch.randint(0, 0x70, (40, k), device="cuda", dtype=torch.uint8)
    scales = torch.rand((k // 128, -(-n // 128)), device="cuda") + 0.5
    x = _normal(1, 2, k, dtype=torch.bfloat16)
    y = ops.linear(x, codes.view(ops.E4M3), scales)
    assert (y[:, :-40] == 0).all()
    q, s = ops.quantize(x)
    wv = codes[-40:].view(ops.E4M3).double() * scales[:, -1].repeat_interleave(128).double()
    want = ops.dequantize(q, s, k).double() @ wv.t()
    assert torch.allclose(y[:, -40:].double(), want, rtol=2.0 ** -7, atol=1e-3 * float(want.abs().max()))
    big = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    big[-3:] = _normal(3, 3, k, dtype=torch.bfloat16)
    q, s = ops.quantize(big)
    q3, s3 = ops.quantize(big[-3:].clone())
    assert torch.equal(q[-3:].view(torch.uint8), q3.view(torch.uint8)) and torch.equal(s[:, -3:], s3)
    assert int(q[:-3].view(torch.uint8).amax()) == 0


def test_graph_and_other_stream():
    """Recorded once, replayed on new inputs with eager work between; and the same on a stream of its own."""
    x, w = _normal(1, 40, 512, dtype=torch.bfloat16), _normal(2, 300, 512, dtype=torch.bfloat16)
    wq, ws = ops.quantize(w, 128)
    one = _normal(3, 1, 512, dtype=torch.bfloat16)

    def step():
        y, saved = ops.linear_forward(x, w)
        return (y,) + tuple(ops.linear_backward(y, saved)) + (ops.linear(one, wq, ws),)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for i in range(4):
        x.copy_(_normal(10 + i, 40, 512, dtype=torch.bfloat16))
        one.copy_(_normal(20 + i, 1, 512, dtype=torch.bfloat16))
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(recorded, eager):
            assert torch.equal(a, b)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
        side.synchronize()
        for a, b in zip(other, eager):
            assert torch.equal(a, b)


def _scales_of(amax):
    """The 32-bit quotient by 448 (by a tensor: a number's reciprocal would be multiplied by)."""
    return amax.clamp_min(2.0 ** -110) / torch.full_like(amax, 448.0)


# A launch counts its threads in 32 bits: 2^24 - 1 workgroups of 256, 2^23 - 1 of 512.  What is more goes into further launches.
def test_more_rows_than_a_launch_takes():
    """16 threads to a row: 2^28 - 16 rows."""
    rows = (1 << 28) - 16 + 37
    x = torch.randint(-1, 2, (rows, 1), device="cuda", dtype=torch.int8).bfloat16()
    q, s = ops.quantize(x)
    top = torch.where(x == 0, torch.zeros((), device="cuda"), torch.full((), 448.0, device="cuda")) * x
    for a in range(0, rows, 1 << 26):
        assert torch.equal(q[a:a + (1 << 26), :1].float(), top[a:a + (1 << 26)])
    assert int(q[-5000:, 1:].view(torch.uint8).amax()) == 0
    assert torch.equal(s[0], _scales_of(x[:, 0].float().abs()))


@pytest.mark.parametrize("block_rows", [1, 128])
def test_more_tiles_than_a_launch_takes(block_rows):
    """A workgroup to 128 rows: (2^24 - 1) * 128 of them."""
    whole = ((1 << 24) - 1) * 128
    rows = whole + 5
    x = torch.zeros((rows, 1), dtype=torch.bfloat16, device="cuda")
    x[:: 77] = 3.0
    x[-300:] = _normal(1, 300, 1, dtype=torch.bfloat16)
    q, s = ops.quantize(x, block_rows, rows=False, transposed=True)
    amax = torch.cat([x[:whole].view(-1, 128).abs().amax(1), x[whole:].abs().amax()[None]]).float()
    assert torch.equal(s[:, 0], _scales_of(amax))
    tail = ops.quantize(x[whole - 640:].clone(), block_rows, rows=False, transposed=True)
    assert torch.equal(q[:, whole - 640:].view(torch.uint8), tail[0].view(torch.uint8)) and torch.equal(s[-6:], tail[1])


def test_more_rows_of_b_than_a_launch_takes():
    """16 rows of B to a workgroup of 512: 2^27 - 128 rows."""
    edge = (1 << 27) - 128
    n, k = edge + 200, 128
    codes = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
    codes[edge - 256:] = torch.randint(0, 0x70, (456, k), device="cuda", dtype=torch.uint8)
    scales = torch.rand((1, -(-n // 128)), device="cuda") + 0.5
    x = _normal(1, 2, k, dtype=torch.bfloat16)
    y = ops.linear(x, codes.view(ops.E4M3), scales)
    assert float(y[:, :edge - 256].abs().amax()) == 0.0
    assert torch.equal(y[:, edge - 256:], ops.linear(x, codes[edge - 256:].view(ops.E4M3), scales[:, edge // 128 - 2:].contiguous()))


def test_more_zeros_than_a_launch_takes():
    """A product over nothing with 5 * 2^30 groups of four zeros."""
    m, n = (1 << 30) + 3, 17
    out = torch.ones((m, n), dtype=torch.bfloat16, device="cuda")
    a, b = (torch.empty((r, 0), dtype=ops.E4M3, device="cuda") for r in (m, n))
    ops.matmul(a, torch.empty((0, m), device="cuda"), b, torch.empty((0, n), device="cuda"), 0, out=out)
    assert float(out.amax()) == 0.0


def test_tiled_product_past_32_bits():
    """Codes, outputs and transposes further than 2^31 elements into their tensors, with more rows than the streaming form takes."""
    m, k = 70000, 32768
    big = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
    big[-200:] = _normal(3, 200, k, dtype=torch.bfloat16)
    q, s, qt, st = ops.quantize(big, transposed=True)
    tail = big[-(m % 128 + 128):].clone()               # the last whole block of rows, and the rest
    q1, s1, qt1, st1 = ops.quantize(tail, transposed=True)
    r = tail.shape[0]
    assert torch.equal(q[-r:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[:, -r:], s1)
    assert torch.equal(qt[:, -256:].view(torch.uint8), qt1.view(torch.uint8)) and torch.equal(st[-2:], st1)
    b, sb = _blocks(5, 96, k, 128)
    y = ops.matmul(q, s, b, sb, k, torch.float32)
    want = ops.dequantize(q[-200:], s[:, -200:], k).double() @ ops.dequantize(b, sb, k).double().t()
    # as in test_matmul_many_tiles
    assert float((y[-200:].double() - want).norm() / want.norm()) < 6e-5 and float(y[:-r].abs().amax()) == 0.0
    del big, qt, st, y
    c, sc = _blocks(6, 33000, 128, 128)
    d, sd = _blocks(7, m, 128, 1)
    y = ops.matmul(d, sd, c, sc, 128, torch.bfloat16)
    want = ops.dequantize(d[-3:], sd[:, -3:], 128).double() @ ops.dequantize(c, sc, 128).double().t()
    assert float((y[-3:].double() - want).norm() / want.norm()) < 4e-3


@pytest.mark.parametrize("tokens", [1, 5, 40, 200])
@pytest.mark.parametrize("hidden", [256, 1000, 4096, 8200])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_into_product(tokens, hidden, kind):
    """A norm's output in 8 bits is the operand of a product as it is: the next linear layer without a pass of its own over x."""
    h, y = _normal(1, tokens, hidden, dtype=torch.bfloat16), _normal(2, tokens, hidden, dtype=torch.bfloat16)
    f = ops.norm_block(h, y, pre_weight=1.0 + _normal(3, hidden, scale=0.2), post=kind, pre=kind, quantized=True)
    w, ws = _blocks(4, 130, hidden, 128, 0.02)
    want, loss = _product64(f.x, f.x_scale, w, ws, hidden)
    got = ops.matmul(f.x, f.x_scale, w, ws, hidden, torch.bfloat16)
    assert ((got.double().cpu() - want).abs() <= loss + want.abs() * ULP[torch.bfloat16]).all()

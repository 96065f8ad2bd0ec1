"""The operators around an 8-bit factored layer on the GPU against their definitions in 64 bits.

Tolerances count roundings: eps = 2^-23 for an fp32 operation (twice the half step, so that sums which the matrix cores round
towards zero are covered), half a step for the rounding of a result: 2^-24 fp32, 2^-9 bf16 relative to a value's power of two
(2^-8 relative to the value at most), e4m3 2^-4 relative, 2^-10 of its scale below its normal numbers."""
import ctypes

import numpy as np
import pytest
import torch

import oracle.scaled as ref
from paper_2510_25977_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def dev():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch.device("cuda:0")


def f64(t):
    return t.detach().cpu().double().numpy()


def bytes_of(codes):
    return codes.contiguous().view(torch.uint8).cpu().numpy()


def rng(*seed):
    return np.random.default_rng([20251208, *seed])


def padded(rows, cols, dtype, extra, fill, offset=0):
    """A [rows, cols] matrix whose rows lie `extra` elements further apart than they are long, inside a buffer full of
    `fill`, and the buffer."""
    ld = cols + extra
    buf = torch.full((offset + rows * ld + 64,), fill, dtype=torch.float32, device=dev()).to(dtype)
    return buf[offset:offset + rows * ld].view(rows, ld)[:, :cols], buf


def put(values, dtype, extra=0, offset=0):
    t, _ = padded(*values.shape, dtype, extra, float("nan"), offset)
    t.copy_(torch.from_numpy(values).to(dtype))
    return t


def code_buffer(rows, cols, extra=0):
    """Rows of codes, NaN codes all around them."""
    ld = -(-cols // 16) * 16 + extra
    buf = torch.full((rows * ld + 32,), 0x7F, dtype=torch.uint8, device=dev()).view(F8)
    return buf[:rows * ld].view(rows, ld)[:, :cols], buf


def check_scaled(got, want, err, what=""):
    """got against the values `want` [R, C] that are quantised, themselves known up to err [R, C]."""
    codes, scales = bytes_of(got.codes), f64(got.scales)
    R, C = want.shape
    cb = -(-C // ref.BLOCK)
    s_want = ref.scales_of(want)
    worst = np.zeros((R, cb * ref.BLOCK))
    worst[:, :C] = err
    worst = worst.reshape(R, cb, ref.BLOCK).max(2).T
    assert scales.shape == s_want.shape
    # the largest magnitude is off by at most the largest error; times 1 / 448 (rounded twice), then rounded to bf16
    assert (np.abs(scales - s_want) <= (worst / ref.LARGEST + s_want * 2 * EPS) * (1 + 2.0 ** -8) + s_want * 2.0 ** -8).all(), what
    s = np.repeat(scales.T, ref.BLOCK, axis=1)[:, :C]
    # v * (1 / s) in fp32 (two roundings), then half a step of e4m3
    tol = err + np.abs(want) * (2.0 ** -4 + 4 * EPS) + s * 2.0 ** -10
    off = np.abs(ref.E4M3[codes] * s - want) - tol
    assert (off <= 0).all(), (what, np.unravel_index(off.argmax(), off.shape), off.max())


def check_float(got, want, err, what=""):
    tol = err + HALF_STEP[got.dtype] * np.abs(want) + 1e-37
    off = np.abs(f64(got) - want) - tol
    assert (off <= 0).all(), (what, np.unravel_index(off.argmax(), off.shape), off.max())


# ------------------------------------------------------------------------------------------------ product
def random_scaled(r, rows, cols, extra, weights=False):
    """Codes of all sizes (no NaN), scales spread over three decades; NaN codes between the rows, NaN scales behind."""
    codes = r.integers(0, 256, (rows, cols), dtype=np.uint8)
    codes[(codes & 0x7F) == 0x7F] ^= 1
    small = r.random((rows, cols)) < 0.7          # most of a block is far below its largest
    codes = np.where(small, (codes & 0x80) | (codes & 0x7F) % 0x40, codes).astype(np.uint8)
    cb = -(-cols // ref.BLOCK)
    shape = (-(-rows // ref.BLOCK), cb) if weights else (cb, rows)
    scales = np.exp(r.normal(size=shape) * 1.5).astype(np.float32) * 1e-2
    q, _ = code_buffer(rows, cols, extra)
    q.view(torch.uint8).copy_(torch.from_numpy(codes))
    if weights:
        s = torch.from_numpy(scales).to(dev())
    else:
        s, _ = padded(*shape, BF16, extra // 16 * 3, float("nan"))
        s.copy_(torch.from_numpy(scales))
        scales = f64(s)
    value = (ref.weights if weights else ref.activations)(codes, scales.astype(np.float64))
    return B.Scaled(q, s), value


def product_error(a, w):
    """What the sums may lose.  The matrix cores add eight products of consecutive codes at a time, each cut off at 2^-13 of
    the power of two of the largest of them: up to 7 x 2^-13 of the group's largest product (the largest itself, of two
    4-bit significands, keeps its bits), which is at most the product of the group's largest operands.  Then a block's
    partial sums and the scaled sum over the blocks in fp32, each rounding at most EPS of the sum of magnitudes."""
    K = a.shape[1]

    def largest(v):
        full = np.zeros((v.shape[0], -(-K // 8) * 8))
        full[:, :K] = np.abs(v)
        return full.reshape(v.shape[0], -1, 8).max(2)

    return 7 * 2.0 ** -13 * (largest(a) @ largest(w).T) + (128 + K / 128 + 8) * EPS * (np.abs(a) @ np.abs(w).T)


MATMULS = [
    # rows, columns, contraction: every remainder of a tile, a block and a 16-byte piece
    (1, 1, 1), (1, 16, 128), (2, 7, 15), (3, 130, 16), (5, 64, 17), (15, 129, 100), (16, 512, 127), (17, 100, 128),
    (16, 300, 129), (31, 128, 255), (32, 257, 256), (33, 96, 257), (47, 200, 640), (64, 512, 1000), (1, 1000, 2304),
    (63, 33, 3000), (65, 384, 513), (100, 127, 2000), (128, 256, 384), (129, 255, 383), (200, 520, 1152), (256, 256, 512),
    (257, 640, 300), (300, 1000, 270), (513, 515, 517), (1000, 700, 1100), (40, 3000, 400), (2, 16, 9000), (130, 40, 9001), (7, 9, 3000),
    (20, 15, 5000), (1, 131, 4000), (64, 259, 4000), (1036, 9, 3647), (2993, 131, 5942), (168, 5463, 7852), (129, 5770, 7063),
    # what else the product's kernels and their cuts of the contraction are chosen for (a host test sees to it that all are here)
    (3, 6000, 300), (700, 500, 1300), (520, 300, 2500), (700, 4100, 400), (90, 1100, 4000), (2741, 2252, 135), (1301, 4999, 300),
    (1290, 5000, 513), (300, 2600, 6000), (2100, 5000, 257), (2111, 4983, 600), (1500, 600, 9000), (3, 66, 555), (284, 1738, 1842),
    (2732, 331, 61), (353, 131, 4010), (2071, 905, 3518), (3585, 2000, 72), (3585, 2830, 120), (2747, 1472, 256),
]


@pytest.mark.parametrize("out", [BF16, F8], ids=["bf16", "f8"])
@pytest.mark.parametrize("M,N,K", MATMULS)
def test_scaled_matmul(M, N, K, out):
    r = rng(1, M, N, K)
    extra = int(r.integers(0, 4)) * 16
    A, a = random_scaled(r, M, K, extra)
    W, w = random_scaled(r, N, K, int(r.integers(0, 3)) * 16, True)
    want, err = a @ w.T, product_error(a, w)
    if out is F8:
        q, buf = code_buffer(M, N, extra)
        s, sbuf = padded(-(-N // 128), M, BF16, 5, -7.0)
        before, sbefore = buf.view(torch.uint8).clone(), sbuf.clone()
        got = B.scaled_matmul(A, W, out=(q, s))
        check_scaled(got, want, err)
        q.view(torch.uint8).fill_(0x7F)
        s.fill_(-7.0)
        assert torch.equal(buf.view(torch.uint8), before) and torch.equal(sbuf, sbefore)     # nothing beside them was written
    else:
        c, buf = padded(M, N, out, 3, -7.0, offset=1)       # rows start anywhere
        before = buf.clone()
        got = B.scaled_matmul(A, W, out=c)
        check_float(got, want, err)
        c.fill_(-7.0)
        assert torch.equal(buf, before)


GATED = [(1, 1, 256), (1, 1400, 512), (5, 130, 256), (16, 512, 1024), (64, 128, 768), (65, 129, 2048), (130, 385, 512), (300, 2600, 512),
         (700, 1100, 1280), (1030, 2000, 256), (2100, 3585, 768), (1999, 4097, 512)]


@pytest.mark.parametrize("out", [BF16, F8], ids=["bf16", "f8"])
@pytest.mark.parametrize("M,N,K", GATED)
def test_gated_product(M, N, K, out):
    """SiLU(G) P of the two halves of the contraction.  G and P are known up to product_error; SiLU's slope is at most 1.1, and its
    own error in fp32 that of an exponential whose argument is rounded (|g| EPS) and a few roundings."""
    r = rng(11, M, N, K)
    A, a = random_scaled(r, M, K, 16)
    W, w = random_scaled(r, N, K, 32, True)
    A.scales.mul_(1 / 16)         # gates of ordinary size and large ones
    a = a / 16
    half = K // 2
    g, p = a[:, :half] @ w[:, :half].T, a[:, half:] @ w[:, half:].T
    dg, dp = product_error(a[:, :half], w[:, :half]), product_error(a[:, half:], w[:, half:])
    with np.errstate(over="ignore"):
        s = ref.silu(g)
    ds = 1.1 * dg + np.abs(s) * (np.abs(g) + dg + 8) * EPS
    want, err = s * p, ds * np.abs(p) + np.abs(s) * dp + ds * dp + np.abs(s * p) * 2 * EPS
    if out is F8:
        q, buf = code_buffer(M, N, 16)
        sc, sbuf = padded(-(-N // 128), M, BF16, 5, -7.0)
        before, sbefore = buf.view(torch.uint8).clone(), sbuf.clone()
        check_scaled(B.scaled_matmul(A, W, gated=True, out=(q, sc)), want, err)
        q.view(torch.uint8).fill_(0x7F)
        sc.fill_(-7.0)
        assert torch.equal(buf.view(torch.uint8), before) and torch.equal(sbuf, sbefore)
    else:
        c, buf = padded(M, N, out, 3, -7.0, offset=1)
        before = buf.clone()
        check_float(B.scaled_matmul(A, W, gated=True, out=c), want, err)
        c.fill_(-7.0)
        assert torch.equal(buf, before)


@pytest.mark.parametrize("M,N", [(40, 200), (300, 4000), (1500, 3600)])
def test_gated_product_keeps_nan_to_its_row(M, N):
    r = rng(12, M, N)
    (A, _), (W, _) = random_scaled(r, M, 768, 0), random_scaled(r, N, 768, 0, True)
    good = B.scaled_matmul(A, W, gated=True).float()
    A.codes.view(torch.uint8)[7, 100] = 0x7F           # in a gate's operand
    A.codes.view(torch.uint8)[M - 2, 700] = 0xFF       # in an up product's
    got = B.scaled_matmul(A, W, gated=True).float()
    bad = torch.isnan(got)
    assert bad[7].all() and bad[M - 2].all() and int(bad.sum()) == 2 * N
    bad[:] = False
    bad[[7, M - 2]] = True
    assert torch.equal(got[~bad], good[~bad]) and torch.isfinite(good).all()


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (16, 512, 14336), (128, 2048, 2048), (300, 1000, 270), (700, 1100, 2688)])
def test_scaled_matmul_gives_the_same_bits_again(M, N, K):
    r = rng(2, M, N, K)
    A, W = random_scaled(r, M, K, 0)[0], random_scaled(r, N, K, 0, True)[0]
    for out in (BF16, F8):
        first = B.scaled_matmul(A, W, out_dtype=out)
        for _ in range(3):
            again = B.scaled_matmul(A, W, out_dtype=out)
            if out is F8:
                assert torch.equal(first.codes.view(torch.uint8), again.codes.view(torch.uint8)) and torch.equal(first.scales, again.scales)
            else:
                assert torch.equal(first, again)


def test_scaled_matmul_passes_nan_on_and_keeps_it_to_its_row():
    """A NaN code in row 3 of A and row 70 of W: those rows and columns are NaN, nothing else is."""
    for M, N, K in ((20, 150, 300), (300, 300, 300)):
        r = rng(3, M)
        A, W = random_scaled(r, M, K, 0)[0], random_scaled(r, N, K, 0, True)[0]
        A.codes.view(torch.uint8)[3, K - 1] = 0x7F
        W.codes.view(torch.uint8)[70, 5] = 0xFF
        c = f64(B.scaled_matmul(A, W))
        bad = np.zeros((M, N), bool)
        bad[3], bad[:, 70] = True, True
        assert np.array_equal(np.isnan(c), bad)


def test_zero_activations_give_zeros_whatever_their_scale():
    A = B.quantize(torch.zeros(20, 400, device=dev()))
    W = B.quantize(torch.randn(300, 400, device=dev()), block_rows=128)
    assert f64(A.scales).max() == 2.0 ** -100
    assert not B.scaled_matmul(A, W).any()
    q = B.scaled_matmul(A, W, out_dtype=F8)
    assert not (q.codes.view(torch.uint8) & 0x7F).any() and f64(q.scales).max() == 2.0 ** -100


# ---------------------------------------------------------------------------------------------- quantiser
QUANTIZE = [(1, 1), (1, 128), (2, 7), (3, 129), (16, 256), (17, 1000), (33, 127), (100, 2687), (130, 385), (257, 136),
            (20, 9), (5, 15), (35, 263), (18, 644)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("R,C", QUANTIZE)
def test_quantize(R, C, gated, dtype):
    r = rng(4, R, C)
    x = put(r.normal(size=(R, C)) * np.exp(r.normal(size=(R, 1)) * 3), dtype, 3, 1)
    u = put(r.normal(size=(R, C)), dtype, 1, 3) if gated else None
    q, buf = code_buffer(R, C, 16)
    s, sbuf = padded(-(-C // 128), R, BF16, 2, -7.0)
    before, sbefore = buf.view(torch.uint8).clone(), sbuf.clone()
    got = B.quantize(x, u, out=(q, s))
    want = f64(x)
    err = 0.0 * want
    if gated:
        # exp of an argument rounded in fp32: |x| 2^-24 relative and a few roundings
        with np.errstate(over="ignore"):
            want, slack = ref.silu(want) * f64(u), (np.abs(want) + 8) * EPS
        err = np.abs(want) * slack
    check_scaled(got, want, err)
    q.view(torch.uint8).fill_(0x7F)
    s.fill_(-7.0)
    assert torch.equal(buf.view(torch.uint8), before) and torch.equal(sbuf, sbefore)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(1, 1), (128, 128), (129, 127), (300, 1000), (7, 400)])
def test_quantize_weights(R, C, dtype):
    r = rng(5, R, C)
    x = put(r.normal(size=(R, C)) * np.exp(r.normal(size=(R, 1))), dtype, 5)
    got = B.quantize(x, block_rows=128)
    v, s_want = f64(x), ref.scales_of(f64(x), 128)
    scales = f64(got.scales)
    assert scales.shape == s_want.shape and (np.abs(scales - s_want) <= 2 * EPS * s_want).all()
    s = np.repeat(np.repeat(scales, 128, 0)[:R], 128, 1)[:, :C]
    assert (np.abs(ref.E4M3[bytes_of(got.codes)] * s - v) <= np.abs(v) * (2.0 ** -4 + 4 * EPS) + s * 2.0 ** -10).all()
    assert np.array_equal(f64(got.to_float()), ref.weights(bytes_of(got.codes), scales).astype(np.float32))


def test_quantize_takes_every_bf16_value():
    """All finite bf16 values, a block of one magnitude each (so the largest code is 448), zeros, denormals; then a block with
    an infinity, which stands for NaN, and one with a NaN, which keeps it to itself."""
    v = torch.arange(0x7F80, dtype=torch.int32).to(torch.int16).view(BF16).to(dev())
    x = v[:, None].expand(-1, 128) * torch.linspace(-1, 1, 128, device=dev())
    x = x.to(BF16).contiguous()
    x[:, 5] = v
    check_scaled(B.quantize(x), f64(x), 0.0 * f64(x))
    y = torch.randn(3, 256, device=dev())
    y[1, 7], y[2, 200] = float("inf"), float("nan")
    got = B.quantize(y).to_float().cpu()
    assert torch.isnan(got[1, :128]).all() and torch.isfinite(got[1, 128:]).all()
    assert torch.isnan(got[2, 200]) and torch.isfinite(got[2]).sum() == 255 and torch.isfinite(got[0]).all()


# -------------------------------------------------------------------------------------------------- norms
def norm_case(r, M, d, dtype, stream, post, gate, branch_scale, bias):
    a = dict(branch=put(r.normal(size=(M, d)) * np.exp(r.normal(size=(M, 1))), dtype, 3, 1),
             residual=put(r.normal(size=(M, d)) * np.exp(r.normal(size=(M, 1))) + 0.3, stream, 1, 5))
    vec = lambda mean: torch.from_numpy(r.normal(size=d) * 0.2 + mean).to(dtype).to(dev())   # noqa: E731
    a["weight"] = vec(1.0) if post != "none" else None
    a["bias"] = vec(0.0) if bias and post != "none" else None
    a["branch_scale"] = vec(0.5) if branch_scale else None
    a["next_weight"], a["next_bias"] = vec(1.0), vec(0.0) if bias else None
    a["gate_rows"] = int(r.integers(1, M + 2)) if gate else 1
    a["gate"] = put(r.normal(size=(-(-M // a["gate_rows"]), d)) * 2, dtype, 2) if gate else None
    return a


KIND = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
ACT = {"plain": B.GATE_PLAIN, "sigmoid": B.GATE_SIGMOID, "tanh": B.GATE_TANH}


def norm_reference(a, post, nxt, act, eps, plus, rs):
    """(h, its error, out, its error) in 64 bits.  c: what the fp32 sums over a row may lose, relative to their terms."""
    d = a["branch"].shape[1] if a["branch"] is not None else a["residual"].shape[1]
    c = (64 + d / 64) * EPS

    def norm(v, dv, kind, w, b):
        n, factor = ref.normalized(v, kind, eps)
        size = np.abs(v) + (np.abs(v).mean(1, keepdims=True) if kind == "layer" else 0)
        rel = np.sqrt((dv * dv).mean(1, keepdims=True)) * factor
        dn = factor * (dv + (dv.mean(1, keepdims=True) if kind == "layer" else 0) + c * size) + np.abs(n) * (c + rel + 4 * EPS)
        w = 1.0 if w is None else f64(w) + plus
        b = 0.0 if b is None else f64(b)
        return n * w + b, dn * np.abs(w) + 2 * EPS * (np.abs(n * w) + np.abs(b))

    b = f64(a["branch"]) if a["branch"] is not None else np.zeros((1, 1))
    db = 0.0 * b
    if post != "none":
        b, db = norm(b, db, post, a["weight"], a["bias"])
    for name in ("branch_scale", "gate"):
        if a[name] is not None:
            g = f64(a[name])
            if name == "gate":
                g = ref.activation(np.repeat(g, a["gate_rows"], 0)[:b.shape[0]], act)
            # sigmoid: exp of an argument of up to 10 rounded in fp32; tanh: a few units in the last place
            db = db * np.abs(g) + np.abs(b * g) * 16 * EPS
            b = b * g
    h = b if a["residual"] is None else np.float64(np.float32(rs)) * f64(a["residual"]) + b
    dh = db + 3 * EPS * (np.abs(b) + np.abs(h))
    n, dn = norm(h, dh, nxt, a["next_weight"], a["next_bias"]) if nxt != "none" else (None, None)
    return h, dh, n, dn


NORMS = [
    # rows, row length, types, norm after, norm before the next, gate, scale per channel, bias
    (1, 1, BF16, BF16, "rms", "rms", None, False, False),
    (1, 4096, BF16, BF16, "none", "rms", None, False, False),
    (5, 7, BF16, F32, "layer", "rms", "tanh", True, True),
    (6, 9, BF16, BF16, "rms", "layer", None, True, True),
    (70, 263, F32, F32, "layer", "layer", "sigmoid", True, True),
    (3, 127, BF16, F32, "rms", "rms", "plain", True, True),
    (5, 129, F32, F32, "layer", "layer", "sigmoid", False, True),
    (7, 511, BF16, BF16, "none", "layer", "tanh", True, False),
    (9, 513, F32, F32, "rms", "rms", "tanh", True, True),
    (4, 1000, BF16, BF16, "layer", "rms", None, False, True),
    (6, 1025, BF16, F32, "rms", "layer", "sigmoid", True, False),
    (17, 2048, BF16, BF16, "rms", "rms", "plain", False, False),
    (5, 2687, F32, F32, "rms", "layer", None, True, True),
    (3, 4097, BF16, BF16, "layer", "layer", "plain", True, True),
    (2, 5120, BF16, F32, "rms", "rms", "tanh", True, False),
    (33, 8191, BF16, BF16, "rms", "rms", None, False, False),
    (2, 8193, F32, F32, "layer", "rms", "plain", False, True),
    (3, 20000, BF16, F32, "rms", "rms", "sigmoid", False, False),
    (2, 32768, BF16, BF16, "rms", "rms", None, True, False),
    (2, 32763, F32, F32, "rms", "layer", "tanh", True, True),
    (700, 384, BF16, BF16, "rms", "rms", "plain", True, False),
    (2100, 1536, BF16, F32, "rms", "rms", "sigmoid", True, False),
    (1030, 4096, BF16, BF16, "rms", "rms", None, False, False),
    (1100, 5120, BF16, F32, "rms", "rms", "tanh", True, False),
    (600, 7000, F32, F32, "layer", "rms", None, True, True),
]


@pytest.mark.parametrize("scaled", [False, True], ids=["float", "f8"])
@pytest.mark.parametrize("M,d,dtype,stream,post,nxt,act,branch_scale,bias", NORMS)
def test_norm_out(M, d, dtype, stream, post, nxt, act, branch_scale, bias, scaled):
    r = rng(6, M, d)
    a = norm_case(r, M, d, dtype, stream, post, act is not None, branch_scale, bias)
    eps, plus, rs = 1e-5, float(r.integers(0, 2)), float(np.float32(r.uniform(0.5, 2)))
    h, hbuf = padded(M, d, stream, 7, -7.0, 2)
    hbefore = hbuf.clone()
    if scaled:
        q, buf = code_buffer(M, d, 16)
        s, sbuf = padded(-(-d // 128), M, BF16, 3, -7.0)
        out, before, sbefore = (q, s), buf.view(torch.uint8).clone(), sbuf.clone()
    else:
        out, buf = padded(M, d, dtype, 9, -7.0, 3)
        before = buf.clone()
    got_h, got = B.norm_out(a["branch"], a["residual"], a["weight"], bias=a["bias"], kind=KIND[post], eps=eps, weight_plus=plus,
                            residual_scale=rs, branch_scale=a["branch_scale"], gate=a["gate"], gate_rows=a["gate_rows"],
                            gate_act=ACT[act or "plain"], next_weight=a["next_weight"], next_bias=a["next_bias"],
                            next_kind=KIND[nxt], h=h, out=out)
    want_h, dh, want, dn = norm_reference(a, post, nxt, act, eps, plus, rs)
    check_float(got_h, want_h, dh, "h")
    (check_scaled if scaled else check_float)(got, want, dn, "out")
    h.fill_(-7.0)
    assert torch.equal(hbuf, hbefore)
    if scaled:
        q.view(torch.uint8).fill_(0x7F)
        s.fill_(-7.0)
        assert torch.equal(buf.view(torch.uint8), before) and torch.equal(sbuf, sbefore)
    else:
        out.fill_(-7.0)
        assert torch.equal(buf, before)


@pytest.mark.parametrize("M,d", [(1, 4096), (40, 1000), (300, 5120), (400, 515), (300, 4099), (40, 2687), (200, 8190)])
def test_norm_in_and_its_in_place_residual(M, d):
    """norm_in without and with what is added; h in the place of x gives the same bits as h elsewhere; norm_out without the
    next norm, the residual's buffer as its h."""
    r = rng(7, M, d)
    a = norm_case(r, M, d, BF16, BF16, "rms", False, False, False)
    x, add, w = a["residual"], a["branch"], a["next_weight"]
    only = dict(branch=None, residual=x, weight=None, bias=None, branch_scale=None, gate=None, next_weight=w, next_bias=None)
    _, _, want, dn = norm_reference(only, "none", "rms", None, 1e-6, 0.0, 1.0)
    check_float(B.norm_in(x, w), want, dn)
    check_scaled(B.norm_in(x, w, scaled=True), want, dn)
    h = torch.empty(M, d, dtype=BF16, device=dev())
    n = B.norm_in(x, w, add=add, h=h, residual_scale=0.5)
    want_h, dh, want, dn = norm_reference(dict(only, branch=add), "none", "rms", None, 1e-6, 0.0, 0.5)
    check_float(h, want_h, dh)
    check_float(n, want, dn)
    x2 = x.clone()
    n2 = B.norm_in(x2, w, add=add, h=x2, residual_scale=0.5)
    assert torch.equal(n2, n) and torch.equal(x2, h)
    x3 = x.clone()
    h3, none = B.norm_out(add, x3, a["weight"], h=x3)
    assert none is None and h3 is x3
    want_h, dh, _, _ = norm_reference(dict(only, branch=add, weight=a["weight"]), "rms", "none", None, 1e-6, 0.0, 1.0)
    check_float(x3, want_h, dh)


def test_rows_of_zeros_and_of_nan():
    x = torch.randn(4, 300, device=dev()).to(BF16)
    x[1] = 0
    x[2, 7] = float("nan")
    n = B.norm_in(x).float().cpu()
    assert not n[1].any() and torch.isnan(n[2]).all() and torch.isfinite(n[[0, 1, 3]]).all()
    q = B.norm_in(x, scaled=True)
    v = q.to_float().cpu()
    assert not v[1].any() and torch.isnan(v[2]).all() and torch.isfinite(v[[0, 1, 3]]).all()


def test_no_rows_do_nothing():
    e = torch.empty(0, 256, dtype=BF16, device=dev())
    assert B.quantize(e).codes.shape == (0, 256)
    W = B.quantize(torch.randn(64, 256, device=dev()), block_rows=128)
    assert B.scaled_matmul(B.quantize(e), W).shape == (0, 64)
    assert B.norm_in(e).shape == (0, 256)
    h, n = B.norm_out(e, e.clone(), scaled=True)
    assert h.shape == (0, 256) and n.codes.shape == (0, 256)


def test_more_rows_than_two_million():
    x = torch.randn((1 << 21) + 5, 16, dtype=BF16, device=dev())
    got = B.norm_in(x)
    for rows in (slice(0, 9), slice(-9, None)):
        assert torch.equal(got[rows], B.norm_in(x[rows]))


def test_offsets_beyond_32_bits():
    """1.1 million rows of 4096: 4.5e9 elements.  The last rows are those of a call of their own; the product's to two bf16
    roundings and what the matrix instruction drops (2.5e-5 of the result's size in either kernel, 1e-3 allowed)."""
    M, d = 1_100_000, 4096
    x = torch.randn(M, d, dtype=BF16, device=dev())
    last = slice(M - 200, M)
    got = B.quantize(x)
    alone = B.quantize(x[last])
    assert torch.equal(got.codes[last].view(torch.uint8), alone.codes.view(torch.uint8)) and torch.equal(got.scales[:, last], alone.scales)
    W = B.quantize(torch.randn(24, d, device=dev()), block_rows=128)
    p, q = B.scaled_matmul(got, W)[last].float(), B.scaled_matmul(alone, W).float()
    assert ((p - q).abs() <= 2 * 2.0 ** -8 * q.abs() + 1e-3 * q.abs().max()).all()
    p = B.scaled_matmul(got, W, out_dtype=torch.float8_e4m3fn).scales[:, last].float()
    q = B.scaled_matmul(alone, W, out_dtype=torch.float8_e4m3fn).scales.float()
    assert ((p - q).abs() <= 3 * 2.0 ** -8 * q).all()      # either rounded to bf16, and the product's difference in the largest
    h = torch.empty_like(x)
    n = B.norm_in(x, h=h)
    assert torch.equal(n[last], B.norm_in(x[last])) and torch.equal(h[last], x[last])


# ---------------------------------------------------------------------------------------------- together
def make_block(r, d, ffn, rank, rank_down):
    f = dict(Ug=(d, rank), Vg=(rank, ffn), Uu=(d, rank), Vu=(rank, ffn), Ud=(ffn, rank_down), Vd=(rank_down, d))
    return {k: torch.from_numpy(r.normal(size=s) / np.sqrt(s[0])).to(BF16).to(dev()) for k, s in f.items()}


def block(x, mlp, w_in, w_out, w_next):
    """A residual block around the 8-bit layer, as a serving loop runs it."""
    n = B.norm_in(x, w_in, scaled=True)
    y = mlp(n)
    return B.norm_out(y, x, w_out, next_weight=w_next, scaled=True)


@pytest.mark.parametrize("M", [1, 5, 40, 200, 600])
def test_a_block_in_8_bits(M):
    """Norm, gated factored layer and norm against the chain in 64 bits.  Each of five quantisations (the norm's output, T, H, Td
    and the weights) is off by at most 2^-4 relative, 0.026 in the root mean square; independent roundings of the terms of
    a sum keep that relative size, so operands contribute 0.026 each: sqrt(8) x 0.026 = 0.074 over the four products in
    a row, SiLU and the product of gate and up at most double it."""
    r = rng(8, M)
    d, ffn, rank, rank_down = 512, 1400, 200, 130
    f = make_block(r, d, ffn, rank, rank_down)
    mlp = B.SvdMlpF8(**f)
    x = torch.from_numpy(r.normal(size=(M, d))).to(BF16).to(dev())
    w = [torch.from_numpy(r.normal(size=d) * 0.1 + 1).to(BF16).to(dev()) for _ in range(3)]
    h, n = block(x, mlp, *w)
    f = {k: f64(v) for k, v in f.items()}
    v = ref.normalized(f64(x), "rms", 1e-6)[0] * f64(w[0])
    y = (ref.silu(v @ f["Ug"] @ f["Vg"]) * (v @ f["Uu"] @ f["Vu"]) @ f["Ud"]) @ f["Vd"]
    got = f64(mlp(B.norm_in(x, w[0], scaled=True)))
    assert np.linalg.norm(got - y) <= 0.15 * np.linalg.norm(y)
    want = f64(x) + ref.normalized(y, "rms", 1e-6)[0] * f64(w[1])
    assert np.linalg.norm(f64(h) - want) <= 0.15 * np.linalg.norm(want)
    want = ref.normalized(want, "rms", 1e-6)[0] * f64(w[2])
    assert np.linalg.norm(f64(n.to_float()) - want) <= 0.15 * np.linalg.norm(want)


@pytest.mark.parametrize("M", [3, 300])
def test_a_linear_layer_in_8_bits(M):
    r = rng(9, M)
    U, V = (torch.from_numpy(r.normal(size=s) / np.sqrt(s[0])).to(F32).to(dev()) for s in ((384, 72), (72, 501)))
    x = torch.from_numpy(r.normal(size=(M, 384))).to(F32).to(dev())
    lin = B.SvdMlpF8(Ug=U, Vg=V, kind=B.SVDMLP_LINEAR)
    out = torch.empty(M, 501, dtype=BF16, device=dev())
    assert lin(x, out=out) is out and lin.out_features() == 501
    want = f64(x) @ f64(U) @ f64(V)
    assert np.linalg.norm(f64(out) - want) <= 0.074 * np.linalg.norm(want)      # four operands of 0.026, and twice that


@pytest.mark.parametrize("M", [2, 70, 300])
def test_a_block_on_a_side_stream_and_in_a_graph(M):
    """The same bits on another stream, and from a graph that is replayed with new inputs between eager work."""
    r = rng(10, M)
    f = make_block(r, 512, 768, 128, 128)
    mlp = B.SvdMlpF8(**f)
    w = [torch.from_numpy(r.normal(size=512) * 0.1 + 1).to(BF16).to(dev()) for _ in range(3)]
    inputs = [torch.from_numpy(r.normal(size=(M, 512))).to(BF16).to(dev()) for _ in range(4)]
    want = [block(x, mlp, *w) for x in inputs]
    torch.cuda.synchronize()

    def same(got, i):
        return (torch.equal(got[0], want[i][0]) and torch.equal(got[1].codes.view(torch.uint8), want[i][1].codes.view(torch.uint8))
                and torch.equal(got[1].scales, want[i][1].scales))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = block(inputs[0], mlp, *w)
    side.synchronize()
    assert same(got, 0)
    n = B.norm_in(inputs[1], w[0], scaled=True, stream=side)
    y = mlp(n, stream=side)
    t = B.scaled_matmul(B.quantize(inputs[2], stream=side), mlp.first, stream=side)
    side.synchronize()
    assert torch.equal(t, B.scaled_matmul(B.quantize(inputs[2]), mlp.first))
    assert torch.equal(y, mlp(B.norm_in(inputs[1], w[0], scaled=True)))
    x = inputs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = block(x, mlp, *w)
    for i in (1, 2, 3, 0, 2):
        x.copy_(inputs[i])
        graph.replay()
        eager = block(inputs[i], mlp, *w)
        torch.cuda.synchronize()
        assert same(captured, i) and same(eager, i), i


def test_a_forward_on_a_side_stream_right_after_construction():
    """The constructor has quantised the factors when it returns, however much its stream had to do before: a forward on another
    stream, which nothing orders after it, gives the bits of one on the same."""
    r = rng(13)
    f = make_block(r, 512, 768, 128, 128)
    x = torch.from_numpy(r.normal(size=(40, 512))).to(BF16).to(dev())
    n = B.quantize(x)
    busy = torch.randn(4096, 4096, device=dev())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        busy = torch.mm(busy, busy).clamp_(-1, 1)
    mlp = B.SvdMlpF8(**f)
    y = mlp(n, stream=side)
    side.synchronize()
    want = mlp(n)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.isfinite(want).all()


def test_a_block_made_in_a_graph():
    """Its factors are quantised by the graph then, and again by each replay."""
    r = rng(14)
    f = make_block(r, 512, 768, 128, 128)
    x = torch.from_numpy(r.normal(size=(40, 512))).to(BF16).to(dev())
    want = B.SvdMlpF8(**f)(x)
    f2 = make_block(r, 512, 768, 128, 128)
    want2 = B.SvdMlpF8(**f2)(x)
    own = {k: v.clone() for k, v in f.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = B.SvdMlpF8(**own)(x)
    for factors, expected in ((f, want), (f2, want2), (f, want)):
        for k, v in factors.items():
            own[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, expected)


def hip_runtime():
    """The HIP runtime that torch and the library have loaded."""
    with open("/proc/self/maps") as f:
        return ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))


def test_an_error_that_an_earlier_call_left_is_not_the_launchs():
    """A call that failed before (here: a device that does not exist) leaves its error with the thread.  The operators launch what
    they are asked for and report their own launches only."""
    x = torch.randn(40, 256, device=dev()).to(BF16)
    W = B.quantize(torch.randn(300, 256, device=dev()), block_rows=128)
    A = B.quantize(x)
    a16, w16 = B.quantize(torch.randn(16, 14336, device=dev())), B.quantize(torch.randn(512, 14336, device=dev()), block_rows=128)
    calls = [lambda: B.quantize(x).scales, lambda: B.quantize(x, x).scales, lambda: B.quantize(x, block_rows=128).scales,
             lambda: B.norm_in(x), lambda: B.norm_out(x, x, scaled=True)[1].scales, lambda: B.scaled_matmul(A, W),
             lambda: B.scaled_matmul(A, W, gated=True), lambda: B.scaled_matmul(a16, w16, out_dtype=F8).scales]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    hip = hip_runtime()
    for call, expected in zip(calls, want):
        assert hip.hipSetDevice(1 << 20) != 0
        try:
            got = call()
        finally:
            hip.hipGetLastError()
        assert torch.equal(got, expected)


def test_operands_side_by_side_in_one_buffer():
    """Column ranges of one buffer, results beside inputs: no byte is shared, so the calls run, with the bits of calls on
    buffers of their own."""
    M, d, N = 70, 256, 128
    r = rng(15)
    whole = torch.zeros(M, 8 * d, dtype=torch.uint8, device=dev())
    x = whole[:, :2 * d].view(BF16)
    y = whole[:, 2 * d:4 * d].view(BF16)
    h = whole[:, 4 * d:6 * d].view(BF16)
    codes = whole[:, 6 * d:7 * d].view(F8)
    c = whole[:, 7 * d:].view(BF16)                  # [M, N]
    for t in (x, y):
        t.copy_(torch.from_numpy(r.normal(size=(M, d))))
    w = torch.from_numpy(r.normal(size=d)).to(BF16).to(dev())
    W = B.quantize(torch.from_numpy(r.normal(size=(N, d))).to(BF16).to(dev()), block_rows=128)
    scales = torch.empty(2, M, dtype=BF16, device=dev())
    x0, y0 = x.clone(), y.clone()
    B.quantize(x, y, out=(codes, scales))
    want = B.quantize(x0, y0)
    assert torch.equal(codes.contiguous().view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(scales, want.scales)
    B.norm_out(y, x, w, h=h, next_weight=w, out=(codes, scales))
    want_h, want = B.norm_out(y0, x0, w, next_weight=w, scaled=True)
    assert torch.equal(h, want_h) and torch.equal(codes.contiguous().view(torch.uint8), want.codes.view(torch.uint8))
    B.scaled_matmul((codes, scales), W, out=c)
    assert torch.equal(c, B.scaled_matmul(want, W))
    assert torch.equal(x, x0) and torch.equal(y, y0) and torch.equal(h, want_h)
    # shifted by a row, results would lie on inputs that other workgroups have yet to read
    with pytest.raises(B.SvdMlpError):
        B.norm_out(y[:-1], x[:-1], w, h=x[1:])
    with pytest.raises(B.SvdMlpError):
        B.quantize(x[:-1], out=(whole[1:, :d].view(F8), scales[:, 1:]))
    assert torch.equal(x, x0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_where_the_quantiser_rounds(dtype):
    """Bit for bit: the scale is the largest magnitude times 1 / 448, the code that of v times 1 / scale, each reciprocal rounded to
    fp32 before its product is.  (Torch on the CPU in fp32, which rounds every operation to nearest even.)"""
    r = rng(16)
    x = torch.from_numpy(r.normal(size=(300, 700)) * np.exp(4 * r.normal(size=(300, 1)))).to(dtype)
    x[7], x[8, :128] = 0, torch.finfo(dtype).tiny
    v = torch.nn.functional.pad(x.float(), (0, 68)).view(300, 6, 128)
    smallest, inv448 = torch.tensor(2.0 ** -100), torch.tensor(1.0) / 448
    for block_rows in (1, 128):
        got = B.quantize(x.to(dev()), block_rows=block_rows)
        amax = v.abs().amax(2)
        if block_rows == 1:
            s = torch.maximum(amax * inv448, smallest).to(BF16)
            assert torch.equal(got.scales.cpu(), s.t())
            s = s.float()
        else:
            amax = torch.nn.functional.pad(amax, (0, 0, 0, 84)).view(3, 128, 6).amax(1)
            s = torch.maximum(amax * inv448, smallest)
            assert torch.equal(got.scales.cpu(), s)
            s = s.repeat_interleave(128, 0)[:300]
        q = (v * (1.0 / s)[:, :, None]).clamp(-448, 448).to(F8).view(300, 768)[:, :700]
        assert np.array_equal(bytes_of(got.codes), bytes_of(q))


def test_a_block_of_strided_factors_that_require_a_gradient():
    """Factors of any strides, parameters among them, give the bits of contiguous ones; results carry no gradient."""
    r = rng(17)
    f = make_block(r, 512, 776, 128, 136)
    x = torch.from_numpy(r.normal(size=(20, 512))).to(BF16).to(dev())
    want = B.SvdMlpF8(**f)(x)
    strided = {}
    for i, (k, v) in enumerate(f.items()):
        if i % 2:
            strided[k] = torch.nn.Parameter(v.t().contiguous()).t()            # columns in one piece
        else:
            wide = torch.zeros(v.shape[0], v.shape[1] + 24, dtype=BF16, device=dev())
            wide[:, 8:8 + v.shape[1]] = v
            strided[k] = torch.nn.Parameter(wide)[:, 8:8 + v.shape[1]]
    got = B.SvdMlpF8(**strided)(x.clone().requires_grad_())
    assert torch.equal(got, want) and not got.requires_grad
    U, V = strided["Ug"], strided["Vg"]
    lin = B.SvdMlpF8(Ug=U, Vg=V, kind=B.SVDMLP_LINEAR)
    assert torch.equal(lin(x), B.SvdMlpF8(Ug=f["Ug"], Vg=f["Vg"], kind=B.SVDMLP_LINEAR)(x))

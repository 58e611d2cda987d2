"""Microscaled 4-bit operators: against the format's definition in 64 bits, and what they refuse."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_11660_amd import binding as B
from tests import mx4ref as R
from tests.gpu_util import dev, host, say

gpu = pytest.mark.gpu
FLOATS = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["f32", "f16", "bf16"]


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
# addresses that are never read: the checks fail before
X, A, S, W, WS, O, V, WK = (i << 32 for i in range(1, 9))


def test_quantize_refuses():
    f = B.lib().mbu_mx4_quantize
    good = [X, 0, 4, 96, 96, 0, A, S, None]

    def call(**other):
        names = ["x", "dtype", "rows", "k", "stride", "across", "codes", "scales", "stream"]
        return f(*[other.get(n, v) for n, v in zip(names, good)])

    assert call(x=None) == B.MBU_ERR_NULL and call(codes=None) == B.MBU_ERR_NULL and call(scales=None) == B.MBU_ERR_NULL
    assert call(dtype=3) == B.MBU_ERR_ARG and call(dtype=-1) == B.MBU_ERR_ARG and call(across=2) == B.MBU_ERR_ARG
    assert call(rows=0) == B.MBU_ERR_SHAPE and call(k=0) == B.MBU_ERR_SHAPE and call(rows=-1) == B.MBU_ERR_SHAPE
    assert call(k=(1 << 23) + 1) == B.MBU_ERR_SHAPE and call(stride=-1) == B.MBU_ERR_SHAPE
    assert call(x=X + 2) == B.MBU_ERR_ALIGN and call(x=X + 1, dtype=2) == B.MBU_ERR_ALIGN
    assert call(codes=A + 4) == B.MBU_ERR_ALIGN and call(scales=S + 8) == B.MBU_ERR_ALIGN
    assert call(codes=X) == B.MBU_ERR_ARG and call(scales=X + 16) == B.MBU_ERR_ARG and call(scales=A + 240) == B.MBU_ERR_ARG
    assert "mbu_mx4_quantize" in B.last_error()


def test_dequantize_refuses():
    f = B.lib().mbu_mx4_dequantize
    assert f(None, S, 4, 96, O, 0, None) == B.MBU_ERR_NULL and f(A, None, 4, 96, O, 0, None) == B.MBU_ERR_NULL
    assert f(A, S, 4, 96, None, 0, None) == B.MBU_ERR_NULL and f(A, S, 0, 96, O, 0, None) == B.MBU_ERR_SHAPE
    assert f(A, S, 4, 96, O, 7, None) == B.MBU_ERR_ARG and f(A, S, 4, 96, A, 0, None) == B.MBU_ERR_ARG
    assert f(A, S, 4, 96, O + 4, 0, None) == B.MBU_ERR_ALIGN


def test_products_refuse():
    L = B.lib()
    f, g = L.mbu_mx4_matmul, L.mbu_mx4_matmul_masked_binary
    assert f(None, S, 4, W, WS, 8, 96, V, O, 0, None) == B.MBU_ERR_NULL
    assert f(A, None, 4, W, WS, 8, 96, V, O, 0, None) == B.MBU_ERR_NULL
    assert f(A, S, 4, None, WS, 8, 96, V, O, 0, None) == B.MBU_ERR_NULL
    assert f(A, S, 4, W, None, 8, 96, V, O, 0, None) == B.MBU_ERR_NULL
    assert f(A, S, 4, W, WS, 8, 96, V, None, 0, None) == B.MBU_ERR_NULL
    for m, n, k in ((0, 8, 96), (4, 0, 96), (4, 8, 0), (4, 8, (1 << 23) + 1), (-4, 8, 96)):
        assert f(A, S, m, W, WS, n, k, V, O, 0, None) == B.MBU_ERR_SHAPE
        assert g(A, S, m, W, n, k, V, V, O, 0, None) == B.MBU_ERR_SHAPE
    assert f(A, S, 4, W, WS, 8, 96, V + 4, O, 0, None) == B.MBU_ERR_ALIGN
    assert g(A, S, 4, W, 8, 96, V + 8, V, O, 0, None) == B.MBU_ERR_ALIGN
    assert f(A, S, 4, W, WS, 8, 96, V, O + 2, 2, None) == B.MBU_ERR_ALIGN
    assert f(A, S, 4, W, WS, 8, 96, V, O, 3, None) == B.MBU_ERR_ARG
    for out in (A, S, W, WS, V, W + 64):
        assert f(A, S, 4, W, WS, 8, 96, V, out, 0, None) == B.MBU_ERR_ARG
    assert g(A, S, 4, W, 8, 96, V, None, W + 1024, 0, None) == B.MBU_ERR_ARG


def test_linear_refuses():
    L = B.lib()
    n = ctypes.c_size_t()
    assert L.mbu_mx4_linear_workspace_bytes(3, 100, None) == B.MBU_ERR_NULL
    assert L.mbu_mx4_linear_workspace_bytes(0, 100, ctypes.byref(n)) == B.MBU_ERR_SHAPE
    assert L.mbu_mx4_linear_workspace_bytes(3, 100, ctypes.byref(n)) == 0 and n.value == 0     # quantised on the way
    assert L.mbu_mx4_linear_workspace_bytes(100, 100, ctypes.byref(n)) == 0 and n.value >= 100 * (64 + 4)
    need = n.value
    f = L.mbu_mx4_linear
    assert f(None, 0, 100, 100, 100, W, WS, 8, V, O, 0, WK, need, None) == B.MBU_ERR_NULL
    assert f(X, 0, 100, 100, 100, W, WS, 8, V, O, 0, None, need, None) == B.MBU_ERR_NULL
    assert f(X, 0, 100, 100, 100, W, WS, 8, V, O, 0, WK, need - 1, None) == B.MBU_ERR_WORKSPACE
    assert f(X, 4, 100, 100, 100, W, WS, 8, V, O, 0, WK, need, None) == B.MBU_ERR_ARG
    assert f(X, 0, 100, 100, -1, W, WS, 8, V, O, 0, WK, need, None) == B.MBU_ERR_SHAPE
    assert f(X, 0, 100, 100, 100, W, WS, 8, V, O, 0, WK + 8, need, None) == B.MBU_ERR_ALIGN
    for out, ws in ((X, WK), (O, X), (O, O), (O, W), (O, V), (X + 39984, WK)):
        assert f(X, 0, 100, 100, 100, W, WS, 8, V, out, 0, ws, need, None) == B.MBU_ERR_ARG
    g = L.mbu_mx4_linear_masked_binary
    assert g(X, 0, 100, 100, 100, None, 8, V, None, O, 0, WK, need, None) == B.MBU_ERR_NULL
    assert g(X, 0, 100, 100, 100, W, 8, V, None, O, 0, WK, 0, None) == B.MBU_ERR_WORKSPACE


def test_packed_masked_binary_size():
    L = B.lib()
    n = ctypes.c_size_t()
    f = L.mbu_mx4_packed_masked_binary_bytes
    assert f(100, 1000, ctypes.byref(n)) == 0 and n.value >= 100 * 1000 / 4
    assert f(4096, 4096, ctypes.byref(n)) == 0 and n.value == 4096 * 4096 // 4
    assert f(100, 1000, None) == B.MBU_ERR_NULL and f(0, 1000, ctypes.byref(n)) == B.MBU_ERR_SHAPE
    assert L.mbu_mx4_pack_masked_binary(None, 100, 1000, O, None) == B.MBU_ERR_NULL
    assert L.mbu_mx4_pack_masked_binary(W, 100, 1000, W, None) == B.MBU_ERR_ARG


def test_host_tensors_are_refused():
    c, s = torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 4), dtype=torch.uint8)
    blob = torch.zeros(2048, dtype=torch.uint8)
    for call in (lambda: B.mx4_quantize(torch.zeros(4, 128)), lambda: B.mx4_dequantize(c, s, 128),
                 lambda: B.mx4_matmul(c, s, c, s), lambda: B.mx4_matmul_masked_binary(c, s, blob, 4),
                 lambda: B.mx4_linear(torch.zeros(4, 128), c, s), lambda: B.mx4_pack_masked_binary(s.view(torch.int8)),
                 lambda: B.mx4_linear_masked_binary(torch.zeros(4, 128), blob, 4)):
        with pytest.raises(ValueError, match="expected a device tensor"):
            call()


# -------------------------------------------------------------------------------------------------- the format (GPU)
def spread(rng, rows, k):
    """Values over many magnitudes, ties of the format, zeros of both signs, a block of zeros."""
    x = rng.standard_normal((rows, k)) * np.exp2(rng.integers(-20, 20, (rows, -(-k // 32)))).repeat(32, 1)[:, :k]
    tie = rng.random((rows, k)) < 0.3
    x = np.where(tie, rng.choice(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0, -0.25, -5.0]), (rows, k)), x)
    x[0, :32] = 0.0
    return x


def check_held(codes, scales, x):
    want, want_scales = R.quantize(x.float().cpu().numpy())
    assert np.array_equal(host(scales), want_scales)
    assert np.array_equal(host(codes), want)


@gpu
@pytest.mark.parametrize("dtype", FLOATS, ids=IDS)
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 32), (3, 33), (1, 4096), (17, 128), (5, 1000), (64, 257), (130, 640),
                                    (2, 9000), (700, 72)])
def test_quantize_and_back(dtype, rows, k):
    say(f"mx4 quantize {rows}x{k} {dtype}")
    rng = np.random.default_rng([rows, k])
    x = dev(spread(rng, rows, k)).to(dtype)
    if dtype == torch.float16:
        x = x.nan_to_num(posinf=60000, neginf=-60000)
    codes, scales = B.mx4_quantize(x)
    check_held(codes, scales, x)
    across = x.t().contiguous().t()
    c2, s2 = B.mx4_quantize(across)
    assert torch.equal(c2, codes) and torch.equal(s2, scales)
    want = R.values(host(codes), host(scales), k)
    for out in FLOATS:
        got = B.mx4_dequantize(codes, scales, k, out)
        assert got.dtype == out and torch.equal(got.cpu(), torch.from_numpy(want).to(out))


@gpu
@pytest.mark.parametrize("dtype", FLOATS, ids=IDS)
def test_quantize_views(dtype):
    """Rows that start anywhere, rows far apart, the same row again and again, across and along."""
    say(f"mx4 quantize views {dtype}")
    x = dev(np.random.default_rng(5).standard_normal((70, 401))).to(dtype)
    for v in (x[:, 1:], x[1::2, 3:259], x[:, :256], x[5:6, 7:], x[:1].expand(9, 401), x.t(), x.t()[3:, 1:], x.t()[:, ::2],
              x[:, 100:101], x[:, :1].expand(70, 1), x[::3].t()):
        codes, scales = B.mx4_quantize(v)
        check_held(codes, scales, v)
    with pytest.raises(ValueError, match="strides"):
        B.mx4_quantize(x[:, ::2])


@gpu
def test_quantize_far_magnitudes():
    """The largest and smallest float32 values, subnormals, infinities and NaN; each spoils its own block only."""
    say("mx4 quantize far magnitudes")
    rng = np.random.default_rng(3)
    x = np.zeros((6, 160), np.float32)
    for i, e in enumerate((127, -126, -127, -140, -149, 0)):
        x[i] = np.clip(rng.standard_normal(160) * 2.0 ** e, -3.4e38, 3.4e38)
    x[0, 3] = np.finfo(np.float32).max
    x[0, 40] = np.finfo(np.float32).min
    x[5, 0], x[5, 33], x[5, 70] = np.inf, -np.inf, np.nan
    t = dev(x)
    codes, scales = B.mx4_quantize(t)
    check_held(codes, scales, t)
    assert host(scales)[5].tolist()[:3] == [255, 255, 255] and 255 not in host(scales)[:5]
    got = host(B.mx4_dequantize(codes, scales, 160))
    np.testing.assert_array_equal(got, R.values(host(codes), host(scales), 160).astype(np.float32))
    assert np.isnan(got[5, :96]).all() and np.isfinite(got[5, 96:]).all()
    for dt in (torch.float16, torch.bfloat16):
        y = torch.tensor([[float("inf")] + [1.0] * 31, [float("nan")] + [1.0] * 31, [1.0] * 32], device="cuda", dtype=dt)
        assert host(B.mx4_quantize(y)[1])[:, 0].tolist() == [255, 255, 125]
        assert host(B.mx4_quantize(y.t().contiguous().t())[1])[:, 0].tolist() == [255, 255, 125]


# ------------------------------------------------------------------------------------------------------ products (GPU)
SHAPES = [(1, 1, 1), (1, 16, 128), (1, 100, 4096), (2, 17, 129), (5, 1000, 640), (16, 64, 512), (16, 33, 5000), (17, 33, 513),
          (31, 40, 32), (33, 100, 640), (64, 256, 2048), (100, 300, 1000), (129, 257, 2050), (300, 520, 1536),
          (513, 1030, 777)]


def rounded(want, dtype):
    return torch.from_numpy(want).to(torch.float32).to(dtype)     # `want` is exact in float32


@gpu
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_are_exact_where_float32_is(m, n, k):
    """Sums of whole multiples of 2^-4 below 2^20: every order gives the same float32, which is rounded once."""
    say(f"mx4 products {m}x{n}x{k}")
    rng = np.random.default_rng([m, n, k])
    (a, sa), (b, sb), w = R.held(rng, m, k), R.held(rng, n, k), R.ternary(rng, n, k)
    w[n // 2] = 0                                                 # an output that the mask leaves nothing
    bias = rng.integers(-64, 65, n).astype(np.float32)
    alpha = np.exp2(rng.integers(-3, 4, n)).astype(np.float32)
    da, dsa, db, dsb, dbias, dalpha = (dev(t) for t in (a, sa, b, sb, bias, alpha))
    va = R.values(a, sa)
    held = va @ R.values(b, sb).T
    masked = va[:, :k] @ w.astype(np.float64).T
    blob = B.mx4_pack_masked_binary(dev(w))
    for dtype in FLOATS:
        got = B.mx4_matmul(da, dsa, db, dsb, dbias, dtype)
        assert got.dtype == dtype and torch.equal(got.cpu(), rounded(held + bias, dtype))
        got = B.mx4_matmul_masked_binary(da, dsa, blob, n, dalpha, dbias, dtype)
        assert got.dtype == dtype and torch.equal(got.cpu(), rounded(masked * alpha + bias, dtype))
    assert torch.equal(B.mx4_matmul(da, dsa, db, dsb, dtype=torch.float32).cpu(), rounded(held, torch.float32))
    assert torch.equal(B.mx4_matmul_masked_binary(da, dsa, blob, n, dtype=torch.float32).cpu(), rounded(masked, torch.float32))
    # the layer: a's values as floats; a block's scale may come out smaller than it was, and holds the same values
    x = torch.from_numpy(va[:, :k])
    q = R.values(*R.quantize(va[:, :k]), k)
    assert np.array_equal(q, va[:, :k])
    for dtype in FLOATS:
        xd = x.to(dtype).cuda()                                   # exact in every type
        got = B.mx4_linear(xd, db, dsb, dbias)
        assert got.dtype == dtype and torch.equal(got.cpu(), rounded(q @ R.values(b, sb, k).T + bias, dtype))
        got = B.mx4_linear_masked_binary(xd, blob, n, dalpha, dbias, torch.float32)
        assert torch.equal(got.cpu(), rounded(q @ w.astype(np.float64).T * alpha + bias, torch.float32))


@gpu
@pytest.mark.parametrize("m,n,k", [(1, 257, 8192), (3, 64, 16000), (16, 130, 4100), (40, 515, 3000), (260, 300, 6000)])
def test_products_of_far_scales(m, n, k):
    """Scales over 2^40: at most K additions, each off by at most 2^-23 of the sum of magnitudes (one unit in the last
    place, in whatever order), then bias and the rounding to the output's type."""
    say(f"mx4 products of far scales {m}x{n}x{k}")
    rng = np.random.default_rng([m, n, k, 1])
    (a, sa), (b, sb), w = R.held(rng, m, k, 107, 147), R.held(rng, n, k, 107, 147), R.ternary(rng, n, k)
    bias, alpha = rng.standard_normal(n).astype(np.float32), rng.random(n).astype(np.float32)
    va, vb = R.values(a, sa), R.values(b, sb)
    for got, want, size in (
            (B.mx4_matmul(dev(a), dev(sa), dev(b), dev(sb), dev(bias), torch.float32), va @ vb.T + bias,
             np.abs(va) @ np.abs(vb).T),
            (B.mx4_matmul_masked_binary(dev(a), dev(sa), B.mx4_pack_masked_binary(dev(w)), n, dev(alpha), dev(bias),
                                        torch.float32), va[:, :k] @ w.T.astype(np.float64) * alpha + bias,
             np.abs(va[:, :k]) @ np.abs(w.T.astype(np.float64)) * alpha)):
        assert (np.abs(host(got) - want) <= (k + 3) * 2.0 ** -23 * (size + np.abs(bias))).all()


@gpu
@pytest.mark.parametrize("m", [1, 20, 300])
def test_not_a_number_stays_in_its_row(m):
    say(f"mx4 NaN blocks M={m}")
    rng = np.random.default_rng(m)
    n, k = 272, 700
    (a, sa), (b, sb), w = R.held(rng, m, k), R.held(rng, n, k), R.ternary(rng, n, k)
    clean = B.mx4_matmul(dev(a), dev(sa), dev(b), dev(sb), dtype=torch.float32)
    sa[m // 2, 21] = 255                                          # last block: 28 values
    w[:, 672:] = 0                                                # masked there: NaN all the same
    sb[5, 0] = 255
    got = host(B.mx4_matmul(dev(a), dev(sa), dev(b), dev(sb), dtype=torch.float32))
    bad = np.zeros((m, n), bool)
    bad[m // 2], bad[:, 5] = True, True
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], host(clean)[~bad])
    blob = B.mx4_pack_masked_binary(dev(w))
    got = host(B.mx4_matmul_masked_binary(dev(a), dev(sa), blob, n, dtype=torch.float32))
    assert np.isnan(got[m // 2]).all() and np.isfinite(np.delete(got, m // 2, 0)).all()
    x = rng.standard_normal((m, k)).astype(np.float32)
    x[m // 2, 400] = np.inf
    got = host(B.mx4_linear_masked_binary(dev(x), blob, n))
    assert np.isnan(got[m // 2]).all() and np.isfinite(np.delete(got, m // 2, 0)).all()


@gpu
@pytest.mark.parametrize("dtype", FLOATS, ids=IDS)
def test_linear_views(dtype):
    """Rows that start anywhere or repeat: what quantisation and product give one after the other, bit for bit."""
    say(f"mx4 linear views {dtype}")
    rng = np.random.default_rng(8)
    x = dev(rng.standard_normal((70, 1290))).to(dtype)
    for v in (x[:, 1:641], x[::2, :640], x[:3, 2:642], x[:1], x[:1].expand(5, 1290), x[4:5, 3:], x[:20, 8:776]):
        k = v.shape[1]
        b, sb = B.mx4_quantize(dev(rng.standard_normal((100, k)).astype(np.float32)))
        blob = B.mx4_pack_masked_binary(dev(R.ternary(rng, 100, k)))
        a, sa = B.mx4_quantize(v)
        assert torch.equal(B.mx4_linear(v, b, sb), B.mx4_matmul(a, sa, b, sb, dtype=dtype))
        assert torch.equal(B.mx4_linear_masked_binary(v, blob, 100),
                           B.mx4_matmul_masked_binary(a, sa, blob, 100, dtype=dtype))
    with pytest.raises(ValueError, match="consecutive"):
        B.mx4_linear(x[:, ::2], b, sb)


@gpu
def test_pack_takes_weights_by_sign():
    say("mx4 pack by sign")
    rng = np.random.default_rng(2)
    w = rng.integers(-128, 128, (50, 300)).astype(np.int8)
    assert torch.equal(B.mx4_pack_masked_binary(dev(w)), B.mx4_pack_masked_binary(dev(np.sign(w))))


@gpu
def test_wrong_tensors_are_refused():
    say("mx4 wrong tensors")
    a, sa = B.mx4_quantize(torch.ones(4, 200, device="cuda"))
    b, sb = B.mx4_quantize(torch.ones(8, 300, device="cuda"))
    blob = B.mx4_pack_masked_binary(torch.ones(8, 200, dtype=torch.int8, device="cuda"))
    bias = torch.ones(8, device="cuda")
    x = torch.ones(4, 200, device="cuda")
    for call in (lambda: B.mx4_matmul(a, sa, b, sb), lambda: B.mx4_matmul(a, sb, a, sa), lambda: B.mx4_matmul(a[:, :32], sa, a, sa),
                 lambda: B.mx4_matmul(a, sa, a, sa, bias), lambda: B.mx4_matmul(a, sa, a, sa, dtype=torch.int32),
                 lambda: B.mx4_matmul(a.t(), sa, a, sa), lambda: B.mx4_dequantize(a, sa, 128), lambda: B.mx4_dequantize(a, sa, 257),
                 lambda: B.mx4_matmul_masked_binary(a, sa, blob, 17), lambda: B.mx4_matmul_masked_binary(b, sb, blob[:-16], 8),
                 lambda: B.mx4_matmul_masked_binary(a, sa, blob, 8, bias[:7]), lambda: B.mx4_linear(x, b, sb),
                 lambda: B.mx4_linear(x.to(torch.int32), a, sa), lambda: B.mx4_linear(x[0], a, sa),
                 lambda: B.mx4_linear_masked_binary(x, blob, 8, bias.half()), lambda: B.mx4_quantize(x.double()),
                 lambda: B.mx4_pack_masked_binary(x.to(torch.int8).t())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.mx4_quantize(x[:0]), lambda: B.mx4_quantize(x[:, :0]), lambda: B.mx4_linear(x[:0], a, sa),
                 lambda: B.mx4_matmul_masked_binary(a, sa, blob, 0)):
        with pytest.raises(B.MbuError) as e:
            call()
        assert e.value.code == B.MBU_ERR_SHAPE


@gpu
def test_offsets_beyond_32_bits():
    """Inputs of more than 2^31 values, held weights and an output of more than 2^31 bytes: the last rows."""
    say("mx4 offsets beyond 32 bits")
    rng = np.random.default_rng(9)
    x = torch.zeros((65540, 32768), dtype=torch.bfloat16, device="cuda")
    last = torch.from_numpy(rng.standard_normal((3, 32768)).astype(np.float32)).to(torch.bfloat16)
    x[-3:] = last.cuda()
    codes, scales = B.mx4_quantize(x)
    check_held(codes[-3:], scales[-3:], last)
    assert int(codes[:-3].max()) == 0 and torch.equal(B.mx4_dequantize(codes, scales, 32768, torch.bfloat16)[-3:],
                                                      B.mx4_dequantize(codes[-3:], scales[-3:], 32768, torch.bfloat16))
    del x
    codes = torch.cat((codes, codes, codes))
    scales = torch.cat((scales, scales, scales))
    assert codes.numel() > 1 << 31
    a, sa = codes[-3:].clone(), scales[-3:].clone()
    for m in (1, 3):
        assert torch.equal(B.mx4_matmul(a[:m], sa[:m], codes, scales)[:, -16:], B.mx4_matmul(a[:m], sa[:m], codes[-16:], scales[-16:]))
    assert torch.equal(B.mx4_matmul(codes, scales, a, sa)[-3:], B.mx4_matmul(a, sa, a, sa))
    del codes, scales
    (b, sb), (c, sc) = R.held(rng, 32800, 64), R.held(rng, 40000, 64)
    got = B.mx4_matmul(dev(c), dev(sc), dev(b), dev(sb), dtype=torch.float16)
    assert got.numel() * 2 > 1 << 31
    want = R.values(c[-20:], sc[-20:]) @ R.values(b, sb).T
    assert torch.equal(got[-20:].cpu(), rounded(want, torch.float16))


# -------------------------------------------------------------------------------------------- as a program uses them
class Layers:
    """Two layers of a feed-forward block: weights in the format, then masked-binary ones."""

    def __init__(self, rng, k, hidden):
        self.w1 = rng.standard_normal((hidden, k)).astype(np.float32)
        self.w2, self.k = R.ternary(rng, k, hidden), k
        self.b, self.sb = B.mx4_quantize(dev(self.w1.T.copy()).t())       # stored input-major
        self.blob = B.mx4_pack_masked_binary(dev(self.w2))
        self.bias, self.alpha = dev(rng.standard_normal(hidden).astype(np.float32)), dev(rng.random(k).astype(np.float32))

    def __call__(self, x):
        h = torch.relu(B.mx4_linear(x, self.b, self.sb, self.bias))
        return x + B.mx4_linear_masked_binary(h, self.blob, self.k, self.alpha)

    def in_parts(self, x):
        h = torch.relu(B.mx4_matmul(*B.mx4_quantize(x), self.b, self.sb, self.bias, x.dtype))
        return x + B.mx4_matmul_masked_binary(*B.mx4_quantize(h), self.blob, self.k, self.alpha, dtype=x.dtype)


@gpu
@pytest.mark.parametrize("m", [1, 24, 200])
def test_layers_in_a_row(m):
    say(f"mx4 layers M={m}")
    net = Layers(np.random.default_rng(4), 640, 1536)
    x = torch.randn((m, 640), device="cuda")
    y = net(x)
    assert torch.equal(y, net.in_parts(x)) and torch.equal(y, net(x))
    q = R.values(*R.quantize(host(x)), 640) @ R.values(*R.quantize(net.w1), 640).T + host(net.bias)
    h = host(torch.relu(B.mx4_linear(x, net.b, net.sb, net.bias)))
    size = np.abs(R.values(*R.quantize(host(x)), 640)) @ np.abs(R.values(*R.quantize(net.w1), 640)).T
    assert (np.abs(h - np.maximum(q, 0)) <= 643 * 2.0 ** -23 * (size + np.abs(host(net.bias)))).all()
    hq = R.values(*R.quantize(h), 1536)
    want = host(x) + hq @ net.w2.T.astype(np.float64) * host(net.alpha)
    size = np.abs(hq) @ np.abs(net.w2.T.astype(np.float64)) * host(net.alpha)
    assert (np.abs(host(y) - want) <= 1540 * 2.0 ** -23 * (size + np.abs(host(x)))).all()


@gpu
@pytest.mark.parametrize("m", [1, 40, 260])
def test_captured_and_on_another_stream(m):
    """Replays on new inputs, with other calls between them, and calls on a second stream give the eager results."""
    say(f"mx4 captured M={m}")
    net = Layers(np.random.default_rng(6), 512, 640)
    x = torch.randn((m, 512), device="cuda", dtype=torch.bfloat16)
    net(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = net(x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, net(x))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = net(x)
        graphs.append((g, out))
    for i in range(4):
        x.copy_(torch.randn((m, 512), device="cuda"))
        want = net(x).clone()
        for g, out in graphs:
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i


@gpu
def test_calls_at_the_same_time_on_two_streams():
    say("mx4 two streams")
    net = Layers(np.random.default_rng(7), 512, 640)
    xs = [torch.randn((m, 512), device="cuda", dtype=torch.bfloat16) for m in (64, 300)]
    want = [net(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(net(xs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])

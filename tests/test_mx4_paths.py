"""Products in the microscaled 4-bit format: every kernel of the automatic choice against exact products, with outputs
that end anywhere in its tiles; and the native calls against the general code."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from paper_2601_11660_amd import binding as B
from tests import mx4ref as R
from tests.gpu_util import dev, say
from tests.test_native_calls import General

pytestmark = pytest.mark.gpu
FEW, WAVE = "mx4_few_kernel", "mx4_wave_kernel"
HELD, MASKED = "mx4_tile_held_kernel", "mx4_tile_masked_kernel"


# rows, inputs, and the kernels of held and of masked-binary weights for about as many outputs as are named
@pytest.mark.parametrize("m, n, k, held, masked", [
    (16, 203, 1000, FEW + "<3, false, 1>", FEW + "<3, true, 1>"),
    (1, 9000, 8192, FEW + "<3, false, 1>", FEW + "<3, true, 1>"),         # three tiles of 16 outputs by one block
    (2, 8701, 520, FEW + "<3, false, 1>", FEW + "<3, true, 1>"),          # two waves a block
    (7, 60, 9000, FEW + "<3, false, 2>", FEW + "<3, true, 2>"),
    (16, 8300, 10000, FEW + "<3, false, 2>", FEW + "<3, true, 2>"),
    (13, 1, 16384, FEW + "<3, false, 2>", FEW + "<3, true, 2>"),
    (13, 300, 16385, WAVE + "<false, 2, 2>", WAVE + "<true, 2, 2>"),      # a step more than fits into registers
    (17, 50, 70, WAVE + "<false, 2, 2>", WAVE + "<true, 2, 2>"),
    (99, 4090, 640, WAVE + "<false, 2, 4>", WAVE + "<true, 2, 4>"),
    (250, 4001, 2050, WAVE + "<false, 4, 4>", WAVE + "<true, 4, 4>"),
    (300, 4040, 1300, HELD + "<1, 4, 4, 2>", MASKED + "<4, 2>"),
    (599, 5021, 640, HELD + "<2, 2, 4, 4>", MASKED + "<4, 2>"),
    (1001, 5002, 250, HELD + "<2, 4, 4, 4>", MASKED + "<8, 4>"),
    (2047, 5009, 600, HELD + "<2, 4, 8, 4>", MASKED + "<8, 4>"),
    (20000, 257, 128, HELD + "<2, 4, 8, 4>", MASKED + "<8, 4>"),
    (33000, 129, 1, HELD + "<2, 4, 8, 4>", MASKED + "<8, 4>"),
])
def test_every_kernel(m, n, k, held, masked):
    """Sums of multiples of 2^-4 below 36 K <= 2^20: exact in float32 in any order.  n and the next multiples of 4 and of
    8 behind it: outputs stored one by one, four and eight at a time."""
    rng = np.random.default_rng([m, n, k])
    a, sa = R.held(rng, m, k, 126, 127)
    va = torch.from_numpy(R.values(a, sa, k)).float()
    da, dsa = dev(a), dev(sa)
    for wide in dict.fromkeys((n, -(-n // 4) * 4 + 4 * (-(-n // 4) % 2 == 0), -(-n // 8) * 8)):
        say(f"mx4 kernels {m}x{wide}x{k}")
        (b, sb), w = R.held(rng, wide, k, 126, 127), R.ternary(rng, wide, k)
        blob, bias = B.mx4_pack_masked_binary(dev(w)), rng.integers(-64, 65, wide).astype(np.float32)
        alpha = np.exp2(rng.integers(-3, 4, wide)).astype(np.float32)
        # exact in float32 as well, as is every partial sum
        want = (va @ torch.from_numpy(R.values(b, sb, k)).float().T + torch.from_numpy(bias))
        want_masked = (va @ torch.from_numpy(w).float().T * torch.from_numpy(alpha))
        for dtype in (torch.float32, torch.float16, torch.bfloat16):
            got = B.mx4_matmul(da, dsa, dev(b), dev(sb), dev(bias), dtype)
            assert B.last_kernel() == held
            assert torch.equal(got.cpu(), want.to(dtype))
            got = B.mx4_matmul_masked_binary(da, dsa, blob, wide, dev(alpha), None, dtype)
            assert B.last_kernel() == masked
            assert torch.equal(got.cpu(), want_masked.to(dtype))


@pytest.mark.parametrize("m, k, kernel", [(1, 16384, "<2, false, 2>"), (4, 8192, "<2, false, 1>"), (16, 4096, "<2, false, 1>"),
                                          (16, 4097, "<3, false, 1>"), (5, 16384, "<3, false, 2>"), (16, 10, "<2, false, 1>")])
def test_floats_are_quantised_on_the_way_or_ahead(m, k, kernel):
    """The same bits either way, and with rows that start anywhere."""
    say(f"mx4 linear on the way {m}x{k}")
    x = torch.randn((m, k + 3), device="cuda").to(torch.bfloat16)[:, 3:]
    b, sb = B.mx4_quantize(torch.randn((5000, k), device="cuda"))
    got = B.mx4_linear(x, b, sb)
    assert B.last_kernel() == FEW + kernel
    assert torch.equal(got, B.mx4_matmul(*B.mx4_quantize(x), b, sb, dtype=torch.bfloat16))


@pytest.mark.parametrize("m, n, k", [(1, 203, 1000), (5, 4500, 8200), (40, 100, 700), (100, 4083, 130), (250, 4004, 300),
                                     (300, 4040, 520), (599, 5021, 140), (1001, 5004, 150), (2000, 5010, 160)])
def test_nothing_else_is_read_or_written(m, n, k):
    """Operands, factors and biases in the middle of NaN, the output in the middle of a mark."""
    say(f"mx4 margins {m}x{n}x{k}")
    rng = np.random.default_rng([m, n, k])
    kp = R.padded(k)

    def inside(t, rows=24, fill=255):
        big = torch.full((t.shape[0] + 2 * rows, *t.shape[1:]), fill, dtype=t.dtype, device="cuda")
        big[rows:rows + t.shape[0]] = t
        return big[rows:rows + t.shape[0]]

    (a, sa), (b, sb), w = R.held(rng, m, k, 126, 127), R.held(rng, n, k, 126, 127), R.ternary(rng, n, k)
    bias, alpha = rng.integers(-64, 65, n).astype(np.float32), np.exp2(rng.integers(-3, 4, n)).astype(np.float32)
    da, dsa, db, dsb = (inside(dev(t)) for t in (a, sa, b, sb))
    dbias, dalpha = (inside(dev(t), 24, float("nan")) for t in (bias, alpha))
    blob = inside(B.mx4_pack_masked_binary(dev(w)), 2048)
    x = inside(dev(R.values(a, sa, k)).float(), 24, float("nan"))
    va = torch.from_numpy(R.values(a, sa, k)).float()
    want = va @ torch.from_numpy(R.values(b, sb, k)).float().T + torch.from_numpy(bias)
    want_masked = va @ torch.from_numpy(w).float().T * torch.from_numpy(alpha) + torch.from_numpy(bias)
    work = torch.full((m * kp + 4096,), 77, dtype=torch.uint8, device="cuda")
    need, L, stream = ctypes.c_size_t(), B.lib(), torch.cuda.current_stream().cuda_stream
    B.check(L.mbu_mx4_linear_workspace_bytes(m, k, ctypes.byref(need)))
    p = lambda t: t.data_ptr()                                                   # noqa: E731
    for code, dtype in enumerate((torch.float32, torch.float16, torch.bfloat16)):
        calls = [
            (want, lambda o: L.mbu_mx4_matmul(p(da), p(dsa), m, p(db), p(dsb), n, k, p(dbias), o, code, stream)),
            (want_masked, lambda o: L.mbu_mx4_matmul_masked_binary(p(da), p(dsa), m, p(blob), n, k, p(dalpha), p(dbias), o, code, stream)),
            (want, lambda o: L.mbu_mx4_linear(p(x), 0, m, k, k, p(db), p(dsb), n, p(dbias), o, code, p(work), need.value, stream)),
            (want_masked, lambda o: L.mbu_mx4_linear_masked_binary(p(x), 0, m, k, k, p(blob), n, p(dalpha), p(dbias), o, code, p(work),
                                                                   need.value, stream))]
        for exact, call in calls:
            out = torch.full((m * n + 128,), 5.5, dtype=dtype, device="cuda")
            B.check(call(p(out) + 64 * out.element_size()))
            assert torch.equal(out[64:-64].view(m, n).cpu(), exact.to(dtype))
            assert bool((out[:64] == 5.5).all()) and bool((out[-64:] == 5.5).all())
            assert bool((work[need.value:] == 77).all())
    # and the conversions
    codes = torch.full((m * kp // 2 + 512,), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((m * kp // 32 + 512,), 77, dtype=torch.uint8, device="cuda")
    across = x.t().contiguous()
    for source, stride, flag in ((x, k, 0), (across, m, 1)):
        codes.fill_(77), scales.fill_(77)
        B.check(L.mbu_mx4_quantize(p(source), 0, m, k, stride, flag, p(codes) + 256, p(scales) + 256, stream))
        assert torch.equal(codes[256:-256].view(m, -1), B.mx4_quantize(x)[0])
        assert torch.equal(scales[256:-256].view(m, -1), B.mx4_quantize(x)[1])
        assert all(bool((t[i] == 77).all()) for t in (codes, scales) for i in (slice(256), slice(-256, None)))
    for code, dtype in enumerate((torch.float32, torch.float16, torch.bfloat16)):
        out = torch.full((m * k + 128,), 5.5, dtype=dtype, device="cuda")
        B.check(L.mbu_mx4_dequantize(p(da), p(dsa), m, k, p(out) + 64 * out.element_size(), code, stream))
        assert torch.equal(out[64:-64].view(m, k).cpu(), va.to(dtype))
        assert bool((out[:64] == 5.5).all()) and bool((out[-64:] == 5.5).all())


@pytest.mark.parametrize("rows, k", [(70000, 1), (40000, 100), (70000, 33), (5000, 1001), (530, 8193), (3, 8200), (16400, 257)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_conversions_of_many_rows(dtype, rows, k):
    """Narrow and wide rows, from four threads a row to several pieces of one; along, across and back."""
    say(f"mx4 conversions {rows}x{k} {dtype}")
    x = torch.randn((rows, k), device="cuda").to(dtype)
    codes, scales = B.mx4_quantize(x)
    at = np.unique(np.random.default_rng(rows).integers(0, rows, 200).tolist() + [0, rows - 1])
    pick = torch.from_numpy(at).cuda()
    want, want_scales = R.quantize(x[pick].float().cpu().numpy())
    assert np.array_equal(codes[pick].cpu().numpy(), want) and np.array_equal(scales[pick].cpu().numpy(), want_scales)
    c2, s2 = B.mx4_quantize(x.t().contiguous().t())
    assert torch.equal(c2, codes) and torch.equal(s2, scales)
    back = B.mx4_dequantize(codes, scales, k, dtype)
    assert torch.equal(back[pick].cpu(), torch.from_numpy(R.values(want, want_scales, k)).to(dtype))
    # quantising what came back changes no value
    assert torch.equal(B.mx4_dequantize(*B.mx4_quantize(back), k, dtype), back)


def test_sign_of_zero_and_infinity_without_factor_and_bias():
    """Zeros stay zeros, and what is beyond the output's type is infinite."""
    say("mx4 signs of zero")
    for m, n in ((3, 40), (40, 40), (300, 5000)):
        a, sa = B.mx4_quantize(torch.full((m, 200), -0.0, device="cuda"))
        b, sb = B.mx4_quantize(torch.full((n, 200), 2.0 ** 60, device="cuda"))
        plain = B.mx4_matmul(a, sa, b, sb, dtype=torch.float32)
        assert int(plain.count_nonzero()) == 0
        with_zero = B.mx4_matmul(a, sa, b, sb, torch.zeros(n, device="cuda"), torch.float32)
        assert int(with_zero.count_nonzero()) == 0 and not bool(torch.signbit(with_zero).any())
        big = B.mx4_matmul(b[:m] if m <= n else b, sb[:m] if m <= n else sb, b, sb, dtype=torch.float16)
        assert bool(torch.isposinf(big).all())


def calls():
    """(function, arguments) of every call that has a native form, as users make them."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((37, 300), device="cuda", generator=g)
    b, sb = B.mx4_quantize(torch.randn((70, 300), device="cuda", generator=g))
    w = torch.randint(-1, 2, (70, 300), device="cuda", generator=g).to(torch.int8)
    a, sa = B.mx4_quantize(x)
    blob, bias, alpha = B.mx4_pack_masked_binary(w), torch.randn(70, device="cuda"), torch.rand(70, device="cuda")
    grad = x.clone().requires_grad_()
    return [(B.mx4_quantize, (x,)), (B.mx4_quantize, (x.half().t(),)), (B.mx4_quantize, (x[1::3, 5:],)), (B.mx4_quantize, (grad,)),
            (B.mx4_dequantize, (a, sa, 300)), (B.mx4_dequantize, (a, sa, 257, torch.bfloat16)),
            (B.mx4_matmul, (a, sa, b, sb)), (B.mx4_matmul, (a, sa, b, sb, bias, torch.float16)),
            (B.mx4_matmul, (a[:5], sa[:5], b, sb, None, torch.float32)),
            (B.mx4_matmul_masked_binary, (a, sa, blob, 70)),
            (B.mx4_matmul_masked_binary, (a, sa, blob, 70, alpha, bias, torch.float32)),
            (B.mx4_linear, (x, b, sb)), (B.mx4_linear, (x[:3].bfloat16(), b, sb, bias)),
            (B.mx4_linear, (x.half(), b, sb, bias, torch.float32)),
            (B.mx4_linear_masked_binary, (x, blob, 70)), (B.mx4_linear_masked_binary, (x[:2], blob, 70, alpha, None, torch.float16)),
            # refused
            (B.mx4_quantize, (x[0],)), (B.mx4_quantize, (x.cpu(),)), (B.mx4_quantize, (x[:0],)), (B.mx4_quantize, (x[:, ::2],)),
            (B.mx4_dequantize, (a, sb, 300)), (B.mx4_dequantize, (a, sa, 385)), (B.mx4_dequantize, (a, sa, 256)),
            (B.mx4_dequantize, (a, sa, -1)), (B.mx4_matmul, (a, sa, b[:, :128], sb)), (B.mx4_matmul, (a, sa, b, sb, bias[1:])),
            (B.mx4_matmul, (a, sa, b, sb, bias.double())), (B.mx4_matmul, (a.cpu(), sa, b, sb)), (B.mx4_matmul, (a, sa, b.cpu(), sb)),
            (B.mx4_matmul_masked_binary, (a, sa, blob[16:], 70)), (B.mx4_matmul_masked_binary, (a, sa, blob, -70)),
            (B.mx4_linear, (x[:, :200], b, sb)), (B.mx4_linear, (x.t(), b, sb)), (B.mx4_linear, (x, b, sb, bias.cpu())),
            (B.mx4_linear_masked_binary, (x, blob, 90)), (B.mx4_linear, (x, b, sb, None, torch.float64))]


def answer(f, args):
    try:
        r = f(*args)
    except (ValueError, B.MbuError) as e:
        return type(e), str(e)
    return r


def test_native_calls_and_general_code_agree(monkeypatch):
    cs = calls()
    native = []
    for i, (f, args) in enumerate(cs):
        say(f"mx4 native {i} {f.__name__}")
        native.append(answer(f, args))
    monkeypatch.setattr(B, "_calls", General())
    refused = 0
    for i, ((f, args), got) in enumerate(zip(cs, native)):
        say(f"mx4 general {i} {f.__name__}")
        want = answer(f, args)
        if isinstance(want, tuple) and isinstance(want[0], type):
            assert got == want
            refused += 1
            continue
        for t, u in zip((got,), (want,)) if torch.is_tensor(want) else zip(got, want):
            assert t.dtype == u.dtype and t.shape == u.shape and t.stride() == u.stride() and not t.requires_grad
            assert torch.equal(t, u)
    assert refused == 20


def test_from_several_threads():
    say("mx4 threads")
    x = torch.randn((100, 2000), device="cuda")
    b, sb = B.mx4_quantize(torch.randn((300, 2000), device="cuda"))
    want, wrong = B.mx4_linear(x, b, sb), []
    torch.cuda.synchronize()

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(30):
                y = B.mx4_linear(x, b, sb)
                torch.cuda.current_stream().synchronize()
                if not torch.equal(y, want):
                    wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong

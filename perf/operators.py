"""The microscaled 4-bit operators, as cases that can be timed and compared.

A row of K values is held as blocks of 32: each value a 4-bit float (sign, two exponent bits, one mantissa bit: 0, 0.5,
1, 1.5, 2, 3, 4, 6), each block a power-of-two scale 2^(s - 127) in one byte, with s - 127 = floor(log2(largest
magnitude)) - 2.  K is padded to a multiple of 128 with zeros.  A weight is held in the same format, or masked-binary
({-1, 0, +1} in two bits, with a float32 factor per output).

Kinds of case, each through the public entry points of `paper_2601_11660_amd.binding`:
  roundtrip      activations or weights into the format and back (quantisation, dequantisation)
  matmul         product of two tensors in the format
  masked         product of activations in the format with masked-binary weights
  linear         product of float activations, quantised within the call, with weights in the format
  linear_masked  the same with masked-binary weights
`m` rows (tokens), `n` outputs, `k` inputs.
"""
import torch

own = False

_DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}


def listed():
    return [
        # the activations of one token
        dict(name="roundtrip_1x4096", kind="roundtrip", m=1, k=4096, dtype="bfloat16", transposed=False),
        # float32 weights stored input-major, an odd size of both: read across their rows
        dict(name="roundtrip_5000x1001_t", kind="roundtrip", m=5000, k=1001, dtype="float32", transposed=True),
        # the activations of a long prompt, or a large weight
        dict(name="roundtrip_8192x8192", kind="roundtrip", m=8192, k=8192, dtype="bfloat16", transposed=False),
        # sixteen sequences decoded together, activations quantised by the layer before
        dict(name="matmul_16x4096x4096", kind="matmul", m=16, n=4096, k=4096, dtype="bfloat16"),
        # a ragged prompt on a layer whose sizes fill no tile
        dict(name="matmul_777x1001x2050", kind="matmul", m=777, n=1001, k=2050, dtype="float32"),
        # a batch of long prompts on a wide layer
        dict(name="matmul_8192x8192x8192", kind="matmul", m=8192, n=8192, k=8192, dtype="bfloat16"),
        # one token on a masked-binary layer
        dict(name="masked_1x11008x4096", kind="masked", m=1, n=11008, k=4096, dtype="float16"),
        # a prompt on a masked-binary layer
        dict(name="masked_2048x8192x8192", kind="masked", m=2048, n=8192, k=8192, dtype="bfloat16"),
        # one token on a square layer: a call whose time is the launch and its latency
        dict(name="linear_1x4096x4096", kind="linear", m=1, n=4096, k=4096, dtype="bfloat16"),
        # eight sequences decoded together on a wide layer: bound by reading the weight
        dict(name="linear_8x28672x8192", kind="linear", m=8, n=28672, k=8192, dtype="bfloat16"),
        # a chunk of a prompt
        dict(name="linear_512x14336x4096", kind="linear", m=512, n=14336, k=4096, dtype="bfloat16"),
        # a hundred sequences decoded together on a masked-binary layer with an odd number of outputs
        dict(name="linear_masked_100x4095x11008", kind="linear_masked", m=100, n=4095, k=11008, dtype="float16"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, evenly spread over its logarithm."""
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random() + 0.5)))


def draw(rng):
    kind = rng.choice(["roundtrip", "matmul", "masked", "linear", "linear", "linear_masked"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if kind == "roundtrip":
        while True:
            m, k = _log(rng, 1, 16384), _log(rng, 32, 16384)
            if m * k <= 1 << 26:
                return dict(kind=kind, m=m, k=k, dtype=dtype, transposed=rng.random() < 0.4)
    while True:
        m, n, k = _log(rng, 1, 8192), _log(rng, 64, 28672), _log(rng, 64, 16384)
        if rng.random() < 0.5:  # sizes of layers are most often whole multiples of a power of two
            n, k = max(64, n // 64 * 64), max(128, k // 128 * 128)
        if n * k <= 28672 * 8192 and m * n * k <= 1 << 39:
            return dict(kind=kind, m=m, n=n, k=k, dtype=dtype)


# ------------------------------------------------------------------------------- inputs
def _activations(g, m, k, dtype):
    """Normal values, one channel in some thirty a good deal larger, as the layers of such models have them."""
    x = torch.randn((m, k), generator=g, device="cuda")
    large = torch.rand((k,), generator=g, device="cuda") < 0.03
    return x.mul_(torch.where(large, 12.0, 1.0)).to(_DTYPES[dtype])


def _to_format(x):
    """Codes [rows, Kp / 2] (two in a byte, the lower index in the low half) and scales [rows, Kp / 32], as uint8."""
    rows, k = x.shape
    kp = -(-k // 128) * 128
    v, e = _quantised(x)
    kb = e.shape[1]
    a = v.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code += (v < 0).to(torch.uint8) * 8
    codes = torch.zeros((rows, kp), dtype=torch.uint8, device=x.device)
    codes[:, :32 * kb] = code.view(rows, 32 * kb)
    scales = torch.zeros((rows, kp // 32), dtype=torch.uint8, device=x.device)
    scales[:, :kb] = (e + 127).to(torch.uint8)
    return codes[:, 0::2] + 16 * codes[:, 1::2], scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, m, k, dtype = case["kind"], case["m"], case["k"], case["dtype"]
    s = dict(case=case)
    x = _activations(g, m, k, dtype)
    if kind == "roundtrip":
        s["x"] = x.t().contiguous().t() if case["transposed"] else x
        return s
    n = case["n"]
    if kind in ("linear", "linear_masked"):
        s["x"] = x
    else:
        s["a"], s["a_scales"] = _to_format(x)
    s["bias"] = torch.randn((n,), generator=g, device="cuda")
    if kind in ("masked", "linear_masked"):
        r = torch.rand((n, k), generator=g, device="cuda")  # 60 % kept, signs even
        s["w"] = (r < 0.3).to(torch.int8) - (r > 0.7).to(torch.int8)
        s["alpha"] = torch.rand((n,), generator=g, device="cuda") * 0.04 + 0.01
        if own:  # a program lays its weights out once
            from paper_2601_11660_amd import binding as B
            s["packed"] = B.mx4_pack_masked_binary(s["w"])
    else:
        s["b"], s["b_scales"] = _to_format(torch.randn((n, k), generator=g, device="cuda").mul_(0.02))
    return s


# ------------------------------------------------------------------------------- plain form
def _quantised(x):
    """Values of the 4-bit format in units of their block's scale [rows, blocks, 32], and the scales' exponents
    [rows, blocks, 1]; the last block is filled up with zeros."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -k % 32)).view(rows, -1, 32)
    e = torch.frexp(x.abs().amax(2, keepdim=True))[1] - 3
    a = torch.ldexp(x.abs(), -e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.where(x < 0, -q, q), e[:, :, 0]


def _dequantised(x):
    """The float32 values that the quantised rows stand for."""
    v, e = _quantised(x)
    return torch.ldexp(v, e[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]]


def _from_format(codes, scales):
    """float32 [rows, Kp]"""
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = value[torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1).int()]
    return torch.ldexp(v.view(codes.shape[0], -1, 32), scales.int()[:, :, None] - 127).view(codes.shape[0], -1)


def _plain(s):
    case = s["case"]
    kind, k, dtype = case["kind"], case["k"], _DTYPES[case["dtype"]]
    if kind == "roundtrip":
        return _dequantised(s["x"]).to(dtype)
    a = _dequantised(s["x"]) if kind in ("linear", "linear_masked") else _from_format(s["a"], s["a_scales"])[:, :k]
    if kind in ("masked", "linear_masked"):
        y = (a @ s["w"].float().t()) * s["alpha"]
    else:
        y = a @ _from_format(s["b"], s["b_scales"])[:, :k].t()
    return (y + s["bias"]).to(dtype)


# ------------------------------------------------------------------------------- the framework's operators
def _own(s):
    from paper_2601_11660_amd import binding as B
    case = s["case"]
    kind, dtype = case["kind"], _DTYPES[case["dtype"]]
    if kind == "roundtrip":
        codes, scales = B.mx4_quantize(s["x"])
        return B.mx4_dequantize(codes, scales, case["k"], dtype)
    if kind == "matmul":
        return B.mx4_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], s["bias"], dtype)
    if kind == "masked":
        return B.mx4_matmul_masked_binary(s["a"], s["a_scales"], s["packed"], case["n"], s["alpha"], s["bias"], dtype)
    if kind == "linear":
        return B.mx4_linear(s["x"], s["b"], s["b_scales"], s["bias"])
    return B.mx4_linear_masked_binary(s["x"], s["packed"], case["n"], s["alpha"], s["bias"])


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------- work and exact results
def work(case):
    m, k, size = case["m"], case["k"], torch.finfo(_DTYPES[case["dtype"]]).bits // 8
    held = k / 2 + -(-k // 32)  # bytes of a row in the format
    if case["kind"] == "roundtrip":  # values read and written, the format written and read
        return {"bytes": 2 * m * (k * size + held), "flops": 0}
    n = case["n"]
    weight = n * k / 4 + 4 * n if case["kind"] in ("masked", "linear_masked") else n * held
    rows = m * k * size if case["kind"] in ("linear", "linear_masked") else m * held
    return {"bytes": rows + weight + 4 * n + m * n * size, "flops": 2 * m * n * k}


def _exact_rows(x):
    """Quantised rows in float64: for every value the nearest of the sixteen, of two equally near the one with an even
    code, by the number of borders between neighbours that its magnitude has passed."""
    rows, k = x.shape
    x = torch.cat((x.double(), x.new_zeros((rows, -k % 32)).double()), 1)
    top = x.abs().view(rows, -1, 32).amax(2).repeat_interleave(32, 1)
    exponent = (top.view(torch.int64) >> 52) - 1023 - 2
    scale = ((exponent + 1023) << 52).view(torch.float64)
    a = (x.abs() / scale).nan_to_num()  # a block of zeros
    q = torch.zeros_like(a)
    for low, high, passed_at_tie in ((0, 0.5, False), (0.5, 1, True), (1, 1.5, False), (1.5, 2, True), (2, 3, False),
                                     (3, 4, True), (4, 6, False)):
        middle = (low + high) / 2
        q += (high - low) * ((a >= middle) if passed_at_tie else (a > middle))
    return (torch.sign(x) * q * scale).nan_to_num()[:, :k]


def _exact_held(codes, scales, k):
    """Held rows in float64, from the fields of each code."""
    code = torch.stack((codes % 16, codes // 16), 2).view(codes.shape[0], -1)[:, :k].long()
    exponent, mantissa = code // 2 % 4, code % 2
    v = torch.where(exponent == 0, mantissa * 0.5, (1 + mantissa * 0.5) * torch.pow(2.0, exponent.double() - 1))
    scale = torch.pow(2.0, scales.double() - 127).repeat_interleave(32, 1)[:, :k]
    return torch.where(code >= 8, -v, v) * scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "roundtrip":
        return _exact_rows(s["x"])
    a = _exact_rows(s["x"]) if "x" in s else _exact_held(s["a"], s["a_scales"], case["k"])
    w = s["w"].double() * s["alpha"].double()[:, None] if "w" in s else _exact_held(s["b"], s["b_scales"], case["k"])
    return torch.addmm(s["bias"].double(), a, w.t())

"""Microscaled storage and products: what training and inference with block-scaled 8- and 4-bit operands have the framework do.

A matrix is held in groups of 32 consecutive elements of a row that share one power of two; an element is an 8-bit (e4m3) or a
4-bit (e2m1) floating-point number.  The scale of a group is the smallest power of two (not below 2^-127) that brings its largest
magnitude to at most 448 or 6, the largest numbers of the two formats; elements are rounded to nearest, ties to even.

Four operators on such matrices:

  store       x -> codes -> x^                   a checkpoint of activations, written and read back whole
  product     y = q(x) W^^T + b                  a layer's transform on 4-bit operands: rows of x are rounded on the way in
  weights     gW = X^^T D, gb = 1^T D            gradient of a layer's weights from the checkpoint of its input
  inputs      gx = D W^                          gradient of its input from the stored weights

Codes of a row: a byte per element (8 bits) or two elements a byte, the even one in the low half (4 bits), the last group filled up
with zeros, row stride a multiple of 16 bytes.  Scales: a byte per group, the exponent plus 127, row stride a multiple of 4 bytes.
"""
import math

import torch

own = False

GROUP = 32
FORMATS = {8: dict(largest=448.0, top=8, carry=0x1FFFFF), 4: dict(largest=6.0, top=2, carry=0x3FFFFF)}


def listed():
    return [
        # checkpoint of a unit-test sized layer: launches and host time count
        dict(op="store", name="store-tiny", bits=8, rows=2048, d=32),
        # checkpoint of a wide layer, width no multiple of a group, in 4 bits (dense social graph)
        dict(op="store", name="store-wide-4bit", bits=4, rows=58241, d=602),
        # checkpoint of a hidden layer of the large co-purchase graph
        dict(op="store", name="store-large", bits=8, rows=612257, d=256),
        # one node's answer: a single row against a hidden layer's weights
        dict(op="product", name="product-row", bits=4, rows=1, d=512, n=512),
        # small graph, widths that are no multiple of anything
        dict(op="product", name="product-odd", bits=4, rows=6000, d=50, n=72),
        # transform of a hidden layer of the citation graph
        dict(op="product", name="product-citation", bits=4, rows=169343, d=256, n=256),
        # weight gradient of a unit-test sized layer
        dict(op="weights", name="weights-tiny", bits=8, rows=2048, d=32, n=16),
        # of the first layer of the dense social graph, features kept in 4 bits
        dict(op="weights", name="weights-wide-4bit", bits=4, rows=58241, d=602, n=256),
        # of a hidden layer of the co-purchase graph
        dict(op="weights", name="weights-large", bits=8, rows=612257, d=256, n=256),
        # input gradient of a mini-batch, odd widths
        dict(op="inputs", name="inputs-odd", bits=4, rows=301, d=100, n=47),
        # of an output layer of the citation graph, weights kept in 8 bits
        dict(op="inputs", name="inputs-last-8bit", bits=8, rows=169343, d=256, n=40),
        # of a hidden layer of the deep multi-label network
        dict(op="inputs", name="inputs-deep", bits=4, rows=179250, d=512, n=512),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one row to the nodes of a large graph, classes to the widest features."""
    limit = {op: [work(c) for c in listed() if c["op"] == op] for op in ("store", "product", "weights", "inputs")}
    while True:
        op = rng.choice(["store", "product", "product", "weights", "weights", "inputs"])
        case = dict(op=op, bits=4 if op == "product" else rng.choice([8, 4]), rows=_log(rng, 1, 610000),
                    d=rng.choice([_log(rng, 1, 1024), rng.randint(16, 640), 32 * rng.randint(1, 16)]))
        if op != "store":
            case["n"] = rng.choice([_log(rng, 3, 1024), rng.randint(16, 640), 32 * rng.randint(1, 16)])
        w = work(case)
        if all(w[k] <= max(x[k] for x in limit[op]) for k in w):
            return case


# ---- the two formats, in elementary operations ------------------------------------------------------------------------------
def _power(byte):
    """2^(byte - 127) in 32 bits; byte 0 is a subnormal number."""
    b = byte.to(torch.int32)
    return torch.where(b > 0, b << 23, torch.full_like(b, 1 << 22)).view(torch.float32)


def _grouped(x):
    pad = -x.shape[1] % GROUP
    return (torch.nn.functional.pad(x, (0, pad)) if pad else x).reshape(x.shape[0], -1, GROUP)


def _rounded(x, bits):
    """(elements as their format's numbers, scale bytes), by groups."""
    f = FORMATS[bits]
    g = _grouped(x)
    amax = g.abs().amax(2)
    byte = (((amax.contiguous().view(torch.int32) + f["carry"]) >> 23) - f["top"]).clamp(min=0)
    v = g * _power(254 - byte)[:, :, None]
    if bits == 8:
        v = v.to(torch.float8_e4m3fn).to(torch.float32)
    else:
        m = v.abs()
        step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
        v = torch.copysign(torch.round(m / step) * step, v)
    return v, byte


def _stored(x, bits):
    """What a matrix's codes stand for."""
    v, byte = _rounded(x, bits)
    return (v * _power(byte)[:, :, None]).reshape(x.shape[0], -1)[:, :x.shape[1]].contiguous()


def _encode(x, bits):
    """Codes and scales as they lie in memory."""
    v, byte = _rounded(x, bits)
    rows, groups = byte.shape
    if bits == 8:
        code = v.reshape(rows, -1).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        m = v.abs()
        c = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
        c = c.reshape(rows, -1, 2)
        code = c[:, :, 0] | (c[:, :, 1] << 4)
    codes = torch.zeros((rows, (code.shape[1] + 15) & ~15), dtype=torch.uint8, device=x.device)
    codes[:, :code.shape[1]] = code
    scales = torch.zeros((rows, (groups + 3) & ~3), dtype=torch.uint8, device=x.device)
    scales[:, :groups] = byte.to(torch.uint8)
    return codes, scales


def _decode(codes, scales, d, bits):
    if bits == 8:
        v = codes.view(torch.float8_e4m3fn).to(torch.float32)
    else:
        c = torch.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1)
        k = (c & 7).to(torch.float32)
        v = torch.where(k < 4, k / 2, torch.where(k < 6, k - 2, 2 * k - 8))
        v = torch.where(c >= 8, -v, v)
    return v[:, :d] * _power(scales).repeat_interleave(GROUP, 1)[:, :d]


# ---- inputs -----------------------------------------------------------------------------------------------------------------
def _padded(rows, d):
    return torch.zeros((rows, (d + 3) & ~3), device="cuda")[:, :d]


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _activations(rows, d, gen):
    """What a ReLU layer and a mean over neighbours leave: about half of the elements zero, some rows much larger than others."""
    x = _padded(rows, d)
    x.normal_(generator=gen).relu_()
    return x.mul_(torch.exp(torch.randn((rows, 1), device="cuda", generator=gen)))


def _gradients(rows, d, gen):
    """Gradients of a mean loss over the rows: small, of very different size from row to row."""
    g = _padded(rows, d)
    g.normal_(generator=gen)
    return g.mul_(torch.exp(2 * torch.randn((rows, 1), device="cuda", generator=gen)) / rows)


def _glorot(a, b, gen):
    return (torch.rand((a, b), device="cuda", generator=gen) * 2 - 1) * math.sqrt(6.0 / (a + b))


def prepare(case, seed):
    gen, rows, d, bits = _gen(seed), case["rows"], case["d"], case["bits"]
    s = dict(case=case)
    if case["op"] == "store":
        s["x"], s["out"] = _activations(rows, d, gen), _padded(rows, d)
        return s
    n = case["n"]
    if case["op"] == "product":
        s["x"], s["bias"], s["out"] = _activations(rows, d, gen), 0.1 * torch.randn(n, device="cuda", generator=gen), _padded(rows, n)
        s["codes"], s["scales"] = _encode(_glorot(n, d, gen), bits)             # weights, a row per output
    elif case["op"] == "weights":
        s["codes"], s["scales"] = _encode(_activations(rows, d, gen), bits)     # the checkpoint of the forward pass
        s["g"] = _gradients(rows, n, gen)
        s["gW"], s["gb"] = torch.zeros((d, n), device="cuda"), torch.zeros(n, device="cuda")
    else:
        s["g"], s["out"] = _gradients(rows, n, gen), _padded(rows, d)
        s["codes"], s["scales"] = _encode(_glorot(n, d, gen), bits)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------
_handle = None


def _library():
    """The binding and a context on the current stream, kept as a program keeps them."""
    global _handle
    import paper_2308_13466_b200.binding as B
    if _handle is None:
        _handle = B.sat_create(0, torch.cuda.current_stream().cuda_stream)
    return B, _handle


def _run_own(s):
    B, ctx = _library()
    case = s["case"]
    if "q" not in s:            # the description of the stored matrix, made once
        fmt = B.SAT_MX8 if case["bits"] == 8 else B.SAT_MX4
        s["q"] = B.new_mx(case["rows"], case["d"], fmt) if case["op"] == "store" else B.make_mx(s["codes"], s["scales"], case["d"], fmt)
    if case["op"] == "store":
        B.sat_mx_quantise(ctx, s["x"], s["q"])
        B.sat_mx_dequantise(ctx, s["q"], s["out"])
    elif case["op"] == "product":
        B.sat_mx_dense_nt(ctx, s["x"], s["q"], s["bias"], s["out"])
    elif case["op"] == "weights":
        B.sat_mx_dense_tn(ctx, s["q"], s["g"], s["gW"], s["gb"])
        return dict(gW=s["gW"], gb=s["gb"])
    else:
        B.sat_mx_dense_nn(ctx, s["g"], s["q"], s["out"])
    return s["out"]


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    d, bits = case["d"], case["bits"]
    if case["op"] == "store":
        return _stored(s["x"], bits)
    w = _decode(s["codes"], s["scales"], d, bits)
    if case["op"] == "product":
        return _stored(s["x"], bits) @ w.t() + s["bias"]
    if case["op"] == "weights":
        return dict(gW=w.t() @ s["g"], gb=s["g"].sum(0))
    return s["g"] @ w


def work(case):
    """Inputs once and outputs once; the checkpoint written and read where it is stored and read back."""
    rows, d, bits = case["rows"], case["d"], case["bits"]
    held = lambda r, c: r * (c * bits / 8 + (c + GROUP - 1) // GROUP)  # noqa: E731  codes and scales
    if case["op"] == "store":
        return {"bytes": int(8 * rows * d + 2 * held(rows, d)), "flops": 3 * rows * d}
    n = case["n"]
    if case["op"] == "product":
        return {"bytes": int(4 * rows * (d + n) + held(n, d) + 4 * n), "flops": 2 * rows * d * n}
    if case["op"] == "weights":
        return {"bytes": int(held(rows, d) + 4 * rows * n + 4 * (d + 1) * n), "flops": 2 * rows * d * n + rows * n}
    return {"bytes": int(4 * rows * (d + n) + held(n, d)), "flops": 2 * rows * d * n}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------
def _numbers(bits):
    """The magnitudes of a format in ascending order, by its definition: (1 + m / 2^M) 2^(e - bias), without the leading one where e = 0."""
    mant, bias, count = (3, 7, 127) if bits == 8 else (1, 1, 8)
    got = []
    for c in range(count):
        e, m = c >> mant, c & ((1 << mant) - 1)
        got.append(m / (1 << mant) * 2.0 ** (1 - bias) if e == 0 else (1 + m / (1 << mant)) * 2.0 ** (e - bias))
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _exact_stored(x, bits):
    x = x.double()
    g = _grouped(x)
    m, e = torch.frexp(g.abs().amax(2))
    lead, width = (0.875, 9) if bits == 8 else (0.75, 3)                        # 448 = 0.875 2^9, 6 = 0.75 2^3
    e = torch.where(m == 0, -127, (e - width + (m > lead)).clamp(min=-127)).double()[:, :, None]
    v = g * torch.exp2(-e)
    table = _numbers(bits)
    a = v.abs()
    hi = torch.searchsorted(table, a).clamp(max=table.numel() - 1)              # the first number not below it
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - a, a - table[lo]
    k = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (torch.sign(v) * table[k] * torch.exp2(e)).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _exact_decode(codes, scales, d, bits):
    table = _numbers(bits)
    table = torch.cat([table, table.new_full((1,), math.nan)]) if bits == 8 else table
    c = codes.long() if bits == 8 else torch.stack([codes.long() % 16, codes.long() // 16], 2).flatten(1)
    half = 128 if bits == 8 else 8
    v = table[c % half] * (1 - 2 * (c // half)).double()
    return v[:, :d] * torch.exp2(scales.double() - 127)[:, torch.arange(d, device="cuda") // GROUP]


def exact(case, seed):
    s = prepare(case, seed)
    d, bits = case["d"], case["bits"]
    if case["op"] == "store":
        return _exact_stored(s["x"], bits)
    w = _exact_decode(s["codes"], s["scales"], d, bits)
    if case["op"] == "product":
        return torch.addmm(s["bias"].double(), _exact_stored(s["x"], bits), w.t())
    g = s["g"].double()
    if case["op"] == "weights":
        return dict(gW=w.t() @ g, gb=g.sum(0))
    return g @ w

"""What is measured of the operators around the signSGD step: gradient norm and clipping over many tensors, microscaled
4-bit quantisation, and products of 4-bit operands.

`run` computes each operator in its plain form (elementary torch operations in 32 bits) or, with `own` set, by this
package's calls; `exact` computes it in 64 bits.  Formats of the 4-bit operands:

  codes   uint8 [rows][row_bytes]: two values a byte, the even column in the low nibble; a nibble is sign, two exponent
          bits, one fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6); a row is padded with zero codes to a multiple of 32 columns
  scales  uint8, one byte for each block of a row: "mx" 32 values and a power of two (exponent + 127), "nv" 16 values and
          an E4M3 number; stored in tiles of 128 rows x 4 blocks, 512 bytes, (row % 32) * 16 + (row / 32) * 4 + block % 4
  tensor scale  "nv" only: a power of two that multiplies every value
"""
import math

import torch

own = False

MX, NV = "mx", "nv"
BLOCK = {MX: 32, NV: 16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # a small perceptron's gradient, one worker: a call of a few microseconds
        {"name": "clip toy", "op": "clip", "layout": "toy", "workers": 1, "type": "f32", "max_norm": 1.0},
        # the Resnet-50 layout of the workloads with its seven workers, fp32 gradients to fp32 rows
        {"name": "clip resnet50 x7", "op": "clip", "layout": "resnet50", "workers": 7, "type": "f32", "max_norm": 5.0},
        # mixed-precision training: bf16 gradients lying end to end in one buffer, odd sizes, so most start off alignment
        {"name": "clip bf16 ragged x3", "op": "clip", "layout": "ragged", "tensors": 97, "top": 400_000, "workers": 3, "type": "bf16", "max_norm": 1.0},
        # the BERT-large-sized vector as its 391 tensors, one worker, bf16 gradients
        {"name": "clip bert-large bf16", "op": "clip", "layout": "bertlarge", "workers": 1, "type": "bf16", "max_norm": 1.0},
        # eight tokens' activations: latency
        {"name": "quantise 8x1024 nv", "op": "quantise", "rows": 8, "cols": 1024, "fmt": NV, "type": "bf16", "out": "bf16", "both": False},
        # a gradient of odd sides in fp32, both directions for the backward products
        {"name": "quantise 1999x4103 mx both", "op": "quantise", "rows": 1999, "cols": 4103, "fmt": MX, "type": "f32", "out": "f32", "both": True},
        # a large layer's activations, both directions
        {"name": "quantise 8192x8192 nv both", "op": "quantise", "rows": 8192, "cols": 8192, "fmt": NV, "type": "bf16", "out": "bf16", "both": True},
        # one token through a BERT-large-sized feed-forward layer with 4-bit weights
        {"name": "token 1x4096x1024 mx", "op": "tokens", "m": 1, "n": 4096, "k": 1024, "fmt": MX, "out": "bf16"},
        # a handful of tokens through a layer of odd width
        {"name": "tokens 17x5003x2600 nv", "op": "tokens", "m": 17, "n": 5003, "k": 2600, "fmt": NV, "out": "f32"},
        # training a BERT-large-sized feed-forward layer: forward and both backward products, fp32 master weights
        {"name": "train 2048x4096x1024 mx", "op": "train", "m": 2048, "n": 4096, "k": 1024, "fmt": MX},
        # the same for sides that no tile divides
        {"name": "train 777x1111x1500 nv", "op": "train", "m": 777, "n": 1111, "k": 1500, "fmt": NV},
        # the product alone at a size where the tensor cores are the bound
        {"name": "product 8192x8192x8192 nv", "op": "product", "m": 8192, "n": 8192, "k": 8192, "fmt": NV, "out": "bf16"},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5 and n > 64:
            n = n // 32 * 32          # as often as not a size that the blocks divide
        return n + 1 if n == 3072 else n

    fmt = rng.choice([MX, NV])
    op = rng.choice(["clip", "quantise", "tokens", "train", "product"])
    if op == "clip":
        c = {"op": op, "layout": "ragged", "tensors": size(1, 500), "top": size(16, 1_000_000), "workers": size(1, 16),
             "type": rng.choice(["f32", "bf16", "f16"]), "max_norm": rng.choice([0.1, 1.0, 5.0])}
        while c["tensors"] * c["top"] * c["workers"] > 100_000_000:
            c["top"] = c["top"] // 2
        return c
    if op == "quantise":
        return {"op": op, "rows": size(1, 8192), "cols": size(16, 8192), "fmt": fmt, "type": rng.choice(["f32", "bf16", "f16"]),
                "out": rng.choice(["f32", "bf16"]), "both": rng.random() < 0.5}
    if op == "tokens":
        return {"op": op, "m": size(1, 64), "n": size(64, 16384), "k": size(64, 8192), "fmt": fmt, "out": rng.choice(["f32", "bf16", "f16"])}
    if op == "train":
        return {"op": op, "m": size(64, 4096), "n": size(64, 6000), "k": size(64, 6000), "fmt": fmt}
    return {"op": op, "m": size(100, 8192), "n": size(100, 8192), "k": size(64, 8192), "fmt": fmt, "out": rng.choice(["f32", "bf16", "f16"])}


# --------------------------------------------------------------------------------------------------------------------
# sizes


def _up(n, k):
    return (n + k - 1) // k * k


def _tensor_sizes(case):
    """Element counts of one worker's gradient tensors."""
    if case["layout"] == "toy":
        return [32 * 64, 64, 64 * 64, 64, 64 * 10, 10]
    if case["layout"] == "resnet50":
        sizes, cin = [3 * 64 * 49, 64, 64], 64
        for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                sizes += [cin * width, width, width, width * width * 9, width, width, width * 4 * width, 4 * width, 4 * width]
                sizes += [cin * 4 * width, 4 * width, 4 * width] if b == 0 else []
                cin = 4 * width
        return sizes + [2048 * 1000, 1000]
    if case["layout"] == "bertlarge":
        h, f = 1024, 4096
        block = [h * h, h] * 4 + [h, h] + [h * f, f, f * h, h] + [h, h]
        return [30522 * h, 512 * h, 2 * h, h, h] + block * 24 + [h * h, h]
    top = case["top"]                 # sizes from 1 to top, spread over their logarithm, the same for every seed
    return [max(1, int(top ** ((37 * i % 101) / 100.0))) | (i % 2) for i in range(case["tensors"])]


def _elements(case):
    return sum(_tensor_sizes(case))


def _scale_bytes(rows, cols, fmt):
    return _up(rows, 128) // 128 * _up(-(-cols // BLOCK[fmt]), 4) // 4 * 512


def _packed_bytes(rows, cols, fmt):
    return rows * cols / 2 + rows * (cols / BLOCK[fmt])


def work(case):
    op = case["op"]
    if op == "clip":
        n = _elements(case) * case["workers"]
        return {"bytes": n * (BYTES[case["type"]] + 4), "flops": 3 * n}
    if op == "quantise":
        n, ways = case["rows"] * case["cols"], 2 if case["both"] else 1
        return {"bytes": n * (BYTES[case["type"]] + ways * BYTES[case["out"]]), "flops": 3 * ways * n}
    m, n, k, fmt = case["m"], case["n"], case["k"], case["fmt"]
    if op == "tokens":                # bf16 activations in, 4-bit weights in
        return {"bytes": 2 * m * k + _packed_bytes(n, k, fmt) + BYTES[case["out"]] * m * n, "flops": 2 * m * n * k}
    if op == "train":                 # x, dy bf16 and w fp32 in; y, dx bf16 and dw fp32 out
        return {"bytes": 2 * (m * k + m * n) + 4 * n * k + 2 * (m * n + m * k) + 4 * n * k, "flops": 6 * m * n * k}
    return {"bytes": _packed_bytes(m, k, fmt) + _packed_bytes(n, k, fmt) + BYTES[case["out"]] * m * n, "flops": 2 * m * n * k}


# --------------------------------------------------------------------------------------------------------------------
# inputs


def _gen(seed, key):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + key) & (2**62 - 1))
    return g


def _activations(rows, cols, gen, scale=1.0):
    """Normal values whose channels differ in size, a few of them by much."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    c = torch.exp(0.5 * torch.randn(cols, generator=gen, device="cuda"))
    return x.mul_(c).mul_(scale)


def _gradients(rows, cols, gen):
    """Heavy-tailed values of the size of a layer's output gradient."""
    z = torch.randn(rows, cols, generator=gen, device="cuda")
    return z.mul_(torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))).mul_(1e-3)


def _stored(v, fmt):
    """A 4-bit operand as it is stored: codes, scales, tensor scale."""
    values, scales, tensor_scale = _plain_quantise(v, fmt)
    rows, cols = v.shape
    b, nb = BLOCK[fmt], scales.shape[1]
    s = scales.repeat_interleave(b, 1)[:, :cols] * tensor_scale
    mag = torch.searchsorted(torch.tensor(LEVELS, device="cuda"), (values.abs() / s).contiguous())
    code = torch.zeros(rows, _up(cols, 32), dtype=torch.uint8, device="cuda")
    code[:, :cols] = (mag + 8 * (values < 0)).to(torch.uint8)
    byte = scales.log2().add_(127).round_().to(torch.uint8) if fmt == MX else scales.to(torch.float8_e4m3fn).view(torch.uint8)
    tiles = torch.zeros(_up(rows, 128), _up(nb, 4), dtype=torch.uint8, device="cuda")
    tiles[:rows, :nb] = byte
    tiles = tiles.view(-1, 4, 32, tiles.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    return {"codes": code[:, 0::2] + 16 * code[:, 1::2], "scales": tiles, "tensor_scale": tensor_scale.reshape(1), "rows": rows, "cols": cols}


def prepare(case, seed):
    op = case["op"]
    s = {"case": case}
    if op == "clip":
        sizes, G, gen = _tensor_sizes(case), case["workers"], _gen(seed, 1)
        count = torch.tensor(sizes, device="cuda")
        sigma = torch.exp(torch.rand(len(sizes), generator=gen, device="cuda") * math.log(1000.0)) * 1e-4
        sigma = sigma.repeat_interleave(count)
        s["g"] = []                   # [worker][tensor], lying end to end or each at a multiple of 32 elements
        starts, o = [], 0
        for n in sizes:
            starts.append(o)
            o += n if case["layout"] == "ragged" else _up(n, 32)
        for _ in range(G):
            flat = torch.randn(sum(sizes), generator=gen, device="cuda").mul_(sigma).to(TYPES[case["type"]])
            buffer = torch.zeros(o, dtype=flat.dtype, device="cuda")
            tensors = [buffer[a:a + n] for a, n in zip(starts, sizes)]
            if case["layout"] == "ragged":
                buffer.copy_(flat)
            else:
                torch._foreach_copy_(tensors, list(flat.split(sizes)))
            s["g"].append(tensors)
        s["pad"] = [torch.zeros(_up(n, 32) - n, device="cuda") for n in sizes]
        ld = sum(_up(n, 32) for n in sizes)
        s["rows"] = torch.zeros(G, ld, device="cuda")
        s["norms"] = torch.zeros(G, device="cuda")
        if own:                       # the table of the tensors, built once for the buffers that the program keeps
            from paper_1802_04434_b200 import binding as B
            dst = [r for row in s["rows"] for r in _row_slices(row, sizes)]
            s["table"] = B.TensorTable([t for w in s["g"] for t in w], dst, [w for w in range(G) for _ in sizes])
    elif op == "quantise":
        s["x"] = _activations(case["rows"], case["cols"], _gen(seed, 2)).to(TYPES[case["type"]])
    elif op == "tokens":
        s["x"] = _activations(case["m"], case["k"], _gen(seed, 3)).to(torch.bfloat16)
        s["w"] = _stored(torch.randn(case["n"], case["k"], generator=_gen(seed, 4), device="cuda").mul_(0.02), case["fmt"])
    elif op == "train":
        s["x"] = _activations(case["m"], case["k"], _gen(seed, 5)).to(torch.bfloat16)
        s["w"] = torch.randn(case["n"], case["k"], generator=_gen(seed, 6), device="cuda").mul_(0.02)
        s["dy"] = _gradients(case["m"], case["n"], _gen(seed, 7)).to(torch.bfloat16)
    else:
        s["a"] = _stored(_activations(case["m"], case["k"], _gen(seed, 8)), case["fmt"])
        s["b"] = _stored(torch.randn(case["n"], case["k"], generator=_gen(seed, 9), device="cuda").mul_(0.02), case["fmt"])
    return s


def _row_slices(row, sizes):
    return [p[:n] for p, n in zip(row.split([_up(n, 32) for n in sizes]), sizes)]


# --------------------------------------------------------------------------------------------------------------------
# the operators


def run(state):
    return (_own if own else _plain)(state, state["case"])


def _own(s, case):
    from paper_1802_04434_b200 import binding as B, fp4
    op = case["op"]
    if op == "clip":
        B.tensors_clip(s["table"], case["max_norm"], s["norms"])
        return {"rows": s["rows"], "norms": s["norms"]}
    fmt = case["fmt"]
    if op == "quantise":
        if case["both"]:
            p, pt = fp4.quantise_both(s["x"], fmt)
            return {"rows": fp4.dequantise(p, TYPES[case["out"]]), "columns": fp4.dequantise(pt, TYPES[case["out"]])}
        return {"rows": fp4.dequantise(fp4.quantise(s["x"], fmt), TYPES[case["out"]])}
    if op == "tokens":
        return fp4.matmul(fp4.quantise(s["x"], fmt), _packed(fp4, s["w"], fmt), TYPES[case["out"]])
    if op == "train":
        y, kept = fp4.linear_forward(s["x"], s["w"], fmt)
        dx, dw = fp4.linear_backward(kept, s["dy"])
        return {"y": y, "dx": dx, "dw": dw}
    return fp4.matmul(_packed(fp4, s["a"], fmt), _packed(fp4, s["b"], fmt), TYPES[case["out"]])


def _packed(fp4, p, fmt):
    return fp4.Packed(p["codes"], p["scales"], p["tensor_scale"] if fmt == NV else None, p["rows"], p["cols"], fmt)


def _plain(s, case):
    op = case["op"]
    if op == "clip":
        rows = torch.stack([torch.cat([p for t, z in zip(w, s["pad"]) for p in (t.float(), z)]) for w in s["g"]])
        norms = rows.square().sum(1).sqrt()
        coef = torch.where(norms > case["max_norm"], case["max_norm"] / norms, torch.ones_like(norms))
        return {"rows": rows * coef[:, None], "norms": norms}
    fmt = case["fmt"]
    if op == "quantise":
        x = s["x"].float()
        out = {"rows": _plain_quantise(x, fmt)[0].to(TYPES[case["out"]])}
        if case["both"]:
            out["columns"] = _plain_quantise(x.t(), fmt)[0].to(TYPES[case["out"]])
        return out
    if op == "tokens":
        return torch.matmul(_plain_quantise(s["x"].float(), fmt)[0], _plain_values(s["w"], fmt).t()).to(TYPES[case["out"]])
    if op == "train":
        x, w, dy = s["x"].float(), s["w"], s["dy"].float()
        q = lambda v: _plain_quantise(v, fmt)[0]  # noqa: E731
        return {"y": torch.matmul(q(x), q(w).t()).to(torch.bfloat16), "dx": torch.matmul(q(dy), q(w.t()).t()).to(torch.bfloat16),
                "dw": torch.matmul(q(dy.t()), q(x.t()).t())}
    return torch.matmul(_plain_values(s["a"], fmt), _plain_values(s["b"], fmt).t()).to(TYPES[case["out"]])


def _power_of_two(e):
    """2^e in fp32 for int32 e >= -127, by its bits."""
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _plain_quantise(v, fmt):
    """Values, block scales and tensor scale of the rows of v (fp32), blocks along the columns."""
    rows, cols = v.shape
    b = BLOCK[fmt]
    x = torch.nn.functional.pad(v, (0, _up(cols, b) - cols)).view(rows, -1, b)
    top = x.abs().amax(2)
    if fmt == MX:
        e = (torch.frexp(top)[1] - 3).clamp(-127, 127)
        scale, tensor_scale = _power_of_two(torch.where(top > 0, e, torch.full_like(e, -127))), torch.ones((), device="cuda")
    else:
        m, e = torch.frexp(top.amax())
        t = torch.where(m <= 0.65625, e - 12, e - 11).clamp(-100, 120)   # 0.65625 * 2^12 = 2688 = 6 * 448
        tensor_scale = _power_of_two(torch.where(m > 0, t, torch.zeros_like(t)))
        scale = (top / tensor_scale / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn).float().clamp(min=2.0 ** -9)
    q = x / (scale * tensor_scale)[:, :, None]
    y = q.abs()
    y = torch.where(y < 2, (y * 2).round() / 2, torch.where(y < 4, y.round(), (y / 2).round() * 2)).clamp(max=6.0)
    values = torch.copysign(y, q) * (scale * tensor_scale)[:, :, None]
    return values.view(rows, -1)[:, :cols], scale, tensor_scale


def _plain_values(p, fmt):
    """The values (fp32) that a stored operand stands for."""
    rows, cols = p["rows"], p["cols"]
    nb = -(-cols // BLOCK[fmt])
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda")
    code = torch.stack((p["codes"] & 15, p["codes"] >> 4), 2).view(rows, -1)[:, :cols]
    byte = p["scales"].view(_up(rows, 128) // 128, -1, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(_up(rows, 128), -1)[:rows, :nb]
    scale = _power_of_two(byte.to(torch.int32) - 127) if fmt == MX else byte.view(torch.float8_e4m3fn).float() * p["tensor_scale"]
    return level[code.int()] * scale.repeat_interleave(BLOCK[fmt], 1)[:, :cols]


# --------------------------------------------------------------------------------------------------------------------
# the same in 64 bits


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "clip":
        G, sizes = case["workers"], _tensor_sizes(case)
        rows = torch.zeros(G, sum(_up(n, 32) for n in sizes), dtype=torch.float64, device="cuda")
        norms = torch.zeros(G, dtype=torch.float64, device="cuda")
        for w in range(G):
            torch._foreach_copy_(_row_slices(rows[w], sizes), s["g"][w])
            norms[w] = torch.linalg.vector_norm(rows[w])
            rows[w] *= min(1.0, case["max_norm"] / max(float(norms[w]), 1e-300))
        return {"rows": rows, "norms": norms}
    fmt = case["fmt"]
    if op == "quantise":
        x = s["x"].double()
        out = {"rows": _exact_quantise(x, fmt)}
        if case["both"]:
            out["columns"] = _exact_quantise(x.t(), fmt)
        return out
    if op == "tokens":
        return _exact_quantise(s["x"].double(), fmt) @ _exact_values(s["w"], fmt).t()
    if op == "train":
        x, w, dy = s["x"].double(), s["w"].double(), s["dy"].double()
        return {"y": _exact_quantise(x, fmt) @ _exact_quantise(w, fmt).t(), "dx": _exact_quantise(dy, fmt) @ _exact_quantise(w.t(), fmt).t(),
                "dw": _exact_quantise(dy.t(), fmt) @ _exact_quantise(x.t(), fmt).t()}
    return _exact_values(s["a"], fmt) @ _exact_values(s["b"], fmt).t()


def _exact_quantise(x, fmt):
    """The nearest 4-bit values, by the midpoints between them; a tie goes to the code whose last bit is 0."""
    rows, cols = x.shape
    b = BLOCK[fmt]
    nb = -(-cols // b)
    blocks = torch.zeros(rows, nb * b, dtype=torch.float64, device="cuda")
    blocks[:, :cols] = x
    blocks = blocks.view(rows, nb, b)
    top = blocks.abs().amax(2, keepdim=True)
    if fmt == MX:
        S = torch.exp2(torch.frexp(top.clamp(min=1e-30))[1].double() - 3)          # 2^(floor(log2 top) - 2)
    else:
        all_top = float(top.max())
        m, e = math.frexp(all_top / 2688.0)
        t = math.ldexp(1.0, e - 1 if m == 0.5 else e) if all_top > 0 else 1.0
        r = (top / t / 6.0).clamp(max=448.0)
        unit = torch.exp2(torch.frexp(r.clamp(min=2.0 ** -6))[1].double() - 4)     # spacing of E4M3 numbers at r
        S = (torch.round(r / unit) * unit).clamp(min=2.0 ** -9) * t
    y = blocks.abs() / S
    count = torch.zeros_like(y, dtype=torch.int32)
    for mid, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        count += (y >= mid) if tie_up else (y > mid)
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    return (level[count] * S * torch.sign(blocks)).view(rows, -1)[:, :cols]


def _exact_values(p, fmt):
    rows, cols = p["rows"], p["cols"]
    r = torch.arange(rows, device="cuda")[:, None]
    c = torch.arange(cols, device="cuda")[None, :]
    code = (p["codes"][r, c // 2].int() >> (4 * (c % 2))) & 15
    exp, frac = (code >> 1) & 3, (code & 1).double()
    mag = torch.where(exp == 0, frac * 0.5, torch.exp2(exp.double() - 1) * (1 + frac * 0.5))
    blk = c // BLOCK[fmt]
    tiles_k = _up(-(-cols // BLOCK[fmt]), 4) // 4
    byte = p["scales"][((r // 128) * tiles_k + blk // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + blk % 4].int()
    if fmt == MX:
        S = torch.exp2(byte.double() - 127)
    else:
        e, f = (byte >> 3) & 15, (byte & 7).double()
        S = torch.where(e == 0, f * 2.0 ** -9, torch.exp2(e.double() - 7) * (1 + f / 8)) * p["tensor_scale"].double()
    return torch.where(code >= 8, -mag, mag) * S

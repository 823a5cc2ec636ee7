"""What the operators on microscaled 4-bit weights are timed on, with their plain forms.

A microscaled stream holds matrices in 4-bit floating point (sign, two exponent bits, one mantissa bit) with one 8-bit
power of two for every 32 neighbouring values of a row (the MXFP4 form of the OCP microscaling formats). Its bytes, in
the order of ``include/enec.h``: a header of 128 bytes, then records of 128 rows x 256 columns, each 16384 bytes of
elements and 1024 bytes of scales. ``prepare`` lays weights out that way, since a serving program has them so.

  op "roundtrip"   quantise a tensor into a stream and bring it back (both operators; returns the values)
  op "dequantize"  bring a stream's values back
  op "matmul"      y = x W^T, x of 16 bits, W a stream
  op "both"        quantise x, then y = x W^T with both as streams (what a prompt's products do)
  op "moe"         a mixture-of-experts layer over expert streams: router, chosen experts, combination

Sizes are those of the Llama-3-8B-shaped layer (4096, 1024, 14336), of the MoE-shaped set (1408 x 2048), of the
OLMo-1B-shaped fp32 layer (2048 x 8192), and odd ones beside them.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_HEADER, _RECORD, _ROWS, _COLS = 128, 17408, 128, 256
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quant(name, dtype, batch, rows, cols, dist="weights"):
    return _named(name, {"op": "roundtrip", "dtype": dtype, "batch": batch, "rows": rows, "cols": cols, "dist": dist})


def _product(name, op, dtype, tokens, rows, cols, gap=0):
    return _named(name, {"op": op, "dtype": dtype, "tokens": tokens, "rows": rows, "cols": cols, "gap": gap})


def _moe(name, dtype, tokens, hidden, inter, experts, top, renormalize=True):
    return _named(name, {"op": "moe", "dtype": dtype, "tokens": tokens, "hidden": hidden, "inter": inter, "experts": experts,
                         "top": top, "renormalize": renormalize})


def _named(name, case):
    return {"name": name, **case} if name else case


def listed():
    return [
        # one token's activations, as they are quantised in front of a product: the smallest call
        _quant("token_roundtrip", "bf16", 1, 1, 4096, "activations"),
        # the largest matrix of a decoder layer, as a checkpoint is converted
        _quant("gate_roundtrip", "bf16", 1, 14336, 4096),
        # a stack of small fp16 matrices whose rows and columns fill no record
        _quant("odd_roundtrip", "fp16", 5, 1411, 2047, "heavy"),
        # an fp32 matrix brought back for a check
        {"name": "fp32_dequantize", "op": "dequantize", "dtype": "fp32", "batch": 1, "rows": 8192, "cols": 2048},
        # decoding one sequence: the square projections
        _product("one_token", "matmul", "bf16", 1, 4096, 4096),
        # decoding eight sequences: the down projection
        _product("eight_tokens", "matmul", "fp16", 8, 4096, 14336),
        # a ragged batch between decoding and prompt, odd sizes, rows of x further apart than they are long
        _product("ragged_tokens", "matmul", "fp16", 77, 1411, 2055, gap=5),
        # a prompt
        _product("prompt", "matmul", "bf16", 2048, 4096, 4096),
        # a prompt with 4-bit activations too: the gate projection, and a ragged short one
        _product("prompt_both", "both", "bf16", 2048, 14336, 4096),
        _product("ragged_both", "both", "fp16", 201, 1411, 2055, gap=1),
        # an MoE layer of the MoE-shaped set while four sequences are decoded, and a wider one with 32 sequences
        _moe("experts_few", "bf16", 4, 2048, 1408, 8, 2),
        _moe("experts_many", "bf16", 32, 2048, 1408, 64, 6),
    ]


def _between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _side(rng, low, high):
    n = _between(rng, low, high)
    return n if rng.random() < 0.4 or n < 64 else n & ~63


def draw(rng):
    op = rng.choice(["roundtrip", "dequantize", "matmul", "matmul", "matmul", "both", "both", "moe", "moe"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op in ("roundtrip", "dequantize"):
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        rows, cols = _side(rng, 1, 14336), _side(rng, 32, 14336)
        while rows * cols * _BYTES[dtype] > 14336 * 4096 * 2:
            rows = max(1, rows // 2)
        batch = rng.randint(1, max(1, min(8, 14336 * 4096 * 2 // (rows * cols * _BYTES[dtype]))))
        if op == "dequantize":
            return {"op": op, "dtype": dtype, "batch": batch, "rows": rows, "cols": cols}
        return _quant(None, dtype, batch, rows, cols, rng.choice(["weights", "activations", "heavy"]))
    if op == "moe":
        hidden, inter = 64 * _between(rng, 8, 64), 64 * _between(rng, 4, 56)
        experts = rng.choice([4, 8, 16, 60, 64, 128])
        while experts * hidden * inter > 64 * 2048 * 1408:
            inter = 64 * max(1, inter // 128)
            if inter == 64:
                experts = max(4, experts // 2)
        return _moe(None, dtype, _between(rng, 1, 32), hidden, inter, experts, rng.randint(1, min(8, experts)), rng.random() < 0.7)
    tokens = _between(rng, 1, 16) if op == "matmul" and rng.random() < 0.5 else _between(rng, 1, 2048)
    rows, cols = _side(rng, 64, 14336), _side(rng, 64, 14336)
    most = 2048 * 4096 * 4096 if op == "matmul" else 2048 * 14336 * 4096
    while tokens * rows * cols > most:
        rows = max(64, rows // 2)
        cols = max(64, cols // 2)
    return _product(None, op, dtype, tokens, rows, cols, rng.choice([0, 0, 8, 5]))


# ---- the stream, laid out with indexing alone -----------------------------------------------------------------------
def _tiles(n, size):
    return (n + size - 1) // size


def _swizzle(device):
    rows, chunks = torch.arange(_ROWS, device=device), torch.arange(8, device=device)
    return (chunks[None, :] ^ (rows[:, None] & 7))[:, :, None].expand(_ROWS, 8, 16)


def _blocks(x):
    """fp32 blocks of 32 of the last dimension, filled with zeros."""
    short = -x.shape[-1] % 32
    x = torch.nn.functional.pad(x.float(), (0, short))
    return x.reshape(*x.shape[:-1], -1, 32)


def _scale_byte(blocks):
    """The exponent of a block's largest magnitude, less that of 4, with 127 added: the scale byte."""
    top = blocks.abs().amax(-1)
    _, exponent = torch.frexp(top)                     # top = m 2^exponent, m in [0.5, 1)
    byte = (exponent - 1 - 2 + 127).clamp(0, 254)
    byte = torch.where(top == 0, torch.zeros_like(byte), byte)
    return torch.where(torch.isfinite(top), byte, torch.full_like(byte, 255))


def _codes(blocks, byte):
    """The four bits of every element: comparisons against the midpoints, ties to the even code."""
    m = torch.ldexp(blocks.double(), (127 - byte)[..., None].to(torch.int32)).abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75).to(torch.uint8) + (m > 1.25).to(torch.uint8) + (m >= 1.75).to(torch.uint8)
            + (m > 2.5).to(torch.uint8) + (m >= 3.5).to(torch.uint8) + (m > 5.0).to(torch.uint8))
    code = code | (torch.signbit(blocks).to(torch.uint8) << 3)
    return torch.where((byte == 255)[..., None], torch.zeros_like(code), code)


def _values(codes, byte):
    """What codes and scale bytes stand for, in 32 bits."""
    grid = torch.tensor(_GRID, device=codes.device)
    v = grid[(codes & 7).long()]
    v = torch.where((codes & 8) != 0, -v, v)
    v = torch.ldexp(v, byte[..., None].to(torch.int32) - 127)
    return torch.where((byte == 255)[..., None], torch.full_like(v, math.nan), v)


def _stream(x):
    """The stream of a tensor [batch, rows, cols] or [rows, cols]."""
    x = x.reshape(-1, *x.shape[-2:])
    batch, rows, cols = x.shape
    down, across = _tiles(rows, _ROWS), _tiles(cols, _COLS)
    blocks = _blocks(x)
    byte = _scale_byte(blocks)
    code = _codes(blocks, byte)
    packed = code[..., 0::2] | (code[..., 1::2] << 4)                                        # [batch, rows, chunks, 16]
    pad = (0, 8 * across - packed.shape[2], 0, _ROWS * down - rows)
    packed = torch.nn.functional.pad(packed, (0, 0) + pad).reshape(batch, down, _ROWS, across, 8, 16).transpose(2, 3)
    elements = torch.gather(packed, 4, _swizzle(x.device).expand(packed.shape)).reshape(batch, down, across, _RECORD - 1024)
    scales = torch.nn.functional.pad(byte.to(torch.uint8), pad).reshape(batch, down, 4, 32, across, 2, 4)
    scales = scales.permute(0, 1, 4, 5, 3, 2, 6).reshape(batch, down, across, 1024)
    body = torch.cat([elements, scales], -1).reshape(-1)
    total = _HEADER + body.numel()
    words = torch.zeros(_HEADER // 4, dtype=torch.int64)
    words[:8] = torch.tensor([0x344D4E45, 1, batch, rows, cols, 0, total & 0xFFFFFFFF, total >> 32])
    head = torch.stack([(words >> s) & 255 for s in (0, 8, 16, 24)], -1).to(torch.uint8).reshape(-1)
    return torch.cat([head.to(x.device), body])


def _records(stream, batch, rows, cols):
    return stream[_HEADER:].reshape(batch, _tiles(rows, _ROWS), _tiles(cols, _COLS), _RECORD)


def _unpacked(records, rows, cols):
    """The values, in 32 bits, of records [batch, row tiles, column tiles, bytes]."""
    batch, down, across = records.shape[:3]
    packed = records[..., :_RECORD - 1024].reshape(batch, down, across, _ROWS, 8, 16)
    packed = torch.gather(packed, 4, _swizzle(records.device).expand(packed.shape))
    code = torch.stack([packed & 15, packed >> 4], -1).reshape(batch, down, across, _ROWS, 8, 32)
    byte = records[..., _RECORD - 1024:].reshape(batch, down, across, 2, 32, 4, 4).permute(0, 1, 2, 5, 4, 3, 6)
    v = _values(code, byte.reshape(batch, down, across, _ROWS, 8))
    return v.transpose(2, 3).reshape(batch, down * _ROWS, across * _COLS)[:, :rows, :cols]


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _normal(shape, generator, std):
    return torch.randn(shape, generator=generator, device="cuda") * std


def _heavy(shape, generator):
    """Laplace with 1 % of the values at 50 standard deviations and some exact zeros, as in the heavy-tailed set."""
    u = torch.rand(shape, generator=generator, device="cuda") - 0.5
    x = -0.02 * torch.sign(u) * torch.log1p(-2 * u.abs().clamp(max=0.4999999))
    r = torch.rand(shape, generator=generator, device="cuda")
    x = torch.where(r < 0.01, torch.sign(u), x)
    return torch.where((r >= 0.01) & (r < 0.015), torch.zeros_like(x), x)


def _apart(x, gap):
    """The same values in rows that are `gap` values further apart than they are long."""
    wide = torch.zeros(x.shape[0], x.shape[1] + gap, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _kept(state, batch, rows, cols, name):
    state[name] = torch.zeros(_HEADER + batch * _tiles(rows, _ROWS) * _tiles(cols, _COLS) * _RECORD, dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _DTYPES[case["dtype"]]
    state = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if case["op"] in ("roundtrip", "dequantize"):
        shape = (case["batch"], case["rows"], case["cols"])
        dist = case.get("dist", "weights")
        x = _heavy(shape, g) if dist == "heavy" else _normal(shape, g, 0.02 if dist == "weights" else 1.0)
        state["out"] = torch.empty(shape, dtype=dtype, device="cuda")
        if case["op"] == "roundtrip":
            state["x"] = x.to(dtype)
            _kept(state, *shape, "stream")
        else:
            state["stream"] = _stream(x)
        return state
    if case["op"] == "moe":
        tokens, hidden, inter, experts = case["tokens"], case["hidden"], case["inter"], case["experts"]
        state["x"] = _normal((tokens, hidden), g, 1.0).to(dtype)
        state["router"] = _normal((experts, hidden), g, hidden ** -0.5).to(dtype)
        for name, rows, cols in (("gate", inter, hidden), ("up", inter, hidden), ("down", hidden, inter)):
            state[name] = _stream(_normal((experts, rows, cols), g, cols ** -0.5).to(dtype))
        state["out"] = torch.empty(tokens, hidden, dtype=dtype, device="cuda")
        return state
    tokens, rows, cols = case["tokens"], case["rows"], case["cols"]
    state["x"] = _apart(_normal((tokens, cols), g, 1.0).to(dtype), case["gap"])
    state["w"] = _stream(_normal((rows, cols), g, cols ** -0.5).to(dtype))
    state["out"] = torch.empty(tokens, rows, dtype=dtype, device="cuda")
    if case["op"] == "both":
        _kept(state, 1, tokens, cols, "stream")
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    dtype = _DTYPES[case["dtype"]]
    if case["op"] == "roundtrip":
        return _quantized(state["x"]).to(dtype)
    if case["op"] == "dequantize":
        return _unpacked(_records(state["stream"], case["batch"], case["rows"], case["cols"]), case["rows"], case["cols"]).to(dtype)
    if case["op"] == "moe":
        return _layer(state).to(dtype)
    x = _quantized(state["x"]) if case["op"] == "both" else state["x"].float()
    w = _unpacked(_records(state["w"], 1, case["rows"], case["cols"]), case["rows"], case["cols"])[0]
    return (x @ w.t()).to(dtype)


def _quantized(x):
    blocks = _blocks(x)
    byte = _scale_byte(blocks)
    v = _values(_codes(blocks, byte), byte)
    return v.reshape(*x.shape[:-1], -1)[..., :x.shape[-1]]


def _layer(state):
    case = state["case"]
    hidden, inter, experts = case["hidden"], case["inter"], case["experts"]
    x = state["x"].float()
    logits = x @ state["router"].float().t()
    p = torch.softmax(logits, -1)
    order = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :case["top"]]   # stable: ties to the lowest index
    weight = torch.gather(p, 1, order)
    if case["renormalize"]:
        weight = weight / weight.sum(-1, keepdim=True)
    share = torch.zeros_like(p).scatter_(1, order, weight)
    used = torch.unique(order)                                                               # experts that no token chose are not read
    gate = _unpacked(_records(state["gate"], experts, inter, hidden)[used], inter, hidden)
    up = _unpacked(_records(state["up"], experts, inter, hidden)[used], inter, hidden)
    down = _unpacked(_records(state["down"], experts, hidden, inter)[used], hidden, inter)
    a = x @ gate.transpose(1, 2)
    h = a / (1 + torch.exp(-a)) * (x @ up.transpose(1, 2))
    y = h @ down.transpose(1, 2)                                                             # [used, tokens, hidden]
    return (y * share[:, used].t()[:, :, None]).sum(0)


def _run_own(state):
    import paper_2604_03298_b200 as enec
    case, status, out = state["case"], state["status"], state["out"]
    dt = {"bf16": enec.BF16, "fp16": enec.FP16, "fp32": enec.FP32}[case["dtype"]]
    if case["op"] in ("roundtrip", "dequantize"):
        shape, stream = (case["batch"], case["rows"], case["cols"]), state["stream"]
        if case["op"] == "roundtrip":
            enec.enec_quantize_microscaled(state["x"], dt, *shape, case["cols"], stream, stream.numel(), status)
        enec.enec_dequantize_microscaled(stream, stream.numel(), dt, *shape, out, case["cols"], status)
        return out
    if case["op"] == "moe":
        need = enec.enec_moe_microscaled_workspace(case["tokens"], case["hidden"], case["inter"], case["experts"], case["top"])
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        gate, up, down = state["gate"], state["up"], state["down"]
        enec.enec_moe_microscaled(state["x"], dt, case["tokens"], case["hidden"], case["hidden"], state["router"], case["experts"], case["top"],
                                  case["renormalize"], gate, gate.numel(), up, up.numel(), down, down.numel(), case["inter"],
                                  out, case["hidden"], workspace, need, status)
        return out
    x, w, tokens, rows, cols = state["x"], state["w"], case["tokens"], case["rows"], case["cols"]
    if case["op"] == "both":
        stream = state["stream"]
        enec.enec_quantize_microscaled(x, dt, 1, tokens, cols, x.stride(0), stream, stream.numel(), status)
        enec.enec_matmul_microscaled_both(stream, stream.numel(), tokens, w, w.numel(), rows, cols, dt, out, rows, status)
    else:
        enec.enec_matmul_microscaled(x, dt, tokens, x.stride(0), w, w.numel(), rows, cols, out, rows, status)
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    b = _BYTES[case["dtype"]]
    bits = 4.25 / 8
    if case["op"] in ("roundtrip", "dequantize"):
        n = case["batch"] * case["rows"] * case["cols"]
        once = n * (b + bits)
        return {"bytes": once * (2 if case["op"] == "roundtrip" else 1), "flops": 0}
    if case["op"] == "moe":
        tokens, hidden, inter, experts, top = (case[k] for k in ("tokens", "hidden", "inter", "experts", "top"))
        used = experts * (1 - (1 - top / experts) ** tokens)          # experts chosen by some token, on average
        return {"bytes": used * 3 * hidden * inter * bits + experts * hidden * b + 2 * tokens * hidden * b,
                "flops": 2 * tokens * experts * hidden + 6 * tokens * top * hidden * inter}
    tokens, rows, cols = case["tokens"], case["rows"], case["cols"]
    extra = 2 * tokens * cols * bits if case["op"] == "both" else 0   # x is written and read once more in 4 bits
    return {"bytes": rows * cols * bits + tokens * cols * b + tokens * rows * b + extra, "flops": 2 * tokens * rows * cols}


# ---- the definition, in 64 bits ------------------------------------------------------------------------------------------
def _nearest(x):
    """MXFP4 values of a tensor by their definition: the nearest grid point of every element, ties to the even one."""
    cols = x.shape[-1]
    flat = x.double().reshape(-1, cols)
    out = torch.empty_like(flat)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    odd = torch.tensor([0.0, 1.0] * 4, dtype=torch.float64, device=x.device) * 1e-9   # of two equally near points, the even code's
    step = max(1, (1 << 23) // cols)
    for first in range(0, flat.shape[0], step):
        part = torch.nn.functional.pad(flat[first:first + step], (0, -cols % 32))
        part = part.reshape(part.shape[0], -1, 32)
        top = part.abs().amax(-1, keepdim=True)
        scale = torch.ldexp(torch.ones_like(top), (torch.frexp(top)[1] - 3).clamp(-127, 127))   # floor(log2 top) is frexp's exponent less 1
        scale = torch.where(top == 0, torch.ones_like(scale), scale)
        q = (part / scale).abs()
        nearest = ((q[..., None] - grid).abs() + odd).argmin(-1)
        v = torch.copysign(grid[nearest], part) * scale
        out[first:first + step] = v.reshape(part.shape[0], -1)[:, :cols]
    return out.reshape(x.shape)


def _matrix64(stream, batch, rows, cols, index):
    """Matrix `index` of a stream in 64 bits, element by element from the byte that holds it."""
    down, across = _tiles(rows, _ROWS), _tiles(cols, _COLS)
    r = torch.arange(rows, device=stream.device)[:, None]
    k = torch.arange(cols, device=stream.device)[None, :]
    record = _HEADER + ((index * down + r // _ROWS) * across + k // _COLS) * _RECORD
    row, chunk = r % _ROWS, k % _COLS // 32
    byte = stream[record + row * 128 + (chunk ^ (row % 8)) * 16 + k % 32 // 2]
    code = torch.where(k % 2 == 1, byte >> 4, byte & 15).long()
    scale = stream[record + _RECORD - 1024 + chunk // 4 * 512 + row % 32 * 16 + row // 32 * 4 + chunk % 4]
    table = torch.tensor(_GRID + tuple(-v for v in _GRID), dtype=torch.float64, device=stream.device)
    return table[code] * torch.exp2(scale.double() - 127)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "roundtrip":
        return _nearest(state["x"])
    if case["op"] == "dequantize":
        return torch.stack([_matrix64(state["stream"], case["batch"], case["rows"], case["cols"], i) for i in range(case["batch"])])
    if case["op"] == "moe":
        x = state["x"].double()
        logits = x @ state["router"].double().t()
        p = torch.exp(logits - logits.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        chosen = torch.argsort(-logits, dim=-1, stable=True)[:, :case["top"]]
        y = torch.zeros_like(x)
        for e in sorted(set(chosen.reshape(-1).tolist())):
            w = torch.where(chosen == e, torch.gather(p, 1, chosen), torch.zeros((), dtype=torch.float64, device="cuda")).sum(-1)
            if case["renormalize"]:
                w = w / torch.gather(p, 1, chosen).sum(-1)
            a = x @ _matrix64(state["gate"], case["experts"], case["inter"], case["hidden"], e).t()
            h = a * torch.sigmoid(a) * (x @ _matrix64(state["up"], case["experts"], case["inter"], case["hidden"], e).t())
            y += w[:, None] * (h @ _matrix64(state["down"], case["experts"], case["hidden"], case["inter"], e).t())
        return y
    x = _nearest(state["x"]) if case["op"] == "both" else state["x"].double()
    return x @ _matrix64(state["w"], 1, case["rows"], case["cols"], 0).t()

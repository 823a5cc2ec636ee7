"""The microscaled 4-bit format and the operators on it in plain numpy and 64 bits, written from the format's definition.
Shared by the tests; nothing of the library is used here."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HEADER, RECORD, ROWS, COLS = 128, 17408, 128, 256


def stream_bytes(batch, rows, cols):
    return HEADER + batch * -(-rows // ROWS) * -(-cols // COLS) * RECORD


def blocks_of(x):
    """float64 [..., cols] -> [..., blocks, 32], zeros behind the row."""
    x = np.asarray(x, dtype=np.float64)
    pad = [(0, 0)] * (x.ndim - 1) + [(0, -x.shape[-1] % 32)]
    x = np.pad(x, pad)
    return x.reshape(*x.shape[:-1], -1, 32)


def encode(x):
    """Scale bytes [..., blocks] and codes [..., blocks, 32]."""
    b = blocks_of(x)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    exponent = np.frexp(top)[1] - 1                                   # floor(log2 top)
    s = np.clip(exponent - 2, -127, 127)
    s = np.where(top == 0, -127, s)
    m = np.abs(b) * np.exp2(-s.astype(np.float64))[..., None]          # exact: powers of two
    distance = np.abs(m[..., None] - GRID)
    nearest = distance.min(-1, keepdims=True)
    tied = distance == nearest
    even = tied & (np.arange(8) % 2 == 0)
    pick = np.where(tied.sum(-1, keepdims=True) > 1, even, tied)
    code = pick.argmax(-1).astype(np.uint8) | (np.signbit(b).astype(np.uint8) << 3)
    code = np.where(bad[..., None], 0, code).astype(np.uint8)
    byte = np.where(bad, 255, s + 127).astype(np.uint8)
    return byte, code


def decode(byte, code, cols):
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * np.exp2(byte.astype(np.float64) - 127)[..., None]
    v = np.where((byte == 255)[..., None], np.nan, v)
    return v.reshape(*v.shape[:-2], -1)[..., :cols]


def values(x):
    """What x becomes in the format."""
    return decode(*encode(x), np.asarray(x).shape[-1])


def stream(x):
    """The stream of a [batch, rows, cols] array, byte by byte from the layout in include/enec.h."""
    x = np.asarray(x, dtype=np.float64)
    batch, rows, cols = x.shape
    down, across = -(-rows // ROWS), -(-cols // COLS)
    out = np.zeros(stream_bytes(batch, rows, cols), dtype=np.uint8)
    out[:32].view(np.uint32)[:] = [0x344D4E45, 1, batch, rows, cols, 0, out.size & 0xFFFFFFFF, out.size >> 32]
    if x.size == 0:
        return out
    byte, code = encode(x)
    b, r, c = np.meshgrid(np.arange(batch), np.arange(rows), np.arange(byte.shape[-1]), indexing="ij")
    record = HEADER + ((b * down + r // ROWS) * across + c // 8) * RECORD
    row, chunk = r % ROWS, c % 8
    at = record + row * 128 + (chunk ^ (row % 8)) * 16
    packed = code[..., 0::2] | (code[..., 1::2] << 4)
    out[(at[..., None] + np.arange(16)).reshape(-1)] = packed.reshape(-1)
    out[(record + 16384 + chunk // 4 * 512 + row % 32 * 16 + row // 32 * 4 + chunk % 4).reshape(-1)] = byte.reshape(-1)
    return out


def layer(x, router, gate, up, down, top, renormalize, chosen=None):
    """The expert layer; gate, up [experts, inter, hidden] and down [experts, hidden, inter] as values. Also the chosen experts, which
    are the largest logits' unless they are given."""
    logits = x @ router.T
    p = np.exp(logits - logits.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    if chosen is None:
        chosen = np.argsort(-logits, axis=-1, kind="stable")[:, :top]
    y = np.zeros_like(x)
    for t in range(x.shape[0]):
        w = p[t, chosen[t]]
        w = w / w.sum() if renormalize else w
        for e, share in zip(chosen[t], w):
            a = gate[e] @ x[t]
            h = a / (1 + np.exp(-a)) * (up[e] @ x[t])
            y[t] += share * (down[e] @ h)
    return y, chosen

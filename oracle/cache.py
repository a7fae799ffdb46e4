"""Float64 restatements of the 4-bit key/value cache and of the attention of drafted
trees over it that include/tv.h declares: the bytes of a page's block, quantising,
reading back, the rows that an acceptance moves, and softmax attention under ancestor masks.
NumPy, literal, slow; shares no code with the CUDA path."""

import numpy as np

from .serving import round_e4m3

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 16


def quantize(x, exponent):
    """(codes 0..15, scales) of rows x [..., d] with the power of two 2^exponent: d values
    and d / 16 scales a row.  The borders between codes are exact products."""
    y = np.asarray(x, np.float64) * 2.0 ** -exponent
    y = np.where(np.isnan(y), 0.0, y)
    y = y.reshape(*y.shape[:-1], -1, GROUP)
    s = round_e4m3(np.minimum(np.abs(y).max(axis=-1) / 6.0, 448.0))
    a = np.abs(y)
    code = np.zeros(a.shape, dtype=np.int64)
    for k in range(7):
        border = (LEVELS[k] + LEVELS[k + 1]) / 2 * s[..., None]
        code += (a > border) if k % 2 == 0 else (a >= border)      # ties to the even code
    code = np.where(s[..., None] > 0, code, 0)
    code = np.where((y < 0) & (code > 0), code + 8, code)
    return code.reshape(*np.shape(x)), s


def held(x, exponent):
    """What the cache holds for rows x."""
    code, s = quantize(x, exponent)
    value = np.where(code >= 8, -1.0, 1.0) * LEVELS[code & 7]
    return value * np.repeat(s, GROUP, axis=-1) * 2.0 ** exponent


def e4m3_value(byte):
    byte = np.asarray(byte).astype(np.int64)
    e, m = (byte >> 3) & 15, byte & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m * 2.0 ** -9)
    return np.where(byte & 128, -v, v)


def e4m3_byte(value):
    """The byte of a value >= 0 that is one of the format's."""
    table = e4m3_value(np.arange(127))
    at = np.searchsorted(table, value)
    assert np.array_equal(table[at], value)
    return at.astype(np.uint8)


def put_row(block, page_size, slot, x, exponent):
    """Writes the bytes of row x [d] into a block [page_size * d * 9 / 16] uint8."""
    code, s = quantize(x, exponent)
    d = len(x)
    b8 = e4m3_byte(s)
    for col in range(0, d, 2):
        at = ((col // 32) * page_size + slot) * 16 + (col % 32) // 2
        block[at] = code[col] | code[col + 1] << 4
    for g in range(d // GROUP):
        block[page_size * d // 2 + ((g // 2) * page_size + slot) * 2 + g % 2] = b8[g]


def get_row(block, page_size, slot, d, exponent):
    """The values of a row of a block."""
    out = np.zeros(d)
    for col in range(d):
        byte = int(block[((col // 32) * page_size + slot) * 16 + (col % 32) // 2])
        code = byte >> 4 if col % 2 else byte & 15
        g = col // GROUP
        s = e4m3_value(block[page_size * d // 2 + ((g // 2) * page_size + slot) * 2 + g % 2])
        out[col] = (-1 if code >= 8 else 1) * LEVELS[code & 7] * s * 2.0 ** exponent
    return out


def visible(parents, length, rows):
    """[rows, length + rows] of truth values: row i of a tree sees what is cached, its
    ancestors and itself; without parents what is cached and rows 0 .. i."""
    m = np.zeros((rows, length + rows), dtype=bool)
    m[:, :length] = True
    for i in range(rows):
        if parents is None:
            m[i, length:length + i + 1] = True
        else:
            j = i
            while j >= 0:
                m[i, length + j] = True
                j = parents[j]
    return m


def attention(q, k, v, mask, scale):
    """[rows, heads, d] of q [rows, heads, d] over k, v [tokens, kv_heads, d] where mask
    [rows, tokens] is true; rows that see nothing are 0."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    group = q.shape[1] // k.shape[1]
    out = np.zeros(q.shape)
    for h in range(q.shape[1]):
        t = q[:, h] @ k[:, h // group].T * scale
        t = np.where(mask, t, -np.inf)
        m = t.max(axis=1, initial=-np.inf, keepdims=True)
        p = np.where(mask, np.exp(t - np.where(np.isfinite(m), m, 0.0)), 0.0)
        s = p.sum(axis=1, keepdims=True)
        out[:, h] = np.divide(p, s, out=np.zeros_like(p), where=s > 0) @ v[:, h // group]
    return out


def accept(path, tau):
    """Tree rows in the order in which they follow the cached tokens after an acceptance."""
    return [0] + [int(n) for n in path[:tau]] if tau >= 0 else []

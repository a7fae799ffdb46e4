"""Float64 restatements of the steps between the target model's last layer and the
verification that include/tv.h declares beside the paper's method: the final norm
with the residual's addition, 8-bit operands with block scales, their product, and
penalties, biases and grammar masks on the logits of a tree's rows.  NumPy, literal,
slow; shares no code with the CUDA path."""

import numpy as np

GROUP = 128
E4M3_MAX = 448.0
LEAST = 2.0 ** -100


def round_e4m3(x):
    """The e4m3 value nearest to x (ties to the even mantissa; magnitudes past 448
    become 448, NaN stays NaN): 3 bits after the leading one, exponents down to -6,
    multiples of 2^-9 below."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.clip(np.rint(x / step) * step, -E4M3_MAX, E4M3_MAX)


def rms_norm(x, residual, weight, eps):
    """(y, h): h = x + residual, y = h w / sqrt(mean(h^2) + eps)."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    return y, h


def row_scales(y):
    """One scale per row and group of 128 columns: [M, ceil(K / 128)]."""
    y = np.asarray(y, np.float64)
    return np.stack([np.maximum(np.abs(y[:, k:k + GROUP]).max(axis=1), LEAST) / E4M3_MAX
                     for k in range(0, y.shape[1], GROUP)], axis=1)


def block_scales(w):
    """One scale per block of 128 rows and 128 columns."""
    w = np.abs(np.asarray(w, np.float64))
    return np.array([[max(w[r:r + GROUP, k:k + GROUP].max(), LEAST) / E4M3_MAX
                      for k in range(0, w.shape[1], GROUP)]
                     for r in range(0, w.shape[0], GROUP)])


def spread(scales, rows, cols, row_group):
    """Scales [.., ..] at every element of a [rows, cols] operand."""
    return np.asarray(scales, np.float64)[np.arange(rows) // row_group][:, np.arange(cols) // GROUP]


def scaled_logits(qa, sa, qw, sw):
    """sum_g sa[i, g] sw[v / 128, g] sum_{k in g} qa[i, k] qw[v, k]."""
    a = np.asarray(qa, np.float64) * spread(sa, *np.shape(qa), 1)
    w = np.asarray(qw, np.float64) * spread(sw, *np.shape(qw), GROUP)
    return a @ w.T


def path_tokens(parents, tokens, i):
    """The drafted tokens from the root (its own excluded) to node i."""
    out = []
    while i > 0:
        out.append(tokens[i])
        i = parents[i]
    return out


def process_row(logits, generated, prompt, bias, penalties, path, allowed):
    """One row: logits, generated counts, prompt marks and biases [V] (the last three may
    be None), penalties (repetition, frequency, presence), the path's tokens, and the
    allowed tokens' truth values (None: all)."""
    l = np.array(logits, np.float64)
    V = l.shape[0]
    n = np.zeros(V) if generated is None else np.array(generated, np.float64)
    for t in path:
        n[t] += 1.0
    seen = n > 0
    if prompt is not None:
        seen = seen | np.asarray(prompt, bool)
    rep, freq, pres = (float(p) for p in penalties)
    l = np.where(seen, np.where(l > 0, l / rep, l * rep), l)
    l = np.where(n > 0, l - freq * n - pres, l)
    if bias is not None:
        l = l + np.asarray(bias, np.float64)
    if allowed is not None:
        l = np.where(np.asarray(allowed, bool), l, -np.inf)
    return l


def row_normaliser(l, temperature):
    """(max, sum of exp((l - max) / T)); (-inf, 0) where nothing is finite or above."""
    l = np.asarray(l, np.float64)
    m = l.max()
    if m == -np.inf:
        return -np.inf, 0.0
    return m, float(np.exp((l - m) / temperature).sum())

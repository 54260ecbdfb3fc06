"""Float64 CPU oracle of the calls on a tied model's table: embedding lookup and gradient, 8-bit rows, log-probs under them.
Test infrastructure only, written from the definitions in include/rapid.h."""
import numpy as np


def embedding_fwd(table, tokens, mask, scale):
    """[N,T,d] float64: scale * table[token], zeros at masked positions and ids out of range."""
    N, T = tokens.shape
    out = np.zeros((N, T, table.shape[1]))
    for n in range(N):
        for t in range(T):
            if (mask is None or mask[n, t]) and 0 <= tokens[n, t] < table.shape[0]:
                out[n, t] = scale * table[tokens[n, t]].astype(np.float64)
    return out


def embedding_bwd(dhidden, tokens, mask, V, scale):
    """(gradient [V,d], sum of magnitudes [V,d], number of terms [V]) in float64."""
    d = dhidden.shape[-1]
    grad, size, terms = np.zeros((V, d)), np.zeros((V, d)), np.zeros(V, np.int64)
    valid = (tokens >= 0) & (tokens < V)
    if mask is not None:
        valid &= mask != 0
    ids, rows = tokens[valid], dhidden[valid].astype(np.float64) * scale
    np.add.at(grad, ids, rows)
    np.add.at(size, ids, np.abs(rows))
    np.add.at(terms, ids, 1)
    return grad, size, terms


def round_e4m3(x):
    """Nearest e4m3 value (ties to even) of |x| <= 448: 3 stored mantissa bits, exponents from 2^-6 on, multiples of 2^-9 below."""
    x = np.asarray(x, np.float64)
    _, exponent = np.frexp(np.maximum(np.abs(x), 2.0 ** -6))       # |x| in [2^(exponent-1), 2^exponent)
    step = np.ldexp(1.0, exponent - 1 - 3)
    return np.rint(x / step) * step


def quantize(rows):
    """Rows [R,d] -> (e4m3 values [R, d up to blocks of 128], exponents [R, blocks]), float64 and int."""
    R, d = rows.shape
    blocks = -(-d // 128)
    x = np.zeros((R, blocks * 128))
    x[:, :d] = rows
    x = x.reshape(R, blocks, 128)
    finite = np.where(np.isfinite(x), x, 0.0)
    most = np.abs(finite).max(axis=2)
    e = np.zeros((R, blocks), np.int64)
    for r, b in zip(*np.nonzero(most)):
        k = -126
        while most[r, b] > np.ldexp(448.0, k):
            k += 1
        e[r, b] = k
    q = np.where(np.isfinite(x), round_e4m3(np.ldexp(finite, -e[:, :, None])), np.nan)
    return q.reshape(R, -1), e


def dequantize(values, exponents):
    R = values.shape[0]
    return np.ldexp(values.reshape(R, -1, 128), exponents[:, :, None]).reshape(R, -1)


def _largest_of_8(x):
    return np.abs(x).reshape(x.shape[0], -1, 8).max(axis=2)


def logprob_fp8(hidden, W, tokens, mask, temperature):
    """(logp, lse, size, top, cut) [N,T] under the head W [V,d], both brought to 8 bits.  What roundings are relative to, each the largest over
    the vocabulary: size, a logit's sum of |terms|; top, the |logit|; cut, the sum over its groups of 8 terms of the group's largest
    |hidden| times its largest |weight|."""
    N, T, d = hidden.shape
    w = dequantize(*quantize(W))
    logp, lse, size, top, cut = (np.zeros((N, T)) for _ in range(5))
    at = np.nonzero(mask)
    if at[0].size == 0:
        return logp, lse, size, top, cut
    h = dequantize(*quantize(hidden[at].astype(np.float64)))
    z = h @ w.T / temperature
    m = z.max(axis=1)
    s = m + np.log(np.exp(z - m[:, None]).sum(axis=1))
    y = tokens[at]
    y = np.where((y >= 0) & (y < W.shape[0]), y, 0)
    lse[at] = s
    logp[at] = z[np.arange(len(y)), y] - s
    size[at] = (np.abs(h) @ np.abs(w).T).max(axis=1) / temperature
    top[at] = np.abs(z).max(axis=1)
    cut[at] = (_largest_of_8(h) @ _largest_of_8(w).T).max(axis=1) / temperature
    return logp, lse, size, top, cut

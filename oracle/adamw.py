"""Oracle: AdamW with the per-parameter clip, and its moments in 8 bits, in fp64.

Test infrastructure (see the package docstring).
"""
import numpy as np

from .precision import F

GROUP = 256
LOW = {"m": 13, "v": 29}


def adamw_step(p, m, v, g, lr, beta1, beta2, eps, clip_k, weight_decay, step):
    """New (p, m, v)."""
    p, m, v, g = (np.asarray(a, F()) for a in (p, m, v, g))
    v = beta2 * v + (1.0 - beta2) * g * g
    root = np.sqrt(v / (1.0 - beta2 ** step))
    gc = np.clip(g, -clip_k * root, clip_k * root) if clip_k > 0 else g
    m = beta1 * m + (1.0 - beta1) * gc
    return (1.0 - lr * weight_decay) * p - lr * (m / (1.0 - beta1 ** step)) / (root + eps), m, v


def value_of(code, exps, which):
    """The values of the codes [n] of moment `which` ("m" or "v") under the groups' exponents."""
    code = np.asarray(code, np.int64)
    a = np.maximum(np.repeat(np.asarray(exps, np.int64), GROUP)[:code.size] - 127, -90)
    mag = code & 127 if which == "m" else code
    e, f = mag >> 3, mag & 7
    x = np.where(e > 0, 8 + f, f) * np.exp2((a - LOW[which] - 4 + np.maximum(e, 1)).astype(F()))
    if which == "m":
        x = np.where(code >= 128, -x, x)
    return np.where(mag == (127 if which == "m" else 255), np.nan, x)


def neighbours(x, which):
    """For each x [n] the two values a code can stand for around it, by its group's largest, and that exponent."""
    x = np.asarray(x, F())
    pad = np.zeros((x.size + GROUP - 1) // GROUP * GROUP)
    pad[:x.size] = np.abs(x)
    top = np.maximum(pad.reshape(-1, GROUP).max(1), 2.0 ** -90)
    a = np.floor(np.log2(top)).astype(np.int64)
    b = np.repeat(a, GROUP)[:x.size]
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -1000)))
    step = np.exp2(np.maximum(e, b - LOW[which]) - 3)
    low = np.floor(np.abs(x) / step) * step
    return low, low + step, a


def philox4x32_7(counter, key):
    """The four words at `counter` (four 32-bit words) and `key` (two)."""
    M = 0xFFFFFFFF
    c, k = [int(w) for w in counter], [int(w) for w in key]
    for _ in range(7):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & M, (p0 >> 32) ^ c[3] ^ k[1], p0 & M]
        k = [(k[0] + 0x9E3779B9) & M, (k[1] + 0xBB67AE85) & M]
    return c


def chances(n, step, tensor, seed):
    """The numbers in [0, 1) that round element 0..n-1's m and v up."""
    words = []
    for i in range((n + 3) // 4):
        words += philox4x32_7((i & 0xFFFFFFFF, i >> 32, step, tensor), (seed & 0xFFFFFFFF, seed >> 32))
    w = np.array(words[:n], np.int64)
    return (w & 0xFFFF) / 65536.0, (w >> 16) / 65536.0


def rounded(x, up, which):
    """The value that stands for each x [n]: the upper neighbour where the cut-off part and `up` fill a step."""
    low, high, _ = neighbours(x, which)
    x = np.asarray(x, F())
    take = (np.abs(x) - low) / (high - low) + up >= 1.0
    mag = np.where(take, high, low)
    if which == "v":
        mag = np.where((x > 0) & (mag == 0), high, mag)
    return np.where(x < 0, -mag, mag)

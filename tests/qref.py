"""Rows of 4 bits and attention over them in float64 numpy, from the format's definition (include/alora.h); shares no code
with the library.  And how far fp32 sums may take a result from it."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # half a rounding step, relative


def quantise(x):
    """x [..., h] float64 (values of the storage type) -> codes [..., h / 2] uint8, exponents [..., ceil(h / 32)] uint8."""
    x = np.asarray(x, dtype=np.float64)
    h = x.shape[-1]
    code = np.zeros(x.shape, dtype=np.uint8)
    exps = np.zeros(x.shape[:-1] + ((h + 31) // 32,), dtype=np.uint8)
    for n in range(exps.shape[-1]):
        b = x[..., 32 * n:32 * n + 32]
        bad = ~np.isfinite(b).all(-1)
        b = np.where(bad[..., None], 0.0, b)
        top = np.abs(b).max(-1)
        m, e = np.frexp(top)                        # top = 2 m * 2^(e - 1)
        ex = np.where(2 * m > 1.75, e - 1 - 1, e - 1 - 2)
        ex = np.where(top == 0, 0, np.clip(ex, -125, 125))
        y = np.abs(b) / np.exp2(ex)[..., None]
        level = np.zeros(b.shape, dtype=np.int64)
        for i, t in enumerate(MIDS):                # a tie goes to the even code
            level += (y >= t) if i % 2 else (y > t)
        c = level + 8 * np.signbit(b)
        code[..., 32 * n:32 * n + 32] = np.where(bad[..., None], 0, c)
        exps[..., n] = np.where(bad, 255, ex + 127)
    return code[..., 0::2] | (code[..., 1::2] << 4), exps


def values(codes, exps):
    h = 2 * codes.shape[-1]
    code = np.empty(codes.shape[:-1] + (h,), dtype=np.int64)
    code[..., 0::2], code[..., 1::2] = codes & 15, codes >> 4
    v = np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7]
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)[..., :h]


def attend(q, K, V, n_q_heads, visible):
    """q [S, n_q_heads * h]; K, V [L, n_kv, h] of one sequence; row i sees the first visible[i] keys.  Returns the result and, for its error:
    sum_j p_j |v_j|, sum_j |v_j| (elementwise) and max_j sum_c |q_c k_jc| / sqrt(h) (per row and head)."""
    L, n_kv, h = K.shape
    G = n_q_heads // n_kv
    out, mag, total = np.empty(q.shape), np.empty(q.shape), np.empty(q.shape)
    spread = np.empty((q.shape[0], n_q_heads))
    for i in range(q.shape[0]):
        n = visible[i]
        for j in range(n_q_heads):
            qv, k, v = q[i, j * h:(j + 1) * h], K[:n, j // G], V[:n, j // G]
            s = k @ qv / np.sqrt(h)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, j * h:(j + 1) * h] = p @ v
            mag[i, j * h:(j + 1) * h] = p @ np.abs(v)
            total[i, j * h:(j + 1) * h] = np.abs(v).sum(0)
            spread[i, j] = (np.abs(k) @ np.abs(qv)).max() / np.sqrt(h)
    return out, mag, total, spread


def tolerance(ref, mag, total, spread, h, L, dtype):
    """|result - ref| is at most
      half a step of the stored type, plus mag = sum p |v| times
      2 * (error of a score): h + 8 fp32 roundings of the terms of q k / sqrt(h), times their sum (spread), its square-root scale included,
          and 2^-22 * spread for the exponent's argument (score less maximum, both at most 1.45 spread in base 2);
      2 * 2^-11 (bf16): a probability rounded to the 11 bits of fp16, at most half a step, in the numerator and the denominator; fp32: 2 * 2^-21, 24 bits and the exponential's own error;
          and what fp16 loses of small ones: half of its smallest number, 2^-25, where the largest probability is 2^7 or more: 2^-32 of sum |v|;
      2 * (L / 8 + 64) * 2^-24: the running sums over keys, eight terms or more at a time, and the joining of partial ones."""
    c = 2 * ((h + 8) * 2.0 ** -24 + 2.0 ** -22) * np.repeat(spread, h, axis=-1) + 2 * 2.0 ** (-11 if dtype == "bf16" else -21) + 2 * (L / 8 + 64) * 2.0 ** -24
    return HALF[dtype] * np.abs(ref) + c * mag + (2.0 ** -32 * total if dtype == "bf16" else 0.0) + 1e-37

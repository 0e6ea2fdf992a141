"""The 4-bit key / value cache in 64 bits on the CPU, from its definition in include/kangaroo.h: quantisation,
the bytes of a page looked up number by number, attention with the tokens' weights, eviction.  Test infrastructure."""
import numpy as np


def bf16_round(x):
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


ROUND = {"f32": lambda x: x.astype(np.float32), "f16": lambda x: x.astype(np.float16).astype(np.float32), "bf16": bf16_round}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}        # half a step, relative to the value


def quantise(x):
    """x float32 [..., D] -> (n, s, m) float64 with s, m per group of 32."""
    g = x.astype(np.float64).reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(g).all(-1)
    g = np.clip(np.nan_to_num(g, nan=0.0, posinf=65504.0, neginf=-65504.0), -65504.0, 65504.0)
    lo, hi = g.min(-1), g.max(-1)
    m = lo.astype(np.float32).astype(np.float16).astype(np.float64)
    s = ((hi.astype(np.float32) - lo.astype(np.float32)) / np.float32(15)).astype(np.float16).astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        n = np.clip(np.rint((g - m[..., None]) / s[..., None]), 0, 15)
    n[(s == 0) | bad] = 0
    return n, np.where(bad, np.nan, s), np.where(bad, 0.0, m)


def values(q):
    n, s, m = q
    v = n * s[..., None] + m[..., None]
    return v.reshape(v.shape[:-2] + (-1,))


class Pages:
    """A page pool in host memory (uint8)."""

    def __init__(self, pool, table, H, D, T, stride):
        self.pool, self.table, self.H, self.D, self.T, self.stride = pool, table, H, D, T, stride
        self.n_pages = (len(pool) - H * T * D * 5 // 4) // stride + 1

    def token(self, s, h, t):
        """(n, s, m) of keys and values [D / 32] of a token; None where it has no page."""
        D, T = self.D, self.T
        G, page, t = D // 32, int(self.table[s][t // T]), t % T
        if page < 0 or page >= self.n_pages:
            return None
        b = self.pool[page * self.stride + h * (T * D * 5 // 4):][:T * D * 5 // 4]
        half = b[T * D:].view(np.float16).astype(np.float64)
        out = []
        for kind in range(2):
            n = np.empty(D)
            for d in range(D):
                if kind == 0:
                    byte = b[t * (D // 2) + ((d % 32 // 8) * G + d // 32) * 4 + d % 8 // 2]
                    n[d] = byte >> 4 if d % 2 else byte & 15
                else:
                    j, r = d // 16, d % 16
                    byte = b[T * D // 2 + (((t // 4) * 16 + r) * (D // 64) + j // 4) * 8 + (t % 4) * 2 + (j % 4) // 2]
                    n[d] = byte >> 4 if j % 2 else byte & 15
            quad = np.array([((t // 4) * G + g) * 4 + t % 4 for g in range(G)])
            if kind == 0:
                s_, m_ = half[quad], half[T * G + t * G + np.arange(G)]
            else:
                s_, m_ = half[2 * T * G + quad], half[3 * T * G + quad]
            out.append((n.reshape(G, 32), s_, m_))
        return out


def token_offsets(H, D, T, h, t):
    """Byte offsets in a page of everything that belongs to head h of token t."""
    G, base, o = D // 32, h * (T * D * 5 // 4), set()
    for i in range(D // 2):
        o.add(base + t * (D // 2) + i)
    for r in range(16):
        for vh in range(D // 64):
            for b in range(2):
                o.add(base + T * D // 2 + (((t // 4) * 16 + r) * (D // 64) + vh) * 8 + (t % 4) * 2 + b)
    for g in range(G):
        for b in range(2):
            quad = (((t // 4) * G + g) * 4 + t % 4) * 2 + b
            o |= {base + T * D + quad, base + T * D + 4 * T * G + quad, base + T * D + 6 * T * G + quad,
                  base + T * D + 2 * T * G + (t * G + g) * 2 + b}
    return o


def attention(q, kq, vq, pos, scale, here=None, halves=False):
    """Rows q [r][heads][D] (float64) over keys / values given as (n, s, m) [len][H][G](32): outputs, tolerance of fp32
    arithmetic (without the output's rounding), probabilities [r][heads][len].  pos[i]: last token that row i sees.
    here [len]: tokens that have a page.

    Tolerance: a score is sum q_d (s n + m) scale, whose terms' absolute sum is A.  Both factors are held to 2^-21 or better and
    added in fp32: the score is off by at most A 2^-20, a probability by twice that and its own rounding; products with the
    values are held to 2^-21, and n terms are added in partial sums of at most 64 + n / 64.
    halves: rows of bf16 may take values and probabilities rounded to fp16, 2^-11 of either at most.  With the largest value V that is
    sum p (1 + 2^-11) v (1 + 2^-11) - sum p v <= (2^-10 + 2^-22) V, an eighth of what rounding V itself to bf16 may cost."""
    r, heads, D = q.shape
    n, H = kq[0].shape[:2]
    g = heads // H
    K, V = values(kq), values(vq)
    Ka = np.abs(kq[0] * kq[1][..., None]) + np.abs(kq[2])[..., None]
    Ka = Ka.reshape(n, H, D)
    Va = 15 * np.abs(vq[1]) + np.abs(vq[2])
    out, tol, prob = np.zeros((r, heads, D)), np.zeros((r, heads, D)), np.zeros((r, heads, n))
    for i in range(r):
        see = np.arange(n) <= pos[i]
        if here is not None:
            see &= here
        if not see.any():
            continue
        for j in range(heads):
            h = j // g
            z = K[see, h] @ q[i, j] * scale
            p = np.exp(z - z.max())
            p /= p.sum()
            A = np.max(Ka[see, h] @ np.abs(q[i, j])) * abs(scale)
            rel = (2.0 ** -10 + 2.0 ** -22 if halves else 0.0) + 2 * A * 2.0 ** -20 + 2.0 ** -20 + (64 + see.sum() / 64) * 2.0 ** -24
            out[i, j] = p @ V[see, h]
            tol[i, j] = rel * np.repeat(Va[see, h].max(0), 32)
            prob[i, j, see] = p
    return out, tol, prob


def evict(w, n, keep, first, recent):
    """Token indices that stay, in order."""
    if n <= keep:
        return np.arange(n)
    key = np.where(np.isnan(w[:n]), np.inf, w[:n])
    nan = np.isnan(w[:n])
    mid = np.arange(first, n - recent)
    order = sorted(mid, key=lambda t: (not nan[t], -key[t], t))
    return np.sort(np.concatenate([np.arange(first), np.array(order[:keep - first - recent], int), np.arange(n - recent, n)])).astype(int)

"""Independent fp64 oracle of the KV cache in 8 bits, in numpy: every e4m3 number is written out, rounding
is a search among them, blocks are dense arrays [slot][d].  Shares no code with the library."""
import numpy as np

P, D = 16, 128
F16, BF16 = 0, 1
LIMITS = {F16: (-15, 8), BF16: (-100, 120)}


def decode16(bits, dtype):
    """fp16 / bf16 bit patterns -> float64"""
    bits = np.asarray(bits, dtype=np.uint16)
    if dtype == F16:
        return bits.view(np.float16).astype(np.float64)
    with np.errstate(invalid="ignore"):
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _numbers():
    """value of each of the 256 codes, from the format's definition"""
    out = np.empty(256)
    for c in range(256):
        sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        if e == 15 and m == 7:
            out[c] = np.nan
        elif e == 0:
            out[c] = sign * m * 2.0 ** -9
        else:
            out[c] = sign * (8 + m) * 2.0 ** (e - 10)
    return out


NUMBERS = _numbers()
POSITIVE = NUMBERS[:127]                       # codes 0 .. 126, rising


def round_codes(x):
    """x (float64, magnitude <= 448 or NaN) -> the nearest code, of two the even one; NaN -> 0x7f."""
    a = np.abs(x)
    with np.errstate(invalid="ignore"):
        hi = np.searchsorted(POSITIVE, a)              # first number >= a
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = POSITIVE[hi] - a, a - POSITIVE[lo]
    pick = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    pick = np.where(hi == lo, hi, pick)
    codes = pick + np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 0x7f, codes).astype(np.uint8)


def scale_exponent(values, dtype):
    """of a block's values (any shape, float64)"""
    lo, hi = LIMITS[dtype]
    finite = np.abs(values[np.isfinite(values)])
    big = finite.max() if finite.size else 0.0
    k = lo
    while k < hi and big > 448.0 * 2.0 ** k:
        k += 1
    return k


def encode(values, k, dtype):
    with np.errstate(invalid="ignore"):
        y = values / 2.0 ** k
    most = 240.0 if k == LIMITS[dtype][1] else 448.0
    y = np.where(np.isfinite(values), np.clip(y, -most, most), np.nan)
    return round_codes(y)


class Pool:
    """codes as [layer][page][K, V][head][slot][d], scale exponents [layer][page][head][K, V]"""

    def __init__(self, layers, pages, heads, dtype, codes=None, scales=None):
        self.dtype, self.heads = dtype, heads
        self.codes = np.zeros((layers, pages, 2, heads, P, D), np.uint8)
        self.k = np.full((layers, pages, heads, 2), LIMITS[dtype][0])
        if codes is not None:
            raw = codes.reshape(layers, pages, 2, heads, P * D)
            self.codes[:, :, 0] = raw[:, :, 0].reshape(layers, pages, heads, P, D)
            self.codes[:, :, 1] = raw[:, :, 1].reshape(layers, pages, heads, D, P).swapaxes(3, 4)
            self.k = np.log2(scales.reshape(layers, pages, heads, 2).astype(np.float64)).astype(int)

    def raw(self):
        """(codes, scales) as they lie in memory"""
        L, N, _, H = self.codes.shape[:4]
        out = np.empty((L, N, 2, H, P * D), np.uint8)
        out[:, :, 0] = self.codes[:, :, 0].reshape(L, N, H, P * D)
        out[:, :, 1] = self.codes[:, :, 1].swapaxes(3, 4).reshape(L, N, H, P * D)
        return out, (2.0 ** self.k).astype(np.float32)

    def put(self, layer, page, kv, head, lo, rows):
        """rows (float64 [n][D]) into slots lo .. of a block, by the rules of the append"""
        k = scale_exponent(rows, self.dtype)
        block = self.codes[layer, page, kv, head]
        if lo > 0:
            old = self.k[layer, page, head, kv]
            k = max(k, old)
            if k > old:
                block[:lo] = round_codes(NUMBERS[block[:lo]] * 2.0 ** (old - k))
        block[lo:lo + len(rows)] = encode(rows, k, self.dtype)
        self.k[layer, page, head, kv] = k

    def append(self, layer, k_new, v_new, begin, pages):
        """bits [n][heads][D] of one sequence's tokens begin .. begin + n"""
        n, t = len(k_new), 0
        while t < n:
            pos = begin + t
            cnt = min(P - pos % P, n - t)
            for kv, new in ((0, k_new), (1, v_new)):
                x = decode16(new[t:t + cnt], self.dtype)
                for h in range(self.heads):
                    self.put(layer, pages[pos // P], kv, h, pos % P, x[:, h])
            t += cnt

    def values(self, layer, pages, n):
        """K and V of tokens [0, n) of the sequence with these pages: [head][n][D] each"""
        pages = np.asarray(pages)[: -(-n // P)]
        x = NUMBERS[self.codes[layer, pages]] * (2.0 ** self.k[layer, pages].swapaxes(1, 2))[..., None, None]
        x = x.transpose(1, 2, 0, 3, 4).reshape(2, self.heads, -1, D)[:, :, :n]
        return x[0], x[1]


def attention(pool, layer, pages, q, begin, scale=None, rows=None):
    """q: bits [n][hq][D].  Returns out, lse and what their error is measured by: A = sum_j p_j |v_j|,
    E = the largest sum_d |q_d k_d| x scale of a row's keys, V = the largest |v| a row sees.  rows: which."""
    n, hq, hkv = q.shape[0], q.shape[1], pool.heads
    G, scale = hq // hkv, D ** -0.5 if scale is None else scale
    rows = np.arange(n) if rows is None else np.asarray(rows)
    K, V = pool.values(layer, pages, begin + n)
    qv = decode16(q, pool.dtype)[rows]
    out, lse = np.empty((len(rows), hq, D)), np.empty((len(rows), hq))
    A, E, VM = np.empty_like(out), np.empty_like(lse), np.empty_like(lse)
    for i, r in enumerate(rows):
        seen = begin + r + 1
        for h in range(hkv):
            k, v = K[h, :seen], V[h, :seen]
            x = qv[i, h * G:(h + 1) * G]
            s = x @ k.T * scale
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            l = p.sum(1, keepdims=True)
            sl = slice(h * G, (h + 1) * G)
            out[i, sl], A[i, sl] = p @ v / l, p @ np.abs(v) / l
            lse[i, sl] = (top + np.log(l))[:, 0]
            E[i, sl] = (np.abs(x) @ np.abs(k).T).max(1) * scale
            VM[i, sl] = np.abs(v).max()
    return out, lse, A, E, VM

"""Oracle of the paged cache's writing side and of the cache in 8 bits (TEST INFRASTRUCTURE ONLY): numpy, 64 bits, one sequence and
one scale block at a time.  bf16 tensors are ``uint16`` bit patterns, e4m3 codes ``uint8``."""
import numpy as np

E4M3_MAX, SCALE_MIN = 448.0, 2.0 ** -126


def bf16_to_f64(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _table():
    """Values of the codes 0 .. 126 (positive, ascending)."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))


POSITIVE = _table()


def e4m3_decode(codes):
    codes = np.asarray(codes, np.uint8)
    v = np.append(POSITIVE, np.nan)[codes & 127]
    return np.where(codes & 128, -v, v)


def e4m3_encode(x):
    """Nearest code, ties to the even one; 127 (NaN) for what is not finite.  |x| is at most 448."""
    x = np.asarray(x, np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    if a.size and a.max() > E4M3_MAX:
        raise ValueError("beyond the largest code")
    hi = np.minimum(np.searchsorted(POSITIVE, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = POSITIVE[hi] - a, a - POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), 127).astype(np.uint8)


def scale_for(amax):
    """Smallest power of two >= 2^-126 with amax <= 448 times it."""
    amax = np.asarray(amax, np.float64)
    mant, exp = np.frexp(amax)  # amax = mant * 2^exp, 448 = 0.875 * 2^9
    return np.where(amax > 0, np.maximum(np.ldexp(1.0, exp - 9 + (mant > 0.875)), SCALE_MIN), SCALE_MIN)


def rope(x, positions, inv_freq, interleaved=False):
    """x [T,H,d] (float64) turned at positions [T]: pairs (i, i + r/2), or (2i, 2i + 1) if interleaved; r = 2 len(inv_freq)."""
    x = np.asarray(x, np.float64)
    out, r = x.copy(), 2 * len(inv_freq)
    phi = np.asarray(positions, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    c, s = np.cos(phi), np.sin(phi)
    one, two = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    with np.errstate(invalid="ignore"):
        out[..., one] = x[..., one] * c - x[..., two] * s
        out[..., two] = x[..., two] * c + x[..., one] * s
    return out


def append_pages(pages, rows, start, block_table):
    """rows [n,Hkv,d] of one sequence into pages [n_pages,page_size,Hkv,d] from logical token `start` on, in place."""
    n_pages, page_size = pages.shape[:2]
    for i, row in enumerate(rows):
        page = int(block_table[(start + i) // page_size])
        if 0 <= page < n_pages:
            pages[page, (start + i) % page_size] = row


def append_quant(codes, scales, rows, start, block_table, valid=None):
    """rows [n,Hkv,d] (float64) of one sequence into codes [n_pages,Hkv,page_size,d] and scales [n_pages,Hkv,blocks] from logical
    token `start` on, in place.  valid [n,Hkv]: rows that are there (all)."""
    n_pages, n_heads, page_size, _ = codes.shape
    block = page_size // scales.shape[2]
    n = rows.shape[0]
    valid = np.ones((n, n_heads), bool) if valid is None else valid
    for tok0 in range(start // block * block, start + n, block):
        page, slot = int(block_table[tok0 // page_size]), tok0 % page_size
        if not 0 <= page < n_pages:
            continue
        first, last = max(tok0, start), min(tok0 + block, start + n)
        for h in range(n_heads):
            put = [t for t in range(first, last) if valid[t - start, h]]
            if not put:  # no row is there: the smallest scale, for what is appended behind
                scales[page, h, slot // block] = SCALE_MIN
                continue
            x = rows[np.array(put) - start, h]
            at = np.array(put) - tok0 + slot
            finite = np.where(np.isfinite(x), np.abs(x), 0.0)
            new = float(scale_for(finite.max()))
            if first > tok0:
                old = float(scales[page, h, slot // block])
                new = max(new, old)
                if new > old:
                    kept = slice(slot, slot + first - tok0)
                    codes[page, h, kept] = e4m3_encode(e4m3_decode(codes[page, h, kept]) * (old / new))
            codes[page, h, at] = e4m3_encode(x / new)
            scales[page, h, slot // block] = new


def dequant(codes, scales, block_table, n):
    """The first n logical tokens of a sequence: [n,Hkv,d] float64."""
    page_size = codes.shape[2]
    block = page_size // scales.shape[2]
    t = np.arange(n)
    page, slot = np.asarray(block_table)[t // page_size], t % page_size
    return e4m3_decode(codes[page, :, slot]) * scales[page, :, slot // block].astype(np.float64)[..., None]


def attend(q, k, v, scale):
    """q [Hq,d], k, v [n,Hkv,d] (float64) -> (out [Hq,d], bound [Hq,d]): softmax attention, zeros without tokens; and how far an evaluation
    may be off that holds products exactly and adds in fp32: a logit by d * 2^-23 of the sum of its products' sizes, hence its weight
    by that much relative, plus 2^-21 for the exponential and its argument's rounding; sums over n tokens, taken in chains of at
    most n / 32 + 192 additions, by 2^-23 for each of those."""
    hq, d = q.shape
    n, hkv = k.shape[:2]
    out, bound = np.zeros((hq, d)), np.zeros((hq, d))
    if n == 0:
        return out, bound
    for h in range(hq):
        g = h // (hq // hkv)
        z = k[:, g] @ q[h] * scale
        size = np.abs(k[:, g]) @ np.abs(q[h]) * scale
        p = np.exp(z - z.max())
        p /= p.sum()
        off = size * (d * 2.0 ** -23) + np.abs(z - z.max()) * 2.0 ** -22 + 2.0 ** -21
        out[h] = p @ v[:, g]
        bound[h] = 2 * (p * off) @ np.abs(v[:, g]) + np.abs(out[h]) * (p @ off) + ((n / 32 + 192) * 2.0 ** -23 + 2.0 ** -20) * (p @ np.abs(v[:, g]))
    return out, bound

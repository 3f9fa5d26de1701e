"""CPU oracle for the paged K/V cache (test infrastructure, not the product; plain numpy in fp64, shares nothing with the CUDA library).

Key t of sequence s is row t % page_size of page table[s, t // page_size].  New rows are turned by their position (every pair of
dimensions is a complex number that is multiplied by e^(i * position * inv_freq)) and put at their slot; one token's attention is the
softmax-weighted mean of its sequence's values.
"""
import numpy as np


def rotate(x, position, inv_freq, interleaved=False):
    """x [..., heads, d] at position [...]; the first 2 * len(inv_freq) dimensions turn."""
    x = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    if half == 0:
        return x
    turn = np.exp(1j * np.asarray(position, np.float64)[..., None, None] * np.asarray(inv_freq, np.float64))
    re, im = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    z = (re + 1j * im) * turn
    if interleaved:
        x[..., 0:2 * half:2], x[..., 1:2 * half:2] = z.real, z.imag
    else:
        x[..., :half], x[..., half:2 * half] = z.real, z.imag
    return x


def slots(first, n, table_row, page_size, n_pages):
    """(page, row) of slots first .. first + n - 1 of one sequence; page -1 where the slot or its page does not exist."""
    out = []
    for t in range(first, first + n):
        page = int(table_row[t // page_size]) if 0 <= t < len(table_row) * page_size else -1
        out.append((page if 0 <= page < n_pages else -1, t % page_size))
    return out


def ordered(pages, table_row, length):
    """Rows 0 .. length - 1 of one sequence, [length, heads, d] in fp64; rows of pages that do not exist are 0."""
    n_pages, page_size = pages.shape[:2]
    rows = [pages[p, r].astype(np.float64) if p >= 0 else np.zeros(pages.shape[2:]) for p, r in slots(0, length, table_row, page_size, n_pages)]
    return np.stack(rows) if rows else np.zeros((0,) + pages.shape[2:])


def token_attention(q, k, v, sm_scale):
    """q [Hq, d], k and v [length, Hkv, d] of one sequence -> out [Hq, d], lse [Hq]; length 0 gives 0 and -inf."""
    Hq, d = q.shape
    length, Hkv = k.shape[:2]
    if length == 0:
        return np.zeros((Hq, d)), np.full(Hq, -np.inf)
    out, lse = np.empty((Hq, d)), np.empty(Hq)
    for h in range(Hq):
        g = h // (Hq // Hkv)
        s = sm_scale * (k[:, g].astype(np.float64) @ q[h].astype(np.float64))
        top = s.max()
        w = np.exp(s - top)
        out[h], lse[h] = w @ v[:, g].astype(np.float64) / w.sum(), top + np.log(w.sum())
    return out, lse

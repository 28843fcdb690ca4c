"""Float64 oracle of the bf16 paged cache's operators for long and shared contexts (test infrastructure only)."""
import numpy as np

PAGE = 16


def reserve(table, seq_len, n_rows, free, taken, share=None):
    """The page table, the slots and n_taken after osprey_kv_reserve of a call without errors."""
    table, slots = table.copy(), []
    for b, (length, n) in enumerate(zip(seq_len, n_rows)):
        held = -(-length // PAGE)
        if share is not None and share[b] not in (-1, b):
            table[b, :held] = table[share[b], :held]
        end = -(-(length + n) // PAGE)
        table[b, held:end] = free[taken:taken + end - held]
        taken += end - held
        slots += [int(table[b, t // PAGE]) * PAGE + t % PAGE for t in range(length, length + n)]
    return table, np.array(slots, np.int64), taken


def reserve_held(table, seq_len, n_rows, free, taken, held, share=None):
    """The page table, the slots, n_taken and held after osprey_kv_reserve_held of a call without errors."""
    table, slots, held = table.copy(), [], list(held)
    for b, (length, n) in enumerate(zip(seq_len, n_rows)):
        if share is not None and share[b] not in (-1, b):
            table[b, :length // PAGE] = table[share[b], :length // PAGE]
            held[b] = max(held[b], length // PAGE)
        while held[b] * PAGE < length + n:
            table[b, held[b]] = free[taken]
            held[b], taken = held[b] + 1, taken + 1
        slots += [int(table[b, t // PAGE]) * PAGE + t % PAGE for t in range(length, length + n)]
    return table, np.array(slots, np.int64), taken, held


def exponent(peak):
    """Smallest e >= -100 with peak <= 127 * 2^e."""
    e = -100
    while peak > 127 * 2.0 ** e:
        e += 1
    return e


def bound(k):
    """Codes [2, hd] and scale of a page's keys k [slots, hd]."""
    if not np.isfinite(k).all():
        return np.zeros((2, k.shape[1])), np.nan
    s = 2.0 ** exponent(np.abs(k).max())
    return np.stack([np.ceil(k.max(0) / s), np.floor(k.min(0) / s)]), s


def scores(q, codes, scale):
    """Scores [pages] of a group's queries q [G, hd] against codes [pages, 2, hd] and scales [pages]."""
    c = np.rint(q / 2.0 ** exponent(np.abs(q).max())) if np.isfinite(q).all() else np.zeros_like(q)
    up, down = np.maximum(c, 0).sum(0), np.minimum(c, 0).sum(0)
    return np.where(np.isnan(scale), np.inf, (codes[:, 0] @ up + codes[:, 1] @ down) * np.where(np.isnan(scale), 1, scale))


def select(score, page, n, first, last):
    """The n pages of 0 .. page to read: the first, the last, then the largest scores, the lower page first."""
    key = [(2 if p < first or p > page - last else 1, score[p]) for p in range(page + 1)]
    return sorted(sorted(range(page + 1), key=lambda p: (-key[p][0], -key[p][1], p))[:n])


def attend(q, k, v, see):
    """Rows q [n, Hq, hd] over keys [T, Hkv, hd], see [n, Hkv, T]: the output, the mean distance of the values from it
    under the weights, and the largest sum of products' magnitudes of a score."""
    n, Hq, hd = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, spread, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, Hq, 1))
    for i in range(n):
        for h in range(Hq):
            on = np.nonzero(see[i, h // G])[0]
            if not len(on):
                continue
            kk, vv = k[on, h // G], v[on, h // G]
            s = kk @ q[i, h] / np.sqrt(hd)
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vv
            spread[i, h] = w @ np.abs(vv - out[i, h])
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() / np.sqrt(hd)
    return out, spread, size

"""The prompt path: blocks of a step's tokens, rotary positions, attention of a chunk.

Block tables and the free list follow Section 3 (paged blocks, a block map per request): request
by request in order, each taking its blocks from the top of the free list, or none once the list
has run short.  Rotary positions turn each pair of dimensions by position times frequency.  A
chunk's query at position p sees the tokens of its request's prefix and those from its first key
to p.
"""
import numpy as np

BLOCK = 16


def plan_blocks(table, owned, lens, indptr, free, free_count, total_q):
    """(table, owned, lens, free_count, granted, slots) after serving the requests in order."""
    table, owned, lens = np.array(table), np.array(owned), np.array(lens)
    left = int(free_count)
    room = left              # less every need so far, granted or not
    granted = np.zeros(len(lens), np.int32)
    slots = np.full(total_q, -1, np.int32)
    for r in range(len(lens)):
        n = int(indptr[r + 1] - indptr[r])
        blocks = -(-(int(lens[r]) + n) // BLOCK)
        if blocks > table.shape[1]:
            continue
        need = max(0, blocks - int(owned[r]))
        room -= need
        if need and room < 0:
            continue
        for _ in range(need):
            left -= 1
            table[r, owned[r]] = free[left]
            owned[r] += 1
        for j in range(n):
            t = int(lens[r]) + j
            slots[indptr[r] + j] = table[r, t // BLOCK] * BLOCK + t % BLOCK
        lens[r] += n
        granted[r] = 1
    return table, owned, lens, left, granted, slots


def trim_blocks(table, owned, keep, free, free_count):
    """(owned, free, free_count): blocks past the kept tokens pushed request by request."""
    owned, free, left = np.array(owned), np.array(free), int(free_count)
    for r in range(len(owned)):
        kept = min(int(owned[r]), -(-int(keep[r]) // BLOCK))
        for b in range(kept, int(owned[r])):
            if left < len(free):
                free[left] = table[r, b]
                left += 1
        owned[r] = kept
    return owned, free, left


def rotate(x, positions, inv_freq, sections=None, interleaved=False):
    """x [rows][heads][D] turned; positions [axes][rows] integers, inv_freq [pairs] as given."""
    x = np.array(x, np.float64)
    positions = np.atleast_2d(positions)
    pairs = len(inv_freq)
    axis = np.repeat(np.arange(len(positions)), [pairs] if sections is None else sections)
    for i in range(pairs):
        angle = positions[axis[i]].astype(np.float64) * float(inv_freq[i])
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        u, w = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        a, b = x[..., u].copy(), x[..., w].copy()
        x[..., u] = a * c - b * s
        x[..., w] = a * s + b * c
    return x


def chunk_attention_request(q, k, v, length, scale, softcap=0.0, slopes=None, first_keys=None,
                            prefix=0, valid=None):
    """q [n][Hq][D] at positions length - n .., k [length][Hkv][D], v [length][Hkv][Dv]; returns
    [n][Hq][Dv].

    first_keys [n]; valid [length] truth values (tokens of an unreadable block are not seen).
    Tokens that a row does not see are left out, not weighted by zero."""
    n, hq, d = q.shape
    hkv = k.shape[1]
    out = np.zeros((n, hq, v.shape[-1]))
    t = np.arange(length)
    for j in range(n):
        p = length - n + j
        lo = 0 if first_keys is None else int(first_keys[j])
        see = (t < prefix) | ((t <= p) & (t >= lo))
        if valid is not None:
            see &= valid
        if not see.any():
            continue
        with np.errstate(all="ignore"):
            x = scale * np.matmul(q[j].reshape(hkv, hq // hkv, d), k[see].transpose(1, 2, 0))
            if softcap:
                x = softcap * np.tanh(x / softcap)
            if slopes is not None:
                x = x - np.reshape(slopes, (hkv, -1, 1)) * np.abs(p - t[see])
            top = x.max(-1, keepdims=True)
            w = np.exp(x - np.where(top == -np.inf, 0.0, top))
            total = w.sum(-1, keepdims=True)
            o = np.matmul(w, v[see].transpose(1, 0, 2)) / total
        out[j] = np.where(total == 0, 0.0, o).reshape(hq, -1)
    return out

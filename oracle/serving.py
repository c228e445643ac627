"""The serving operators in numpy fp64: paged cache write with head norms and rotation, attention of one new token
per row over the paged cache, block and slot assignment.

The paper fine-tunes by forward passes and evaluates the tuned model by letting it answer (Sec. 4.1); a paged cache is
this library's way of serving that.  The linear of a decode step is linear.perturbed_linear at sign 0.

A cache is a pair of arrays [n_blocks][n_kv_heads][block_size][head_dim] holding values (an 8-bit cache: code * scale).
"""
import numpy as np


def rotate(x, positions, theta):
    """x [T][H][dh]: rotate pairs (i, i + dh/2) by position * theta**(-2i/dh)."""
    dh = x.shape[-1]
    half = dh // 2
    ang = np.asarray(positions, np.float64)[:, None] * theta ** (-np.arange(half) * 2.0 / dh)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def head_norm(x, gain, eps):
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * gain


def qk_norm_rope(q, k, positions, q_gain, k_gain, eps, theta):
    """The new rows' queries and keys as they enter the attention; gains or theta None = left out."""
    q, k = np.asarray(q, np.float64), np.asarray(k, np.float64)
    if q_gain is not None:
        q = head_norm(q, np.asarray(q_gain, np.float64), eps)
    if k_gain is not None:
        k = head_norm(k, np.asarray(k_gain, np.float64), eps)
    if theta is not None:
        q, k = rotate(q, positions, theta), rotate(k, positions, theta)
    return q, k


def write_cache(pages, rows, slots):
    """pages[slot // block][:][slot % block] = rows, in place; negative slots are padding."""
    block = pages.shape[2]
    for t, slot in enumerate(slots):
        if slot >= 0:
            pages[slot // block, :, slot % block] = rows[t]


def paged_attention(q, k_pages, v_pages, table, row_seq, positions, scale):
    """out [R][H][dh] and, for error bounds, sum_j p_j |v_j|; a row with a negative position gives zeros."""
    R, H, dh = q.shape
    n_blocks, Hkv, block, _ = k_pages.shape
    out, spread = np.zeros((R, H, dh)), np.zeros((R, H, dh))
    for r in range(R):
        if positions[r] < 0:
            continue
        j = np.arange(positions[r] + 1)
        page = table[row_seq[r]][j // block]
        for h in range(H):
            kv = h // (H // Hkv)
            k = k_pages[page, kv, j % block].astype(np.float64)
            v = v_pages[page, kv, j % block].astype(np.float64)
            s = k @ q[r, h].astype(np.float64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h], spread[r, h] = p @ v, p @ np.abs(v)
    return out, spread


def assign_slots(lens, new, table, free, free_count, block, max_rows):
    """One request after the other: finished ones push their blocks, growing ones pop what they lack, rows are numbered.
    Returns a dict of the new state, or None when the step cannot be served (nothing changes then)."""
    lens, table, free = list(map(int, lens)), np.array(table), np.array(free)
    width, top = table.shape[1], int(free_count)
    held = [-(-n // block) for n in lens]
    need = sum(-(-(n + a) // block) - h for n, a, h in zip(lens, new, held) if a > 0)
    back = sum(h for a, h in zip(new, held) if a < 0)
    rows = sum(int(a) for a in new if a > 0)
    too_wide = any(n < 0 or -(-(n + max(int(a), 0)) // block) > width for n, a in zip(lens, new))
    if too_wide or top < 0 or top + back > len(free) or need > top + back or rows > max_rows:
        return None
    for r, a in enumerate(new):
        if a < 0:
            for j in range(held[r]):
                free[top] = table[r, j]
                top += 1
    row_seq, positions, slots = [], [], []
    for r, a in enumerate(new):
        if a < 0:
            lens[r] = 0
            continue
        for _ in range(int(a)):
            if lens[r] % block == 0:
                top -= 1
                table[r, lens[r] // block] = free[top]
            row_seq.append(r)
            positions.append(lens[r])
            slots.append(int(table[r, lens[r] // block]) * block + lens[r] % block)
            lens[r] += 1
    pad = [-1] * (max_rows - rows)
    return {"row_seq": row_seq + pad, "positions": positions + pad, "slots": slots + pad, "lens": lens, "free_count": top,
            "table": table, "free": free}

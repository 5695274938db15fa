"""The key/value cache of an inference engine, as the engine knobs see it:
places of a step's new tokens in a cache of blocks, the 8-bit storage of keys
and values, and attention over what the blocks hold.  The knobs (block size,
most requests and tokens per step, chunked prefill) are those of the paper's
Table 1; the operations are the usual ones of such engines, written from their
definitions, request by request, in float64 and Python integers.
"""
import numpy as np

INT32_MAX = 2 ** 31 - 1


def assign(context_len, new_len, block_table, free_blocks, block_size, max_tokens):
    """Returns (block_table, query_start, seq_len, positions, slots, counts).

    Requests are taken in order.  A request whose tokens would end past
    max_tokens or whose blocks exceed the table's columns asks for no blocks
    and is not admitted; otherwise its new blocks come from the front of what
    the requests before it asked for, and it is admitted if they are there."""
    table = np.array(block_table, dtype=np.int64)
    rows, cols = table.shape
    start, asked, admitted, taken, tok = [0], 0, 0, 0, 0
    seq_len = []
    positions = np.full(max_tokens, -1, dtype=np.int64)
    slots = np.full(max_tokens, -1, dtype=np.int64)
    for r in range(rows):
        c, n = max(int(context_len[r]), 0), max(int(new_len[r]), 0)
        first, tok = tok, tok + n
        start.append(min(tok, INT32_MAX))
        used, total = -(-c // block_size), -(-(c + n) // block_size)
        if tok > max_tokens or total > cols:
            seq_len.append(0)
            continue
        mine = (asked, asked + total - used)
        asked = mine[1]
        if total > used and asked > len(free_blocks):
            seq_len.append(0)
            continue
        admitted += 1
        taken = asked if total > used else taken
        seq_len.append(c + n)
        table[r, used:total] = free_blocks[mine[0]:mine[1]]
        for j in range(n):
            p = c + j
            positions[first + j] = p
            b = table[r, p // block_size]
            if b >= 0:
                slots[first + j] = b * block_size + p % block_size
    counts = [min(tok, INT32_MAX), admitted, taken, min(asked, INT32_MAX)]
    return table, np.array(start), np.array(seq_len), positions, slots, np.array(counts)


def round_e4m3(x):
    """Nearest OCP e4m3 value (ties to even), limited to +-448; NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.floor(np.log2(np.abs(np.where(x == 0, 1.0, x))))
        e = np.clip(np.where(np.isfinite(e), e, 0), -6, 8)
        q = np.exp2(e - 3)
        y = np.round(np.where(np.isfinite(x), x, 0) / q) * q
    y = np.where(np.isinf(x), np.sign(x) * 448.0, y)
    return np.where(np.isnan(x), np.nan, np.clip(y, -448.0, 448.0))


def write(x, slots, cache, store):
    """cache (blocks, heads, block_size, dim) with x (tokens, heads, dim), passed
    through ``store``, at its slots; slots outside are skipped."""
    out = np.array(cache, dtype=np.float64)
    bs = out.shape[2]
    for t, s in enumerate(slots):
        if 0 <= s < out.shape[0] * bs:
            out[s // bs, :, s % bs] = store(x[t])
    return out


def attention(q, k_cache, v_cache, block_table, query_start, seq_len, scale, window=0):
    """Attention of every request's queries over its cached positions.

    Returns (out, spread, reach): out (tokens, heads, dim), NaN rows where no
    request owns the row; spread = sum of the weights times |v| per element,
    and reach (tokens, heads) = the largest scale * sum |q k| of a visible key,
    for error bounds."""
    tokens, heads, dim = q.shape
    blocks, kv_heads, bs, _ = k_cache.shape
    out = np.full((tokens, heads, dim), np.nan)
    spread = np.full((tokens, heads, dim), np.nan)
    reach = np.zeros((tokens, heads))
    for r in range(len(seq_len)):
        lo, hi = min(int(query_start[r]), tokens), min(int(query_start[r + 1]), tokens)
        n = int(query_start[r + 1]) - int(query_start[r])
        held = min(int(seq_len[r]), block_table.shape[1] * bs)
        at = np.arange(max(held, 0))
        block = np.asarray(block_table[r], dtype=np.int64)[at // bs]
        real = (block >= 0) & (block < blocks)
        at, block = at[real], block[real]
        for t in range(lo, hi):
            p = int(seq_len[r]) - n + (t - int(query_start[r]))
            see = at <= p
            if window:
                see &= at > p - window
            a, b = at[see], block[see]
            for h in range(heads):
                g = h // (heads // kv_heads)
                if a.size == 0:
                    out[t, h] = spread[t, h] = 0.0
                    continue
                k, v = k_cache[b, g, a % bs], v_cache[b, g, a % bs]
                s = scale * (k @ q[t, h])
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ v
                spread[t, h] = w @ np.abs(v)
                reach[t, h] = scale * (np.abs(k) @ np.abs(q[t, h])).max()
    return out, spread, reach


def attention_bound(out, spread, reach, keys, dim, out_bits, weight_bits, v_max):
    """How far a result may be off that sums in float (24 bits), rounds the
    softmax's weights to ``weight_bits`` and the result to ``out_bits``.

    * the result's own rounding: 2^-out_bits |out|;
    * every weight is off by at most 2^-weight_bits of itself (numerator and,
      summed, denominator): 2^-weight_bits (spread + |out|);
    * weights below the 16-bit formats' normal range (2^-14 of the largest)
      are off by at most 2^-25 of the largest: keys 2^-25 v_max;
    * a score is a float sum of dim products: off by (dim + 4) 2^-24 reach at
      most, and the exponential by 2^-21, in numerator and denominator;
    * the sums over the keys, keys 2^-24 of spread (and of the denominator)."""
    weight = 2.0 ** -weight_bits + (dim + 4) * 2.0 ** -24 * reach[..., None] + 2.0 ** -21 + keys * 2.0 ** -24
    return 1.05 * (2.0 ** -out_bits * np.abs(out) + weight * (spread + np.abs(out))) + keys * 2.0 ** -25 * v_max + 1e-30



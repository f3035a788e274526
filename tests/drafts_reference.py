"""Plain implementations of the calls on drafted tokens, from their definitions (NumPy, on the host, 64 bits)."""
import numpy as np

import q8_reference as ref


def above(parents, t):
    """Draft t and the drafts above it, t first."""
    line = [t]
    while 0 <= parents[line[-1]] < line[-1] and line[-1] > 0:
        line.append(parents[line[-1]])
    return line


def prepare(parents, n_drafts, first):
    """parents [B, T] -> bits [B, T, T], positions [B, T]."""
    B, T = parents.shape
    bits, positions = np.zeros((B, T, T), bool), np.zeros((B, T), np.int64)
    for b in range(B):
        positions[b] = first[b]
        for t in range(min(max(n_drafts[b], 0), T)):
            line = above(parents[b], t)
            bits[b, t, line] = True
            positions[b, t] += len(line) - 1
    return bits, positions


def words(bits):
    """[.., T] truth values -> i32 words [.., ceil(T / 32)]."""
    T = bits.shape[-1]
    w = -(-T // 32)
    full = np.zeros(bits.shape[:-1] + (32 * w,), np.uint64)
    full[..., :T] = bits
    v = (full.reshape(*bits.shape[:-1], w, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return v.astype(np.uint32).view(np.int32)


def accept(parents, n_drafts, tokens, target):
    """-> per sequence the list of accepted drafts."""
    found = []
    for b in range(len(parents)):
        n = min(max(n_drafts[b], 0), parents.shape[1])
        path = [0] if n else []
        while path:
            at = path[-1]
            children = [t for t in range(at + 1, n) if parents[b, t] == at and tokens[b, t] == target[b, at]]
            if not children:
                break
            path.append(children[0])
        found.append(path)
    return found


def attend(q, keys, scale):
    """q [rows, 128]; keys: a list of (k [n, 128], v [n, 128], seen [rows, n] or None, scales of v [n]).

    -> out, lse, and how far the outputs and lse may be off, from the arithmetic:
    - a score is a sum of 128 products in fp32 (each operand exact), times two factors: off by 130 roundings of sum |q k|;
    - the score in base 2 plus the value's scale's logarithm is rounded once, the difference to the maximum once: 2^-23 of its size, and
      that logarithm is off by 2^-22 of itself (a function of the GPU);
    - so a probability is off by d = the sum of these times ln 2 of itself, the exponential by 2^-22 more, and where it multiplies a
      value by 2^-11 (f16), or 2^-33 of the largest of its row if that is more (f16's subnormals end at 2^-25, the largest is 2^8 or more);
    - fp32 sums of n terms: n 2^-24 of the sum of their magnitudes.
    """
    rows = len(q)
    k = np.concatenate([x[0] for x in keys])
    v = np.concatenate([x[1] for x in keys])
    sv = np.concatenate([x[3] for x in keys])
    seen = np.concatenate([np.ones((rows, len(x[0])), bool) if x[2] is None else x[2] for x in keys], 1)
    n = k.shape[0]
    out, lse = np.zeros((rows, 128)), np.full(rows, -np.inf)
    off, off_lse = np.zeros((rows, 128)), np.zeros(rows)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for r in range(rows):
            s = np.flatnonzero(seen[r])
            if not len(s):
                continue
            kk, vv, vs = k[s], v[s], sv[s]
            x = kk @ q[r] * scale
            m = x.max()
            p = np.exp(x - m)
            l = p.sum()
            w = p / l
            out[r], lse[r] = w @ vv, m + np.log(l)
            size = np.abs(x) / np.log(2) + np.abs(np.log2(vs))
            d = (np.abs(kk) @ np.abs(q[r]) * scale * 132 * 2.0 ** -24 + np.log(2) * (size + size.max()) * 2.0 ** -22 + 2.0 ** -21).max()
            weight = w * vs                                       # what is largest decides where f16 ends
            tail = 2.0 ** -33 * weight.max() / vs
            mean = w @ np.abs(vv)
            off[r] = mean * (2 * d + 2.0 ** -11 + (n + 64) * 2.0 ** -23) + tail @ np.abs(vv)
            off[r] += np.abs(out[r]) * 2.0 ** -11 + 2.0 ** -25     # the output's own rounding
            off_lse[r] = d + (n + 64) * 2.0 ** -23 + np.abs(lse[r]) * 2.0 ** -22
    return out, lse, off, off_lse


def commit(codes, scales, table, old, new, rows):
    """In place: rows[b][:new[b]] ([T, H, 128], 64-bit values) behind old[b] tokens of sequence b, as q8_reference.append; the scale of a page
    that is appended to, if it is no power of two, goes to the next one, and the product of a code and the factor is rounded in fp32 first."""
    n_pages, H, P, _ = codes.shape
    for b in range(len(old)):
        held = min(max(old[b], 0), table.shape[1] * P)
        o, n = held % P, min(new[b], table.shape[1] * P - held)
        if o and n > 0 and 0 <= table[b, held // P] < n_pages:
            page = table[b, held // P]
            for h in range(H):
                s = abs(np.float32(scales[page, h]))
                top = max(ref.scale_of(rows[b][:min(n, P - o), h]), 2.0 ** np.ceil(np.log2(max(float(s), 2.0 ** -64))))
                v = ref.VALUES[codes[page, h, :o]].astype(np.float32) * np.float32(np.float32(scales[page, h]) / np.float32(top))
                codes[page, h, :o] = np.where(np.isnan(v), codes[page, h, :o], ref.encode(v))
                scales[page, h] = top
        ref.append(codes, scales, table[b:b + 1], [old[b]], [new[b]], [0], rows[b])

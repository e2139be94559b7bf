"""64-bit references of the 8-bit cache's operators, from their definitions, on the CPU.

Codes are E4M3 bytes, scales E8M0 bytes; pools [layer][page][slot][kv_head][channel], scales
[layer][page][block][kv_head]."""
import numpy as np

import oracle


def code_values():
    """Value of every E4M3 byte."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (8.0 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v[(c & 127) == 127] = np.nan
    return np.where(c & 128, -v, v)


VALUES = code_values()


def encode(x):
    """E4M3 byte nearest to x, ties to even; NaN for what is not finite.  |x| <= 448."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -30))), -6.0)
    n = np.rint(a * 2.0 ** (3 - e))                     # in steps of 2^(e - 3); 16 carries into the next binade
    code = np.where(e > -6, (e + 7) * 8 + n - 8, n).astype(np.int64)   # below 2^-6 and in [2^-6, 2^-5): n itself
    assert (code <= 126).all()
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(codes, exponents):
    """Values of codes under exponent bytes that broadcast against them."""
    return VALUES[codes] * 2.0 ** (exponents.astype(np.float64) - 127)


def need(top):
    """Smallest exponent byte in [1, 254] whose scale holds `top`."""
    e = 1
    while 448.0 * 2.0 ** (e - 127) < top:
        e += 1
    return e


def logical(pool, scale, row, n):
    """[layer][kv_head][n][channel] values of one sequence through its block-table row."""
    p = np.arange(n)
    page, block = pool.shape[2], pool.shape[2] // scale.shape[2]
    ids, at = row[p // page], p % page
    return decode(pool[:, ids, at], scale[:, ids, at // block][..., None]).transpose(0, 2, 1, 3)


def bf16_bits(x):
    """bf16 bit patterns of values that bf16 holds exactly."""
    f = np.asarray(x, np.float32)
    assert np.array_equal(f.astype(np.float64), x, equal_nan=True)
    u = np.ascontiguousarray(f).view(np.uint32)
    assert not np.any((u & 0xffff)[~np.isnan(f)])
    return (u >> 16).astype(np.uint16)


def turned(x, delta, omega, offset, style):
    """Rows [..., channel] with the rotary slice at `offset` turned by delta positions, and the bound of the fp32
    rotation's error: c and s are rounded (2^-24 each, the angle's own error is smaller still), the product and
    the sum are rounded, together below 2^-22 (|a| + |b|)."""
    r = 2 * len(omega)
    x = x.copy()
    err = np.zeros_like(x)
    if delta == 0:
        return x, err
    c, s = np.cos(delta * omega), np.sin(delta * omega)
    ia = offset + (np.arange(r // 2) if style == 0 else 2 * np.arange(r // 2))
    ib = ia + (r // 2 if style == 0 else 1)
    a, b = x[..., ia].copy(), x[..., ib].copy()
    with np.errstate(invalid="ignore"):
        x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
        err[..., ia] = err[..., ib] = 2.0 ** -22 * (np.abs(a) + np.abs(b))
    return x, err


def store(src, pool, scale, segs, kv_len, table, omega, offset, style, capacity, turn):
    """One tensor's splice: the expected pool, scales and, per byte, the lowest and highest code that the fp32
    rotation's error allows.  segs: (src_slot0, seq, n_tokens, src_pos0, dst_pos0)."""
    L, P, page, H, d = pool.shape
    block = page // scale.shape[2]
    pool, scale = pool.copy(), scale.copy()
    lo, hi = pool.copy(), pool.copy()
    for seq in range(table.shape[0]):
        where = {}                                       # slot -> (source slot, delta)
        for src0, sq, n, pos0, dst0 in reversed(segs):
            if sq == seq:
                for i in range(n):
                    if 0 <= dst0 + i < capacity and 0 <= src0 + i < src.shape[2]:
                        where[dst0 + i] = (src0 + i, dst0 - pos0)
        for b in sorted({t // block for t in where}):
            pg, first = table[seq, b * block // page], b * block % page
            if not 0 <= pg < P:
                continue
            got = [t for t in range(b * block, (b + 1) * block) if t in where]
            kept = [t for t in range(b * block, min((b + 1) * block, kv_len[seq], capacity)) if t not in where]
            rows = [turned(src[:, :, where[t][0]], where[t][1] if turn else 0, omega, offset, style) for t in got]
            x, err = np.stack([r[0] for r in rows], 1), np.stack([r[1] for r in rows], 1)   # [L, rows, H, d]
            for l in range(L):
                for h in range(H):
                    v = x[l, :, h]
                    e = need(np.abs(v[np.isfinite(v)]).max(initial=0.0))
                    old = int(scale[l, pg, first // block, h])
                    if kept:
                        e = max(e, old)
                    up = 2.0 ** (127 - e)
                    at = [t % page for t in got]
                    with np.errstate(invalid="ignore"):
                        pool[l, pg, at, h] = encode(v * up)
                        lo[l, pg, at, h] = encode((v - err[l, :, h]) * up)
                        hi[l, pg, at, h] = encode(np.clip((v + err[l, :, h]) * up, -448, 448))
                    if kept and e > old:
                        at = [t % page for t in kept]
                        for z in (pool, lo, hi):
                            z[l, pg, at, h] = encode(VALUES[pool[l, pg, at, h]] * 2.0 ** (old - e))
                    scale[l, pg, first // block, h] = e
    return pool, scale, lo, hi


def check_codes(got, want, lo, hi, what=""):
    """Every code is the expected one, or (near a rounding boundary) between those that the error allows.  Returns
    how many are not the expected one.  (NaN codes compare by being NaN; a zero's sign is free where both are 0.)"""
    g, w = VALUES[got], VALUES[want]
    same = (got == want) | (np.isnan(g) & np.isnan(w)) | (g == w)
    a, b = VALUES[lo], VALUES[hi]
    ok = same | ((g >= np.minimum(a, b)) & (g <= np.maximum(a, b)))
    assert ok.all(), "%s: %d codes wrong, e.g. got %s want %s" % (what, (~ok).sum(), g[~ok][:4], w[~ok][:4])
    return int((~same).sum())


def attention(q_bits, pool_k, pool_v, ks, vs, row, vrow, q_pos, kv, scale, window=0):
    """The oracle's attention of one layer's queries [rows][H][d] over one sequence, each pool [page][slot][kv_head][d]."""
    k = bf16_bits(logical(pool_k[None], ks[None], row, kv))[0]
    v = bf16_bits(logical(pool_v[None], vs[None], vrow, kv))[0]
    return oracle.attention(np.ascontiguousarray(q_bits), k, v, q_pos, kv, scale, window=window)


# ---- pages ----------------------------------------------------------------------

def free(ref, table, seqs, keep, page):
    ref, table, bad = ref.copy(), table.copy(), False
    for i, s in enumerate(seqs):
        if not 0 <= s < len(table):
            bad = True
            continue
        first = 0 if keep is None else -(-max(int(keep[i]), 0) // page)
        for e in range(first, table.shape[1]):
            p, table[s, e] = table[s, e], -1
            if p == -1:
                continue
            if 0 <= p < len(ref) and ref[p] > 0:
                ref[p] -= 1
            else:
                bad = True
    return ref, table, bad


def fork(ref, table_in, table_out, forks, page, same):
    """Counts, table, copies (source, destination, slots) and whether anything is flagged."""
    ref, out, bad, copies = ref.copy(), table_out.copy(), False, []
    n, width = table_in.shape

    def fine(f):
        return 0 <= f[0] < n and 0 <= f[1] < n and 0 <= f[2] <= width * page

    children = [f[1] for f in forks if fine(f)]
    free_pages = iter(np.nonzero(ref == 0)[0].tolist())
    for i, f in enumerate(forks):
        if not fine(f) or f[1] in [g[1] for g in forks[:i] if fine(g)] or (same and f[0] in children):
            bad = True
            continue
        whole, tail = f[2] // page, f[2] % page
        row = np.full(width, -1, np.int32)
        row[:whole] = table_in[f[0], :whole]
        for p in row[:whole]:
            if 0 <= p < len(ref):
                ref[p] += 1
            else:
                bad = True
        if tail:
            p, new = table_in[f[0], whole], None
            if 0 <= p < len(ref):
                new = next(free_pages, None)
            if new is None:
                bad = True
            else:
                row[whole] = new
                ref[new] = 1
                copies.append((int(p), new, tail))
        out[f[1]] = row
    return ref, out, copies, bad


def compact(ref, table):
    n = int((ref > 0).sum())
    to = np.full(len(ref), -1, np.int32)
    holes = iter([p for p in range(n) if ref[p] <= 0])
    copies, after = [], np.zeros_like(ref)
    for p in range(len(ref)):
        if ref[p] > 0:
            to[p] = p if p < n else next(holes)
            after[to[p]] = ref[p]
            if to[p] != p:
                copies.append((p, int(to[p])))
    inside = (table >= 0) & (table < len(ref))
    renamed = np.where(inside, to[np.clip(table, 0, len(ref) - 1)], table)
    return after, renamed.astype(np.int32), copies, n, bool((inside & (renamed == -1)).any())

"""The 4-bit KV cache in plain numpy, 64 bits: its rows, and attention over the
values they stand for (the definitions in include/wide.h; no code shared with
the library)."""
import numpy as np

HD = 128


def row_bytes(qg):
    return HD // 2 + 4 * (HD // qg)


def bf16_bits_to_f64(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _next_down_bf16(f64):
    """Largest bf16 value <= f64 (finite, below 2^127 in size), by stepping the pattern."""
    bits = f64.astype(np.float32).view(np.uint32) >> 16        # towards zero
    val = bf16_bits_to_f64(bits)
    return np.where(val > f64, bf16_bits_to_f64(bits + 1), val)  # (negative: one pattern further from zero)


def _nearest_bf16(w, div):
    """w / div (w >= 0) to the nearest bf16, ties to even, decided on products."""
    guess = (w / div).astype(np.float32).view(np.uint32) >> 16
    best = None
    for cand in (np.maximum(guess.astype(np.int64) - 1, 0), guess.astype(np.int64), guess.astype(np.int64) + 1):
        v = bf16_bits_to_f64(cand.astype(np.uint32))
        dist = np.abs(w - div * v)                             # exact: few bits either side near the candidates
        if best is None:
            best, bd, bb = v, dist, cand
        else:
            take = (dist < bd) | ((dist == bd) & (cand % 2 == 0) & (bb % 2 == 1))
            best, bd, bb = np.where(take, v, best), np.where(take, dist, bd), np.where(take, cand, bb)
    return best


def _bf16_bytes(f64):
    return (f64.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def quantize(x, qg):
    """fp64 rows [...][128] -> uint8 rows [...][row_bytes]."""
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, HD)
    ng = HD // qg
    out = np.zeros((flat.shape[0], row_bytes(qg)), np.uint8)
    bad = ~(np.abs(flat) < 2.0 ** 127).all(1)
    grp = np.where(bad[:, None], 0.0, flat).reshape(-1, ng, qg)
    low = _next_down_bf16(grp.min(2))
    with np.errstate(invalid="ignore", over="ignore"):
        scale = _nearest_bf16(grp.max(2) - low, 15.0)
    scale = np.where(scale < 2.0 ** -126, 0.0, scale)
    d = grp - low[..., None]
    code = np.zeros(d.shape, np.int64)
    for k in range(15):
        border = scale[..., None] * (k + 0.5)
        code += np.where(k % 2 == 1, d >= border, d > border) & (scale[..., None] > 0)
    code = code.reshape(-1, HD)
    for dim in range(HD):
        l, e, m = dim % 32 // 2, dim % 2, dim // 32
        n = m + 4 * e
        out[:, 4 * l + n // 2] |= (code[:, dim] << (4 * (n % 2))).astype(np.uint8)
    sb, lb = _bf16_bytes(scale), _bf16_bytes(low)
    lb = np.where((low == 0) & np.signbit(grp.min(2)), 0x8000, lb).astype(np.uint16)
    out[bad] = 0
    sb[bad], lb[bad] = 0, 0x7fc0
    out[:, 64:] = np.concatenate([sb, lb], 1).view(np.uint8)
    return out.reshape(x.shape[:-1] + (row_bytes(qg),))


def parts(rows, qg):
    """uint8 rows -> (scale, low, code), fp64, each [...][128]."""
    ng = HD // qg
    dim = np.arange(HD)
    n = dim // 32 + 4 * (dim % 2)
    code = rows[..., 4 * (dim % 32 // 2) + n // 2] >> (4 * (n % 2)).astype(np.uint8) & 15
    meta = np.ascontiguousarray(rows[..., 64:]).view(np.uint16)
    scale = np.repeat(bf16_bits_to_f64(meta[..., :ng]), qg, -1)
    low = np.repeat(bf16_bits_to_f64(meta[..., ng:]), qg, -1)
    return scale, low, code.astype(np.float64)


def values(rows, qg):
    s, low, c = parts(rows, qg)
    return low + s * c


def where_rows(n_seq, T, L, pos, kv_len):
    """[(row, sequence, position)] of the rows a call touches."""
    out = []
    for b in range(n_seq):
        end = L if kv_len is None else min(int(kv_len[b]), L)
        for i in range(T):
            p = (0 if pos is None else int(pos[b])) + i
            if 0 <= p < end:
                out.append((b * T + i, b, p))
    return out


def attention(q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, head_major):
    """o and its allowed error, fp64 [B][n_q*128].

    The error, with u = 2^-24 and every product exact but for fp32 sums:
      scores: a sum of 128 terms up to (16 + 15) s|q| and of the groups' low and
        offset terms (|low| + 16 s) sum|q|, in fp32, in any order: each of at
        most 160 additions off by u of at most E = sum_d (47 s + |low|)|q|; one
        more rounding of the scaled exponent.  The three bf16 parts of sum(q)
        hold 24 bits of it: u of the same again.
        Of q, its two e4m3 terms leave up to 2^-22 of the head's largest value
        where a value is below 2^-14 of it: at most 15 s 2^-22 max|q| in each
        dimension, no more than the sums' bound even if one dimension holds all
        of |q| (15/47 * 128 * 4/162 = 1.0), and then the sums are short.
      p: exp2 to 2^-22 relative, times the error of its exponent; the maximum
        cancels in the quotient but for p's own exponent (twice the error).
      P.V: p s in two bf16 parts, 2^-16 of it, over terms up to (16 + 15) s p;
        fp32 sums over the keys: (keys + 64) u; all of sum_j w_j (47 s_j + |low_j|).
      the quotient 4 u, and half a step (2^-8) of the stored bf16 value.
    """
    B = q.shape[0]
    qpk, hpg = n_q // n_kv, group // HD
    out = np.zeros((B, n_q, HD))
    tol = np.zeros((B, n_q, HD))
    L = kc.shape[2 if head_major else 1]
    u = 2.0 ** -24
    for b in range(B):
        n = L if kv_len is None else max(0, min(L, int(kv_len[b])))
        for h in range(n_q):
            if n == 0 or not mask[b, h // hpg]:
                continue
            rows = [c[b, h // qpk, :n] if head_major else c[b, :n, h // qpk] for c in (kc, vc)]
            ks, kl, kcode = parts(rows[0], qg)
            vs, vl, vcode = parts(rows[1], qg)
            qh = q[b].reshape(n_q, HD)[h]
            sc = (kl + ks * kcode) @ qh / np.sqrt(HD)
            w = np.exp(sc - sc.max())
            w /= w.sum()
            out[b, h] = w @ (vl + vs * vcode)
            size = (47 * ks + np.abs(kl)) @ np.abs(qh) / np.sqrt(HD)
            e_sc = float(size.max()) * 162 * u
            mag = w @ (47 * vs + np.abs(vl))
            tol[b, h] = (2 * e_sc + 2.0 ** -22 + 2.0 ** -16 + (n + 64 + 4) * u) * mag * 1.01
    tol += 2.0 ** -8 * np.abs(out) + 2.0 ** -133
    return out.reshape(B, -1), tol.reshape(B, -1)

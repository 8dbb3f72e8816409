"""Plain 64-bit reference of the KV-page operators (numpy only), and the error bounds that their tests use."""
import numpy as np

E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}  # largest relative rounding error of a 16-bit type


def _e4m3_table():
    t = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        t[b] = np.nan if (b & 127) == 127 else (-v if b > 127 else v)
    return t


E4M3 = _e4m3_table()


def nearest_even(x, table):
    """Index into an increasing table of the nearest value, ties to the even index, saturating."""
    x = np.asarray(x, np.float64)
    i = np.clip(np.searchsorted(table, x), 1, len(table) - 1)
    lo, hi = table[i - 1], table[i]
    up = (x - lo > hi - x) | ((x - lo == hi - x) & (i % 2 == 0))
    return np.where(x >= table[-1], len(table) - 1, np.where(up, i, i - 1))


def quantise(x, g):
    """float32 [..., D] -> (codes uint8 [..., D], scale bytes uint8 [..., D/16]), by the format's 32-bit definition."""
    x = np.asarray(x, np.float32)
    g = np.float32(g)
    b = x.reshape(*x.shape[:-1], -1, 16)
    fin = np.isfinite(b).all(-1)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        a = np.abs(b).max(-1)
        want = np.minimum((a * np.float32(1 / 6)) / g, np.float32(448))
        s = nearest_even(np.where(fin, want, 0), E4M3[:127]).astype(np.uint8)
        den = (E4M3[s].astype(np.float32) * g)[..., None]
        live = fin[..., None] & (den > 0)
        y = np.where(live, b / np.where(live, den, 1), 0).astype(np.float32)
    code = nearest_even(np.abs(y), E2M1[:8]).astype(np.uint8) | (np.signbit(b).astype(np.uint8) << 3)
    code = np.where(fin[..., None], code, np.signbit(b).astype(np.uint8) << 3).astype(np.uint8)
    s = np.where(fin, s, 0x7F).astype(np.uint8)
    return code.reshape(x.shape), s


def dequantise(code, s, g):
    """float64 values, rounded as the format says: code * fl32(scale * g)."""
    den = (E4M3[s].astype(np.float32) * np.float32(g)).astype(np.float64)
    return (E2M1[code].reshape(*code.shape[:-1], -1, 16) * den[..., None]).reshape(code.shape)


def page_bytes(C, H, D):
    return C * H * (D + D // 8)


def put_token(pool, slot, pos_in_page, head, C, H, D, kc, ks, vc, vs):
    """Write one token's codes and scales of one head into pool (uint8 [slots, page_bytes])."""
    gb = 16 * (D + D // 8)
    base = (head * (C // 16) + pos_in_page // 16) * gb
    t = pos_in_page % 16
    for off, code in ((0, kc), (8 * D, vc)):
        pool[slot, base + off + t * (D // 2): base + off + (t + 1) * (D // 2)] = code[0::2] | (code[1::2] << 4)
    for off, s in ((16 * D, ks), (17 * D, vs)):
        pool[slot, base + off + t * (D // 16): base + off + (t + 1) * (D // 16)] = s


def get_tokens(pool, slots, n, C, H, D, gk=1.0, gv=1.0):
    """k, v float64 [n, H, D] of the first n positions behind a list of slots."""
    gb = 16 * (D + D // 8)
    raw = pool[np.asarray(slots, np.int64)].reshape(len(slots), H, C // 16, gb)
    out = []
    for j, g in ((0, gk), (1, gv)):
        by = raw[..., 8 * D * j: 8 * D * (j + 1)].reshape(len(slots), H, C, D // 2)
        code = np.stack((by & 15, by >> 4), -1).reshape(len(slots), H, C, D)
        s = raw[..., 16 * D + D * j: 16 * D + D * (j + 1)].reshape(len(slots), H, C, D // 16)
        x = dequantise(code, s, g).transpose(0, 2, 1, 3).reshape(len(slots) * C, H, D)
        out.append(x[:n])
    return out


def attend(q, k, v, last, scale):
    """q [n, D], k, v [m, D] float64, query i sees keys 0..last[i]: out, lse, p, and p @ |v|; 0 and -inf without a key."""
    n, m = q.shape[0], k.shape[0]
    out, lse, p = np.zeros((n, v.shape[1])), np.full(n, -np.inf), np.zeros((n, m))
    mag = np.zeros_like(out)
    for i in range(n):
        e = min(int(last[i]) + 1, m)
        if e <= 0:
            continue
        s = (k[:e] @ q[i]) * scale
        t = s.max()
        x = np.exp(s - t)
        lse[i] = t + np.log(x.sum())
        p[i, :e] = x / x.sum()
        out[i] = p[i, :e] @ v[:e]
        mag[i] = p[i, :e] @ np.abs(v[:e])
    return out, lse, p, mag


def score_error(q, k, scale):
    """Bound on the error of a score: D products summed in 32 bits in any order (each partial sum may lose a unit in
    the last place of the whole sum's magnitude), the scaling and the exponent's argument."""
    D = q.shape[-1]
    return (D + 8) * 2.0 ** -23 * float(np.abs(q).sum(-1).max() * np.abs(k).max()) * abs(scale) + 2.0 ** -20


def out_bound(ref, mag, u_p, u_out, err, n):
    """Weights off by the scores' error (numerator and denominator), their rounding u_p, 32-bit sums over n keys, and
    the output's own rounding."""
    rel = 2 * np.expm1(err) + u_p + (n + 64) * 2.0 ** -24
    return rel * mag * (1 + u_out) + u_out * np.abs(ref) + 2.0 ** -24


def lse_bound(lse, err, n):
    return err + (n + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0)) + 2.0 ** -20

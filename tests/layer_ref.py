"""Plain 64-bit references of the gated linear recurrence and of the norms
around a block, in numpy, and the sums of magnitudes that bound the rounding
of each output."""
import numpy as np

BLOCK = 512
START = -87.0  # log decays below it start a sequence


def live_positions(B, L, lengths):
    n = np.full(B, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)
    return np.arange(L)[None, None, :] < n[:, None, None]


def scan_states(a, start, live, u, h0):
    """The state behind every position, [B, C, L], and the one before it."""
    B, C, L = u.shape
    h, after, before = h0.copy(), np.empty((B, C, L)), np.empty((B, C, L))
    for t in range(L):
        before[..., t] = h
        step = np.where(start[..., t], 0.0, a[..., t] * np.where(start[..., t], 0.0, h)) + u[..., t]
        h = np.where(live[..., t], step, h)
        after[..., t] = h
    return after, before


def scan(x1, x2, v, log_a, D, h0=None, lengths=None, gy=None, gh_last=None):
    """Outputs of the recurrence and, with gy, its gradients: dict of arrays."""
    B, C, L = x1.shape
    live = np.broadcast_to(live_positions(B, L, lengths), (B, C, L))
    x1, x2, v, log_a = (np.where(live, x, 0.0) for x in (x1, x2, v, log_a))
    start = log_a < START
    a = np.where(start, 0.0, np.exp(np.where(start, 0.0, log_a)))
    u = x1 * v
    first = np.zeros((B, C)) if h0 is None else np.asarray(h0, np.float64)
    after, before = scan_states(a, start, live, u, first)
    z = after + D[:, None] * u
    out = dict(y=np.where(live, x2 * z, 0.0), h_last=after[..., -1].copy(), states=before[..., ::BLOCK].copy())
    if gy is None:
        return out
    gy = np.where(live, gy, 0.0)
    gz = gy * x2
    c = np.zeros((B, C)) if gh_last is None else np.asarray(gh_last, np.float64).copy()
    gh, handed = np.zeros((B, C, L)), np.zeros((B, C, L))
    for t in range(L - 1, -1, -1):
        g = gz[..., t] + c
        step = np.where(start[..., t], 0.0, a[..., t] * np.where(start[..., t], 0.0, g))
        gh[..., t] = g
        c = np.where(live[..., t], step, c)
        handed[..., t] = c
    gu = gh + D[:, None] * gz
    with np.errstate(invalid="ignore"):
        gla = np.where(start, 0.0, handed * before)
    out.update(gx1=np.where(live, gu * v, 0.0), gx2=np.where(live, gy * z, 0.0), gv=np.where(live, gu * x1, 0.0),
               glog_a=np.where(live, gla, 0.0), gD=(gz * u).sum((0, 2)), gh0=c)
    return out


def scan_magnitudes(x1, x2, v, log_a, D, h0=None, lengths=None, gy=None, gh_last=None):
    """The same with every term in its magnitude: what the roundings of an output are relative to."""
    absent = lambda x: None if x is None else np.abs(x)  # noqa: E731
    return scan(np.abs(x1), np.abs(x2), np.abs(v), log_a, np.abs(D), absent(h0), lengths, absent(gy), absent(gh_last))


def scan_roundings(L):
    """fp32 roundings (of 2^-23) on the way of one contribution, at most: 8 positions of a lane, 6 + 1 steps over the
    lanes, 4 + 2 over the wavefronts, 6 + 2 over the segments, and one for each tile that its row has; each step is an
    exponential, a product and a sum (2 roundings).  The argument of an exponential is a sum of rounded logs, off by
    S 2^-23 for a decay of 2^-S, which weighs at most S 2^-S < 0.6."""
    return 2.0 * (8 + 7 + 6 + 8 + -(-L // BLOCK)) + 4.0


_M = (0xD2511F53, 0xCD9E8D57)
_W = (0x9E3779B9, 0xBB67AE85)


def philox(counter, key):
    """Philox4x32-10 of one counter (four 32-bit words) and key (two), in plain integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = c[0] * _M[0], c[2] * _M[1]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + _W[0]) & 0xFFFFFFFF, (k[1] + _W[1]) & 0xFFFFFFFF]
    return c


def keep_factors(B, C, P, p, seed, offset):
    """0 where a point is dropped, 1 / (1 - p) where it is kept (p to a multiple of 2^-16)."""
    drop = min(65535, int(np.floor(p * 65536 + 0.5)))
    seed, offset, groups = seed % (1 << 64), offset % (1 << 64), -(-P // 8)
    bits = np.empty((B * C, groups, 8))
    for r in range(B * C):
        for g in range(groups):
            i = r * groups + g
            w = philox((i & 0xFFFFFFFF, i >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
            bits[r, g] = [(w[j // 2] >> (16 * (j % 2))) & 0xFFFF for j in range(8)]
    bits = bits.reshape(B, C, groups * 8)[..., :P]
    return (bits >= drop) * (65536.0 / (65536 - drop))


def block_norm(x, z=None, gate=None, w_post=None, scale=None, w_pre=None, eps_post=1e-6, eps_pre=1e-6, keep=None):
    """(x_out, n) of [B, C, P] arrays; keep: the factors of the points."""
    col = lambda w: 1.0 if w is None else w[None, :, None]  # noqa: E731
    out = x
    if z is not None:
        t = z if gate is None else z / (1 + np.exp(-gate))
        out = x + col(scale) * (1.0 if keep is None else keep) * (t * inverse_rms(t, eps_post) * col(w_post))
    return out, None if w_pre is None else out * inverse_rms(out, eps_pre) * col(w_pre)


def inverse_rms(t, eps):
    r = np.sqrt((t * t).mean(1, keepdims=True) + eps)
    with np.errstate(divide="ignore"):
        return np.where(r > 0, 1 / r, 0.0)


def block_norm_backward(x_out, z=None, gate=None, w_post=None, scale=None, w_pre=None, gx_out=None, gn=None,
                        eps_post=1e-6, eps_pre=1e-6, keep=None):
    """Gradients, and for each the magnitude that its roundings are relative to: dict name -> (value, magnitude)."""
    col = lambda w: 1.0 if w is None else w[None, :, None]  # noqa: E731
    gx, mag = (np.zeros_like(x_out),) * 2 if gx_out is None else (gx_out, np.abs(gx_out))
    out = {}
    if gn is not None:
        q = inverse_rms(x_out, eps_pre)
        unit, g = x_out * q, gn * col(w_pre)
        gx = gx + q * (g - unit * (g * unit).mean(1, keepdims=True))
        mag = mag + np.abs(q) * (np.abs(g) + np.abs(unit) * np.abs(g * unit).mean(1, keepdims=True))
        out["gw_pre"] = (gn * unit).sum((0, 2)), np.abs(gn * unit).sum((0, 2))
    out["gx"] = gx, mag
    if z is None:
        return out
    sig = np.ones_like(z) if gate is None else 1 / (1 + np.exp(-gate))
    t = sig * z
    r = inverse_rms(t, eps_post)
    unit = t * r
    k = 1.0 if keep is None else keep
    g, gmag = gx * k * col(scale) * col(w_post), mag * k * np.abs(col(scale) * col(w_post))
    gt = r * (g - unit * (g * unit).mean(1, keepdims=True))
    gtmag = r * (gmag + np.abs(unit) * (gmag * np.abs(unit)).mean(1, keepdims=True))
    out["gz"] = gt * sig, gtmag * sig
    if gate is not None:
        rest = 1 / (1 + np.exp(gate))
        out["ggate"] = gt * t * rest, gtmag * np.abs(t) * rest
    s, smag = (gx * k * unit), mag * k * np.abs(unit)
    out["gw_post"] = (s * col(scale)).sum((0, 2)), (smag * np.abs(col(scale))).sum((0, 2))
    if scale is not None:
        out["gscale"] = (s * col(w_post)).sum((0, 2)), (smag * np.abs(col(w_post))).sum((0, 2))
    return out

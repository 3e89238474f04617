"""Plain 64-bit references of the operators for batches of many requests, and
the bounds of what fp32 may lose on the way.

The reference of the scan is the recurrence, token by token.  Beside every
value it carries a bound on the error of an fp32 evaluation, propagated from
the roundings of each step (u = 2^-24):

  conv     v = b + four products: 6 roundings of the sum of magnitudes
  silu     slope <= 1.1; exp, add, divide: 8 u, and 2 |v| u from the argument
           of exp
  dt       softplus: argument rounded once, exp and log1p: (10 + 3 |a|) u of dt
  A        exp: (3 + 2 |A_log|) u of A
  decay    exp of a sum of dt A over a span, all of one sign and at most 14
           roundings deep: relative |a_t| (rel dt + rel A + 16 u) per token (with
           the products by A and log2 e), and 8 u for the exps and products of
           a term
  products each operand may be held as two 11-bit halves, three of the four
           products of halves taken: 12 u of the term
  sums     at most 128 terms over the state and 64 + 3 over a chunk, any order:
           195 u of the sum of magnitudes

Worst cases add up to `err`; the typical error is that of independent
roundings, so the root mean square over a tensor is held to 16 u of the sums
of magnitudes, and one error that is not independent: an exponent c is a sum in
fp32, of up to 14 roundings of partial sums up to |c|, each at most u / 2 of one and
about a third of that in the root mean square: sqrt(14) / 6 < 2 / 3 of u |c|, up
to 2 u |c| at three times it.  Every element of a head's state has the same c, so
this does not average out; `sys` carries 2 u |a_t| per token of what a term has
decayed, which adds up to 2 u |c|.
"""
import numpy as np

U = 2.0 ** -24


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1.0 + np.exp(-v))


def softplus(v):
    return np.where(v > 20.0, v, np.log1p(np.exp(np.minimum(v, 20.0))))


def scan(zx, p, ring, state, pos, N):
    """One sequence: zx [L, >= ld], ring [4, conv_dim], state [H, 64, N] (before
    it), pos its position (<= 0: new).  Returns dict(y, ring, state, and for y
    and state `_err` worst-case and `_abs` sum of magnitudes)."""
    f = lambda a: np.asarray(a, np.float64)
    H = p["dt_bias"].shape[0]
    di = 64 * H
    cd = di + 2 * N
    L = zx.shape[0]
    zx, w, b = f(zx), f(p["conv_w"]), f(p["conv_b"])
    ring, h = np.array(ring, np.float64), f(state).copy()
    if pos <= 0:
        ring[:] = 0.0
        h[:] = 0.0
    A = -np.exp(f(p["A_log"]))
    relA = (3 + 2 * np.abs(f(p["A_log"]))) * U
    Dh = f(p["D"])
    habs, herr, hsys = np.abs(h), np.zeros_like(h), np.zeros_like(h)
    y = np.zeros((L, di))
    yerr, yabs, ysys = np.zeros((L, di)), np.zeros((L, di)), np.zeros((L, di))
    raw = zx[:, di + cd:di + cd + H] + f(p["dt_bias"])
    dt = softplus(raw)
    reldt = (10 + 3 * np.abs(raw)) * U
    a = dt * A
    absa = np.abs(a)
    for t in range(L):
        ring[(pos + t) & 3] = zx[t, di:di + cd]
        taps = np.stack([ring[(pos + t + 1 + j) & 3] for j in range(4)], 1)
        v = (w * taps).sum(1) + b
        verr = 6 * U * ((np.abs(w * taps)).sum(1) + np.abs(b))
        s = silu(v)
        serr = 1.1 * verr + (8 + 2 * np.abs(v)) * U * np.abs(s)
        x, xe = s[:di].reshape(H, 64), serr[:di].reshape(H, 64)
        B, Be, C, Ce = s[di:di + N], serr[di:di + N], s[di + N:], serr[di + N:]
        dA = np.exp(a[t])[:, None, None]
        # more than 150 in the exponent leaves nothing of a term
        rel = (np.minimum(absa[t], 150.0) * (reldt[t] + relA + 16 * U))[:, None, None]
        dx = dt[t][:, None] * x
        dxe = dt[t][:, None] * xe + np.abs(dx) * (reldt[t][:, None] + U)
        add = dx[:, :, None] * B
        adderr = dxe[:, :, None] * np.abs(B) + np.abs(dx)[:, :, None] * Be + np.abs(add) * (12 + 8) * U
        herr = dA * (herr + habs * rel) + adderr
        hsys = dA * (hsys + habs * (2 * U * np.minimum(absa[t], 150.0))[:, None, None])
        h = h * dA + add
        habs = habs * dA + np.abs(add)
        aC = np.abs(C)
        y[t] = ((h * C).sum(-1) + Dh[:, None] * x).reshape(-1)
        ya = (habs * aC).sum(-1) + np.abs(Dh[:, None] * x)
        yabs[t] = ya.reshape(-1)
        ysys[t] = (hsys * aC).sum(-1).reshape(-1)
        yerr[t] = ((herr * aC).sum(-1) + (habs * Ce).sum(-1) + np.abs(Dh)[:, None] * xe + (12 + 195) * U * ya).reshape(-1)
    serr_ = herr + 195 * U * habs
    tiny = 1e-37
    return dict(y=y, y_err=yerr + tiny, y_rms=16 * U * yabs + ysys + tiny, ring=ring, state=h, state_err=serr_ + tiny,
                state_rms=16 * U * habs + hsys + tiny)


def wide(zx, p, ring, state, pos, N):
    """What scan's bounds leave out: the prompts' products take an operand as fp16
    halves under an exponent that it shares, so that beside 2^-22 of itself a value
    is off by up to half of fp16's smallest step there, 2^-25 where the largest is
    in [2^14, 2^15): 2^-39 of the largest, or 2^-85 (the exponent is 60 at most).
    An exponent is shared by the B, and by the C, of 64 tokens, by a channel's x in
    them, weighted or not, by a channel's state, and by a head's M in them, whose
    largest is taken to be max |C . B| max dt + |D|.  Tokens behind the last one
    count: their B and C repeat the last input, their x goes on from zeros.
    Returns (y, state): bounds to add to scan's."""
    f = lambda a: np.asarray(a, np.float64)
    H = p["dt_bias"].shape[0]
    di = 64 * H
    cd = di + 2 * N
    L = zx.shape[0]
    zx, w, b, Dh = f(zx), f(p["conv_w"]), f(p["conv_b"]), np.abs(f(p["D"]))
    h = np.zeros((H, 64, N)) if pos <= 0 else f(state).copy()
    eh = np.zeros_like(h)
    before = np.zeros((3, cd)) if pos <= 0 else f(ring)[[(pos + 1 + j) & 3 for j in range(3)]]
    u = np.concatenate([before, zx[:, di:di + cd]])
    dt_all = softplus(zx[:, di + cd:di + cd + H] + f(p["dt_bias"]))
    A = -np.exp(f(p["A_log"]))
    step = lambda m: np.maximum(1.01 * 2.0 ** -39 * m, 1.01 * 2.0 ** -85)
    y_err = np.zeros((L, H, 64))
    conv = lambda v: silu(b + sum(w[:, j] * v[j:j + 64] for j in range(4)))
    for c0 in range(0, L, 64):
        n = min(64, L - c0)
        seg = u[c0:c0 + n + 3]
        zeros = conv(np.concatenate([seg, np.zeros((64 - n, cd))]))
        last = conv(np.concatenate([seg, np.repeat(seg[-1:], 64 - n, 0)]))
        xg = zeros[:, :di].reshape(64, H, 64)
        Bg, Cg = last[:, di:di + N], last[:, di + N:]
        x, B, C, dt = xg[:n], np.abs(Bg[:n]), np.abs(Cg[:n]), dt_all[c0:c0 + n]
        c = np.cumsum(dt * A, 0)
        dB, dC = step(np.abs(Bg).max()), step(np.abs(Cg).max())
        G = Cg @ Bg.T
        tile = np.arange(64) // 16
        gmax = np.abs(G[tile[:, None] >= tile]).max()
        eG = dC * B.sum(1) + dB * C.sum(1)[:, None] + 2 * N * dB * dC                    # [i, j]
        low = np.tril(np.ones((n, n)))
        decay = np.exp(np.where(low > 0, c.T[:, :, None] - c.T[:, None, :], 0.0)) * low  # [H, i, j]
        M = np.abs(decay * G[:n, :n] * dt.T[:, None]) + Dh[:, None, None] * np.eye(n)
        eM = decay * eG * dt.T[:, None] + low * step(gmax * dt.max(0) + Dh)[:, None, None]
        ax = np.abs(x).transpose(1, 0, 2)                                                # [H, j, p]
        dx = step(np.abs(xg).max(0))                                                     # [H, p]
        dM = step(gmax * dt.max(0) + Dh)
        y1 = eM @ ax + M.sum(-1)[:, :, None] * dx[:, None] + 128 * dM[:, None, None] * dx[:, None]
        ah = np.abs(h)
        dh = step(ah.max(-1))
        y2 = dC * ah.sum(-1)[:, None] + C.sum(1)[:, None] * dh[:, None] + 2 * N * dC * dh[:, None]
        y2 = y2 + np.matmul(C, eh.transpose(0, 2, 1))
        y_err[c0:c0 + n] = (y1 + np.exp(c.T)[:, :, None] * y2).transpose(1, 0, 2)
        xw = (x * (dt * np.exp(c[-1] - c))[:, :, None]).transpose(1, 2, 0)               # [H, p, j]
        dw = step(np.abs(xw).max(-1))
        end = np.exp(c[-1])[:, None, None]
        eh = end * eh + dw[..., None] * B.sum(0) + (np.abs(xw).sum(-1) * dB + 128 * dw * dB)[..., None]
        h = end * h + xw @ Bg[:n]
    return y_err.reshape(L, di), eh


def assert_close(got, want, err, typical, what):
    got = np.asarray(got, np.float64)
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    d = np.abs(got - want)
    worst = float((d / err).max()) if d.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound, at {np.unravel_index((d / err).argmax(), d.shape)}"
    if d.size:
        rms, lim = float(np.sqrt((d ** 2).mean())), float(np.sqrt((typical ** 2).mean()))
        assert rms <= lim, f"{what}: rms error {rms:.3g} > {lim:.3g}"


def unpack4(p):
    p = np.asarray(p, np.uint8)
    v = np.stack([p & 15, p >> 4], -1).reshape(*p.shape[:-1], -1).astype(np.int64)
    return np.where(v >= 8, v - 16, v)


def adapters(q, s, ids, A, B, beta, y):
    """The integers in 64 bits, then the fp32 operations in their order."""
    out = np.array(y, np.float32)
    for m, a in enumerate(np.asarray(ids)):
        if 0 <= a < len(A):
            low = np.asarray(A[a], np.int64) @ np.asarray(q[m], np.int64)
            acc = np.asarray(B[a], np.int64) @ low
            t = np.asarray(beta[a], np.float32) * acc.astype(np.float32)
            out[m] = out[m] + np.float32(s[m]) * t
    return out

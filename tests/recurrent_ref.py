"""Plain 64-bit references of the recurrent operators, with bounds on what the kernels may be off.

Every bound follows the definition step by step before anything runs: u is the unit roundoff of the element type for
the one rounding of a result, E = 2^-20 covers a step's fp32 operations (16 units: the exponential, the softplus and
the sigmoid are good to a few 2^-23 each, products and sums to 2^-24), and what a state or a gradient carries on is carried
on in its bound by the same recurrence.  An argument v of softplus or sigmoid is itself rounded: its relative error is up
to |v| 2^-24 and enters as E (1 + |v|).  Sums over many terms get E times the sum of their absolute values, more by
1/256 a term for their order.  fp32 (and bf16) end at 2^-126: an exponential or a product below that may come as 0, which is
an error of at most 2^-126 (LEAST) in that term, carried on like any other."""
import torch

from encoder_ref import TINY, U, within  # noqa: F401

E = 2.0 ** -20
LEAST = 2.0 ** -126


def _d(t):
    return None if t is None else t.detach().double().cpu()


def scan(x, delta, A, Bt, Ct, D=None, z=None, delta_bias=None, softplus=True, lengths=None, state=None, dy=None, dstate=None):
    """{"y", "state", "dx", "ddelta", "dA", "dBt", "dCt", "dD", "dz", "dbias", "dstate"} -> (want, bound), 64-bit on the CPU.
    What lies behind a sequence's length never enters."""
    dt = x.dtype
    u, tiny = U[dt], TINY[dt]
    x, delta, A, Bt, Ct, D, z, delta_bias, state, dy, dstate = (_d(t) for t in (x, delta, A, Bt, Ct, D, z, delta_bias, state, dy, dstate))
    B, L, C, T = x.shape
    G, N = Bt.shape[2:]
    zero = torch.zeros
    n = torch.full((B,), L) if lengths is None else lengths.cpu().long().clamp(0, L)
    inside = (torch.arange(L)[None] < n[:, None])[:, :, None, None]
    x, delta, z, dy = (None if t is None else torch.where(inside, t, 0.0) for t in (x, delta, z, dy))
    Bt, Ct = torch.where(inside, Bt, 0.0), torch.where(inside, Ct, 0.0)
    per = lambda t: t.repeat_interleave(C // G, 2)[:, :, :, None]  # [B, L, C, 1, N]
    b, c = per(Bt), per(Ct)
    v = delta + (0.0 if delta_bias is None else delta_bias[:, None])
    d = torch.logaddexp(v, torch.zeros(())) if softplus else v
    derr = E * (1 + v.abs()) * d.abs()
    d, derr = torch.where(inside, d, 0.0), torch.where(inside, derr, 0.0)
    D_ = zero(C, 1, dtype=torch.float64) if D is None else D[:, None]
    An = A[:, None]  # [C, 1, N]
    a = torch.exp(d[..., None] * An)
    aerr = a * (An.abs() * derr[..., None] + E * (1 + (d[..., None] * An).abs())) + LEAST
    h = zero(B, C, T, N, dtype=torch.float64) if state is None else state
    herr = zero(B, C, T, N, dtype=torch.float64)
    H, Herr, P, Perr = [], [], [], []
    for l in range(L):
        P.append(h)
        Perr.append(herr)
        add = d[:, l, :, :, None] * b[:, l] * x[:, l, :, :, None]
        live = inside[:, l, :, :, None]
        new = a[:, l] * h + add
        err = a[:, l] * herr + aerr[:, l] * h.abs() + (b[:, l] * x[:, l, :, :, None]).abs() * derr[:, l, :, :, None] \
            + E * ((a[:, l] * h).abs() + add.abs()) + LEAST
        h, herr = torch.where(live, new, h), torch.where(live, err, herr)
        H.append(h)
        Herr.append(herr)
    out = {"state": (h, herr)}
    if L == 0:
        out["y"] = (x, x)
        return out
    H, Herr, P, Perr = (torch.stack(t, 1) for t in (H, Herr, P, Perr))
    y0 = (c * H).sum(-1) + D_ * x
    y0err = (c.abs() * Herr + LEAST).sum(-1) + 4 * E * ((c * H).abs().sum(-1) + (D_ * x).abs())
    sil = torch.ones_like(x) if z is None else z * torch.sigmoid(z)
    silerr = 0.0 * sil if z is None else 4 * E * sil.abs() + E * (z * z).abs() * torch.sigmoid(z)
    y = torch.where(inside, y0 * sil, 0.0)
    out["y"] = (y, u * y.abs() + (1 + u) * (sil.abs() * y0err + y0.abs() * silerr) + tiny)
    if dy is None and dstate is None:
        return out
    dy = torch.zeros_like(x) if dy is None else dy
    s, serr = dy * sil, dy.abs() * silerr + E * (dy * sil).abs()
    r = zero(B, C, T, N, dtype=torch.float64) if dstate is None else dstate
    rerr = 0.0 * r
    g, gerr, R, Rerr = ([None] * L for _ in range(4))
    for l in reversed(range(L)):
        cs = c[:, l] * s[:, l, :, :, None]
        g[l] = cs + r
        gerr[l] = c[:, l].abs() * serr[:, l, :, :, None] + rerr + E * (cs.abs() + r.abs()) + LEAST
        live = inside[:, l, :, :, None]
        nr = a[:, l] * g[l]
        ne = a[:, l] * gerr[l] + aerr[:, l] * g[l].abs() + E * nr.abs() + LEAST
        r, rerr = torch.where(live, nr, r), torch.where(live, ne, rerr)
        R[l], Rerr[l] = torch.where(live, r, 0.0), torch.where(live, rerr, 0.0)
        g[l], gerr[l] = torch.where(live, g[l], 0.0), torch.where(live, gerr[l], 0.0)
    out["dstate"] = (r, rerr)
    g, gerr, R, Rerr = (torch.stack(t, 1) for t in (g, gerr, R, Rerr))
    sums = lambda t, dims: t.sum(dims)
    grp = lambda t: t.reshape(B, L, G, C // G, T, N).sum((3, 4))  # over a group's columns
    many = lambda k: E * (1 + k / 256)
    dx_ = (d * x)[..., None]
    dxerr = ((derr * x.abs()) + E * (d * x).abs())[..., None]
    K = C // G * T
    for name, val, err in (("dBt", g * dx_, gerr * dx_.abs() + g.abs() * dxerr + LEAST),
                           ("dCt", H * s[..., None], Herr * s.abs()[..., None] + H.abs() * serr[..., None] + LEAST)):
        w = grp(val)
        out[name] = (w, u * w.abs() + (1 + u) * (grp(err) + many(K) * grp(val.abs())) + tiny)
    gB, gBabs = (g * b).sum(-1), (g * b).abs().sum(-1)
    gBerr = (gerr * b.abs() + LEAST).sum(-1) + 4 * E * gBabs
    w = torch.where(inside, d * gB + D_ * s, 0.0)
    out["dx"] = (w, u * w.abs() + (1 + u) * (d.abs() * gBerr + derr * gB.abs() + D_.abs() * serr
                                             + E * ((d * gB).abs() + (D_ * s).abs()) + LEAST) + tiny)
    m, merr = R * P, Rerr * P.abs() + R.abs() * Perr + E * (R * P).abs() + LEAST
    dd = (An * m).sum(-1) + x * gB
    dderr = (An.abs() * (merr + 4 * E * m.abs())).sum(-1) + x.abs() * gBerr + E * (x * gB).abs()
    sg = torch.sigmoid(v) if softplus else torch.ones_like(v)
    dv = torch.where(inside, dd * sg, 0.0)
    dverr = torch.where(inside, (1 + E) * dderr * sg + dv.abs() * E * (1 + v.abs()) + LEAST, 0.0)
    out["ddelta"] = (dv, u * dv.abs() + (1 + u) * dverr + tiny)
    k = B * L * T
    val = d[..., None] * m
    out["dA"] = (val.sum((0, 1, 3)), (d.abs()[..., None] * merr + derr[..., None] * m.abs() + LEAST).sum((0, 1, 3))
                 + many(k) * val.abs().sum((0, 1, 3)))
    out["dD"] = ((s * x).sum((0, 1, 3)), (serr * x.abs() + LEAST).sum((0, 1, 3)) + many(k) * (s * x).abs().sum((0, 1, 3)))
    out["dbias"] = (dv.sum((0, 1, 3)), dverr.sum((0, 1, 3)) + many(k) * dv.abs().sum((0, 1, 3)))
    if z is not None:
        sz = torch.sigmoid(z)
        ds = sz * (1 + z * (1 - sz))
        w = torch.where(inside, dy * y0 * ds, 0.0)
        dserr = 4 * E * sz * (1 + z.abs()) ** 2
        out["dz"] = (w, u * w.abs() + (1 + u) * dy.abs() * (y0err * ds.abs() + y0.abs() * dserr) + 2 * E * w.abs() + LEAST + tiny)
    return out


def conv(x, weight, bias=None, activation="none", lengths=None, state=None, dy=None, dstate=None):
    """{"y", "state", "dx", "dw", "db", "dstate"} -> (want, bound)."""
    dt = x.dtype
    u, tiny = U[dt], TINY[dt]
    x, weight, bias, state, dy, dstate = (_d(t) for t in (x, weight, bias, state, dy, dstate))
    B, L, C, T = x.shape
    W = weight.shape[1]
    n = [L] * B if lengths is None else [min(max(int(k), 0), L) for k in lengths]
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)
    out = {k: [z(*s), z(*s)] for k, s in (("y", x.shape), ("state", (B, W - 1, C, T)), ("dx", x.shape), ("dw", (C, W)),
                                          ("db", (C,)), ("dstate", (B, W - 1, C, T)))}
    b_ = z(C, 1) if bias is None else bias[:, None]
    for i in range(B):
        full = torch.cat((z(W - 1, C, T) if state is None else state[i], x[i, :n[i]]))
        win = torch.stack([full[w:w + n[i]] for w in range(W)])  # [W, n, C, T]
        ww = weight.T[:, None, :, None]
        v = b_ + (win * ww).sum(0)
        verr = 2 * E * (b_.abs() + (win * ww).abs().sum(0))
        sg = torch.sigmoid(v)
        if activation == "silu":
            y, slope, bend = v * sg, sg * (1 + v * (1 - sg)), 4 * E * sg * (1 + v.abs()) ** 2
            yerr = 1.2 * verr + 4 * E * y.abs() + E * v * v * sg
        else:
            y, slope, bend, yerr = v, torch.ones_like(v), torch.zeros_like(v), verr
        out["y"][0][i, :n[i]], out["y"][1][i, :n[i]] = y, u * y.abs() + (1 + u) * yerr
        out["state"][0][i] = full[n[i]:]
        if dy is None and dstate is None:
            continue
        dv = z(n[i], C, T) if dy is None else dy[i, :n[i]] * slope
        dverr = 0 * dv if dy is None else dy[i, :n[i]].abs() * (0.5 * verr + bend) + E * dv.abs()
        df, dferr = z(W - 1 + n[i], C, T), z(W - 1 + n[i], C, T)
        for w in range(W):
            df[w:w + n[i]] += weight[:, w, None] * dv
            dferr[w:w + n[i]] += weight[:, w, None].abs() * (dverr + 2 * E * dv.abs())
        if dstate is not None:
            df[n[i]:] += dstate[i]
            dferr[n[i]:] += E * dstate[i].abs()
        dferr = u * df.abs() + (1 + u) * dferr + tiny
        out["dstate"][0][i], out["dstate"][1][i] = df[:W - 1], dferr[:W - 1]
        out["dx"][0][i, :n[i]], out["dx"][1][i, :n[i]] = df[W - 1:], dferr[W - 1:]
        k = E * (1 + n[i] * T / 256)
        out["dw"][0] += (win * dv).sum((1, 3)).T
        out["dw"][1] += (win.abs() * (dverr + k * dv.abs())).sum((1, 3)).T
        out["db"][0] += dv.sum((0, 2))
        out["db"][1] += (dverr + k * dv.abs()).sum((0, 2))
    for k in ("dw", "db"):
        out[k][1] += u * out[k][0].abs() + tiny
    out["y"][1] += tiny
    return {k: tuple(v) for k, v in out.items()}


def _norm(v, verr, w, b, kind, eps):
    """(normalised, its error, factor, its relative error, affine, its error) over the last two axes."""
    mean = lambda t: t.mean((-2, -1), keepdim=True)
    if kind == "layer":
        verr = verr + mean(verr) + 2 * E * mean(v.abs())
        v = v - mean(v)
    f = 1 / torch.sqrt(mean(v * v) + eps)
    frel = f * f * mean(v.abs() * verr) + 2 * E
    n = v * f
    nerr = verr * f + n.abs() * (frel + E)
    out = n * w[:, None] + b[:, None]
    return n, nerr, f, frel, out, nerr * w.abs()[:, None] + E * ((n * w[:, None]).abs() + b.abs()[:, None])


def _back(g, gerr, n, nerr, f, frel, kind):
    mean = lambda t: t.mean((-2, -1), keepdim=True)
    m1 = mean(g) if kind == "layer" else 0 * mean(g)
    m1err = (mean(gerr) + 2 * E * mean(g.abs())) if kind == "layer" else 0 * mean(g)
    m2, m2err = mean(g * n), mean(g.abs() * nerr + gerr * n.abs()) + 2 * E * mean((g * n).abs())
    q = g - m1 - n * m2
    qerr = gerr + m1err + n.abs() * m2err + nerr * m2.abs() + E * (g.abs() + m1.abs() + (n * m2).abs())
    return f * q, f * qerr + (frel + E) * (f * q).abs()


def residual(x, branch=None, weight=None, bias=None, scale=None, gate=None, post_weight=None, post_bias=None, kind="layer",
             eps=1e-6, dr=None, dh=None):
    """{"r", "h", "dx", "dbranch", "dweight", ..} -> (want, bound); x [B, L, C, T]."""
    dt = x.dtype
    u, tiny = U[dt], TINY[dt]
    x, v, w, b, scale, gate, pw, pb, dr, dh = (_d(t) for t in (x, branch, weight, bias, scale, gate, post_weight, post_bias, dr, dh))
    B, L, C, T = x.shape
    zeros = torch.zeros(C, dtype=torch.float64)
    out = {}
    rnd = lambda t, e: (t, u * t.abs() + (1 + u) * e + tiny)
    r, rerr = x, 0 * x
    if v is not None:
        verr = 0 * v
        if pw is not None:
            uh, uherr, fu, furel, v, verr = _norm(v, verr, pw, zeros if pb is None else pb, kind, eps)
        k = torch.ones(1, 1, C, 1, dtype=torch.float64)
        k = k if scale is None else k * scale[:, None]
        k = k if gate is None else k * gate[:, None, :, None]
        r = x + k * v
        rerr = k.abs() * verr + E * (x.abs() + (k * v).abs())
        out["r"] = rnd(r, rerr)
    if w is not None:
        rh, rherr, fr, frrel, h, herr = _norm(r, rerr, w, zeros if b is None else b, kind, eps)
        out["h"] = rnd(h, herr)
    if dr is None and dh is None:
        return out
    g, gerr = (torch.zeros_like(x) if dr is None else dr), torch.zeros_like(x)
    many = E * (1 + B * L * T / 256)
    col = lambda val, err: rnd(val.sum((0, 1, 3)), (err + many * val.abs()).sum((0, 1, 3)))
    if dh is not None:
        out["dweight"] = col(dh * rh, dh.abs() * rherr)
        out["dbias"] = col(dh, 0 * dh)
        q = dh * w[:, None]
        q, qerr = _back(q, E * q.abs(), rh, rherr, fr, frrel, kind)
        g, gerr = g + q, qerr + E * (g.abs() + q.abs())
    out["dx"] = rnd(g, gerr)
    if v is None:
        return out
    gv, gverr = g * v, gerr * v.abs() + g.abs() * verr
    # sums of g v come from those of g uh and g where there is a norm before: the terms of both count
    if pw is not None:
        gverr = gverr + many * ((g * uh * pw[:, None]).abs() + (g * (zeros if pb is None else pb)[:, None]).abs())
    one = torch.ones(1, 1, C, 1, dtype=torch.float64)
    gs, ss = one if gate is None else gate[:, None, :, None], one if scale is None else scale[:, None]
    if scale is not None:
        out["dscale"] = col(gs * gv, (gs * gverr).abs())
    if gate is not None:
        t = ss * gv
        out["dgate"] = rnd(t.sum((1, 3)), ((ss * gverr).abs() + many * t.abs()).sum((1, 3)))
    dv, dverr = k * g, k.abs() * gerr + E * (k * g).abs()
    if pw is not None:
        out["dpost_weight"] = col(dv * uh, dverr * uh.abs() + dv.abs() * uherr)
        out["dpost_bias"] = col(dv, dverr)
        q = dv * pw[:, None]
        dv, dverr = _back(q, dverr * pw.abs()[:, None] + E * q.abs(), uh, uherr, fu, furel, kind)
    out["dbranch"] = rnd(dv, dverr)
    return out

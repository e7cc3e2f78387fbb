"""Plain 64-bit references of the encoder operators, with bounds on what the kernels may be off.

Every bound is formed from the definition before anything runs: u is the unit roundoff of the element type, E32 covers
the fp32 sums, exponentials and statistics (measured bars of this library's fp32 outputs are a few 1e-7 of the sum of
absolute terms; 2^-16 = 1.5e-5 leaves room for the longest sums and largest scores drawn here)."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
E32 = 2.0 ** -16
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# smallest step of a result in fp16's subnormal range
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -24, torch.bfloat16: 0.0}


def within(name, got, want, bound):
    """got (any type, any device) against want and its elementwise bound, both 64-bit on the CPU."""
    g = got.detach().double().cpu()
    assert g.shape == want.shape, (name, g.shape, want.shape)
    if g.numel() == 0:
        return
    bad = ~((g - want).abs() <= bound)
    if bad.any():
        i = int(torch.nonzero(bad.reshape(-1))[0])
        raise AssertionError("%s: %d of %d outside the bound, first at %d: got %r, want %r, bound %r" % (
            name, int(bad.sum()), bad.numel(), i, g.reshape(-1)[i].item(), want.reshape(-1)[i].item(),
            bound.reshape(-1)[i].item()))


def visible(Lq, Lk, length, start, left, right, sinks):
    """[Lq, Lk] truth values of the definition, written out."""
    p = (start + torch.arange(Lq))[:, None]
    j = torch.arange(Lk)[None, :]
    seen = (p < length) & (j < length)
    if right >= 0:
        seen &= j <= p + right
    if left >= 0:
        seen &= (j >= p - left) | (j < sinks)
    return seen


def attention(q, k, v, do=None, left=-1, right=-1, sinks=0, scale=None, lengths=None, starts=None):
    """Values and bounds: {"o", "dq", "dk", "dv"} -> (want, bound), 64-bit on the CPU.  Invisible rows of k, v, q and do
    never enter a sum, whatever they hold."""
    dt = q.dtype
    u = U[dt]
    B, Lq, H, D = q.shape
    Lk, Hkv = k.shape[1:3]
    G = H // Hkv
    scale = D ** -0.5 if scale is None else scale
    q, k, v = (t.detach().double().cpu() for t in (q, k, v))
    out = {n: [torch.zeros(s, dtype=torch.float64) for _ in range(2)] for n, s in (
        ("o", (B, Lq, H, D)), ("dq", (B, Lq, H, D)), ("dk", (B, Lk, Hkv, D)), ("dv", (B, Lk, Hkv, D)))}
    if do is not None:
        do = do.detach().double().cpu()
    for b in range(B):
        n = Lk if lengths is None else min(max(int(lengths[b]), 0), Lk)
        st = Lk - Lq if starts is None else int(starts[b])
        seen = visible(Lq, Lk, n, st, left, right, sinks)
        rows, cols = seen.any(1), seen.any(0)
        for h in range(H):
            hk = h // G
            Q = torch.where(rows[:, None], q[b, :, h], 0.0)
            # a key outside a row's view must not touch it: infinities and NaN are cut pair by pair
            K, V = (torch.where(cols[:, None], t[b, :, hk], 0.0) for t in (k, v))
            S = torch.where(seen, pairdot(Q, K, seen) * scale, -math.inf)
            m = S.amax(1, keepdim=True) if Lk else torch.zeros(Lq, 1, dtype=torch.float64)
            e = torch.where(seen, torch.exp(S - torch.where(m == -math.inf, 0.0, m)), 0.0)
            P = e / e.sum(1, keepdim=True)
            P = torch.where(seen, P, 0.0)
            o, ob = pairsum(P, V, seen), pairsum(P, V.abs(), seen)
            out["o"][0][b, :, h] = o
            out["o"][1][b, :, h] = (2.5 * u + E32) * ob + TINY[dt]
            if do is None:
                continue
            g = torch.where(rows[:, None], do[b, :, h], 0.0)
            dP = torch.where(seen, pairdot(g, V, seen), 0.0)
            delta = (g * o).sum(1, keepdim=True)
            dS = torch.where(seen, P * (dP - delta), 0.0)
            # a rounded o moves delta by u |do| |o|; dP - delta cancels, so fp32 errors go by the terms' sizes
            terms = P * (torch.where(seen, pairdot(g.abs(), V.abs(), seen), 0.0) + (g.abs() * ob).sum(1, keepdim=True))
            dSb = u * dS.abs() + (u + E32) * P * (g.abs() * o.abs()).sum(1, keepdim=True) + E32 * terms + TINY[dt] * seen
            out["dq"][0][b, :, h] = scale * pairsum(dS, K, seen)
            out["dq"][1][b, :, h] = 1.5 * (scale * pairsum(dSb, K.abs(), seen) + u * out["dq"][0][b, :, h].abs()) + TINY[dt]
            out["dv"][0][b, :, hk] += pairsum(P.T, g, seen.T)
            out["dv"][1][b, :, hk] += (2.5 * u + E32) * pairsum(P.T, g.abs(), seen.T) + TINY[dt] * (
                1 + pairsum(seen.T.double(), g.abs(), seen.T))
            dk, dkb = scale * pairsum(dS.T, Q, seen.T), scale * pairsum(dSb.T, Q.abs(), seen.T)
            out["dk"][0][b, :, hk] += dk
            out["dk"][1][b, :, hk] += 1.5 * dkb + 1.5 * u * dk.abs() + TINY[dt]
    return {n: tuple(t) for n, t in out.items()}


def pairdot(a, b, seen):
    """a [M, D] . b [N, D] -> [M, N]; plain where all is finite, pair by pair where not."""
    if torch.isfinite(a).all() and torch.isfinite(b).all():
        return a @ b.T
    return torch.where(seen, (a[:, None] * b[None]).sum(-1), 0.0)


def pairsum(w, x, seen):
    """sum_j w[i, j] x[j] over the pairs that are seen."""
    if torch.isfinite(w).all() and torch.isfinite(x).all():
        return w @ x
    return torch.where(seen[:, :, None], w[:, :, None] * x[None], 0.0).sum(1)


def rotary(x, positions, freqs, sections, T, interleaved, inverse=False):
    """(want, bound)."""
    u = U[x.dtype]
    B, L, N, D = x.shape
    n = sum(sections)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    pos = positions.cpu().double().expand(B, L, len(sections))
    y = x.detach().double().cpu().view(B, L, N, D // T, T).clone()
    size = torch.zeros_like(y)
    for c in range(n):
        phi = pos[:, :, axis[c]] * freqs[c].double().cpu()
        if inverse:
            phi = -phi
        co, si = torch.cos(phi)[:, :, None, None], torch.sin(phi)[:, :, None, None]
        lo, hi = (2 * c, 2 * c + 1) if interleaved else (c, c + n)
        a, b = y[:, :, :, lo].clone(), y[:, :, :, hi].clone()
        y[:, :, :, lo], y[:, :, :, hi] = a * co - b * si, b * co + a * si
        size[:, :, :, lo] = size[:, :, :, hi] = a.abs() + b.abs()
    # products and sines in fp32 (a few units of 2^-24 of either term), one rounding; passed channels exactly
    bound = torch.where(size > 0, u * y.abs() + 2.0 ** -20 * size + TINY[x.dtype], 0.0)
    return y.view(B, L, N, D), bound.view(B, L, N, D)


def group_norm_act(x, w, b, groups, act, eps, dy=None):
    """{"y", "dx", "dw", "db"} -> (want, bound)."""
    dt = x.dtype
    u = U[dt]
    shape = x.shape
    B, C, T = shape[0], shape[-2], shape[-1]
    x = x.detach().double().cpu().view(B, -1, C, T)
    w, b = w.detach().double().cpu()[:, None], b.detach().double().cpu()[:, None]
    S = x.shape[1]
    g = x.view(B, S, groups, C // groups * T)
    mean = g.mean((1, 3), keepdim=True)
    var = (g - mean).pow(2).mean((1, 3), keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    xh = ((g - mean) * rstd).view(B, S, C, T)
    # the spread of x about its group's first element limits the sums' accuracy
    far = ((mean - g[:, :1, :, :1]).abs() * rstd).clamp(min=1.0)
    kappa = (far * far).expand(B, S, groups, C // groups * T).reshape(B, S, C, T)
    z = xh * w + b
    ez = E32 * kappa * (1.0 + xh.abs()) * w.abs() + E32 * z.abs()
    phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
    sg = torch.sigmoid(z)
    y = {"none": z, "relu": torch.clamp(z, min=0.0), "silu": z * sg, "gelu": z * phi}[act]
    out = {"y": (y.view(shape), (u * y.abs() + 1.2 * ez + E32 * (1 if act in ("silu", "gelu") else 0) + TINY[dt]).view(shape))}
    if dy is None:
        return out
    dy = dy.detach().double().cpu().view(B, S, C, T)
    d = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": sg * (1 + z * (1 - sg)),
         "gelu": phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[act]
    dz = dy * d
    edz = dy.abs() * ((0.0 if act in ("none", "relu") else 1.0) * ez + E32)
    n = S * (C // groups) * T
    grp = lambda t: t.view(B, S, groups, -1)
    mean_of = lambda t: grp(t).sum((1, 3), keepdim=True).expand(B, S, groups, C // groups * T).reshape(B, S, C, T) / n
    rs = rstd.expand(B, S, groups, C // groups * T).reshape(B, S, C, T)
    gw = dz * w
    dx = rs * (gw - mean_of(gw) - xh * mean_of(gw * xh))
    e = edz * w.abs()
    edx = rs * (e + mean_of(e) + E32 * (gw.abs() + mean_of(gw.abs())) + xh.abs() * mean_of(e * xh.abs() + E32 * kappa * (gw * xh).abs())
                + E32 * kappa * (1 + xh.abs()) * mean_of((gw * xh).abs()) + E32 * kappa * mean_of(gw.abs()))
    sums = lambda t: t.sum((0, 1, 3))
    dw, db = sums(dz * xh), sums(dz)
    out["dx"] = (dx.view(shape), (u * dx.abs() + 1.2 * edx + TINY[dt]).view(shape))
    out["dw"] = (dw, u * dw.abs() + sums(edz * xh.abs() + E32 * kappa * dz.abs() * (1 + xh.abs())) + TINY[dt])
    out["db"] = (db, u * db.abs() + sums(edz + E32 * dz.abs()) + TINY[dt])
    return out

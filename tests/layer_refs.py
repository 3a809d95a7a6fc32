"""Plain implementations in 64 bits of the convolution, the selective scan and their
gradients, one token after the other, with a bound on what a 32-bit evaluation may be off.

Bounds are first order in EPS = 2^-24, the relative error of one float32 operation, and
follow the formulas: each line of arithmetic below has its line of error.  What an
exponential, a reciprocal or a sigmoid loses is counted as a few EPS (the hardware's are good
to one unit in the last place, two EPS).
"""
import torch

EPS = 2.0 ** -24
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


def sigmoid(v):
    return torch.where(v >= 0, 1 / (1 + torch.exp(-v.abs())),
                       torch.exp(-v.abs()) / (1 + torch.exp(-v.abs())))


def rounded(bound, ref, dtype):
    """A bound before the one rounding to the storage format, and the rounding's."""
    return bound + U[dtype] * (ref.abs() + bound) + TINY[dtype]


# ------------------------------------------------------------------ convolution


def conv_table(x, state, offsets, K):
    """Every sequence behind its state's rows: a list of [K - 1 + length][D]."""
    out = []
    for s in range(len(offsets) - 1):
        head = state[s] if state is not None else x.new_zeros(K - 1, x.shape[1])
        out.append(torch.cat([head, x[offsets[s]:offsets[s + 1]]]))
    return out


def conv(x, w, b, offsets, state, silu):
    """(y, last, bound of y) for x[tokens][D], w[D][K], b[D] or None."""
    K = w.shape[1]
    ys, lasts, errs = [], [], []
    for seq in conv_table(x, state, offsets, K):
        n = len(seq) - (K - 1)
        u = torch.zeros(n, x.shape[1], dtype=x.dtype) + (0 if b is None else b)
        size = u.abs()
        for k in range(K):
            u = u + seq[k:k + n] * w[:, k]
            size = size + (seq[k:k + n] * w[:, k]).abs()
        err = (K + 1) * EPS * size
        if silu:
            s = sigmoid(u)
            slope = s * (1 + u * (1 - s))
            err = err * slope.abs() + 8 * EPS * (u * s).abs()
            u = u * s
        ys.append(u)
        errs.append(err)
        lasts.append(seq[n:])
    return torch.cat(ys), torch.stack(lasts), torch.cat(errs)


def conv_grad(x, w, b, dy, offsets, state, dlast, silu):
    """(dx, dw, db, dstate) and their bounds."""
    K, D = w.shape[1], x.shape[1]
    dxs, dstates, exs, estates = [], [], [], []
    dw, db = torch.zeros_like(w), torch.zeros(D, dtype=x.dtype)
    ew, eb = torch.zeros_like(w), torch.zeros(D, dtype=x.dtype)
    tokens = max(1, x.shape[0])
    for i, seq in enumerate(conv_table(x, state, offsets, K)):
        n = len(seq) - (K - 1)
        g = dy[offsets[i]:offsets[i + 1]]
        eg = torch.zeros_like(g)
        if silu:
            u = torch.zeros(n, D, dtype=x.dtype) + (0 if b is None else b)
            size = u.abs()
            for k in range(K):
                u = u + seq[k:k + n] * w[:, k]
                size = size + (seq[k:k + n] * w[:, k]).abs()
            s = sigmoid(u)
            # the slope s (1 + u (1 - s)) changes by at most 1/2 for each unit of u
            eu = (K + 1) * EPS * size
            slope = s * (1 + u * (1 - s))
            eg = g.abs() * (0.5 * eu + 8 * EPS * s * (1 + (u * (1 - s)).abs())
                            + 3 * EPS * s * u.abs())
            g = g * slope
        back, eback = torch.zeros_like(seq), torch.zeros_like(seq)
        for k in range(K):
            back[k:k + n] += g * w[:, k]
            eback[k:k + n] += (eg + (K + 2) * EPS * g.abs()) * w[:, k].abs()
            dw[:, k] += (g * seq[k:k + n]).sum(0)
            ew[:, k] += ((eg + EPS * tokens * g.abs()) * seq[k:k + n].abs()).sum(0)
        db += g.sum(0)
        eb += (eg + EPS * tokens * g.abs()).sum(0)
        if dlast is not None:
            back[n:] += dlast[i]
            eback[n:] += 2 * EPS * dlast[i].abs()
        dxs.append(back[K - 1:])
        dstates.append(back[:K - 1])
        exs.append(eback[K - 1:])
        estates.append(eback[:K - 1])
    return ((torch.cat(dxs), dw, db, torch.stack(dstates)),
            (torch.cat(exs), ew, eb, torch.stack(estates)))


# ------------------------------------------------------------------ selective scan


def heads(v, D, N):
    """[tokens][groups N] as [tokens][D][N]."""
    n, G = v.shape[0], v.shape[1] // N
    return v.view(n, G, 1, N).expand(n, G, D // G, N).reshape(n, D, N)


def step_size(delta, bias, soft):
    """s, its slope, and the relative error of s."""
    v = delta + (0 if bias is None else bias)
    rel = torch.full_like(v, EPS if bias is not None else 0.0)
    if not soft:
        return v, torch.ones_like(v), rel
    s = v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    # the sum's rounding moves s by its slope, at most |v| + 1 of s; the rest are some twelve
    # operations
    return s, sigmoid(v), (13 + v.abs()) * EPS


def selective(x, delta, A, B, C, offsets, h0, skip, z, bias, soft, cut, grad=None):
    """(y, last) with bounds, or with grad = (dy, dlast) also the gradients and theirs, as
    dicts by name.  cut: the tokens of the longest range whose decay may be taken as one, the
    exponential of a sum of so many steps."""
    D, N = A.shape
    n = x.shape[0]
    s, slope, rel = step_size(delta, bias, soft)
    Bw, Cw = heads(B, D, N), heads(C, D, N)
    arg = s.unsqueeze(2) * A
    a = torch.exp(arg)
    # the step's error, log2 e times A, the product, the exponential; a range's sum
    ea = a * (arg.abs() * (rel.unsqueeze(2) + (3 + cut) * EPS) + 2 * EPS)
    u = (s * x).unsqueeze(2) * Bw
    eu = u.abs() * (rel.unsqueeze(2) + 2 * EPS)
    h, eh = torch.zeros(n, D, N, dtype=x.dtype), torch.zeros(n, D, N, dtype=x.dtype)
    hp, ehp = torch.zeros_like(h), torch.zeros_like(h)
    last, elast = [], []
    for i in range(len(offsets) - 1):
        state = h0[i] if h0 is not None else torch.zeros(D, N, dtype=x.dtype)
        e = torch.zeros_like(state)
        for t in range(offsets[i], offsets[i + 1]):
            hp[t], ehp[t] = state, e
            e = a[t] * e + ea[t] * state.abs() + eu[t]
            state = a[t] * state + u[t]
            e = e + EPS * (state.abs() + 0)
            h[t], eh[t] = state, e
        last.append(state)
        elast.append(e)
    k0 = skip if skip is not None else torch.zeros(D, dtype=x.dtype)
    v = (Cw * h).sum(2) + k0 * x
    ev = (Cw.abs() * (eh + (N + 2) * EPS * h.abs())).sum(2) + 2 * EPS * (k0 * x).abs()
    y, ey = v, ev
    if z is not None:
        sg = sigmoid(z)
        y = v * z * sg
        ey = (z * sg).abs() * ev + 8 * EPS * y.abs()
    out = {"y": y, "last": torch.stack(last)}
    err = {"y": ey, "last": torch.stack(elast)}
    if grad is None:
        return out, err
    dy, dlast = grad
    dv, edv = dy, torch.zeros_like(dy)
    if z is not None:
        dzs = sg * (1 + z * (1 - sg))
        out["z"] = dy * v * dzs
        err["z"] = (dy * dzs).abs() * ev + (dy * v).abs() * sg * (1 + (z * (1 - sg)).abs() + z.abs()) \
            * 12 * EPS
        dv = dy * z * sg
        edv = 8 * EPS * dv.abs()
    lam, elam = torch.zeros_like(h), torch.zeros_like(h)
    mus, emus = torch.zeros_like(h), torch.zeros_like(h)
    dh0, edh0 = [], []
    into = dv.unsqueeze(2) * Cw
    einto = (edv + EPS * dv.abs()).unsqueeze(2) * Cw.abs()
    for i in range(len(offsets) - 1):
        mu = dlast[i] if dlast is not None else torch.zeros(D, N, dtype=x.dtype)
        e = torch.zeros_like(mu)
        for t in range(offsets[i + 1] - 1, offsets[i] - 1, -1):
            l = into[t] + mu
            lam[t], elam[t] = l, einto[t] + e + EPS * l.abs()
            e = a[t] * elam[t] + ea[t] * l.abs()
            mu = a[t] * l
            e = e + EPS * mu.abs()
            mus[t], emus[t] = mu, e
        dh0.append(mu)
        edh0.append(e)
    q = mus * hp
    eq = emus * hp.abs() + mus.abs() * ehp + EPS * q.abs()
    ex = (lam * Bw).sum(2)
    eex = ((elam + (N + 2) * EPS * lam.abs()) * Bw.abs()).sum(2)
    out["x"] = s * ex + k0 * dv
    err["x"] = s.abs() * eex + (rel + 3 * EPS) * (s * ex).abs() + k0.abs() * (edv + 2 * EPS * dv.abs())
    ds = (q * A).sum(2)
    eds = ((eq + (N + 5) * EPS * q.abs()) * A.abs()).sum(2)
    dd = ds + x * ex
    out["delta"] = dd * slope
    # a sigmoid changes by at most itself for each unit of its argument
    es = (8 + (0 if not soft else 1) * (delta.abs() + 1)) * EPS if soft else 0.0
    err["delta"] = slope * (eds + x.abs() * (eex + EPS * ex.abs()) + 3 * EPS * dd.abs()) \
        + (dd * slope).abs() * es
    long = (n + 4) * EPS
    out["A"] = (q * s.unsqueeze(2)).sum(0)
    err["A"] = (eq * s.abs().unsqueeze(2) + (q * s.unsqueeze(2)).abs() * (rel.unsqueeze(2) + long)).sum(0)
    out["skip"] = (dv * x).sum(0)
    err["skip"] = ((edv + dv.abs() * long) * x.abs()).sum(0)
    out["delta_bias"] = out["delta"].sum(0)
    err["delta_bias"] = (err["delta"] + out["delta"].abs() * long).sum(0)
    G = B.shape[1] // N
    wide = (D // G + 4) * EPS
    f = lam * (s * x).unsqueeze(2)
    ef = elam * (s * x).abs().unsqueeze(2) + f.abs() * (rel.unsqueeze(2) + wide)
    out["B"] = f.view(n, G, D // G, N).sum(2).reshape(n, G * N)
    err["B"] = ef.view(n, G, D // G, N).sum(2).reshape(n, G * N)
    f = dv.unsqueeze(2) * h
    ef = edv.unsqueeze(2) * h.abs() + dv.abs().unsqueeze(2) * eh + f.abs() * wide
    out["C"] = f.view(n, G, D // G, N).sum(2).reshape(n, G * N)
    err["C"] = ef.view(n, G, D // G, N).sum(2).reshape(n, G * N)
    out["state"], err["state"] = torch.stack(dh0), torch.stack(edh0)
    return out, err


# ------------------------------------------------------------------ beams


def beam(scores, total, lse, beams, picks, finished=None, end=0):
    """The picks by the definition: 32-bit sums, ties to the lowest place."""
    import numpy as np
    rows, V = scores.shape
    base = total.astype(np.float32)
    if lse is not None:
        with np.errstate(invalid="ignore"):
            base = (base - lse.astype(np.float32)).astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        c = (scores.astype(np.float32) + base[:, None]).astype(np.float32)
    if finished is not None:
        over = finished != 0
        c[over] = -np.inf
        c[over, end] = total[over]
    c = np.where(np.isnan(c), np.float32(-np.inf), c) + np.float32(0)
    groups = rows // beams
    parent = np.empty((groups, picks), np.int32)
    token, out = np.empty_like(parent), np.empty((groups, picks), np.float32)
    for g in range(groups):
        flat = c[g * beams:(g + 1) * beams].reshape(-1)
        order = np.argsort(-flat, kind="stable")[:picks]
        for j in range(picks):
            at = int(order[j]) if j < len(order) else -1
            if at < 0 or flat[at] == -np.inf:
                parent[g, j], token[g, j], out[g, j] = g * beams + j % beams, -1, -np.inf
            else:
                parent[g, j], token[g, j], out[g, j] = g * beams + at // V, at % V, flat[at]
    return parent, token, out

"""Layer norm and the gated delta rule in binary64, step by step from their definitions (numpy, no code of the package), with the sizes that binary32's
roundings of them are counted in."""
import numpy as np

from seq_oracle import U, _length, sigmoid


# ---- layer norm -----------------------------------------------------------------------------------------------------
def norm(x, w, b, eps, dy=None, add=None):
    """A dict of the outputs, and of how far a computation in binary32 may be from them (besides an output's own rounding).

    A sum of n terms in any order is within n u of the sum of their sizes.  E: of x - mean; R: relative, of r (half the variance's own, in which E enters twice)."""
    F = x.shape[1]
    w = np.ones(F) if w is None else w
    mean = x.mean(1, keepdims=True)
    d = x - mean
    s = np.sqrt((d * d).mean(1, keepdims=True) + eps)
    r = 1 / s
    h = d * r
    E = U * (np.abs(x) + np.abs(mean) + (F + 8) * np.abs(x).mean(1, keepdims=True))
    R = E.max(1, keepdims=True) * r + (F / 2 + 8) * U
    off_h = r * E + np.abs(h) * (R + 2 * U)
    out = {"y": h * w + (0 if b is None else b)}
    off = {"y": np.abs(w) * off_h + 4 * U * np.abs(h * w) + (0 if b is None else U * np.abs(b))}
    if dy is None:
        return out, off
    g = dy * w
    m1, m2 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    off1 = (F + 8) * U * np.abs(g).mean(1, keepdims=True)
    off2 = (F + 10) * U * np.abs(g * h).mean(1, keepdims=True) + (np.abs(g) * off_h).mean(1, keepdims=True)
    out["dx"] = r * (g - m1 - h * m2) + (0 if add is None else add)
    off["dx"] = r * (U * np.abs(g) + off1 + np.abs(h) * off2 + np.abs(m2) * off_h) + (R + 6 * U) * r * (np.abs(g) + np.abs(m1) + np.abs(h * m2)) + (0 if add is None else U * np.abs(add))
    out["dw"], out["db"] = (dy * h).sum(0), dy.sum(0)
    M = len(x)
    off["dw"] = (np.abs(dy) * off_h).sum(0) + (M + 8) * U * np.abs(dy * h).sum(0)
    off["db"] = (M + 8) * U * np.abs(dy).sum(0)
    return out, off


# ---- gated delta rule -------------------------------------------------------------------------------------------------
def unit(x):
    return 1 / np.sqrt((x * x).sum(-1, keepdims=True) + 1e-6)


def delta(q, k, v, a, b, A, a_bias=None, scale=1.0, normalize=True, softplus=True, starts=None, lengths=None, h_in=None, dy=None, dh_out=None):
    """A dict of the outputs; with dy the gradients too; and sizes of a head's sequence: "state" [N,H,V], the most that a column of the state and a value have together,
    "grad" [N,H,V], the same of the state's gradient and the output's."""
    T, N, G, K = q.shape
    H, V = v.shape[2:]
    per = H // G
    group = np.arange(H) // per
    qu, ku = (unit(x) if normalize else np.ones((T, N, G, 1)) for x in (q, k))
    x = a + (0 if a_bias is None else a_bias)
    step = np.logaddexp(0, x) if softplus else x
    rise = sigmoid(x) if softplus else np.ones_like(x)
    alpha, beta = np.exp(step * A), sigmoid(b)
    S = np.zeros((N, H, K, V)) if h_in is None else h_in.astype(float).copy()
    out, kept = {"y": np.zeros_like(v)}, {}
    length = [_length(lengths, n, T) for n in range(N)]
    state = np.zeros((N, H, V))
    for t in range(T):
        for n in range(N):
            if t >= length[n]:
                continue
            begin = starts is not None and bool(starts[t, n])
            kt, qt = (k[t, n] * ku[t, n])[group], (q[t, n] * qu[t, n])[group] * scale          # [H,K]
            past = np.zeros((H, K, V)) if begin else S[n].copy()
            al = np.zeros(H) if begin else alpha[t, n]
            moved = al[:, None, None] * past
            z = v[t, n] - np.einsum("hk,hkv->hv", kt, moved)
            state[n] = np.maximum(state[n], np.abs(v[t, n]) + np.sqrt((past ** 2).sum(1)))
            S[n] = moved + (beta[t, n][:, None] * kt)[:, :, None] * z[:, None, :]
            out["y"][t, n] = np.einsum("hk,hkv->hv", qt, S[n])
            kept[t, n] = (kt, qt, past, al, z, S[n].copy(), begin)
    out["h_out"] = S
    sizes = {"state": state + np.sqrt((S ** 2).sum(2))}
    if dy is None:
        return out, sizes
    g = np.zeros((N, H, K, V)) if dh_out is None else dh_out.astype(float).copy()
    grad = np.sqrt((g ** 2).sum(2))
    dqu, dku = np.zeros((T, N, G, K)), np.zeros((T, N, G, K))
    out["dv"], out["da"], out["db"], out["dA"] = np.zeros_like(v), np.zeros_like(a), np.zeros_like(a), np.zeros(H)
    for t in reversed(range(T)):
        for n in range(N):
            if t >= length[n]:
                continue
            kt, qt, past, al, z, now, begin = kept[t, n]
            gt = g[n] + qt[:, :, None] * dy[t, n][:, None, :]
            dq = scale * np.einsum("hkv,hv->hk", now, dy[t, n])
            gk = np.einsum("hkv,hk->hv", gt, kt)
            dz = beta[t, n][:, None] * gk
            dk = beta[t, n][:, None] * np.einsum("hkv,hv->hk", gt, z) - al[:, None] * np.einsum("hkv,hv->hk", past, dz)
            np.add.at(dqu[t, n], group, dq)
            np.add.at(dku[t, n], group, dk)
            out["dv"][t, n] = dz
            out["db"][t, n] = (gk * z).sum(1) * beta[t, n] * (1 - beta[t, n])
            back = gt - kt[:, :, None] * dz[:, None, :]
            if not begin:
                dlog = al * (back * past).sum((1, 2))
                out["dA"] += dlog * step[t, n]
                out["da"][t, n] = dlog * A * rise[t, n]
            g[n] = 0 if begin else al[:, None, None] * back
            grad[n] = np.maximum(grad[n], np.sqrt((g[n] ** 2).sum(1)) + np.sqrt((gt ** 2).sum(1)))
    out["da_bias"], out["dh_in"] = out["da"].sum((0, 1)), g
    if normalize:
        for name, x, r, d in (("dq", q, qu, dqu), ("dk", k, ku, dku)):
            n = x * r
            out[name] = r * (d - n * (n * d).sum(-1, keepdims=True))
    else:
        out["dq"], out["dk"] = dqu, dku
    sizes["grad"] = grad
    return out, sizes


def allowed(sizes, shapes, T, K, A, alpha=None, dy=None, scale=1.0, normalize=True, k=None, q=None):
    """How far each output may be off besides its own rounding, from the sizes of its head's sequence.

    A step adds to a column of the state what is rounded of the sums that it takes part in: over the K entries of a key, over the up to 64 steps before it in its chunk, and in
    the substitution for their inverse again.  The products' factors are lengths (by Cauchy and Schwarz), so each rounding is at most u times the column's size, and since
    decays and 1 - be k k^T lengthen nothing the later steps carry it on without growth.  These are roundings of either sign: T (64 x 64 + K) of them are off by their root, and
    eight such deviations are more than any of the tests' entries has.  A gradient along the values is a sum over V of products of the state's and the gradient's columns;
    that of a decay's logarithm is one over pairs of steps on both sides, and every term has the decay as a factor."""
    R = 8 * np.sqrt(T * (64 * 64 + K)) * U
    s, off = sizes["state"], {}
    off["y"], off["h_out"] = np.broadcast_to(R * scale * s, shapes["y"]), R * s[:, :, None, :] * np.ones((1, 1, K, 1))
    if "grad" not in sizes:
        return off
    g, H = sizes["grad"], s.shape[1]
    both = np.sqrt((s ** 2).sum(2)) * np.sqrt((g ** 2).sum(2))               # [N,H]
    asked = scale * np.sqrt((dy ** 2).sum(3)).max(0) * np.sqrt((s ** 2).sum(2))
    G = shapes["dq"][2]
    grouped = lambda x: x.reshape(len(x), G, H // G).sum(2)  # noqa: E731
    qu, ku = (unit(x) if normalize else np.ones((*x.shape[:3], 1)) for x in (q, k))
    off["dv"] = np.broadcast_to(2 * R * g, shapes["dv"])
    off["dq"], off["dk"] = 2 * R * grouped(asked)[None, :, :, None] * qu * np.ones(K), 4 * R * grouped(both)[None, :, :, None] * ku * np.ones(K)
    off["db"] = np.broadcast_to(2 * R * both, shapes["db"])
    off["dlog"] = 8 * R * both * alpha                                       # [T,N,H]
    off["da"] = off["dlog"] * np.abs(A)
    off["da_bias"] = off["da"].sum((0, 1))
    off["dh_in"] = 2 * R * g[:, :, None, :] * np.ones((1, 1, K, 1))
    return off

"""The attention block's operators in 64 bits on the CPU, from their formulas,
with what bounds the rounding of the GPU's results.

u = 2^-8 is the unit roundoff of bf16.  What the kernels round to bf16 are the
probabilities P (before they meet v or dout), dS (before k or q) and every
stored result; sums are fp32.  So, with B_i = sum_j P_ij |v_j|,

  |out error|   <= u (|out| + B)                     (inference)
                   u |out| + u^2 B                   (a training step: P in parts)
  |delta error| <= eps_i = u^2 sum |dout| B          (rows' sums of dout out)
  |dv error|    <= u (|dv| + P^T |dout|)
  |dq error|    <= u (|dq| + scale |dS| |k|) + scale P eps |k|, dk likewise
  |dtable error| <= sum over the bucket of P eps

each with fp32's own error on top: 1e-5 of the largest sum of the terms'
absolute values (lengths here are a few hundred; a result may cancel, dS = P (dP
- delta) above all, its terms P dP and P delta do not).
"""
import numpy as np

U = 2.0 ** -8
F32 = 1e-5


def heads_of(x, heads):
    """[N, 4, C, H, W] -> [N, heads, H W, 4 dq]"""
    n, _, c, h, w = x.shape
    dq = c // heads
    return x.transpose(0, 3, 4, 1, 2).reshape(n, h * w, 4, heads, dq).transpose(0, 3, 1, 2, 4).reshape(n, heads, h * w, 4 * dq)


def map_of(t, h, w):
    n, heads, _, d = t.shape
    return t.reshape(n, heads, h, w, 4, d // 4).transpose(0, 4, 1, 5, 2, 3).reshape(n, 4, heads * (d // 4), h, w)


def buckets(hq, wq, hk, wk, by, bx, nx, pos):
    """[hq wq, hk wk] bucket of every pair of pixels."""
    ky, kx = np.divmod(np.arange(hk * wk), wk)
    qy, qx = np.divmod(np.arange(hq * wq), wq)
    out = np.zeros((hq * wq, hk * wk), np.int64)
    for b, k, q, p, mul in ((by, ky, qy, pos[0], nx), (bx, kx, qx, pos[1], 1)):
        if b is None:
            continue
        r = len(b) // 2
        out += mul * np.asarray(b)[np.clip(k[None, :] - q[:, None] - p, -r, r) + r]
    return out


def attention(q, k, v, heads, table=None, by=None, bx=None, kv_len=None, pos=None, scale=None, dout=None):
    """Outputs and error bounds (for bf16 maps) of forward and backward:
    dicts with out, stats, and with dout dq, dk, dv, dtable."""
    n, _, c, hq, wq = q.shape
    _, _, ckv, hk, wk = k.shape
    dq_ = c // heads
    kvh = ckv // dq_
    group = heads // kvh
    scale = 1.0 / np.sqrt(4 * dq_) if scale is None else scale
    Q, K, V = heads_of(q, heads), heads_of(k, kvh), heads_of(v, kvh)
    G = None if dout is None else heads_of(dout, heads)
    lk = hk * wk
    out, B, Bt = np.zeros_like(Q), np.zeros_like(Q), None
    lse = np.full(Q.shape[:3], -np.inf)
    names = ("dq", "dk", "dv")
    res, err, size = {}, {}, {}
    if G is not None:
        g = {"dq": np.zeros_like(Q), "dk": np.zeros_like(K), "dv": np.zeros_like(V)}
        e = {m: np.zeros_like(t) for m, t in g.items()}
        z = {m: np.zeros_like(t) for m, t in g.items()}
        nb = None if table is None else table.reshape(heads, -1).shape[1]
        dt = None if table is None else np.zeros((heads, nb))
        et = None if table is None else np.zeros((heads, nb))
        zt = None if table is None else np.zeros((heads, nb))
    for i in range(n):
        m = lk if kv_len is None else int(min(max(kv_len[i], 0), lk))
        idx = None
        if table is not None:
            nx = table.shape[2]
            idx = buckets(hq, wq, hk, wk, by, bx, nx, (0, 0) if pos is None else pos[i])[:, :m]
        if m == 0:
            continue
        for h in range(heads):
            kh, vh = K[i, h // group, :m], V[i, h // group, :m]
            s = scale * Q[i, h] @ kh.T
            if idx is not None:
                s = s + table.reshape(heads, -1)[h][idx]
            top = s.max(1, keepdims=True)
            p = np.exp(s - np.where(np.isneginf(top), 0, top))
            tot = p.sum(1, keepdims=True)
            with np.errstate(divide="ignore"):
                lse[i, h] = (np.where(np.isneginf(top), 0, top) + np.log(tot))[:, 0]
            p = p / np.where(tot == 0, 1, tot)
            out[i, h] = p @ vh
            B[i, h] = p @ np.abs(vh)
            if G is None:
                continue
            go = G[i, h]
            dp = go @ vh.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            eps = U * U * (np.abs(go) * B[i, h]).sum(1, keepdims=True)
            pe = p * eps
            g["dq"][i, h] = scale * ds @ kh
            g["dk"][i, h // group, :m] += scale * ds.T @ Q[i, h]
            g["dv"][i, h // group, :m] += p.T @ go
            e["dq"][i, h] = scale * (U * np.abs(ds) + pe) @ np.abs(kh)
            e["dk"][i, h // group, :m] += scale * (U * np.abs(ds) + pe).T @ np.abs(Q[i, h])
            e["dv"][i, h // group, :m] += U * p.T @ np.abs(go)
            terms = p * (np.abs(go) @ np.abs(vh).T + (np.abs(go) * B[i, h]).sum(1, keepdims=True))
            z["dq"][i, h] = scale * terms @ np.abs(kh)
            z["dk"][i, h // group, :m] += scale * terms.T @ np.abs(Q[i, h])
            z["dv"][i, h // group, :m] += p.T @ np.abs(go)
            if dt is not None:
                np.add.at(zt[h], idx.reshape(-1), terms.reshape(-1))
                np.add.at(dt[h], idx.reshape(-1), ds.reshape(-1))
                np.add.at(et[h], idx.reshape(-1), pe.reshape(-1))
    res["out"], res["lse"] = map_of(out, hq, wq), lse
    size["out"] = B
    err["out"] = U * (np.abs(res["out"]) + (U if G is not None else 1.0) * map_of(B, hq, wq))
    if G is not None:
        for name, (h, w) in zip(names, ((hq, wq), (hk, wk), (hk, wk))):
            res[name] = map_of(g[name], h, w)
            err[name] = U * np.abs(res[name]) + map_of(e[name], h, w)
            size[name] = z[name]
        if table is not None:
            res["dtable"], err["dtable"], size["dtable"] = dt.reshape(table.shape), et.reshape(table.shape), zt
    for name in err:
        err[name] = (err[name], F32 * float(np.abs(size[name]).max()))
    return res, err


def check(got, ref, err, bf16, what):
    """|got - ref| <= the bf16 bound (if any) + fp32's."""
    got = np.asarray(got, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.all(np.isfinite(got)), f"{what}: non-finite values"
    bound = err[1] + (1.01 * err[0] if bf16 else 0.0)
    off = np.abs(got - ref) - bound
    if np.any(off > 0):
        i = np.unravel_index(np.argmax(off), off.shape)
        raise AssertionError(f"{what}: {int((off > 0).sum())} of {off.size} outside; worst at {i}: got {got[i]:.8g}, "
                             f"ref {ref[i]:.8g}, bound {np.broadcast_to(bound, off.shape)[i]:.3g}")


MUL, WEYL = (0xD2511F53, 0xCD9E8D57), (0x9E3779B9, 0xBB67AE85)


def philox(counter, key, rounds=7):
    """Philox 4x32 in plain integers: four words."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = MUL[0] * c[0], MUL[1] * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[i] + WEYL[i]) & 0xFFFFFFFF for i in range(2)]
    return c


def drop_factors(n, c, h, w, p, seed, offset):
    """[N, 4, C, H, W] factors 0 or 1 / (1 - p')."""
    cut = int(round(float(np.float32(p)) * 65536))
    if cut == 0:
        return np.ones((n, 4, c, h, w))
    rows = np.zeros((n * h * w, 4 * c))
    for m in range(n * h * w):
        for ch in range((4 * c + 7) // 8):
            words = philox((ch, m, offset & 0xFFFFFFFF, offset >> 32 & 0xFFFFFFFF), (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
            for j in range(8 * ch, min(8 * ch + 8, 4 * c)):
                bits = words[j % 8 // 2] >> (16 * (j % 2)) & 0xFFFF
                rows[m, j] = 65536.0 / (65536 - cut) if bits >= cut else 0.0
    return rows.reshape(n, h, w, 4, c).transpose(0, 3, 4, 1, 2)


def _col(t):
    return 1.0 if t is None else t[None, :, :, None, None]


def residual(x, y, gamma, gate, scale, next_gamma, factors, eps):
    def norm(t):
        return t / np.sqrt((t * t).mean((1, 2), keepdims=True) + eps)
    z = y if gamma is None else norm(y) * _col(gamma)
    out = x + _col(scale) * (1.0 if gate is None else gate) * factors * z
    return out, None if next_gamma is None else norm(out) * _col(next_gamma)


def residual_gradients(y, dout, gamma, gate, scale, next_gamma, out, dh, factors, eps):
    res = {}
    G = dout.copy()
    if next_gamma is not None:
        r = 1 / np.sqrt((out * out).mean((1, 2), keepdims=True) + eps)
        hat, u = out * r, dh * _col(next_gamma)
        res["dnext_gamma"] = (dh * hat).sum((0, 3, 4))
        G = G + r * (u - hat * (u * hat).mean((1, 2), keepdims=True))
    res["dx"] = G
    r = 1 / np.sqrt((y * y).mean((1, 2), keepdims=True) + eps) if gamma is not None else 1.0
    hat, gm = y * r, G * factors
    gt = 1.0 if gate is None else gate
    if gamma is not None:
        res["dgamma"] = (gm * hat * gt * _col(scale)).sum((0, 3, 4))
    if scale is not None:
        res["dscale"] = (gm * hat * gt * _col(gamma)).sum((0, 3, 4))
    if gate is not None:
        res["dgate"] = (gm * hat * _col(gamma) * _col(scale)).sum((3, 4), keepdims=True)
    u = gm * gt * _col(scale) * _col(gamma)
    res["dy"] = r * (u - hat * (u * hat).mean((1, 2), keepdims=True)) if gamma is not None else u
    return res

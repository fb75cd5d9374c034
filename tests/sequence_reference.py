"""The operators on sequences of pixels in 64 bits on the CPU, from their
formulas, with what bounds the rounding of the GPU's results.

u = 2^-8 is the unit roundoff of bf16.  With bf16 maps, B_i = sum_j P_ij |v_j|:

cache attention (probabilities keep 16 bits: u^2 of each)
  |out error|   <= u |out| + u^2 B
packed attention (probabilities and dS rounded to bf16 before a product, but in a
training step's forward pass probabilities keep 16 bits too)
  |out error|   <= u (|out| + B)                        (inference)
                   u |out| + u^2 B                      (a training step)
  |delta error| <= eps_i = u^2 sum |dout| B             (rows' sums of dout out)
  |dv error|    <= u (|dv| + P^T |dout|)
  |dq error|    <= u (|dq| + scale |dS| |k|) + scale P eps |k|, dk likewise

each with fp32's own error on top, all there is with fp32 maps: 1e-5 of the
largest sum of the terms' absolute values (lengths here are a few hundred, of
the cache a few thousand with a term each of 1 / length; a result may cancel,
dS = P (dP - delta) above all, its terms P dP and P delta do not).
"""
import numpy as np

U = 2.0 ** -8
F32 = 1e-5


def rows_of(x, heads):
    """[N, 4, C, H, W] -> [N H W, heads, 4 dq]"""
    n, _, c, h, w = x.shape
    return x.transpose(0, 3, 4, 1, 2).reshape(n * h * w, 4, heads, c // heads).transpose(0, 2, 1, 3).reshape(n * h * w, heads, -1)


def map_of(t, n, h, w):
    _, heads, d = t.shape
    return t.reshape(n, h, w, heads, 4, d // 4).transpose(0, 4, 3, 5, 1, 2).reshape(n, 4, heads * (d // 4), h, w)


def quantise(x):
    """[..., reals] -> (elements' values, bytes e + 127), e4m3 with the least e >=
    -117 whose 448 2^e no magnitude exceeds; with e = 120 at most 240 (256 2^120 is
    beyond fp32)."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(top)
    mant, e = np.frexp(np.where(bad | (top == 0), 1.0, top))  # [1/2, 1) 2^e; 448 = 7/8 2^9
    e = np.where(top == 0, -117, np.maximum(e - 9 + (mant > 0.875), -117))
    y = np.where(bad[..., None], 0.0, x) * 2.0 ** -e[..., None].astype(np.float64)
    _, ye = np.frexp(np.where(y == 0, 1.0, y))
    step = 2.0 ** (np.maximum(ye - 1, -6) - 3).astype(np.float64)
    y = np.round(y / step) * step  # (half to even)
    most = np.where(e == 120, 240.0, 448.0)[..., None]
    return np.where(bad[..., None], np.nan, np.clip(y, -most, most)), np.where(bad, 255, e + 127)


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int)


def cache_attention(q, keys, values, lens, heads, table=None, by=None, bx=None, pos=None, width=1, scale=None):
    """q [n, heads, d]; keys, values: per sequence [positions, kv heads, d].
    (out [n, heads, d], bf16 bound, size for fp32's)"""
    n, _, d = q.shape
    out, bound = np.zeros_like(q), np.zeros_like(q)
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    for i in range(n):
        m = min(max(int(lens[i]), 0), len(keys[i]))
        here = [j for j in range(m) if keys[i][j] is not None]
        if not here:
            continue
        at = np.array(here)
        k, v = np.stack([keys[i][j] for j in here]), np.stack([values[i][j] for j in here])
        for h in range(heads):
            g = h // (heads // k.shape[1])
            s = scale * k[:, g] @ q[i, h]
            if table is not None:
                idx = np.zeros(len(at), int)
                for b, a, p, mul in ((by, at // width, 0 if pos is None else pos[i][0], table.shape[2]),
                                     (bx, at % width, 0 if pos is None else pos[i][1], 1)):
                    if b is not None:
                        r = len(b) // 2
                        idx += mul * np.asarray(b)[np.clip(a - int(p), -r, r) + r]
                s = s + table[h].reshape(-1)[idx]
            top = s.max()
            if np.isneginf(top):
                continue
            p = np.exp(s - top)
            p /= p.sum()
            out[i, h], bound[i, h] = p @ v[:, g], p @ np.abs(v[:, g])
    return out, U * np.abs(out) + U * U * bound, float(bound.max())


def packed(q, k, v, lq, lk, causal=True, scale=None, dout=None):
    """Rows [tokens, heads, d] of packed sequences of lq queries and lk keys.
    (results, bounds): dicts of out, lse and with dout dq, dk, dv; a bound is
    (of bf16 maps, of fp32 on top)."""
    heads, d = q.shape[1:]
    kvh = k.shape[1]
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    res = {"out": np.zeros_like(q), "lse": np.full(q.shape[:2], -np.inf)}
    if dout is not None:
        res.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v))
    err = {m: np.zeros_like(t) for m, t in res.items() if m != "lse"}
    size = {m: 0.0 for m in err}
    terms_k = {"dk": np.zeros_like(k), "dv": np.zeros_like(v)}
    for a, nq, b, nk in zip(starts(lq), lq, starts(lk), lk):
        sees = np.ones((nq, nk), bool)
        if causal:
            sees = np.arange(nk)[None, :] <= np.arange(nq)[:, None] + nk - nq
        if nq == 0 or nk == 0:
            continue
        for h in range(heads):
            g = h // (heads // kvh)
            qh, kh, vh = q[a:a + nq, h], k[b:b + nk, g], v[b:b + nk, g]
            s = np.where(sees, scale * qh @ kh.T, -np.inf)
            top = s.max(1, keepdims=True)
            p = np.where(sees, np.exp(s - np.where(np.isneginf(top), 0, top)), 0.0)
            tot = p.sum(1, keepdims=True)
            with np.errstate(divide="ignore"):
                res["lse"][a:a + nq, h] = (np.where(np.isneginf(top), 0, top) + np.log(tot))[:, 0]
            p = p / np.where(tot == 0, 1, tot)
            out, B = p @ vh, p @ np.abs(vh)
            res["out"][a:a + nq, h] = out
            err["out"][a:a + nq, h] = U * (np.abs(out) + (1.0 if dout is None else U) * B)
            size["out"] = max(size["out"], float(B.max()))
            if dout is None:
                continue
            go = dout[a:a + nq, h]
            dp = go @ vh.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            pe = p * (np.abs(go) * U * U * B).sum(1, keepdims=True)
            off = abs(scale) * (U * np.abs(ds) + pe)
            terms = p * (np.abs(go) @ np.abs(vh).T + (np.abs(go) * B).sum(1, keepdims=True))
            res["dq"][a:a + nq, h] = scale * ds @ kh
            res["dk"][b:b + nk, g] += scale * ds.T @ qh
            res["dv"][b:b + nk, g] += p.T @ go
            err["dq"][a:a + nq, h] = off @ np.abs(kh)
            err["dk"][b:b + nk, g] += off.T @ np.abs(qh)
            err["dv"][b:b + nk, g] += U * p.T @ np.abs(go)
            size["dq"] = max(size["dq"], float((abs(scale) * terms @ np.abs(kh)).max()))
            terms_k["dk"][b:b + nk, g] += abs(scale) * terms.T @ np.abs(qh)
            terms_k["dv"][b:b + nk, g] += p.T @ np.abs(go)
    for m in ("dq", "dk", "dv"):
        if m in res:
            err[m] += U * np.abs(res[m])
            if m in terms_k and terms_k[m].size:
                size[m] = float(terms_k[m].max())
    return res, {m: (err[m], F32 * size[m]) for m in err}


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

"""Differential attention in 64 bits (numpy), one head after the other, with the error bounds that the GPU tests use:
test infrastructure, written from the formulas."""
import numpy as np

U32, U16 = 2.0 ** -24, 2.0 ** -8          # half a step of fp32 and of bf16, relative


def lens(given, B, full):
    return [full] * B if given is None else [min(max(int(x), 0), full) for x in given]


def visible(ql, kl, Nq, Nk, causal):
    t, u = np.arange(Nq)[:, None], np.arange(Nk)[None, :]
    vis = (t < ql) & (u < kl)
    return vis & (u <= kl - ql + t) if causal else vis


def softmax(s, vis):
    s = np.where(vis, s, -np.inf)
    m = s.max(-1, keepdims=True)
    e = np.where(vis, np.exp(s - np.where(np.isfinite(m), m, 0.0)), 0.0)
    z = e.sum(-1, keepdims=True)
    return np.divide(e, z, out=np.zeros_like(e), where=z > 0)


def clean(x, n):
    """Rows from n on do not count, whatever stands there."""
    x = np.array(x, dtype=np.float64)
    x[n:] = 0.0
    return x


def run(q, k, v, lam, causal, q_lens=None, kv_lens=None, scale=None, dout=None, bf16=True, tensor_cores=True):
    """Returns {name: (value, tolerance)} for out (and dq, dk, dv, dlam when dout is given).

    Bounds, to first order.  Scores: a dot product of d terms and the scaling, (d + 3) steps of |q| |k|.  A weight is off
    by twice the largest score error of its row (it is a quotient), by the exponential's 2 ulp and by the sum's roundings,
    relative: rel.  Weights rounded to 16 bits for the tensor cores add 2^-8 of themselves.  Sums of n products add
    n steps of the sum of magnitudes.  Results are rounded to storage once; the backward reads out and A_2 V in storage."""
    B, H, Nq, D = q.shape
    Hk, Nk = k.shape[1], k.shape[2]
    g, d = H // Hk, D // 2
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    lam = np.broadcast_to(np.asarray(lam, dtype=np.float64), (H,))
    QL, KL = lens(q_lens, B, Nq), lens(kv_lens, B, Nk)
    wr = U16 if bf16 and tensor_cores else 0.0        # rounding of the weights
    sr = U16 if bf16 else U32                         # rounding of results to storage
    res = {"out": (np.zeros(q.shape), np.zeros(q.shape))}
    if dout is not None:
        for name, x in (("dq", q), ("dk", k), ("dv", v)):
            res[name] = (np.zeros(x.shape), np.zeros(x.shape))
        res["dlam"] = (np.zeros(H), np.zeros(H))
    for b in range(B):
        vis = visible(QL[b], KL[b], Nq, Nk, causal)
        for h in range(H):
            qq, kk, vv = clean(q[b, h], QL[b]), clean(k[b, h // g], KL[b]), clean(v[b, h // g], KL[b])
            halves = [slice(0, d), slice(d, D)]
            P, rel = [], []
            for c in halves:
                P.append(softmax(qq[:, c] @ kk[:, c].T * scale, vis))
                es = (d + 3) * U32 * abs(scale) * np.where(vis, np.abs(qq[:, c]) @ np.abs(kk[:, c]).T, 0).max(-1, keepdims=True)
                rel.append(2 * es + (Nk + 8) * U32)
            o1, o2 = P[0] @ vv, P[1] @ vv
            av = np.abs(vv)
            t1 = ((rel[0] + wr + Nk * U32) * P[0]) @ av
            t2 = ((rel[1] + wr + Nk * U32) * P[1]) @ av
            L = abs(lam[h])
            out = o1 - lam[h] * o2
            tol = t1 + L * t2 + 4 * U32 * (np.abs(o1) + L * np.abs(o2))
            res["out"][0][b, h], res["out"][1][b, h] = out, tol + sr * np.abs(out)
            if dout is None:
                continue
            do = clean(dout[b, h], QL[b])
            ado = np.abs(do)
            dA = do @ vv.T
            edA = (D + 2) * U32 * (ado @ av.T)
            delta = [(do * o1).sum(-1, keepdims=True), (do * o2).sum(-1, keepdims=True)]
            t_out, t_o2 = tol + sr * np.abs(out), t2 + sr * np.abs(o2) + 4 * U32 * np.abs(o2)
            e2 = (ado * (t_o2 + D * U32 * np.abs(o2))).sum(-1, keepdims=True)
            e1 = (ado * (t_out + D * U32 * np.abs(out))).sum(-1, keepdims=True) + L * e2
            sign = [1.0, -lam[h]]
            A = P[0] - lam[h] * P[1]
            eA = rel[0] * P[0] + L * rel[1] * P[1] + 4 * U32 * (P[0] + L * P[1]) + wr * np.abs(A)
            kv = (b, h // g)
            res["dv"][0][kv] += A.T @ do
            res["dv"][1][kv] += eA.T @ ado + Nq * U32 * (np.abs(A).T @ ado)
            for i, c in enumerate(halves):
                w = P[i]
                ds = sign[i] * scale * w * (dA - delta[i])
                eds = abs(sign[i] * scale) * w * ((rel[i] + 8 * U32) * np.abs(dA - delta[i]) + edA + (e1, e2)[i]
                                                  + U32 * np.abs(delta[i])) + wr * np.abs(ds)
                ak, aq = np.abs(kk[:, c]), np.abs(qq[:, c])
                res["dq"][0][b, h][:, c] = ds @ kk[:, c]
                res["dq"][1][b, h][:, c] = eds @ ak + Nk * U32 * (np.abs(ds) @ ak)
                res["dk"][0][kv][:, c] += ds.T @ qq[:, c]
                res["dk"][1][kv][:, c] += eds.T @ aq + Nq * g * U32 * (np.abs(ds).T @ aq)
            terms = P[1] * dA
            res["dlam"][0][h] -= terms.sum()
            # (a thread's running sum is shorter than the row; 1024 steps cover what it adds up in fp32)
            res["dlam"][1][h] += (P[1] * (rel[1] * np.abs(dA) + edA) + 1024 * U32 * np.abs(terms)).sum()
    if dout is not None:
        for name in ("dq", "dk", "dv"):
            val, tol = res[name]
            res[name] = (val, tol + sr * np.abs(val))
    return res

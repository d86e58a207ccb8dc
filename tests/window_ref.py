"""The decoder stack in float64 with a sliding attention window: plain numpy, token by token of the formulas.

Sync block: R = X + sum_i Y_i, out = R + sum_i Z_i(R); SPD block: Z_i sees X + Y_i, out = X + sum_i Y_i + sum_i Z_i.
"""
import numpy as np

import oracle


def stack_forward(w, mask, layers, x, pos0, kc, vc, window=0, sinks=0):
    """x [B, S, H]; kc, vc [n_layers, B, max_len, nkv, d] are written at pos0[b] on.  Returns [B, S, H]."""
    x = np.asarray(x, dtype=np.float64)
    B, S, H = x.shape
    nq, nkv, d, T = w.n_q_heads, w.n_kv_heads, w.head_dim, w.T
    for l, lw in enumerate(layers):
        W = {n: np.asarray(t, dtype=np.float64) for n, t in lw.items()}

        def norm(t, g):
            return t / np.sqrt(np.mean(t * t, -1, keepdims=True) + w.rms_eps) * g

        h = norm(x, W["attn_norm"])
        q, k, v = ((h @ W[n].T).reshape(B, S, -1, d) for n in ("wq", "wk", "wv"))
        a = np.zeros((B, S, nq, d))
        for b in range(B):
            for i in range(S):
                p = int(pos0[b]) + i
                if w.rope_base > 0:
                    for t in (q, k):
                        for j in range(t.shape[2]):
                            t[b, i, j] = oracle.rope(t[b, i, j], p, w.rope_base)
                kc[l, b, p], vc[l, b, p] = k[b, i], v[b, i]
                t = np.arange(p + 1)
                seen = (t > p - window) | (t < sinks) if window else t >= 0
                K, V = kc[l, b, :p + 1][seen], vc[l, b, :p + 1][seen]
                for j in range(nq):
                    s = K[:, j * nkv // nq] @ q[b, i, j] / np.sqrt(d)
                    e = np.exp(s - s.max())
                    a[b, i, j] = e @ V[:, j * nkv // nq] / e.sum()
        a = a.reshape(B, S, nq * d)
        qs, fs = nq * d // T, w.ffn // T
        Y = [a[..., i * qs:(i + 1) * qs] @ W["wo"][:, i * qs:(i + 1) * qs].T for i in range(T)]
        r = x + sum(Y)
        out = r.copy()
        for i in range(T):
            u = norm(r if mask[l] else x + Y[i], W["mlp_norm"])
            g, up = (u @ W[n][i * fs:(i + 1) * fs].T for n in ("w_gate", "w_up"))
            out += (g / (1 + np.exp(-g)) * up) @ W["w_down"][:, i * fs:(i + 1) * fs].T
        x = out
    return x

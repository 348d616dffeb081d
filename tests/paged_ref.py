"""Plain float64 forms of the paged cache's operators, and a pool to run them on, for the GPU tests."""
from __future__ import annotations

import numpy as np

from paper_2604_21215_amd import inputs as gen


def quantise(u):
    """Rows of 64 (last axis) -> (codes float64, bytes): definition of an 8-bit row, by search over the exponents."""
    u = np.asarray(u, dtype=np.float64)
    top = np.abs(u).max(-1)
    byte = np.zeros(top.shape, dtype=np.int64)
    codes = np.zeros(u.shape)
    for i in np.ndindex(top.shape):
        if not np.isfinite(top[i]):
            byte[i] = 255
            continue
        if top[i] == 0:
            continue
        e = max(-126, int(np.floor(np.log2(top[i]))) - 8)
        while top[i] > 127 * 2.0 ** e:
            e += 1
        byte[i] = e + 127
        codes[i] = np.rint(u[i] / 2.0 ** e)
    return codes, byte.astype(np.uint8)


def values(codes, byte):
    b = np.asarray(byte).astype(np.float64)
    step = np.where(b == 255, np.nan, np.where(b == 0, 0.0, np.exp2(b - 127)))
    return np.asarray(codes, dtype=np.float64) * step[..., None]


def attention(q, K, V, k_t, v_t, scale, alibi, half_step):
    """One sequence: q [H, 64], K, V [n, H, 64], pair [H, 64] or None -> out [H, 64], lse [H], bounds of both.

    Bounds: a logit is a sum of 64 products and a product with the scale, 70 roundings of 2^-24 of the sum of magnitudes, and the bias
    adds two more of its own size; a weight is off by twice the largest such error, by 2^-21 for the exponential and its argument, and
    the sums over the keys by 2^-24 for each addition; out is rounded to the storage type."""
    H, n = q.shape[0], K.shape[0]
    slopes = np.array([2.0 ** (-alibi * (h + 1) / H) if alibi > 0 else 0.0 for h in range(H)])
    z = np.einsum("hc,nhc->hn", q, K) * scale - slopes[:, None] * np.arange(n, 0, -1)[None]
    mag = np.einsum("hc,nhc->hn", np.abs(q), np.abs(K)) * abs(scale) * 70 + 4 * slopes[:, None] * np.arange(n, 0, -1)[None]
    vals = V.transpose(1, 0, 2)
    if k_t is not None:
        z = np.concatenate((z, (q * k_t).sum(-1)[:, None] * scale), 1)
        mag = np.concatenate((mag, (np.abs(q) * np.abs(k_t)).sum(-1)[:, None] * abs(scale) * 70), 1)
        vals = np.concatenate((vals, v_t[:, None]), 1)
    if z.shape[1] == 0:
        return np.zeros(q.shape), np.full(H, -np.inf), np.zeros(q.shape), np.zeros(H)
    top = z.max(1, keepdims=True)
    w = np.exp(z - top)
    l = w.sum(1, keepdims=True)
    out = np.einsum("hn,hnc->hc", w / l, vals)
    delta = (mag.max(1) + np.abs(top[:, 0])) * 2.0 ** -24
    rel = 2 * delta + 2.0 ** -21 + (z.shape[1] + 16) * 2.0 ** -24
    bound = half_step * np.abs(out) + rel[:, None] * np.einsum("hn,hnc->hc", w / l, np.abs(vals)) * 1.01
    lse = top[:, 0] + np.log(l[:, 0])
    return out, lse, bound, 2 * rel + 4 * 2.0 ** -24 * np.abs(lse)


def rms(u, g, eps):
    return u / np.sqrt((u * u).mean(-1, keepdims=True) + eps) * g


def layer_step(w, g, x, caches, H, scale=1.0, alibi=0.0, alpha=1.0, eps=1e-6, norm_free=False):
    """x [S, d]; caches: per sequence (K, V) [n, H, 64].  Returns y, k, v of the step (no rounding)."""
    from scipy.special import erf
    S, d = x.shape
    norm = (lambda u, gg: u) if norm_free else (lambda u, gg: rms(u, gg, eps))  # noqa: E731
    head = lambda u, gg: norm(u.reshape(S, H, 64), gg.reshape(H, 64))  # noqa: E731
    n = norm(x, g["g_attn"])
    q, kt, vt = head(n @ w["Wq"].T, g["g_q"]), head(n @ w["Wk"].T, g["g_k"]), (n @ w["Wv"].T).reshape(S, H, 64)
    a = np.stack([attention(q[s], *caches[s], kt[s], vt[s], scale, alibi, 0.0)[0] for s in range(S)]).reshape(S, d)
    h = x + alpha * a @ w["Wo"].T
    u = norm(h, g["g_mlp"]) @ w["W1"].T
    z = h + alpha * (0.5 * u * (1 + erf(u / np.sqrt(2.0)))) @ w["W2"].T
    m = norm(z, g["g_kv"])
    return z, head(m @ w["Wk"].T, g["g_k"]), (m @ w["Wv"].T).reshape(S, H, 64)


class Pool:
    """A pool on the device whose rows outside the filled positions hold NaN (codes of a byte 255), its table with wrong entries behind
    each sequence's last page, and the values of every sequence on the host."""

    def __init__(self, rng, dtype, bits, S, H, lens, page, spare=2, room=0):
        import torch
        from paper_2604_21215_amd import torch_io as tio
        self.dtype, self.bits, self.page, self.H = dtype, bits, page, H
        lens = [int(n) for n in lens]
        need = [max(0, -(-max(n, 0) // page)) + room for n in lens]
        per, pages = max(max(need), 1) + 1, sum(need) + spare
        order = rng.permutation(pages)
        table = rng.integers(-3, 2 * pages, (S, per)).astype(np.int32)      # entries that nobody looks at
        shape = (pages, H, page, 64)
        Kh, Vh = np.full(shape, np.nan, dtype=np.float32), np.full(shape, np.nan, dtype=np.float32)
        self.K, self.V, at = [], [], 0
        for s, n in enumerate(lens):
            mine = order[at:at + need[s]]
            at += need[s]
            table[s, :need[s]] = mine
            k = rng.standard_normal((max(n, 0), H, 64)).astype(np.float32)
            k /= np.sqrt((k * k).mean(-1, keepdims=True)) if n > 0 else 1
            v = (rng.standard_normal((max(n, 0), H, 64)) * 0.6).astype(np.float32)
            if dtype == "bf16":
                k, v = gen.round_to_bf16(k), gen.round_to_bf16(v)
            for p in range(max(n, 0)):
                Kh[mine[p // page], :, p % page] = k[p]
                Vh[mine[p // page], :, p % page] = v[p]
            self.K.append(k.astype(np.float64)); self.V.append(v.astype(np.float64))
        self.table = torch.from_numpy(table).to("cuda:0")
        self.K_exp = self.V_exp = None
        if bits:
            ck, bk = quantise(np.where(np.isnan(Kh), np.inf, Kh)); cv, bv = quantise(np.where(np.isnan(Vh), np.inf, Vh))
            ck[bk == 255] = 99; cv[bv == 255] = 99
            self.Kd, self.Vd = (torch.from_numpy(c.astype(np.int8)).to("cuda:0") for c in (ck, cv))
            self.K_exp, self.V_exp = (torch.from_numpy(b).to("cuda:0") for b in (bk, bv))
            for s in range(S):
                for name in ("K", "V"):
                    c, b = quantise(getattr(self, name)[s])
                    getattr(self, name)[s] = values(c, b)
        else:
            nan = lambda a: np.where(np.isnan(a), np.float32(0), a)  # noqa: E731
            self.Kd, self.Vd = tio.to_device(nan(Kh), dtype), tio.to_device(nan(Vh), dtype)
            for h, dev in ((Kh, self.Kd), (Vh, self.Vd)):
                dev[torch.from_numpy(np.isnan(h)).to("cuda:0")] = float("nan")

    def cache(self):
        from paper_2604_21215_amd import binding
        return binding.make_cache(self.Kd, self.Vd, self.table, self.K_exp, self.V_exp)

    def bits_of(self):
        """Everything the pool holds, as integers."""
        import torch
        out = [t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).cpu().numpy().copy()
               for t in (self.Kd, self.Vd)]
        return out + [t.cpu().numpy().copy() for t in (self.K_exp, self.V_exp) if t is not None]

"""One decoder layer over a prefix forest in the shared layout (Sec. 6, prefix-sharing training
runtime): every shared token is one row, computed once, whatever number of samples read it.

Forward (also the forward-only pass of the reference model and of the old-policy log-probs,
Sec. 6): h = rmsnorm(x) g1; q, k, v = h Wq, h Wk, h Wv; rotary embedding of q and k by each row's
sequence position (psattn_rope); k, v into their pool slots (psattn_kv_scatter); prefix-shared
attention (psattn_fwd); y = x + o Wo; z = rmsnorm(y) g2; out = y + (silu(z W1) * (z W3)) W2.

Backward: one pass over the accumulated adjoints (Sec. 6): the upstream gradient of a shared row
is the sum over the samples that read it (advantage_adjoint, Sec. 2.5 advantage masking), and the
layer's backward runs once on the shared rows (psattn_bwd for the attention, psattn_kv_gather and
the inverse rotation for its inputs).  The dense products are plain library GEMMs (torch on the
GPU); the tree-dependent steps are the library's kernels.
"""
from __future__ import annotations

from typing import Callable, Dict, Sequence, Tuple

import numpy as np

from . import psattn as P


def advantage_adjoint(parent, seg_len, row_off, sample_end, adv: Sequence[float],
                      loss_mask: Callable[[int, np.ndarray], np.ndarray], c: np.ndarray) -> np.ndarray:
    """Upstream gradient of every shared row for the loss sum_s A_s sum_t m_{s,t} <c, out_{s,t}>:
    row t collects A_s m_{s,t} c from every sample s whose path holds it (the earliest use of a
    shared token carries the loss terms of every later sample, Sec. 4.1.1).  loss_mask(s, rows)
    gives sample s's mask along its sequence (rows: the packed row of each position)."""
    parent = np.asarray(parent)
    seg_len = np.asarray(seg_len)
    row_off = np.asarray(row_off)
    ns = int(seg_len[row_off >= 0].sum())
    w = np.zeros(ns)
    for s, e in enumerate(sample_end):
        path = []
        n = int(e)
        while n >= 0:
            path.append(n)
            n = int(parent[n])
        rows = np.concatenate([np.arange(int(row_off[m]), int(row_off[m]) + int(seg_len[m])) for m in reversed(path)])
        w[rows] += float(adv[s]) * np.asarray(loss_mask(s, rows), dtype=np.float64)
    return w[:, None] * np.asarray(c, dtype=np.float64)[None, :]


class SharedLayer:
    """Weights W (torch tensors on the GPU, fp32 or bf16 like the tree): g1 [H], Wq [H, Hq d],
    Wk, Wv [H, Hkv d], Wo [Hq d, H], g2 [H], W1, W3 [H, F], W2 [F, H]."""

    def __init__(self, W: Dict[str, "torch.Tensor"], hq: int, hkv: int, head_dim: int, theta: float = 10000.0,
                 eps: float = 1e-6):
        self.W, self.hq, self.hkv, self.d, self.theta, self.eps = W, hq, hkv, head_dim, theta, eps

    def _rms(self, x):
        import torch
        return torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + self.eps)

    def forward(self, tree: P.Tree, X, K_pool, V_pool):
        """out [Ns, H] and what the backward needs.  K_pool / V_pool receive this layer's K/V."""
        import torch
        W, ns, hq, hkv, d = self.W, tree.num_rows, self.hq, self.hkv, self.d
        dt = X.dtype
        r1 = self._rms(X)
        h = (X.float() * r1).to(dt) * W["g1"]
        q = (h @ W["Wq"]).view(ns, hq, d).contiguous()
        k = (h @ W["Wk"]).view(ns, hkv, d).contiguous()
        v = (h @ W["Wv"]).view(ns, hkv, d).contiguous()
        P.psattn_rope(tree, q, self.theta)
        P.psattn_rope(tree, k, self.theta)
        P.psattn_kv_scatter(tree, k, v, K_pool, V_pool)
        o_lo = torch.empty_like(q) if dt == torch.bfloat16 else None   # O's rounding residual (Delta)
        o, lse = P.psattn_fwd(tree, q, K_pool, V_pool, O_lo=o_lo)
        y = X + o.view(ns, hq * d) @ W["Wo"]
        r2 = self._rms(y)
        z = (y.float() * r2).to(dt) * W["g2"]
        a, b = z @ W["W1"], z @ W["W3"]
        m = torch.nn.functional.silu(a) * b
        out = y + m @ W["W2"]
        saved = dict(X=X, r1=r1, h=h, q=q, o=o, o_lo=o_lo, lse=lse, y=y, r2=r2, z=z, a=a, b=b, m=m, K=K_pool, V=V_pool)
        return out, saved

    def _products(self, dt):
        """(weight gradient x^T g, input gradient g w^T, planes of g) for fp32 g and x, w of the layer's
        dtype.  fp32: library fp32 products.  bf16: g goes in as its three bf16 planes (psattn_split_planes) and
        the products run on the bf16 matrix cores with fp32 sums, which an fp32 product of the same
        numbers, x and w widened first, takes three times as long for.  The input gradient comes as the
        planes' three terms."""
        import torch
        f32 = torch.float32
        if dt != torch.bfloat16:
            return (lambda x, g: x.t() @ g), (lambda g, w, add=None: g @ w.t() if add is None else add + g @ w.t()), (lambda g: g)

        def wgrad(x3, g3):
            return torch.mm(x3.detach().t(), g3, out_dtype=f32)

        def igrad(g3, w, add=None):
            wt = w.detach().t()
            return torch.mm(g3, wt, out_dtype=f32) if add is None else torch.addmm(add, g3, wt, out_dtype=f32, out=add)
        return wgrad, igrad, (lambda g: P.psattn_split_planes(g.detach().contiguous()))

    def backward(self, tree: P.Tree, saved, dout):
        """dX [Ns, H] and the weight gradients for the summed upstream gradient dout [Ns, H]."""
        import torch
        W, ns, hq, hkv, d = self.W, tree.num_rows, self.hq, self.hkv, self.d
        s = saved
        dt = s["q"].dtype
        bf16 = dt == torch.bfloat16
        f = lambda t: t.float()
        wgrad, igrad, planes = self._products(dt)
        rows = (lambda x: x.repeat(3, 1)) if bf16 else (lambda x: x)      # x against each plane of a gradient
        total = (lambda t: t.view(3, ns, -1).sum(0)) if bf16 else (lambda t: t)
        g = {}
        dout = f(dout)
        p = planes(dout)
        g["W2"] = wgrad(rows(s["m"]), p)
        dm = igrad(p, W["W2"])
        a, b = s["a"], s["b"]
        if bf16:
            da, db = P.psattn_silu_bwd(dm, a.detach(), b.detach())
        else:
            sig = torch.sigmoid(a)
            da = dm * b * (sig + a * sig * (1 - sig))
            db = dm * a * sig
        z = rows(s["z"])
        g["W1"], g["W3"] = wgrad(z, da), wgrad(z, db)
        dz = total(igrad(db, W["W3"], igrad(da, W["W1"])))
        yn = f(s["y"]) * s["r2"]
        g["g2"] = (dz * yn).sum(0)
        dzh = dz * f(W["g2"])
        dy = dout + (dzh - yn * (dzh * yn).mean(-1, keepdim=True)) * s["r2"]
        o = s["o"]
        p = planes(dy)
        g["Wo"] = wgrad(rows(o.view(ns, hq * d)), p)
        do = total(igrad(p, W["Wo"])).view(ns, hq, d).to(o.dtype).contiguous()
        dq, dKp, dVp = P.psattn_bwd(tree, s["q"], s["K"], s["V"], o, s["lse"], do, O_lo=s["o_lo"])
        dk, dv = P.psattn_kv_gather(tree, dKp, dVp)
        P.psattn_rope(tree, dq, self.theta, inverse=True)
        P.psattn_rope(tree, dk, self.theta, inverse=True)
        h = rows(s["h"])
        dq2, dk2, dv2 = planes(dq.view(ns, hq * d)), planes(dk.view(ns, hkv * d)), planes(dv.view(ns, hkv * d))
        g["Wq"], g["Wk"], g["Wv"] = wgrad(h, dq2), wgrad(h, dk2), wgrad(h, dv2)
        dh = total(igrad(dv2, W["Wv"], igrad(dk2, W["Wk"], igrad(dq2, W["Wq"]))))
        xn = f(s["X"]) * s["r1"]
        g["g1"] = (dh * xn).sum(0)
        dhh = dh * f(W["g1"])
        dX = dy + (dhh - xn * (dhh * xn).mean(-1, keepdim=True)) * s["r1"]
        return dX, g


def row_targets(parent, seg_len, row_off, tokens):
    """The next tokens of every shared row, as lists by row: (tgt_ptr [Ns + 1], tgt, entry [Ns]), int32 numpy arrays, for
    psattn_logprob_fwd.  A row inside a node has one, the node's next token; a node's last row has the first token of
    each of its children (in node order), none at a leaf.  tokens [Ns]: the token of each row.  entry[r] is the list entry
    that predicts row r's token, -1 where no row of this call does (a root's first token, and that of a node behind a
    cached one)."""
    parent, seg_len, row_off, tokens = (np.asarray(x) for x in (parent, seg_len, row_off, tokens))
    ns = int(seg_len[row_off >= 0].sum())
    if tokens.shape != (ns,):
        raise ValueError(f"expected {ns} tokens, got {tokens.shape}")
    src = np.full(ns, -1, dtype=np.int64)         # the row behind which each row's token comes
    for n in range(len(parent)):
        a = int(row_off[n])
        if a < 0:
            continue
        src[a + 1:a + int(seg_len[n])] = np.arange(a, a + int(seg_len[n]) - 1)
        p = int(parent[n])
        if p >= 0 and row_off[p] >= 0:
            src[a] = int(row_off[p]) + int(seg_len[p]) - 1
    first = np.asarray([int(a) for a in row_off if a >= 0], dtype=np.int64)
    node_rank = np.zeros(ns, dtype=np.int64)      # order among the rows behind one row: that of their nodes
    node_rank[first] = np.arange(len(first))
    dst = np.flatnonzero(src >= 0)
    dst = dst[np.lexsort((node_rank[dst], src[dst]))]
    ptr = np.zeros(ns + 1, dtype=np.int32)
    ptr[1:] = np.cumsum(np.bincount(src[dst], minlength=ns))
    entry = np.full(ns, -1, dtype=np.int32)
    entry[dst] = np.arange(len(dst))
    return ptr, tokens[dst].astype(np.int32), entry


def advantage_dlogp(parent, seg_len, row_off, sample_end, adv: Sequence[float],
                    loss_mask: Callable[[int, np.ndarray], np.ndarray], entry: np.ndarray) -> np.ndarray:
    """Adjoint of the log-probabilities for the loss -sum_s A_s sum_t m_{s,t} logp(token t of sample s): a shared token collects
    the terms of every sample that holds it (Sec. 2.5, Sec. 4.1.1).  loss_mask as for advantage_adjoint; entry is row_targets'."""
    parent, seg_len, row_off = np.asarray(parent), np.asarray(seg_len), np.asarray(row_off)
    w = np.zeros(int(entry.max(initial=-1)) + 1)
    for s, e in enumerate(sample_end):
        path = []
        n = int(e)
        while n >= 0:
            path.append(n)
            n = int(parent[n])
        rows = np.concatenate([np.arange(int(row_off[m]), int(row_off[m]) + int(seg_len[m])) for m in reversed(path) if row_off[m] >= 0])
        m = np.asarray(loss_mask(s, rows), dtype=np.float64)
        known = entry[rows] >= 0
        w[entry[rows][known]] -= float(adv[s]) * m[known]
    return w


class SharedHead:
    """What follows the last layer: h = rmsnorm(x) g, and the log-probabilities of each shared row's next tokens over the
    vocabulary (psattn_logprob_fwd / _bwd).  Weights W: g [H], W [V, H]."""

    def __init__(self, W: Dict[str, "torch.Tensor"], logit_scale: float = 1.0, eps: float = 1e-6):
        self.W, self.scale, self.eps = W, logit_scale, eps

    def forward(self, X, tgt_ptr, tgt):
        """logp [targets] (fp32) and what the backward needs."""
        import torch
        r = torch.rsqrt(X.float().pow(2).mean(-1, keepdim=True) + self.eps)
        h = (X.float() * r).to(X.dtype) * self.W["g"]
        logp, lse = P.psattn_logprob_fwd(h, self.W["W"], tgt_ptr, tgt, logit_scale=self.scale)
        return logp, dict(X=X, r=r, h=h, lse=lse, tgt_ptr=tgt_ptr, tgt=tgt)

    def backward(self, saved, dlogp):
        """dX [Ns, H] (fp32, the dout of the last layer's backward) and the weight gradients."""
        s = saved
        dh, dW = P.psattn_logprob_bwd(s["h"], self.W["W"], s["tgt_ptr"], s["tgt"], s["lse"], dlogp, logit_scale=self.scale)
        dh = dh.float()
        xn = s["X"].float() * s["r"]
        dhh = dh * self.W["g"].float()
        dX = (dhh - xn * (dhh * xn).mean(-1, keepdim=True)) * s["r"]
        return dX, {"g": (dh * xn).sum(0), "W": dW}


def adamw(layers, head, state_bits: int = 32) -> P.AdamW:
    """The optimizer of a stack of layers and its head: every weight in train_step's order, no decay on the norms' gains."""
    weights = [(k, w) for part in (*layers, head) for k, w in part.W.items()]
    return P.AdamW([w for _, w in weights], state_bits=state_bits, decay=[0.0 if k in ("g", "g1", "g2") else 1.0 for k, _ in weights])


def train_step(layers, head, opt: P.AdamW, tree: P.Tree, X, pools, tgt_ptr, tgt, adjoint, **hyper):
    """One training step over the shared rows: the layers and the head forward, adjoint(logp) -> dlogp (the gradient of the
    loss by the log-probabilities), their backward, and opt.step(..., **hyper) on every weight.  pools: (K, V) per layer.
    Returns (logp, dX, what opt.step returns)."""
    saved, x = [], X
    for layer, (K, V) in zip(layers, pools):
        x, s = layer.forward(tree, x, K, V)
        saved.append(s)
    logp, s = head.forward(x, tgt_ptr, tgt)
    dx, gh = head.backward(s, adjoint(logp))
    grads = [gh[k] for k in head.W]
    for layer, s in zip(reversed(list(layers)), reversed(saved)):
        dx, g = layer.backward(tree, s, dx)
        grads = [g[k] for k in layer.W] + grads
    return logp, dx, opt.step(grads, **hyper)

"""Attention with a bias by relative position and dropout from its formulas in 64 bits, with what 32-bit sums and words of 16 bits may be
off by, for the tests.

Tolerances, per number.  u = 2^-24, a rounding in 32 bits; W, that of the words between the products (16-bit tensors; 0 for 32-bit ones).
A sum of m numbers made in 32 bits is off by at most m u times the sum of magnitudes, in any order.  So
  s     is off by es = (dim + 4) u scale |q|.|k| + 4 u (|s| + |bias| + |max|)   (products, scale, bias, times log2 e, less the maximum)
  P     by the share ep = es + max es of the row + (len + 24) u               (exp2's own rounding, the sum's, its reciprocal, rescaling)
  o     by sum_j P' |v| (ep + W + (len + 24) u),  P' = m P / (1 - p)
  dP    by edp = (dim + 4) u m / (1 - p) |do|.|v|
  delta by ed = sum_j P (edp + |dP| (ep + (len + 4) u))                         (it is added up as sum_j P dP)
  dS    by eds = P (edp + ed) + |dS| (ep + 4 u)
  dq, dk by scale sum (eds + |dS| (W + (len + 24) u)) |k| or |q|; dv by sum P' (ep + W + (len + 24) u) |do|; dbias by sum eds + |dS| N u, N terms
and every output by its own rounding.  A word of a 16-bit float that was scaled is off by 2^-38 of its column's largest, where it is subnormal."""
import numpy as np
import torch

from tests import philox

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -140, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U = 2.0 ** -24


def bucket_of(starts, length):
    """[query][key]: the bucket of every distance, by its definition."""
    distance = np.arange(length)[None, :] - np.arange(length)[:, None]
    return torch.from_numpy(np.sum(distance[..., None] >= np.asarray(starts[1:], dtype=np.int64), -1) if len(starts) > 1 else np.zeros_like(distance))


def rounded(value, tol, kind):
    return tol + HALF_ULP[kind] * (value.abs() + tol) + TINY[kind]


def formulas(q, k, v, bias, starts, do=None, seqs=1, lengths=None, causal=True, scale=None, rng=None, p=0.0, heads=1, kv_heads=1, kind=None):
    """Outputs and gradients, and what each may be off by (with its rounding).  Tensors on the CPU, [n][t][heads * dim]."""
    kind, (n, t, wide) = kind or q.dtype, q.shape
    dim, length, group = wide // heads, t // seqs, heads // kv_heads
    scale = float(np.float32(dim ** -0.5 if scale is None else scale))
    word = 0.0 if kind == torch.float32 else HALF_ULP[kind]
    tiny = 2.0 ** -38 if kind == torch.float16 else 0.0
    starts = list(starts or [])
    out = {"o": torch.zeros(n, seqs, length, heads, dim, dtype=torch.float64)}
    if do is not None:
        out.update({"dq": torch.zeros(n, seqs, length, heads, dim, dtype=torch.float64), "dk": torch.zeros(n, seqs, length, kv_heads, dim, dtype=torch.float64),
                    "dv": torch.zeros(n, seqs, length, kv_heads, dim, dtype=torch.float64), "dbias": torch.zeros(n, heads, len(starts), dtype=torch.float64)})
    tol = {name: torch.zeros_like(x) for name, x in out.items()}
    parts = {}
    for name, x, h in (("q", q, heads), ("k", k, kv_heads), ("v", v, kv_heads), ("do", do, heads)):
        if x is not None:
            parts[name] = x.double().unflatten(2, (h, dim)).unflatten(1, (seqs, length))
    share = 1 - philox.least(p) / 65536
    for i in range(n):
        for s in range(seqs):
            l = length if lengths is None else min(max(int(lengths[i][s]), 0), length)
            if l == 0:
                continue
            allowed = torch.ones(l, l, dtype=torch.bool).tril() if causal else torch.ones(l, l, dtype=torch.bool)
            bucket = bucket_of(starts, l) if starts else None
            keep = torch.ones(heads, l, l, dtype=torch.bool)
            if p:
                keep = torch.from_numpy(philox.keep_pairs(rng, (i * seqs + s) * heads + np.arange(heads), l, p))
            for h in range(heads):
                Q, K, V = parts["q"][i, s, :l, h], parts["k"][i, s, :l, h // group], parts["v"][i, s, :l, h // group]
                b = bias[h].double()[bucket] if starts else torch.zeros(l, l, dtype=torch.float64)
                logits = torch.where(allowed, scale * (Q @ K.t()) + b, -torch.inf)
                top = logits.amax(1, keepdim=True)
                some = torch.isfinite(top)
                safe = torch.where(some, top, 0.0)
                P = torch.exp(logits - safe)
                P = torch.where(some, P / P.sum(1, keepdim=True).clamp(min=1e-300), 0.0)
                finite = lambda x: torch.where(torch.isfinite(x), x.abs(), 0.0)
                es = torch.where(allowed, (dim + 4) * U * abs(scale) * (Q.abs() @ K.abs().t()) + 4 * U * (finite(logits) + finite(b) + safe.abs()), 0.0)
                ep = es + es.amax(1, keepdim=True) + (l + 24) * U
                more = word + (l + 24) * U
                m = keep[h].double() / share
                PD = P * m
                o = PD @ V
                eo = (PD * (ep + more)) @ V.abs() + tiny * V.abs().sum(0) / share
                out["o"][i, s, :l, h] = o
                tol["o"][i, s, :l, h] = rounded(o, eo, kind)
                if do is None:
                    continue
                dO = parts["do"][i, s, :l, h]
                dP = (dO @ V.t()) * m
                delta = (dO * o).sum(1, keepdim=True)
                dS = P * (dP - delta)
                edp = (dim + 4) * U * m * (dO.abs() @ V.abs().t())
                ed = (P * (edp + dP.abs() * (ep + (l + 4) * U))).sum(1, keepdim=True)
                eds = P * (edp + ed) + dS.abs() * (ep + 4 * U)
                # dq is made with do . o for delta, of which o's rounding is taken back at the end by sum P k, whose P's are words
                ew = eds + dS.abs() * more
                eo_k = more * (dO.abs() * rounded(o, eo, kind)).sum(1, keepdim=True) * (P @ K.abs())
                out["dq"][i, s, :l, h] = scale * (dS @ K)
                tol["dq"][i, s, :l, h] = abs(scale) * (eo_k + (ew + more * P * (dO.abs() * rounded(o, eo, kind)).sum(1, keepdim=True) + tiny * dS.abs().amax(1, keepdim=True)) @ K.abs())
                out["dk"][i, s, :l, h // group] += scale * (dS.t() @ Q)
                tol["dk"][i, s, :l, h // group] += abs(scale) * ((ew + tiny * dS.abs().amax(0, keepdim=True)).t() @ Q.abs())
                out["dv"][i, s, :l, h // group] += PD.t() @ dO
                tol["dv"][i, s, :l, h // group] += (PD * (ep + more)).t() @ dO.abs() + tiny * dO.abs().sum(0) / share
                if starts:
                    for c in range(len(starts)):
                        here = bucket == c
                        out["dbias"][i, h, c] += torch.where(here, dS, 0.0).sum()
                        tol["dbias"][i, h, c] += torch.where(here, eds + dS.abs() * (int(here.sum()) + 64) * U, 0.0).sum()
    if do is not None:
        tol["dq"] = rounded(out["dq"], tol["dq"], kind)
        # the heads that share a key are added up in 32 bits
        for name in ("dk", "dv"):
            tol[name] = rounded(out[name], tol[name] * (1 + group * U), kind)
        tol["dbias"] = rounded(out["dbias"], tol["dbias"] + (seqs + 8) * U * out["dbias"].abs(), torch.float32)
    for x in (out, tol):
        for name in ("o", "dq", "dk", "dv"):
            if name in x:
                x[name] = x[name].reshape(n, t, -1)
    return out, tol


def check(got, want, tol, what):
    got = got.cpu().double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    off = (got - want).abs()
    assert (off <= tol).all(), (what, float((off / tol.clamp(min=1e-300)).max()), float(off.max()))

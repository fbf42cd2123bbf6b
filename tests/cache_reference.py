"""Plain float64 evaluation of causal FMA for one sequence, with the error
bounds that the paged cache's tests allow.

With h the half step of a type (fp32 2^-24, bf16 2^-8) and u = 2^-24, for one
query: scores s_i = tau q . x_i, weights p_i = exp(s_i) / sum, output o = sum p_i y_i.
 - A far row x is a sum of up to s_l products in fp32: at most `chain` additions
   deep, off by chain u sum |pi| |x_j|; the kernels round it to the type, h |x|.
 - A score is off by ds_i = tau sum_c |q_c| (e_x + (d + 8) u |x|)_c, so a weight
   by a factor of exp(2 max ds); its rounding to the type adds h (bf16 products
   take the weights in bf16, their sum is fp32), exp and the sums 64 + sources / 8 u.
 - The output rounds once: h |o|.
So |error| <= h |o| + (exp(2 ds) - 1 + h + more u) sum p |y| + sum p e_y.
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def levels_of(max_len, r):
    blocks, L = -(-max_len // r), 0
    while (1 << L) < blocks:
        L += 1
    return max(L - 1, 0)


def weight_len(max_len, r, rank):
    return rank * r * ((1 << levels_of(max_len, r)) - 1)


def set_weights(w, r, rank, l, s):
    """pi of basis s of the level with groups of r << l tokens."""
    o = rank * r * ((1 << l) - 1) + s * (r << l)
    return w[o:o + (r << l)].double()


def running_sums(x, w, r, rank, levels):
    """[blocks, sets, d] sums S_e(b) of every complete block, and of the magnitudes."""
    n, d = x.shape
    nb = n // r
    out = torch.zeros(nb, levels * rank, d, dtype=torch.float64)
    mag = torch.zeros_like(out)
    x = x[:nb * r].double()
    for l in range(levels):
        for s in range(rank):
            size = r << l
            pi = set_weights(w, r, rank, l, s).repeat(-(-nb * r // size) or 1)[:nb * r]
            for dst, y in ((out, pi[:, None] * x), (mag, (pi[:, None] * x).abs())):
                for g in range(-(-nb * r // size)):
                    c = y[g * size:(g + 1) * size].cumsum(0)
                    b0 = g << l
                    b1 = min(nb, (g + 1) << l)
                    dst[b0:b1, l * rank + s] = c[r - 1::r][:b1 - b0]
    return out, mag


def far_rows(b, levels, rank):
    """(block, set) of the far field of queries in block b, by the definition:
    the groups under the neighbourhood of the parent that are not next to
    the query's own, and in the past."""
    rows = []
    for l in range(levels):
        own = b >> l
        for g in range(2 * ((own >> 1) - 1), 2 * ((own >> 1) + 2)):
            if 0 <= g < own - 1:
                rows += [(((g + 1) << l) - 1, l * rank + s) for s in range(rank)]
    return rows


def attend(q, k, v, wk, wv, r, rank, levels, scale, dtype, lo=0, missing=()):
    """Queries at positions lo .. n - 1 of one head: (output, bound) [n - lo, d].
    missing: blocks whose token rows are not there (nor their own token's)."""
    n, d = k.shape
    h = HALF[dtype]
    ks, km = running_sums(k, wk, r, rank, levels)
    vs, vm = running_sums(v, wv, r, rank, levels)
    k, v, q = k.double(), v.double(), q.double()
    out, bound = [], []
    for b in range(lo // r, -(-n // r)):
        p0, p1 = max(lo, b * r), min(n, (b + 1) * r)
        near = [j for x in (b - 1, b) if x >= 0 and x not in missing for j in range(x * r, min(p1, (x + 1) * r))]
        far = far_rows(b, levels, rank)
        chain = (r + (1 << max(levels - 1, 0)) + 8) * U
        K, V = k[near], v[near]
        eK, eV = torch.zeros_like(K), torch.zeros_like(V)
        if far:
            fb, fe = torch.tensor([x[0] for x in far]), torch.tensor([x[1] for x in far])
            K, V = torch.cat([K, ks[fb, fe]]), torch.cat([V, vs[fb, fe]])
            hr = 0 if dtype == torch.float32 else h
            eK = torch.cat([eK, hr * ks[fb, fe].abs() + chain * km[fb, fe]])
            eV = torch.cat([eV, hr * vs[fb, fe].abs() + chain * vm[fb, fe]])
        pos = torch.tensor(near + [-1] * len(far), dtype=torch.long)
        vis = pos[None, :] <= torch.arange(p0, p1)[:, None]
        qq = q[p0 - lo:p1 - lo]
        sc = (qq @ K.T * scale).masked_fill(~vis, -math.inf)
        ds = abs(scale) * (qq.abs() @ (eK + (d + 8) * U * K.abs()).T) + 4 * U * sc.abs().masked_fill(~vis, 0)
        ds = ds.masked_fill(~vis, 0).amax(1, keepdim=True) if K.shape[0] else torch.zeros(p1 - p0, 1, dtype=torch.float64)
        if K.shape[0] == 0:
            out.append(torch.zeros(p1 - p0, d, dtype=torch.float64))
            bound.append(torch.zeros(p1 - p0, d, dtype=torch.float64))
            continue
        p = torch.exp(sc - sc.amax(1, keepdim=True).clamp(min=-1e300)).masked_fill(~vis, 0)
        z = p.sum(1, keepdim=True)
        p = torch.where(z > 0, p / z.clamp(min=1e-300), torch.zeros_like(p))
        o = p @ V
        rel = torch.expm1(2 * ds) + (h if dtype == torch.bfloat16 else 0) + (64 + K.shape[0] / 8) * U
        out.append(o)
        bound.append(h * o.abs() + rel * (p @ V.abs()) + p @ eV + 1e-37)
    return torch.cat(out), torch.cat(bound)

"""Windowed attention in 64 bits, element by element with a dense mask per segment, and
how far a kernel's result may be from it by its roundings."""
import math

import torch


def visible(length, window, n_sink):
    i = torch.arange(length)[:, None]
    j = torch.arange(length)[None]
    see = j <= i
    if window:
        see &= (j > i - window) | (j < n_sink)
    return see


def reference(qkv, lens, hq, hkv, hd, window, n_sink, dout=None, scale=None, bf16=False):
    """{name: (value, allowed error)} of out, lse (log2 units) and, with dout, dqkv.

    Relative roundings: u of every weight p and score gradient ds as an operand of the
    next product and of every result (bfloat16: 2^-8, half a step; float32: none, the
    operands are the float32 values), and f of the float32 arithmetic: a sum of m terms is
    off by at most m 2^-24 of the sum of their magnitudes, so a score is off by
    (hd + 4) 2^-24 of c |q||k|, and 2^x of it by that much relatively, with two units in the
    last place of the exponential and the |x| 2^-24 of its scaled argument."""
    n, G = qkv.shape[0], hq // hkv
    c = scale or 1.0 / math.sqrt(hd)
    x = qkv.double()
    q, k, v = (t.reshape(n, -1, hd).transpose(0, 1) for t in
               x.split([hq * hd, hkv * hd, hkv * hd], 1))
    do = None if dout is None else dout.double().reshape(n, hq, hd).transpose(0, 1)
    u, e = (2.0 ** -8 if bf16 else 0.0), 2.0 ** -24
    new = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    o, oe, lse, le = new(hq, n, hd), new(hq, n, hd), new(hq, n), new(hq, n)
    d = [new(*t.shape) for t in (q, k, v)]
    de = [new(*t.shape) for t in (q, k, v)]
    a = 0
    for L in lens:
        if L == 0:
            continue
        r = slice(a, a + L)
        see = visible(L, window, n_sink)
        for h in range(hq):
            g = h // G
            Q, K, V = q[h, r], k[g, r], v[g, r]
            s = (Q @ K.T * c).masked_fill(~see, -math.inf)
            ls = torch.logsumexp(s, 1)
            p = torch.exp(s - ls[:, None])
            # relative error of a row's weights: scores, exponentials and their sum
            size = (Q.abs() @ K.abs().T * c).masked_fill(~see, 0.0).amax(1, keepdim=True)
            w = e * (2 * (hd + 4) * size + 4 * size + 8 + L)
            O = p @ V
            mag = p @ V.abs()
            o[h, r], lse[h, r] = O, ls * math.log2(math.e)
            oe[h, r] = (u + 2 * w) * mag + u * (O.abs() + (u + 2 * w) * mag)
            le[h, r] = (w[:, 0] * 2 + 4 * e * (1 + ls.abs())) * math.log2(math.e)
            if do is None:
                continue
            D = do[h, r]
            dp, dl = D @ V.T, (D * O).sum(1, keepdim=True)
            # dP and delta are products of hd terms; delta reads the rounded output
            b = e * (hd + 4) * (D.abs() @ V.abs().T + (D.abs() * O.abs()).sum(1, keepdim=True)) \
                + (D.abs() * oe[h, r]).sum(1, keepdim=True)
            ds = p * (dp - dl)
            dse = p * b + (u + 3 * w) * p * (dp - dl).abs() + u * p * b
            pe = (u + 3 * w) * p
            sums = e * (L * G + 8)
            d[0][h, r] = ds @ K * c
            de[0][h, r] = (dse + sums * ds.abs()) @ K.abs() * c
            d[1][g, r] += ds.T @ Q * c
            de[1][g, r] += (dse + sums * ds.abs()).T @ Q.abs() * c
            d[2][g, r] += p.T @ D
            de[2][g, r] += (pe + sums * p).T @ D.abs()
        a += L
    flat = lambda t: t.transpose(0, 1).reshape(n, -1)  # noqa: E731
    res = {"out": (flat(o), flat(oe)), "lse": (lse, le)}
    if do is not None:
        val, err = (torch.cat([flat(t) for t in ts], 1) for ts in (d, de))
        res["dqkv"] = (val, err + u * (val.abs() + err) + 2 * e * val.abs())
    return res

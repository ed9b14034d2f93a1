"""Cross attention of segments and its gradients in 64 bits, from the definition, with bounds on what rounding may add.

Test infrastructure only; shares nothing with the CUDA path. Segments are (q_begin, q_len, k_begin, k_len); q
[rows][Hq][d], k / v [key rows][Hkv][d] (any float type and device, taken to float64); query head h reads KV head
h / (Hq / Hkv)."""
import math

import torch

# A weight below the smallest normal number, 2^-126, may become 0: one relative to the row's largest as well as one
# relative to the log-sum-exp, a largest that lags by up to 2^8 and a sum of up to 2^1 (or fewer keys) apart. So each
# weight is off by 2^-117 at most where the bounds relative to it say less.
FLUSHED = 2.0 ** -117
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


def _pairs(segments, hq, hkv):
    for qb, qn, kb, kn in segments:
        for h in range(hq):
            if qn and kn:
                yield slice(qb, qb + qn), slice(kb, kb + kn), h, h // (hq // hkv)


def forward(segments, q, k, v, scale):
    """(out, lse, rows): rows marks the query rows of the segments (the others' out and lse are 0 here)."""
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    rows = torch.zeros(q.shape[0], dtype=torch.bool, device=q.device)
    for qb, qn, kb, kn in segments:
        rows[qb:qb + qn] = True
        if kn == 0:
            lse[qb:qb + qn] = -math.inf
    for a, b, h, g in _pairs(segments, q.shape[1], k.shape[1]):
        s = scale * q[a, h] @ k[b, g].T
        top = s.max(1, keepdim=True).values
        w = torch.exp(s - top)
        total = w.sum(1, keepdim=True)
        out[a, h] = (w / total) @ v[b, g]
        lse[a, h] = (top + total.log())[:, 0]
    return out, lse, rows


def backward(segments, q, k, v, dout, scale):
    """(dq, dk, dv), written out (not by autograd)."""
    q, k, v, dout = q.double(), k.double(), v.double(), dout.double()
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, b, h, g in _pairs(segments, q.shape[1], k.shape[1]):
        p = torch.softmax(scale * q[a, h] @ k[b, g].T, 1)
        dp = dout[a, h] @ v[b, g].T
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        dq[a, h] = scale * ds @ k[b, g]
        dk[b, g] += scale * ds.T @ q[a, h]
        dv[b, g] += p.T @ dout[a, h]
    return dq, dk, dv


def forward_bounds(segments, q, k, v, scale):
    """Largest |error| of out and lse for inputs held in their own type, products and sums in fp32, P rounded to the
    inputs' type before its product, one rounding at the end.

    A score is off by e = (d + 4) 2^-24 scale |q|.|k| (a sum of d products, the products with scale and log2 e) and
    a weight by 2 e + 2^-20 of itself (the largest score is off too; exp2). With a = sum_j p_j |v_j|:
      |out error| <= a (r + 2 e + 2^-20 + (n + 16) 2^-24) + r |out|, r the type's half step (fp32: r a counts P's own)
      |lse error| <= e + 2^-20 + n 2^-24 + |lse| 2^-22."""
    r = HALF[q.dtype]
    q, k, v = q.double(), k.double(), v.double()
    bo, bl = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    for a, b, h, g in _pairs(segments, q.shape[1], k.shape[1]):
        s = scale * q[a, h] @ k[b, g].T
        e = ((q.shape[2] + 4) * 2.0 ** -24 * scale * (q[a, h].abs() @ k[b, g].abs().T).max(1, keepdim=True).values)
        p, n = torch.softmax(s, 1), s.shape[1]
        out, lse = p @ v[b, g], torch.logsumexp(s, 1, keepdim=True)
        bo[a, h] = FLUSHED * v[b, g].abs().sum(0) + (p @ v[b, g].abs()) * (r + 2 * e + 2.0 ** -20 + (n + 16) * 2.0 ** -24) + r * out.abs()
        bl[a, h] = (e + 2.0 ** -20 + n * 2.0 ** -24 + lse.abs() * 2.0 ** -22)[:, 0]
    return bo, bl


def backward_bounds(segments, q, k, v, out, dout, scale, off=None):
    """Largest |error| of dq, dk and dv for an out given in the inputs' type (r its half step; off by at most `off` more) and
    an lse in fp32.

    P is off by eP = 2 e + (|lse| + 4) 2^-21 of itself; D = dout . out by r |dout|.|out| (out's rounding) and d 2^-24
    of that; dP by d 2^-24 |dout|.|v|; dS = P (dP - D) by P (those) + eP |dS|, and by r |dS| when it is rounded; so
      |dq error| <= scale sum_j (|dS error|_ij + r |dS_ij|) |k_j| + r |dq|, sums of n terms adding n 2^-24 of |.|."""
    r = HALF[q.dtype]
    q, k, v, out, dout = (t.double() for t in (q, k, v, out, dout))
    off = torch.zeros_like(out) if off is None else off
    bq, bk, bv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    d = q.shape[2]
    rows = sum(s[1] for s in segments) * q.shape[1]     # (no key's sum has more terms)
    for a, b, h, g in _pairs(segments, q.shape[1], k.shape[1]):
        s = scale * q[a, h] @ k[b, g].T
        e = (d + 4) * 2.0 ** -24 * scale * (q[a, h].abs() @ k[b, g].abs().T).max(1, keepdim=True).values
        lse = torch.logsumexp(s, 1, keepdim=True)
        ep = 2 * e + (lse.abs() + 4) * 2.0 ** -21
        p, dp = torch.softmax(s, 1), dout[a, h] @ v[b, g].T
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        dd = ((r + (d + 4) * 2.0 ** -24) * dout[a, h].abs() * out[a, h].abs() + dout[a, h].abs() * off[a, h]).sum(1, keepdim=True)
        eds = p * (dd + (d + 4) * 2.0 ** -24 * (dout[a, h].abs() @ v[b, g].abs().T)) + (ep + 2.0 ** -22) * \
            (p * (dp.abs() + (p * dp).sum(1, keepdim=True).abs())) + \
            FLUSHED * (1 + dp.abs() + (p * dp).sum(1, keepdim=True).abs())
        n = rows + s.shape[1]
        eds = eds + (r + n * 2.0 ** -24) * (ds.abs() + eds)
        bq[a, h] = scale * eds @ k[b, g].abs() + r * (scale * ds @ k[b, g]).abs()
        bk[b, g] += scale * eds.T @ q[a, h].abs()
        bv[b, g] += (p * (r + ep + n * 2.0 ** -24) + FLUSHED).T @ dout[a, h].abs()
    dq, dk, dv = backward(segments, q, k, v, dout, scale)
    return bq + r * dq.abs(), bk + r * dk.abs(), bv + r * dv.abs()

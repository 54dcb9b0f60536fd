"""Plain 64-bit forms of the operators in front of the cache, and the bounds that their outputs are held to."""
import math

import torch

from paper_2601_13684_amd import binding as hc

DEV = "cuda:0"
D = 128


def context(B, Hkv, G, max_ctx):
    return hc.hc_create(hc.hc_config(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, max_ctx=(max_ctx + 63) // 64 * 64, max_k=8, window=1, metric=0, tau_num=1, tau_den=2,
                                     agg=0, window_mode=0))


def blocks(room, Hkv, gap=0):
    """Offsets of the heads' K and V blocks, `gap` elements (a multiple of 8) apart, and the size of the buffer."""
    k_off, v_off, at = [], [], gap
    for rows in room:
        for _ in range(Hkv):
            k_off.append(at)
            v_off.append(at + rows * D + gap)
            at += 2 * (rows * D + gap)
    return k_off, v_off, at


def turned(x, weight, eps, pos, rope):
    """Norm and rotation of x [T, H, 128] at positions pos [T], 64 bits; and of |.|: what the 32-bit arithmetic's errors scale with."""
    x = x.double()
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + eps) ** -0.5 * weight.double()
    r = rope.rot_dim
    y, scale = x.clone(), x.abs()
    if r:
        f = torch.tensor([rope.freq[i] for i in range(r // 2)], dtype=torch.float64, device=x.device)
        a = (pos.double()[:, None] * f)[:, None]
        i = torch.arange(r // 2, device=x.device)
        one, two = (i, i + r // 2) if rope.layout == hc.HC_ROPE_HALF else (2 * i, 2 * i + 1)
        u, v = x[..., one], x[..., two]
        y[..., one] = rope.gain * (u * a.cos() - v * a.sin())
        y[..., two] = rope.gain * (v * a.cos() + u * a.sin())
        s = abs(rope.gain) * (u.abs() + v.abs())
        scale[..., one], scale[..., two] = s, s
    return y, scale


def check_turned(got, y, scale, where):
    """Half a step of bf16, 2^-8 of the value, and the 32-bit arithmetic.  cos and sin: the reduced angle is rounded to 2^-26 turns, 2^-23.3 rad,
    sincospi is good to 2^-23 and the gain's product to 2^-24: 2^-21.9.  Norm: twelve additions, halved by the root, the root 2^-23, three
    products: 2^-20.6.  Product and sum: 2^-23.  Together below 2^-19.9 of |u| + |v|: 2^-19."""
    err = (got.double() - y).abs()
    tol = y.abs() * 2.0 ** -8 + scale * 2.0 ** -19 + 1e-38
    assert (err <= tol).all(), (where, float((err - tol).max()))


def attention(q, kv, k_off, v_off, first, count, Hkv, G):
    """out, lse, sum p |v| and sqrt(sum p^2 v^2) in 64 bits; q [T, Hq, 128]."""
    T = q.shape[0]
    res = [torch.zeros((T, Hkv * G, D), dtype=torch.float64, device=q.device) for _ in range(3)]
    lse = torch.zeros((T, Hkv * G), dtype=torch.float64, device=q.device)
    t = 0
    for b, (f, n) in enumerate(zip(first, count)):
        for h in range(Hkv if n else 0):
            k, v = (kv[o[b * Hkv + h]:o[b * Hkv + h] + (f + n) * D].view(f + n, D).double() for o in (k_off, v_off))
            step = max(1, (1 << 26) // ((f + n) * G))
            for i in range(0, n, step):
                m = min(step, n - i)
                s = q[t + i:t + i + m, h * G:(h + 1) * G].double().reshape(m * G, D) @ k.t().contiguous() / math.sqrt(D)
                hidden = torch.arange(f + n, device=q.device)[None] > torch.arange(f + i, f + i + m, device=q.device).repeat_interleave(G)[:, None]
                s[hidden] = -math.inf
                l = torch.logsumexp(s, -1)
                p = (s - l[:, None]).exp()
                at = (slice(t + i, t + i + m), slice(h * G, (h + 1) * G))
                lse[at] = l.view(m, G)
                for r, x in zip(res, (p @ v, p @ v.abs(), (p.square() @ v.square()).sqrt())):
                    r[at] = x.view(m, G, D)
        t += n
    return res[0], lse, res[1], res[2]


def check_attention(out, lse, want, where):
    """A weight is off by at most half a step of bf16, 2^-8 of it, the output by its own rounding, 2^-8 of it; the rest is 32-bit: the logits (128
    products, 2^-17 of sum |q k| / sqrt(128), below 2^-12 for these inputs, twice in a ratio), 2^-10 of sum p |v| with the sums.  Single values are
    held to the sum of these; the 2-norm to what independent roundings of at most that size come to.  lse: see gpu_util."""
    o, l, pv, p2 = want
    err = (out.double() - o).abs()
    tol = 2.0 ** -8 * (pv + o.abs()) + 2.0 ** -10 * pv
    assert (err <= tol).all(), (where, float((err - tol).max()))
    assert float(err.norm()) <= 2.0 ** -8 * float((p2.square() + o.square()).sum().sqrt()) + 2.0 ** -10 * float(pv.norm()), (where, "2-norm")
    assert ((lse.double() - l).abs() <= 1e-4 + 1e-6 * l.abs()).all(), (where, "lse", float((lse.double() - l).abs().max()))

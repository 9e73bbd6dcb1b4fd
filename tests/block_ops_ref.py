"""64-bit definitions of the block operators beside the step (not a test module): rotary positions, differential attention and activations
in 8 bits, written from their formulas with torch in double precision, with the error bounds of their 16-bit forms."""
import math

import numpy as np
import torch

UB = 2.0 ** -8          # half a step of bf16, relative
U32 = 2.0 ** -24


def f64(t):
    return t.detach().double()


# ------------------------------------------------------------------ rotary positions
def rope_frequencies(rot, base, scaling=0, factor=1.0, orig_len=1.0, fast=32.0, slow=1.0):
    """Angle per position of each pair, and what cosines and sines are multiplied by."""
    if scaling == 2 and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    out = []
    for j in range(rot // 2):
        f = base ** (-2.0 * j / rot)
        if scaling == 1:
            f /= factor
        elif scaling == 3:
            def index(turns):
                return rot * math.log(orig_len / (turns * 2 * math.pi)) / (2 * math.log(base))
            lo, hi = max(math.floor(index(fast)), 0), min(math.ceil(index(slow)), rot - 1)
            ramp = min(max((j - lo) / (hi - lo if hi > lo else 0.001), 0.0), 1.0)
            f = f * (1 - ramp) + f / factor * ramp
        elif scaling == 4:
            turns = orig_len * f / (2 * math.pi)
            w = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            f = (1 - w) * f / factor + w * f
        out.append(f)
    return out, (0.1 * math.log(factor) + 1.0 if scaling == 3 else 1.0)


def rope_table(n_pos, rot, base=10000.0, **kw):
    f, mag = rope_frequencies(rot, base, **kw)
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    return torch.stack([ang.cos(), ang.sin()]) * mag


def rope(x, layout, n_heads, d_head, rot, cs, pos, inverse):
    """x [rows, >= n_heads d_head] fp64, cs [2, n_pos, rot/2] fp64, pos [rows] (outside the table: unturned)."""
    out = x[:, :n_heads * d_head].clone().view(len(x), n_heads, d_head)
    ok = (pos >= 0) & (pos < cs.shape[1])
    at = torch.where(ok, pos, 0).long()
    c = torch.where(ok[:, None], cs[0][at], 1.0)[:, None]
    s = torch.where(ok[:, None], cs[1][at], 0.0)[:, None] * (-1 if inverse else 1)
    i = torch.arange(rot // 2, device=x.device)
    a, b = (i, i + rot // 2) if layout == 0 else (2 * i, 2 * i + 1)
    x1, x2 = out[..., a].clone(), out[..., b].clone()
    out[..., a], out[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
    return out.reshape(len(x), -1)


# ------------------------------------------------------------------ differential attention
def dattn_split(qkv, B, S, H, K, D):
    x = qkv.view(B, S, H + 2 * K, D).transpose(1, 2)
    group = torch.arange(H, device=qkv.device) // (H // K)
    return x[:, :H], x[:, H:H + K][:, group], x[:, H + K:][:, group], group


def dattn_seen(B, S, causal, lens, device):
    seen = torch.ones(B, 1, S, S, dtype=torch.bool, device=device)
    if causal:
        seen = seen.tril()
    if lens is not None:
        n = lens.to(device).long().clamp(0, S)
        seen = seen & (torch.arange(S, device=device) < n[:, None])[:, None, None]
    return seen


def dattn_fwd(qkv, lam, gain, eps, c, B, S, H, K, D, causal, lens, u=0.0):
    """o, o2, y (rows [B S, H D]), lse [2, B, H, S], and bounds on the errors of o, o2, y when probabilities are rounded by u relative."""
    q, k, v, _ = dattn_split(qkv, B, S, H, K, D)
    seen = dattn_seen(B, S, causal, lens, qkv.device)
    o, lse, spread, score = [], [], [], 0.0
    for m in range(2):
        a, b = q[..., m * D // 2:(m + 1) * D // 2], k[..., m * D // 2:(m + 1) * D // 2]
        z = torch.where(seen, a @ b.mT / math.sqrt(D / 2), -math.inf)
        score = max(score, float((a.abs() @ b.abs().mT).max()) / math.sqrt(D / 2))
        top = z.amax(-1, keepdim=True)
        e = torch.where(seen, torch.exp(z - torch.where(top == -math.inf, 0.0, top)), 0.0)
        n = e.sum(-1, keepdim=True)
        p = torch.where(n > 0, e / torch.where(n > 0, n, 1.0), 0.0)
        o.append(p @ v)
        spread.append(p @ v.abs())
        lse.append((top + n.log())[..., 0])
    w = lam[:, None, None]
    full = o[0] - w * o[1]
    # a sum of D/2 products in fp32 moves a score by (D/2) 2^-24 of its terms' sum at most, a probability by as much
    slack = 2 * (D // 2 + 8) * U32 * (1 + score) + S * U32
    d_o = (u + slack) * (spread[0] + w.abs() * spread[1])
    d_o2 = (u + slack) * spread[1]
    rows = lambda t: t.transpose(1, 2).reshape(B * S, H * D)     # noqa: E731
    y = dy = None
    if gain is not None:
        r = 1.0 / torch.sqrt((full ** 2).mean(-1, keepdim=True) + eps)
        y = full * r * gain * c
        # y = g o r: |dy| <= |g| r (|do| + |o| r |do|_rms): (|o|_rms r <= 1)
        dy = (gain * c).abs() * r * (d_o + full.abs() * r * (d_o ** 2).mean(-1, keepdim=True).sqrt()) + slack * y.abs()
        y, dy = rows(y), rows(dy)
    return rows(full), rows(o[1]), y, torch.stack(lse), rows(d_o), rows(d_o2), dy, slack * (1 + score)


def dattn_bwd(qkv, lam, gain, eps, c, o, o2, lse, dy, B, S, H, K, D, causal, lens, u=0.0):
    """dqkv, dlam, dgain from the forward pass's saved values, and a bound on dqkv's error when dS, P and (with a norm) the gradient of o are
    rounded by u relative."""
    q, k, v, group = dattn_split(qkv, B, S, H, K, D)
    seen = dattn_seen(B, S, causal, lens, qkv.device)
    heads = lambda t: t.view(B, S, H, D).transpose(1, 2)         # noqa: E731
    g, o, o2 = heads(dy), heads(o), heads(o2)
    dgain, w, ug = None, lam[:, None, None], 0.0
    if gain is not None:
        r = 1.0 / torch.sqrt((o ** 2).mean(-1, keepdim=True) + eps)
        dgain = (g * o * r * c).sum((0, 1, 2))
        t = g * gain * c
        g = r * (t - o * r * r * (t * o).mean(-1, keepdim=True))
        ug = u
    dlam = -(g * o2).sum((0, 2, 3))
    dlam_terms = (g * o2).abs().sum((0, 2, 3))
    held = [o + w * o2, o2]
    out = torch.zeros(B, S, H + 2 * K, D, dtype=torch.float64, device=qkv.device)
    bound = torch.zeros_like(out)
    dp, adp = g @ v.mT, g.abs() @ v.abs().mT
    mix, each = 0.0, 0.0
    # an fp32 sum of n products is off by n 2^-24 of its terms' sum at most: n = S keys (dq) or the queries of all heads of a group (dk, dv),
    # and 8 roundings of a term's factors
    n_sum = (S * (H // K) + 8) * U32
    for m in range(2):
        at = slice(m * D // 2, (m + 1) * D // 2)
        a, b = q[..., at], k[..., at]
        z = a @ b.mT / math.sqrt(D / 2)
        score = (a.abs() @ b.abs().mT) / math.sqrt(D / 2)
        p = torch.where(seen, torch.exp(torch.where(seen, z, 0.0) - torch.where(lse[m] == -math.inf, 0.0, lse[m])[..., None]), 0.0)
        slack = 4 * (D + 8) * U32 * (1 + float(score.max()))
        sign = 1.0 if m == 0 else -w
        d = (g * held[m]).sum(-1, keepdim=True)
        ad = (g * held[m]).abs().sum(-1, keepdim=True)
        ds = sign * p * (dp - d)
        e = (sign * p).abs() if m else p
        dds = (u + n_sum) * ds.abs() + e * (ug + slack) * (adp + ad)       # its own rounding; that of g, and fp32 sums, in dP and D
        mix, each = mix + sign * p, each + slack * e             # what a probability is off by, as its score is
        scale = 1 / math.sqrt(D / 2)
        out[:, :, :H, at] = (ds @ b * scale).transpose(1, 2)
        bound[:, :, :H, at] = (dds @ b.abs() * scale).transpose(1, 2)
        out[:, :, H:H + K, at].index_add_(2, group, (ds.mT @ a * scale).transpose(1, 2))
        bound[:, :, H:H + K, at].index_add_(2, group, (dds.mT @ a.abs() * scale).transpose(1, 2))
    pm = mix.abs()
    out[:, :, H + K:].index_add_(2, group, (mix.mT @ g).transpose(1, 2))
    bound[:, :, H + K:].index_add_(2, group, (((u + ug + n_sum) * pm + each).mT @ g.abs()).transpose(1, 2))
    return out.view(B * S, -1), dlam, dgain, bound.view(B * S, -1), dlam_terms


# ------------------------------------------------------------------ 8 bits
def pow2(e):
    """2 ** e of whole numbers, exactly."""
    return torch.from_numpy(np.ldexp(1.0, e.cpu().numpy().astype(np.int64))).to(e.device)


def pack(x, fmt, parts=1):
    """Values in range and scale exponents' bytes; x [rows, parts * f] fp64 of finite values (non-finite blocks: byte 255, zeros)."""
    rows, f = x.shape[0], x.shape[1] // parts
    x = torch.nn.functional.pad(x.view(rows, parts, f), (0, -f % 32)).view(rows, parts, -1, 32)
    bad = ~x.isfinite().all(-1)
    x = torch.where(bad[..., None], 0.0, x)
    top = x.abs().amax(-1)
    e = torch.full(top.shape, -110, dtype=torch.int64, device=x.device)
    for n in range(-110, 128):                                   # the least power of two that brings it into range
        e = torch.where(top > (448.0 if fmt else 127.0) * 2.0 ** n, n + 1, e)
    v = x / pow2(e)[..., None]
    if fmt == 0:
        v = v.round()
    else:
        step = pow2(torch.frexp(v)[1].clamp(min=-5) - 4)
        v = (v / step).round() * step
    byte = torch.where(bad, 255, e + 127)
    return v.flatten(2)[..., :f].reshape(rows, parts * f), byte.flatten(1)


def unpack(q, byte, parts=1):
    """What 8-bit values [rows, parts * f] (as numbers) stand for."""
    rows, f = q.shape[0], q.shape[1] // parts
    s = pow2(byte.int() - 127)
    s = torch.where(byte == 255, math.nan, s).view(rows, parts, -1).repeat_interleave(32, 2)[..., :f]
    return q.double() * s.reshape(rows, parts * f)


def activation(kind, x):
    """Value, and its derivatives by each part of x."""
    if kind == 1:
        cdf = torch.special.ndtr(x)
        return x * cdf, [cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)]
    f = x.shape[1] // 2
    a, u = x[:, :f], x[:, f:]
    s = torch.sigmoid(a)
    return a * s * u, [u * s * (1 + a * torch.sigmoid(-a)), a * s]

"""The cache operators from their definitions, in 64 bits on the CPU: what tests compare the library with."""
import math

import torch

E4M3 = [(m if e == 0 else (8 + m) * 2.0 ** (e - 1)) * 2.0 ** -9 for e in range(16) for m in range(8)][:127]
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def half_step(dtype):
    """Largest relative error of one rounding."""
    return torch.finfo(dtype).eps / 2


def nearest(x, table):
    """Index of the nearest entry of an ascending table, the even one of two."""
    table = torch.tensor(table, dtype=torch.float64)
    middle = (table[1:] + table[:-1]) / 2
    low = torch.searchsorted(middle, x.contiguous())
    tie = (low < len(middle)) & (middle[low.clamp(max=len(middle) - 1)] == x)
    return torch.where(tie & (low % 2 == 1), low + 1, low)


def held(x, exp):
    """(codes with sign, scale codes, values) of x [..., d]; elements that are not finite count as 0."""
    y = torch.where(torch.isfinite(x), x, 0).double() / 2.0 ** exp
    y = y.unflatten(-1, (-1, 16))
    s_code = nearest(y.abs().amax(-1, keepdim=True), [6 * s for s in E4M3])
    s = torch.tensor(E4M3, dtype=torch.float64)[s_code]
    code = nearest(torch.where(s > 0, y.abs() / s, 0), E2M1)
    value = y.sign() * torch.tensor(E2M1, dtype=torch.float64)[code] * s * 2.0 ** exp
    return code.flatten(-2), s_code.squeeze(-1), value.flatten(-2)


def appended(k, v, k_exp, v_exp):
    """Values of keys and values as the cache holds them."""
    kv, vv = held(k, k_exp)[2], held(v, v_exp)[2]
    bad = ~(torch.isfinite(k).all(-1) & torch.isfinite(v).all(-1))
    kv[..., :16] = torch.where(bad[..., None], math.nan, kv[..., :16])
    return kv, vv


def decode(data, pages, page_size, heads, d):
    """Keys and values of every slot, [pages * page_size, heads, d] float64, from the bytes by the header's layout."""
    raw = data[:pages * heads * (page_size // 16) * 18 * d].cpu().view(pages, heads, page_size // 16, 18 * d).int()
    codes = torch.tensor(E2M1 + [-x for x in E2M1], dtype=torch.float64)
    scales = torch.tensor(E4M3 + [math.nan] + [-x for x in E4M3] + [math.nan], dtype=torch.float64)
    out = [torch.empty(pages, page_size // 16, 16, heads, d, dtype=torch.float64) for _ in range(2)]
    for i in range(16):
        half, g, t, e = i // 8, i % 8, i % 8 // 2, i % 2
        for c in range(d):
            lane_g, byte = c // (d // 8), c % (d // 8) // 2
            at = [i * (d // 2) + c // 2, 8 * d + (((half * 8 + lane_g) * 4 + t) * 2 + e) * (d // 16) + byte]
            group = c // 16
            t4, x = group // (d // 64), group % (d // 64)
            sc = [16 * d + ((g * 4 + t4) * 2 + half) * (d // 64) + x, 17 * d + ((group * 4 + t) * 2 + half) * 2 + e]
            for side in range(2):
                out[side][:, :, i, :, c] = (codes[raw[..., at[side]] >> (4 * (c % 2)) & 15] * scales[raw[..., sc[side]]]).transpose(1, 2)
    return [x.reshape(pages * page_size, heads, d) for x in out]


def tables(old, new, free, count, table, page_size, max_tokens):
    """sol_attn_block_tables, one token after another. Returns table, cu_q, kv_lens, slots, positions, result."""
    table = [list(r) for r in table]
    stack = list(free)[:max(0, min(count, len(free)))]
    cu, kv, slots, positions = [0], [], [], []
    for b, (o, n) in enumerate(zip(old, new)):
        o, n = max(0, o), max(0, n)
        for p in range(o, o + n):
            j, slot = p // page_size, -1
            if j < len(table[b]):
                if p % page_size == 0:
                    taken = table[b][j] = stack.pop() if stack else -1
                else:
                    taken = table[b][j] if p == o or j == o // page_size else taken
                if taken >= 0:
                    slot = taken * page_size + p % page_size
            slots.append(slot if len(slots) < max_tokens else -1)
            positions.append(p)
        cu.append(cu[-1] + n)
        kv.append(o + n)
    return table, cu, kv, slots[:max_tokens], positions[:max_tokens], [len(stack), sum(s < 0 for s in slots)]


def norm_rope(x, weight, cos, sin, positions, eps, interleaved):
    """x [B, N, H, d] -> (result, tolerance before the last rounding), float64."""
    d = x.shape[-1]
    y = x.double()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
    if weight is not None:
        y = y * weight.double()
    z, size = y.clone(), y.abs()
    if cos is not None:
        half = cos.shape[1]
        at = positions.long().clamp(0, cos.shape[0] - 1)
        co, si = cos.double()[at][:, :, None], sin.double()[at][:, :, None]
        first = torch.arange(half) * (2 if interleaved else 1)
        second = first + (1 if interleaved else half)
        a, b = y[..., first], y[..., second]
        z[..., first], z[..., second] = a * co - b * si, a * si + b * co
        size = size.clone()
        size[..., first] = size[..., second] = a.abs() + b.abs()
    # d + 2 roundings of the sum of squares count half (root), 6 more: rsqrt (2 ulp), its products, the rotation
    return z, size * (d + 16) * 2.0 ** -24


def attention(q, cu, kv_lens, table, k, v, page_size, causal, scale, k_all_pages):
    """q [T, H, d]; k, v [slots, Hk, d] float64.  Returns out, lse, tolerance of out before its last rounding, tolerance of lse.

    Error of a weight, relative: 2^-11 for its rounding to fp16; 2^-18 for exp2 (2.6e-6 of a polynomial, d = 64; the instruction 2^-21) and the
    subtraction's result; and the error of its
    logit, d products of exact operands summed in fp32 with an error of 2^-23 of the partial sums at each step, the scaling
    (2^-23) and the subtraction of the maximum (2^-24 of its result, at most 2 largest logits).  Numerator and denominator both
    have the logits' error.  The sums over n keys in fp32: 2^-23 for each of the tree's n / 16 + 64 steps of its magnitude sum p |v|.
    Weights are held as 2^11 times their ratio to an earlier maximum, which is no larger than the row's: fp16's subnormal numbers, below
    2^-14, are 2^-24 apart, so small weights are off by 2^-25 / 2^11 = 2^-36 of the largest each."""
    T, H, d = q.shape
    Hk = k.shape[1]
    out, lse = torch.zeros(T, H, d, dtype=torch.float64), torch.full((T, H), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros(T, H, d, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    touched = torch.zeros(T, dtype=torch.bool)
    for b in range(len(kv_lens)):
        lo, hi = cu[b], cu[b + 1]
        n = min(max(kv_lens[b], 0), len(table[b]) * page_size)
        pos = torch.arange(n)
        pages = torch.tensor(table[b], dtype=torch.long)[pos // page_size] if n else torch.zeros(0, dtype=torch.long)
        there = (pages >= 0) & (pages < k_all_pages)
        slots = torch.where(there, pages * page_size + pos % page_size, 0)
        touched[lo:hi] = True
        m = hi - lo
        sees = (n - m + torch.arange(m) + 1).clamp(min=0) if causal else torch.full((m,), n)
        hidden = (pos[None, :] >= sees[:, None]) | ~there[None, :]
        for h in range(H):
            kk, vv = k[slots, h * Hk // H], v[slots, h * Hk // H]
            x = q[lo:hi, h].double()
            z = torch.where(hidden, -math.inf, x @ kk.T * scale)
            top = z.amax(-1) if n else torch.full((m,), -math.inf, dtype=torch.float64)
            some = (~hidden).any(-1)
            w = torch.exp(z - torch.where(some, top, 0.0)[:, None])
            w = torch.where(hidden, 0.0, w)
            total = w.sum(-1)
            vz = torch.where(hidden.all(0)[:, None] if m else torch.zeros(n, 1, dtype=torch.bool), 0.0, vv)
            o = torch.where(some[:, None], w @ vz / torch.where(some, total, 1.0)[:, None], 0.0)
            out[lo:hi, h] = o
            lse[lo:hi, h] = torch.where(some, top + torch.log(torch.where(some, total, 1.0)), -math.inf)
            size = torch.where(hidden, 0.0, x.abs() @ kk.abs().T * scale).nan_to_num(0)
            logit = (size.amax(-1) if n else torch.zeros(m, dtype=torch.float64)) * (d + 8) * 2.0 ** -23
            wn = (w / torch.where(some, total, 1.0)[:, None]).nan_to_num(0)
            mass = wn @ vz.abs().nan_to_num(0)
            tol[lo:hi, h] = mass * (2.0 ** -11 + 2.0 ** -18 + 2 * logit[:, None] + (n / 16 + 64) * 2.0 ** -23) + \
                n * 2.0 ** -36 * (vz.abs().nan_to_num(0).max() if n else 0)
            tol_lse[lo:hi, h] = 2.0 ** -18 + 2 * logit + (n / 16 + 80) * 2.0 ** -23 + 2.0 ** -22 * lse[lo:hi, h].abs().nan_to_num(0, 0, 0)
    return out, lse, tol, tol_lse, touched

"""The operators around the linear layer from their definitions, on the CPU: in 64 bits, and where every operation's rounding is part
of the definition, in 32 bits operation by operation."""
import math

import torch


def f64(t):
    return t.detach().cpu().double()


# ---- norm ----------------------------------------------------------------------------------------

def add_rms_norm(x, residual, weight, eps):
    """(h bf16, y fp64): h = bf16(x + residual) in one fp32 addition, y its norm."""
    x = x.cpu()
    h = x if residual is None else (x.float() + residual.cpu().float()).to(torch.bfloat16)
    d = h.double()
    return h, d / torch.sqrt((d * d).mean(1, keepdim=True) + eps) * weight.cpu().double()


# ---- rotary positions, rotation, quantiser -------------------------------------------------------

def rope_table(positions, rot, base, scaling=0, factor=1.0, low=1.0, high=32.0, original_len=8192.0):
    f = [base ** (-2.0 * j / rot) for j in range(rot // 2)]
    amplitude = 1.0
    if scaling == 1:
        f = [v / factor for v in f]
    elif scaling == 2:
        out = []
        for v in f:
            wavelength = 2 * math.pi / v
            if wavelength < original_len / high:
                out.append(v)
            elif wavelength > original_len / low:
                out.append(v / factor)
            else:
                smooth = (original_len / wavelength - low) / (high - low)
                out.append((1 - smooth) * v / factor + smooth * v)
        f = out
    elif scaling == 3:
        pair = lambda turns: rot * math.log(original_len / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
        ramp = [min(max((j - lo) / max(hi - lo, 0.001), 0.0), 1.0) for j in range(rot // 2)]
        f = [v / factor * r + v * (1 - r) for v, r in zip(f, ramp)]
        amplitude = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    return torch.cat([angle.cos(), angle.sin()], 1) * amplitude


def turn(x, cos_sin, positions, interleaved, rotate, dtype=torch.float32):
    """rope and rotation of heads [T, H, D] in `dtype`, each operation rounded on its own."""
    x = x.cpu().to(dtype)
    D = x.shape[-1]
    if cos_sin is not None:
        rot = cos_sin.shape[1]
        row = cos_sin.cpu().to(dtype)[positions.cpu().long().clamp(0, cos_sin.shape[0] - 1)][:, None]
        cos, sin = row[..., :rot // 2], row[..., rot // 2:]
        at = torch.arange(rot // 2)
        i, j = (2 * at, 2 * at + 1) if interleaved else (at, at + rot // 2)
        a, b = x[..., i], x[..., j]
        x = x.clone()
        x[..., i], x[..., j] = a * cos - b * sin, b * cos + a * sin
    if rotate:
        step = 1
        while step < D:
            y = x.reshape(*x.shape[:-1], -1, 2, step)
            a, b = y[..., 0, :].clone(), y[..., 1, :].clone()
            x = torch.stack([a + b, a - b], -2).reshape(x.shape)
            step *= 2
        x = x * torch.tensor(1.0 / math.sqrt(D), dtype=torch.float64).to(torch.float32).to(dtype)
    return x


def quantise(x, clip_lo, clip_hi):
    """(codes, scale, lo) of the last axis of fp32 x; fused multiply-adds through fp64 (products of fp32 are exact there)."""
    c_lo, c_hi = torch.tensor(clip_lo, dtype=torch.float32), torch.tensor(clip_hi, dtype=torch.float32)
    lo, hi = c_lo * x.amin(-1, keepdim=True), c_hi * x.amax(-1, keepdim=True)
    s = (hi - lo) / torch.tensor(15.0)
    s = torch.where((s > 0) & torch.isfinite(s), s, torch.ones_like(s))
    inv = torch.ones_like(s) / s
    t = (x.double() * inv.double() + (-(lo * inv)).double()).float()
    return t.clamp(0, 15).round().nan_to_num(0.0), s, lo


def dequantise(codes, s, lo):
    return (s.double() * codes.double() + lo.double()).float()


# ---- cache ---------------------------------------------------------------------------------------

def cache_views(cache, D):
    """(codes uint8 [pages, heads, 2, P, D/2], ranges fp32 [pages, heads, 2, P, 2]) of a cache; they share its memory."""
    P = cache.shape[2] // (D + 16)
    return cache[..., :P * D].unflatten(-1, (2, P, D // 2)), cache.view(torch.float32)[..., P * D // 4:].unflatten(-1, (2, P, 2))


def put(cache, D, slots, which, codes, s, lo):
    """Stores the vectors of tokens at `slots`; negative slots and those past the cache are left out."""
    P = cache.shape[2] // (D + 16)
    all_codes, all_ranges = cache_views(cache, D)
    b = codes.to(torch.uint8)
    packed = b[..., 0::2] | (b[..., 1::2] << 4)
    for t, slot in enumerate(slots.tolist()):
        if 0 <= slot < cache.shape[0] * P:
            all_codes[slot // P, :, which, slot % P] = packed[t]
            all_ranges[slot // P, :, which, slot % P] = torch.cat([s, lo], -1)[t]


def values(cache, D):
    """What the cache stands for, fp64 [pages, heads, 2, P, D], and the codes with their scales alone."""
    codes, ranges = cache_views(cache, D)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
    r = ranges.double()
    return c * r[..., :1] + r[..., 1:], c * r[..., :1]


def paged_attention(q, cache, page_table, lengths, max_len, scale, q_len, softcap, window):
    """(out, lse, slack of out, slack of lse), fp64 [rows, heads, D] and [rows, heads].

    The slacks follow from how the kernel may round.  Weights times scales go to the value product in fp16 (2^-11 of each), so an
    output may be off by 2^-11 of the sum of weight x scale x code, taken twice for what else there is (fp32 scores, the matrix
    cores' sums), before it is stored.  A score is a sum of D products of magnitude |q| (15 scale + |lo|) in arithmetic
    that keeps 2^-20 of their sum at least, taken four times."""
    q, cache, page_table, lengths = q.cpu(), cache.cpu(), page_table.cpu(), lengths.cpu()
    rows, heads, D = q.shape
    kv_heads = cache.shape[1]
    P = cache.shape[2] // (D + 16)
    group = heads // kv_heads
    val, part = values(cache, D)
    _, ranges = cache_views(cache, D)
    out = torch.zeros(rows, heads, D, dtype=torch.float64)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64)
    slack_out, slack_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(lengths.numel()):
        n = min(max(int(lengths[b]), 0), max_len)
        at = torch.arange(n)
        page = page_table[b].long()[at // P] if n else at
        there = (page >= 0) & (page < cache.shape[0])
        for j in range(q_len):
            end = n - (q_len - 1 - j)
            seen = there & (at < end)
            if window:
                seen &= at >= end - window
            t = at[seen]
            if t.numel() == 0:
                continue
            k, v = val[page[t], :, 0, t % P].transpose(0, 1), val[page[t], :, 1, t % P].transpose(0, 1)       # [kv heads, tokens, D]
            w = part[page[t], :, 1, t % P].transpose(0, 1)
            rk = ranges.double()[page[t], :, 0, t % P].transpose(0, 1)
            x = q[b * q_len + j].double().reshape(kv_heads, group, D)
            s = x @ k.transpose(1, 2) * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            r = b * q_len + j
            out[r] = (p @ v / total).reshape(heads, D)
            lse[r] = (top + torch.log(total)).reshape(heads)
            slack_out[r] = 2.0 ** -10 * (p @ w / total).reshape(heads, D) + 1e-30
            widest = (15 * rk[..., 0].abs() + rk[..., 1].abs()).amax(-1)
            slack_lse[r] = 2.0 ** -18 * abs(scale) * (x.abs().sum(-1) * widest[:, None]).reshape(heads) + 2.0 ** -20 * (1 + lse[r].abs())
            # (an error of the scores changes the weights by as much, relatively)
            slack_out[r] += slack_lse[r][:, None] * 2 * (p @ v.abs() / total).reshape(heads, D)
    return out, lse, slack_out, slack_lse

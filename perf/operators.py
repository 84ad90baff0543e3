"""The operators around the W4A4 linear layer of a served model, as cases that can be timed and compared.

Four kinds of pass:

  norm    basq_add_rms_norm: the residual's addition, the root-mean-square norm, and its output in bf16 or in 8 bits
          (e4m3) with a scale per token
  append  basq_rope_append: rotary positions on q and k, their online per-head Hadamard rotation, and the INT4 quantisation
          of k and v into a paged cache
  attend  basq_paged_attention: new tokens' attention over that cache
  step    the three in a row for one new token of each sequence, as a decode step has them between its linear layers

`own` chooses between the plain form, in elementary torch operations, and the library's kernels.

The cache is one uint8 tensor [pages, kv heads, P * (D + 16)] for pages of P tokens and heads of D channels.  One head of one
page holds the codes of its keys, [P, D/2] with the even channel in the low nibble, those of its values, then the ranges of
the keys, fp32 [P, 2] = (scale, lo), and those of the values; a value is scale * code + lo.
"""
from __future__ import annotations

import math
import random

import torch

own = False

CLIP = 0.9                       # the range clip ratio of the library's own workloads
EPS = 1e-5
MOST_TOKENS = 64 * 4096          # in all contexts of the largest listed attention, about, which has 64 heads over 8 kv heads


def _norm(name, M, K, out8):
    return {"name": name, "kind": "norm", "M": M, "K": K, "out8": out8}


def _append(name, T, heads, kv_heads, D, page, rot, interleaved, rotate, values):
    return {"name": name, "kind": "append", "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "page": page, "rot": rot,
            "interleaved": interleaved, "rotate": rotate, "values": values}


def _attend(name, B, longest, heads, kv_heads, D, page, q_len=1, softcap=0.0, window=0, ragged=True, kind="attend"):
    return {"name": name, "kind": kind, "B": B, "longest": longest, "heads": heads, "kv_heads": kv_heads, "D": D, "page": page,
            "q_len": q_len, "softcap": softcap, "window": window, "ragged": ragged}


def listed():
    return [
        # one decoded token in front of a 4096-wide layer: the smallest call, all latency
        _norm("norm_token", 1, 4096, False),
        # a ragged batch of decoded tokens in front of a projection in 8 bits
        _norm("norm_batch_61_fp8", 61, 8192, True),
        # a long prefill of the widest model
        _norm("norm_prefill", 4096, 8192, False),
        # one new token of sixteen sequences, as many kv heads as heads
        _append("append_token_16", 16, 32, 32, 128, 64, 128, False, True, False),
        # a ragged prompt of a small model: 64-channel heads, half of each rotated, pairs of neighbours
        _append("append_prompt_333", 333, 32, 8, 64, 16, 32, True, True, True),
        # a long prefill, eight heads to a kv head, with the values that the cache stands for, for the prompt's own attention
        _append("append_prefill", 4096, 64, 8, 128, 64, 128, False, True, True),
        # one sequence just begun, as many kv heads as heads: the smallest attention, latency
        _attend("attend_short", 1, 129, 32, 32, 128, 64, ragged=False),
        # a batch in the middle of its answers, lengths from a few tokens to 4096
        _attend("attend_batch_16", 16, 4096, 32, 8, 128, 64),
        # one document of 131072 tokens: has to be split over its length
        _attend("attend_long", 1, 131072, 64, 8, 128, 64, ragged=False),
        # a server's batch, up to 8192 tokens each: the largest call, one pass over 340 MB
        _attend("attend_serving", 64, 8192, 64, 8, 128, 64),
        # four drafted tokens to check, capped scores, a sliding window, 64-channel heads, seven heads to a kv head
        _attend("attend_draft_window", 8, 2048, 28, 4, 64, 16, q_len=4, softcap=50.0, window=1024),
        # what a decode step has between its linear layers: norm, append and attention of sixteen sequences
        _attend("step_16", 16, 2048, 32, 32, 128, 64, kind="step"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, mostly odd or ragged."""
    pick = rng.random()
    if pick < 0.25:
        K = 8 * _log_uniform(rng, 1024 // 8, 14336 // 8)
        M = _log_uniform(rng, 1, max(1, 4096 * 8192 // K))
        case = _norm("", M, K, rng.random() < 0.4)
    elif pick < 0.5:
        D = rng.choice([64, 128, 128])
        heads, kv_heads = rng.choice([(32, 32), (32, 8), (64, 8), (28, 4), (40, 40), (16, 1)])
        rot = rng.choice([D, D, D // 2, 16 * rng.randint(1, D // 16)])
        case = _append("", _log_uniform(rng, 1, 4096 * 80 // (heads + 2 * kv_heads)), heads, kv_heads, D,
                       rng.choice([16, 32, 64, 128]), rot, rng.random() < 0.3, rng.random() < 0.8, rng.random() < 0.5)
    else:
        D = rng.choice([64, 128, 128])
        heads, kv_heads = rng.choice([(32, 32), (32, 8), (64, 8), (28, 4), (40, 40), (16, 1), (71, 1)])
        B = _log_uniform(rng, 1, 64)
        step = rng.random() < 0.25
        q_len = 1 if step or rng.random() < 0.7 else rng.randint(2, 8)
        longest = _log_uniform(rng, q_len, min(131072, MOST_TOKENS * 8 // (B * kv_heads), MOST_TOKENS * 64 // (B * heads * q_len)))
        plain = step or rng.random() < 0.6
        case = _attend("", B, longest, heads, kv_heads, D, rng.choice([16, 32, 64, 128]), q_len,
                       0.0 if plain else rng.choice([0.0, 30.0, 50.0]), 0 if plain else rng.choice([0, 128, 1000, 4096]),
                       B > 1, "step" if step else "attend")
    del case["name"]
    return case


def _lengths(case):
    """Context lengths of the sequences, the new tokens among them; by the case alone, so that the work is known without a seed."""
    if not case["ragged"]:
        return [case["longest"]] * case["B"]
    rng = random.Random(case["B"] * 1000003 + case["longest"])
    most, least = case["longest"], min(case["longest"], case["q_len"])
    return [most] + [max(least, int(most * rng.uniform(0.05, 1.0))) for _ in range(case["B"] - 1)]


def _table(positions, rot):
    """cos and sin of position * 500000^(-2j/rot), j < rot/2: fp32 [positions, rot], cosines first."""
    inv = 500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _qkv(gen, T, heads, kv_heads, D):
    """One token's q, k and v heads side by side, as a fused projection leaves them: keys have a few channels of large mean."""
    x = torch.randn((T, heads + 2 * kv_heads, D), generator=gen, device="cuda")
    loud = torch.randperm(D, generator=gen, device="cuda")[:4]
    x[:, heads:heads + kv_heads, loud] += 6.0
    x = x.to(torch.bfloat16)
    return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]


def _full_cache(gen, pages, kv_heads, D, P):
    """A pool of pages that earlier tokens have filled: codes bell-shaped around the middle of their range."""
    cache = torch.empty((pages, kv_heads, P * (D + 16)), dtype=torch.uint8, device="cuda")
    low, high = (torch.randn((pages, kv_heads, P * D), generator=gen, device="cuda").mul_(2.6).add_(7.5).round_().clamp_(0, 15).to(torch.uint8)
                 for _ in range(2))
    cache[..., :P * D] = low | (high << 4)
    scale = torch.exp(0.2 * torch.randn((pages, kv_heads, 2 * P), generator=gen, device="cuda")) * 0.36
    lo = scale * (-7.5 + 0.5 * torch.randn(scale.shape, generator=gen, device="cuda"))
    cache.view(torch.float32)[..., P * D // 4:] = torch.stack([scale, lo], -1).flatten(2)
    return cache


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) + 20250615)
    s = {"case": case}
    dev = {"device": "cuda"}
    if case["kind"] == "norm":
        _norm_state(s, gen, case["M"], case["K"], case["out8"])
        return s
    heads, kv_heads, D, P = case["heads"], case["kv_heads"], case["D"], case["page"]
    if case["kind"] == "append":
        T = case["T"]
        s["q"], s["k"], s["v"] = _qkv(gen, T, heads, kv_heads, D)
        # prompts of up to 1000 tokens packed one behind the other, each in pages of its own
        at = torch.arange(T, **dev)
        seq, pos = at // 1000, at % 1000
        per_seq = -(-min(T, 1000) // P)
        pages = (T + 999) // 1000 * per_seq
        order = torch.randperm(pages, generator=gen, **dev)
        s["positions"] = (pos + 17).to(torch.int32)
        s["slots"] = (order[seq * per_seq + pos // P] * P + pos % P).to(torch.int32)
        s["cos_sin"] = _table(1024 + 17, case["rot"])
        s["cache"] = torch.zeros((pages, kv_heads, P * (D + 16)), dtype=torch.uint8, **dev)
        s["q_out"] = torch.empty((T, heads, D), dtype=torch.bfloat16, **dev)
        s["k_hat"], s["v_hat"] = (torch.empty((T, kv_heads, D), dtype=torch.bfloat16, **dev) if case["values"] else None for _ in range(2))
        return s

    B, q_len = case["B"], case["q_len"]
    lengths = _lengths(case)
    used = [-(-n // P) for n in lengths]
    order = torch.randperm(sum(used), generator=gen, **dev).to(torch.int32)
    table = torch.zeros((B, max(used)), dtype=torch.int32, **dev)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    s["page_table"], s["lengths"] = table, torch.tensor(lengths, dtype=torch.int32, **dev)
    s["cache"] = _full_cache(gen, sum(used), kv_heads, D, P)
    s["longest"] = max(lengths)
    s["out"] = torch.empty((B * q_len, heads, D), dtype=torch.bfloat16, **dev)
    s["lse"] = torch.empty((B * q_len, heads), dtype=torch.float32, **dev)
    if case["kind"] == "attend":
        # scores of standard deviation 2 or so: some tokens count far more than others
        s["q"] = (1.8 * torch.randn((B * q_len, heads, D), generator=gen, **dev)).to(torch.bfloat16)
    else:
        s["q"], s["k"], s["v"] = _qkv(gen, B, heads, kv_heads, D)
        last = s["lengths"].long() - 1
        s["positions"] = last.to(torch.int32)
        s["slots"] = (table.long().gather(1, (last // P)[:, None])[:, 0] * P + last % P).to(torch.int32)
        s["cos_sin"] = _table(s["longest"], D)
        s["q_out"] = torch.empty((B, heads, D), dtype=torch.bfloat16, **dev)
        _norm_state(s, gen, B, heads * D, False)
    # a program keeps the attention's workspace: as many bytes as the library asks for, 64 MiB hold every case here
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, **dev)
    return s


def _norm_state(s, gen, M, K, out8):
    dev = {"device": "cuda"}
    loud = torch.ones(K, **dev)
    loud[torch.randperm(K, generator=gen, **dev)[:max(1, K // 256)]] = 20.0
    s["x"] = torch.randn((M, K), generator=gen, **dev).to(torch.bfloat16)
    s["residual"] = (torch.randn((M, K), generator=gen, **dev) * loud).to(torch.bfloat16)
    s["weight"] = (1.0 + 0.1 * torch.randn(K, generator=gen, **dev)).to(torch.bfloat16)
    s["res_out"] = torch.empty((M, K), dtype=torch.bfloat16, **dev)
    s["y"] = None if out8 else torch.empty((M, K), dtype=torch.bfloat16, **dev)
    s["y8"] = torch.empty((M, K), dtype=torch.float8_e4m3fn, **dev) if out8 else None
    s["y8_scale"] = torch.empty(M, **dev) if out8 else None


# ---- the library's operators ------------------------------------------------------------------

def _own_norm(s):
    from paper_2506_15689_amd import binding as B
    B.basq_add_rms_norm(s["x"], s["residual"], s["weight"], EPS, s["y"], s["res_out"], Y8=s["y8"], y8_scale=s["y8_scale"])
    return [s["res_out"]] + [t for t in (s["y"], s["y8"], s["y8_scale"]) if t is not None]


def _own_append(s):
    from paper_2506_15689_amd import binding as B
    c = s["case"]
    B.basq_rope_append(s["q"], s["k"], s["v"], s["positions"], s["cos_sin"], s["slots"], s["cache"], CLIP, CLIP, s["q_out"],
                       s.get("k_hat"), s.get("v_hat"), interleaved=c.get("interleaved", False), rotate=c.get("rotate", True))
    return [s["q_out"], s["cache"]] + [t for t in (s.get("k_hat"), s.get("v_hat")) if t is not None]


def _own_attend(s, q):
    from paper_2506_15689_amd import binding as B
    c = s["case"]
    B.basq_paged_attention(q, s["cache"], s["page_table"], s["lengths"], s["longest"], 1.0 / math.sqrt(c["D"]), s["out"],
                           s["workspace"], q_len=c["q_len"], softcap=c["softcap"], window=c["window"], lse=s["lse"])
    return [s["out"], s["lse"]]


# ---- the same in elementary operations, 32 bits throughout, rounded where an operator stores -------------------------

def _plain_norm(s):
    h = (s["x"].float() + s["residual"].float()).to(torch.bfloat16)
    f = h.float()
    y = f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * s["weight"].float()
    if s["y"] is not None:
        return [h, y.to(torch.bfloat16)]
    scale = y.abs().amax(1, keepdim=True) / 448.0
    return [h, (y / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale[:, 0]]


def _butterflies(x, step):
    """Hadamard transform of the last axis: sums and differences of channels 1, 2, 4, ... apart."""
    if step == x.shape[-1]:
        return x
    y = x.unflatten(-1, (-1, 2, step))
    a, b = y[..., 0, :], y[..., 1, :]
    return _butterflies(torch.stack([a + b, a - b], -2).flatten(-3), 2 * step)


def _turned(x, cos_sin, positions, interleaved, rotate):
    x = x.float()
    rot = cos_sin.shape[1]
    half = rot // 2
    row = cos_sin[positions.long()][:, None]
    cos, sin = row[..., :half], row[..., half:]
    first, second = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :half], x[..., half:rot])
    a, b = first * cos - second * sin, second * cos + first * sin
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    x = torch.cat([turned, x[..., rot:]], -1)
    # 1/sqrt(D) as the nearest 32-bit number
    return _butterflies(x, 1) * float(torch.tensor(x.shape[-1] ** -0.5, dtype=torch.float32)) if rotate else x


def _multiply_add(a, b, c):
    """a * b + c rounded to 32 bits once."""
    return (a.double() * b.double() + c.double()).float()


def _quantised(x):
    """Codes, scale and lower bound of each vector along the last axis, operation by operation as the library's quantiser."""
    lo, hi = CLIP_32 * x.amin(-1, keepdim=True), CLIP_32 * x.amax(-1, keepdim=True)
    # a division of two tensors is rounded once; one by a number may be a product with its reciprocal
    scale = (hi - lo) / torch.full_like(lo, 15.0)
    scale = torch.where((scale > 0) & torch.isfinite(scale), scale, torch.ones_like(scale))
    inv = torch.ones_like(scale) / scale
    codes = _multiply_add(x, inv, -(lo * inv)).clamp(0.0, 15.0).round()
    return codes, scale, lo


CLIP_32 = float(torch.tensor(CLIP, dtype=torch.float32))


def _plain_append(s):
    c = s["case"]
    P, D = c["page"], c["D"]
    turn = (s["cos_sin"], s["positions"], c.get("interleaved", False), c.get("rotate", True))
    q, k, v = _turned(s["q"], *turn), _turned(s["k"], *turn), s["v"].float()
    codes, scale, lo = _quantised(torch.stack([k, v], 2))                       # [T, kv heads, 2, D]
    bytes_ = codes.to(torch.uint8)
    packed = bytes_[..., 0::2] | (bytes_[..., 1::2] << 4)
    page, at = s["slots"].long() // P, s["slots"].long() % P
    all_codes = s["cache"][..., :P * D].unflatten(-1, (2, P, D // 2))
    all_codes[page, :, :, at] = packed
    all_ranges = s["cache"].view(torch.float32)[..., P * D // 4:].unflatten(-1, (2, P, 2))
    all_ranges[page, :, :, at] = torch.cat([scale, lo], -1)
    outputs = [q.to(torch.bfloat16), s["cache"]]
    if c.get("values"):
        hat = _multiply_add(scale, codes, lo).to(torch.bfloat16)
        outputs += [hat[:, :, 0], hat[:, :, 1]]
    return outputs


def _plain_attend(s, q):
    c = s["case"]
    B, q_len, heads, kv_heads, D, P = c["B"], c["q_len"], c["heads"], c["kv_heads"], c["D"], c["page"]
    group = heads // kv_heads
    pages = s["cache"][s["page_table"].long()].transpose(1, 2)                   # [B, kv heads, pages, bytes of a page]
    codes = pages[..., :P * D].unflatten(-1, (2, P, D // 2))
    codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()       # [B, kv heads, pages, 2, P, D]
    ranges = pages[..., P * D:].contiguous().view(torch.float32).unflatten(-1, (2, P, 2))
    values = codes * ranges[..., :1] + ranges[..., 1:]
    k, v = values[:, :, :, 0].flatten(2, 3), values[:, :, :, 1].flatten(2, 3)
    # rows of a kv head: its heads for the first new token, then for the next
    rows = q.float().view(B, q_len, kv_heads, group, D).transpose(1, 2).reshape(B, kv_heads, q_len * group, D)
    scores = torch.matmul(rows, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    if c["softcap"]:
        scores = c["softcap"] * torch.tanh(scores / c["softcap"])
    at = torch.arange(k.shape[2], device=k.device)
    end = (s["lengths"][:, None] - (q_len - 1) + torch.arange(q_len, device=k.device)).repeat_interleave(group, 1)[:, None, :, None]
    seen = at < end
    if c["window"]:
        seen = seen & (at >= end - c["window"])
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = torch.exp(scores - top.masked_fill(top == -math.inf, 0.0))
    total = weights.sum(-1, keepdim=True)
    # what is masked may hold anything, also what is no number
    v = v.masked_fill(~(at < s["lengths"][:, None])[:, None, :, None], 0.0)
    out = torch.matmul(weights, v) / total.masked_fill(total == 0, 1.0)
    lse = (top + torch.log(total))[..., 0]
    back = lambda t: t.unflatten(2, (q_len, group)).transpose(1, 2).reshape(B * q_len, heads, *t.shape[3:])  # noqa: E731
    return [back(out).to(torch.bfloat16), back(lse)]


def run(s):
    kind = s["case"]["kind"]
    norm, append, attend = (_own_norm, _own_append, _own_attend) if own else (_plain_norm, _plain_append, _plain_attend)
    if kind == "norm":
        return norm(s)
    if kind == "append":
        return append(s)
    if kind == "attend":
        return attend(s, s["q"])
    normed = norm(s)
    appended = append(s)
    return normed + appended + attend(s, appended[0])


# ---- the same from its definition, in 64 bits -----------------------------------------------------

def _exact_norm(s):
    h = (s["x"].double() + s["residual"].double()).to(torch.bfloat16)           # the sum is stored, and the norm is the stored sum's
    d = h.double()
    y = d / torch.sqrt(d.pow(2).sum(1, keepdim=True) / d.shape[1] + EPS) * s["weight"].double()
    if s["y"] is not None:
        return [h.double(), y]
    scale = y.abs().max(1, keepdim=True).values / 448.0
    return [h.double(), y / scale, scale[:, 0]]


def _exact_turn(x, cos_sin, positions, interleaved, rotate):
    T, H, D = x.shape
    x = x.double()
    rot = cos_sin.shape[1]
    table = cos_sin.double()[positions.long()]
    z = torch.complex(table[:, :rot // 2], table[:, rot // 2:])[:, None]
    pairs = x[..., :rot].reshape(T, H, rot // 2, 2) if interleaved else x[..., :rot].reshape(T, H, 2, rot // 2).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
    x = torch.cat([z.reshape(T, H, rot) if interleaved else z.transpose(2, 3).reshape(T, H, rot), x[..., rot:]], -1)
    if not rotate:
        return x
    i = torch.arange(D, device=x.device)
    common = i[:, None] & i[None]
    parity = sum((common >> b) & 1 for b in range(8)) % 2
    return x @ (1.0 - 2.0 * parity.double()) / math.sqrt(D)


def _exact_append(s):
    c = s["case"]
    turn = (s["cos_sin"], s["positions"], c.get("interleaved", False), c.get("rotate", True))
    q = _exact_turn(s["q"], *turn)
    outputs = [q, None]                                                         # (the pages are whole bytes)
    for x in (_exact_turn(s["k"], *turn), s["v"].double()) if c.get("values") else ():
        lo = CLIP_32 * x.min(-1, keepdim=True).values
        scale = (CLIP_32 * x.max(-1, keepdim=True).values - lo) / 15.0
        outputs.append(((x - lo) / scale).round().clamp(0, 15) * scale + lo)
    return outputs


def _exact_attend(s, q, cache):
    c = s["case"]
    q_len, heads, kv_heads, D, P = c["q_len"], c["heads"], c["kv_heads"], c["D"], c["page"]
    group = heads // kv_heads
    outs, lses = [], []
    for b, n in enumerate(_lengths(c)):
        used = -(-n // P)
        pages = cache[s["page_table"][b, :used].long()]                          # [pages, kv heads, bytes]
        numbers = pages.view(torch.float32)[..., P * D // 4:].double().view(used, kv_heads, 2, P, 2)
        kv = []
        for part in range(2):
            raw = pages[..., part * P * D // 2:(part + 1) * P * D // 2].reshape(used, kv_heads, P, D // 2)
            x = torch.empty((used, kv_heads, P, D), dtype=torch.float64, device=raw.device)
            x[..., 0::2] = raw % 16
            x[..., 1::2] = raw // 16
            x = x * numbers[:, :, part, :, :1] + numbers[:, :, part, :, 1:]
            kv.append(x.transpose(0, 1).reshape(kv_heads, used * P, D)[:, :n])
        k, v = kv
        for j in range(q_len):
            end = n - (q_len - 1) + j
            begin = max(0, end - c["window"]) if c["window"] else 0
            rows = q[b * q_len + j].double().reshape(kv_heads, group, D)
            scores = rows @ k[:, begin:end].transpose(1, 2) / math.sqrt(D)
            if c["softcap"]:
                scores = torch.tanh(scores / c["softcap"]) * c["softcap"]
            lses.append(torch.logsumexp(scores, -1).reshape(heads))
            outs.append((torch.softmax(scores, -1) @ v[:, begin:end]).reshape(heads, D))
    return [torch.stack(outs), torch.stack(lses)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "attend":
        return _exact_attend(s, s["q"], s["cache"])
    # the new tokens' q is stored in bf16 and their k and v as codes with ranges: the attention's inputs are the stored ones
    q, k, v = _exact_append(s)[0], _exact_turn(s["k"], s["cos_sin"], s["positions"], False, True), s["v"].double()
    P, D = case["page"], case["D"]
    for b, slot in enumerate(s["slots"].tolist()):
        for part, x in enumerate((k[b], v[b])):
            lo = (CLIP_32 * x.min(-1, keepdim=True).values).float()
            scale = ((CLIP_32 * x.max(-1, keepdim=True).values - lo.double()) / 15.0).float()
            codes = ((x - lo.double()) / scale.double()).round().clamp(0, 15).to(torch.uint8)
            start = (part * P + slot % P) * D // 2
            s["cache"][slot // P, :, start:start + D // 2] = codes[:, 0::2] + 16 * codes[:, 1::2]
            start = P * D // 4 + 2 * (part * P + slot % P)
            s["cache"].view(torch.float32)[slot // P, :, start:start + 2] = torch.cat([scale, lo], 1)
    return _exact_norm(s) + [q, None] + _exact_attend(s, q.to(torch.bfloat16), s["cache"])


# ---- what a pass cannot do without ---------------------------------------------------------------

def _norm_work(M, K, out8):
    return 2 * 3 * M * K + (M * K + 4 * M if out8 else 2 * M * K) + 2 * K, 8 * M * K


def _append_work(T, heads, kv_heads, D, rot, table_rows, rotate, values):
    nbytes = T * (4 * heads * D + 2 * kv_heads * (2 * D + D // 2 + 8) + 8) + 4 * rot * table_rows
    if values:
        nbytes += T * 2 * kv_heads * 2 * D
    turn = (heads + kv_heads) * (3 * rot + (D * math.log2(D) + D if rotate else 0))
    return nbytes, T * (turn + 2 * kv_heads * 6 * D)


def _attend_work(case):
    q_len, window = case["q_len"], case["window"]
    tokens = pairs = 0
    for n in _lengths(case):
        tokens += min(n, window + q_len - 1) if window else n
        pairs += sum(min(n - (q_len - 1) + j, window or n) for j in range(q_len))
    rows = case["B"] * q_len * case["heads"]
    nbytes = tokens * case["kv_heads"] * (case["D"] + 16) + rows * (4 * case["D"] + 4)
    return nbytes, pairs * case["heads"] * 4 * case["D"]


def work(case):
    if case["kind"] == "norm":
        parts = [_norm_work(case["M"], case["K"], case["out8"])]
    elif case["kind"] == "append":
        parts = [_append_work(case["T"], case["heads"], case["kv_heads"], case["D"], case["rot"], min(case["T"], 1000),
                              case["rotate"], case["values"])]
    else:
        parts = [_attend_work(case)]
        if case["kind"] == "step":
            B, heads, D = case["B"], case["heads"], case["D"]
            parts += [_norm_work(B, heads * D, False), _append_work(B, heads, case["kv_heads"], D, D, B, True, False)]
    return {"bytes": sum(p[0] for p in parts), "flops": sum(p[1] for p in parts)}

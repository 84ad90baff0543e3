"""The two ends of a served model's step, as cases that can be timed and compared: where its tokens go in the cache, their embeddings,
the last vectors' logits, and the tokens drawn from them.

Five kinds of pass:

  product  basq_w4a16_gemm: few tokens in bf16 times 4-bit weights with a scale and a zero point for each group of channels (an output
           head, a layer whose activations are not quantised)
  lookup   basq_w4a16_lookup: rows of such a matrix, in bf16 (the embeddings of tokens)
  sample   basq_sample: a token for each row of logits, with temperature, top-k, top-p and min-p, from given random numbers: of the tokens
           in the order of their logits, equal ones by their index, the first at which the running probability is beyond the number
  tables   basq_kv_extend: pages, positions and slots of new tokens in a paged cache, pages of tokens that go back, the batch's page table
  step     tables, lookup, product and sample, as a decode step has them around its layers

`own` chooses between the plain form, in elementary torch operations, and the library's kernels.

Weights are uint8 [N, K/2], the even channel in the low nibble; scales and zero points bf16 [N, K/G] for groups of G channels; a weight is
scale * (code - zero point).  `streamed` weights lie in the library's streaming layout instead: for blocks of 16 rows and 128 channels,
16 bytes of each row after the other, then the next 16 bytes.
"""
from __future__ import annotations

import math
import random

import torch

own = False

MOST_WEIGHTS = 128000 * 8192     # of the largest listed product
MOST_LOGITS = 256 * 128000       # of the largest listed draw


def _product(name, M, K, N, G, streamed, f32, bias=False):
    return {"name": name, "kind": "product", "M": M, "K": K, "N": N, "G": G, "streamed": streamed, "f32": f32, "bias": bias}


def _lookup(name, T, K, N, G, streamed):
    return {"name": name, "kind": "lookup", "T": T, "K": K, "N": N, "G": G, "streamed": streamed}


def _sample(name, B, V, f32, filters):
    """filters: "free" (a temperature only), "top_k", "top_p", "min_p", "greedy", or "mixed": each row its own"""
    return {"name": name, "kind": "sample", "B": B, "V": V, "f32": f32, "filters": filters}


def _tables(name, B, page, longest, new, packed):
    """up to `new` tokens more of each sequence, packed from one on; of more than one, some sequences are cut instead"""
    return {"name": name, "kind": "tables", "B": B, "page": page, "longest": longest, "new": new, "packed": packed}


def listed():
    return [
        # one token through a square layer: the smallest product, latency
        _product("product_token", 1, 4096, 4096, 128, True, False),
        # a ragged batch through the widest contraction, weights as the quantiser leaves them, small groups, a bias
        _product("product_batch_13", 13, 14336, 4096, 64, False, False, True),
        # drafted tokens of a batch, the smallest groups
        _product("product_draft_48", 48, 4096, 11008, 32, True, False),
        # the output head of a large model for a batch: 560 MB of weights, the largest case
        _product("product_head_16", 16, 8192, 128000, 128, True, True),
        # the embeddings of a decode step
        _lookup("lookup_step_16", 16, 4096, 32000, 64, True),
        # ... and of a long prompt, from the head's matrix
        _lookup("lookup_prompt_4096", 4096, 8192, 128000, 128, True),
        # one sequence's next token out of a small vocabulary: latency
        _sample("sample_one", 1, 32000, False, "top_p"),
        # a server's batch: every request with choices of its own
        _sample("sample_batch_64", 64, 128000, True, "mixed"),
        # many samples without a filter: the whole mass counts
        _sample("sample_free_256", 256, 128000, False, "free"),
        # a decode step's places: one more token of each sequence
        _tables("tables_step_64", 64, 64, 8192, 1, False),
        # prompts of a batch, packed one behind the other, small pages, among sequences that end
        _tables("tables_prompts_48", 48, 16, 8192, 4096, True),
        # everything around the layers of a decode step of sixteen sequences
        {"name": "step_16", "kind": "step", "B": 16, "K": 4096, "V": 32000, "G": 128, "page": 64, "longest": 4096},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, mostly odd or ragged."""
    pick = rng.random()
    if pick < 0.35:
        streamed = rng.random() < 0.6
        K = 128 * _log_uniform(rng, 8, 112) if streamed else 32 * _log_uniform(rng, 32, 448)
        G = rng.choice([g for g in (32, 64, 128, 256, K) if K % g == 0])
        N = _log_uniform(rng, 1000, min(128000, MOST_WEIGHTS // K))
        M = _log_uniform(rng, 1, min(64, max(1, 16 * MOST_WEIGHTS // (N * K))))
        case = _product("", M, K, N, G, streamed, rng.random() < 0.4, rng.random() < 0.3)
    elif pick < 0.45:
        streamed = rng.random() < 0.6
        K = 128 * _log_uniform(rng, 8, 64) if streamed else 32 * _log_uniform(rng, 32, 256)
        G = rng.choice([g for g in (32, 64, 128, K) if K % g == 0])
        case = _lookup("", _log_uniform(rng, 1, 4096 * 8192 // K), K, _log_uniform(rng, 1000, 128000), G, streamed)
    elif pick < 0.75:
        V = _log_uniform(rng, 1000, 200000)
        B = _log_uniform(rng, 1, min(256, MOST_LOGITS // V))
        case = _sample("", B, V, rng.random() < 0.5, rng.choice(["free", "top_k", "top_p", "min_p", "greedy", "mixed", "mixed"]))
    elif pick < 0.9:
        packed = rng.random() < 0.5
        case = _tables("", _log_uniform(rng, 1, 512), rng.choice([16, 32, 64, 128]), _log_uniform(rng, 64, 8192),
                       _log_uniform(rng, 1, 4096) if packed else rng.randint(1, 8), packed)
        case["B"] = min(case["B"], max(1, 400000 // case["longest"], 64))
        case["new"] = min(case["new"], max(1, 200000 // case["B"]))
    else:
        K = 128 * _log_uniform(rng, 8, 64)
        case = {"kind": "step", "B": _log_uniform(rng, 1, 32), "K": K, "V": _log_uniform(rng, 1000, 64000), "G": rng.choice([64, 128]),
                "page": rng.choice([16, 64]), "longest": _log_uniform(rng, 64, 8192)}
    case.pop("name", None)
    return case


# ---- what a program has in hand --------------------------------------------------------------------

def _weights(s, gen, N, K, G, streamed):
    """4-bit weights with group scales of roughly normal weights, of a standard deviation that keeps outputs near that of inputs."""
    dev = {"device": "cuda"}
    # codes of two bytes' sum: bell-shaped, all sixteen values
    raw = torch.randint(0, 256, (N, K // 2), generator=gen, dtype=torch.uint8, **dev)
    other = torch.randint(0, 256, (N, K // 2), generator=gen, dtype=torch.uint8, **dev)
    mean = ((raw & 15) + (other & 15) + 1) // 2
    mean |= (((raw >> 4) + (other >> 4) + 1) // 2) << 4
    s["codes"] = mean
    scale = torch.exp(0.3 * torch.randn((N, K // G), generator=gen, **dev)) / (3.3 * math.sqrt(K))
    s["w_scale"] = scale.to(torch.bfloat16)
    s["w_zero"] = (7.5 + 1.2 * torch.randn((N, K // G), generator=gen, **dev)).clamp_(0, 15).to(torch.bfloat16)
    s["Wq"] = s["codes"]
    if streamed:
        rows = -(-N // 16) * 16
        padded = torch.zeros((rows, K // 2), dtype=torch.uint8, **dev)
        padded[:N] = s["codes"]
        s["Wq"] = padded.view(rows // 16, 16, K // 128, 4, 16).permute(0, 2, 3, 1, 4).contiguous().view(-1)


def _choices(s, gen, B, filters):
    """Each request's temperature, top-k, top-p, min-p, and its random number."""
    dev = {"device": "cuda"}
    row = torch.arange(B, **dev)
    uniform = lambda: torch.rand(B, generator=gen, **dev)  # noqa: E731
    s["temperature"] = 0.6 + 0.6 * uniform()
    k = torch.tensor([1, 5, 20, 50, 200, 1000], dtype=torch.int32, **dev)[torch.randint(0, 6, (B,), generator=gen, **dev)]
    p, m = 0.7 + 0.29 * uniform(), 0.02 + 0.1 * uniform()
    kind = {"free": 0, "top_k": 1, "top_p": 2, "min_p": 3, "greedy": 4}.get(filters)
    kind = (row + torch.randint(0, 6, (1,), generator=gen, **dev)) % 6 if kind is None else torch.full((B,), kind, **dev)
    both = kind == 5                                             # top-k and top-p together
    s["temperature"][kind == 4] = 0.0
    s["top_k"] = torch.where((kind == 1) | both, k, 0).to(torch.int32)
    s["top_p"] = torch.where((kind == 2) | both, p, 1.0)
    s["min_p"] = torch.where(kind == 3, m, 0.0)
    s["u"] = torch.rand(B, generator=gen, dtype=torch.float64, **dev)
    s["token"], s["kept"] = (torch.empty(B, dtype=torch.int32, **dev) for _ in range(2))
    s["logprob"] = torch.empty(B, **dev)
    # a program keeps a workspace: as many bytes as the library asks for, 64 MiB hold every case here
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, **dev)


def _logits(gen, B, V, f32):
    """A wide bell with a few dozen tokens that stand out, more in some rows than in others, and some tokens forbidden."""
    dev = {"device": "cuda"}
    z = 2.2 * torch.randn((B, V), generator=gen, **dev)
    few = min(64, V // 4)
    at = (torch.randint(0, V, (B, 1), generator=gen, **dev) + torch.arange(few, **dev) * (V // few)) % V
    up = 9.0 * torch.rand((B, 1), generator=gen, **dev) + 4.0 * torch.rand((B, few), generator=gen, **dev)
    z.scatter_(1, at, up)
    z.scatter_(1, torch.randint(0, V, (B, few), generator=gen, **dev), -math.inf)
    return z if f32 else z.to(torch.bfloat16)


def _places(s, gen, case, B, new, packed):
    """A pool of pages, twice as many sequences as the batch has, and what each of them holds already."""
    dev = {"device": "cuda"}
    P, longest = case["page"], case["longest"]
    rng = random.Random(B * 7919 + longest)                      # by the case alone, so that the work is known without a seed
    counts, before = _new_tokens(case, B, new, packed)
    width = -(-(longest + max(counts)) // P) + 1
    rows = 2 * B
    held = [rng.randint(0, longest) for _ in range(rows - B)]
    order = torch.randperm(rows, generator=gen, **dev)
    seqs = order[:B]
    lengths = torch.empty(rows, dtype=torch.int64, **dev)
    lengths[order] = torch.tensor(before + held, **dev)
    used = (lengths + P - 1) // P
    want = int(used.sum()) + sum(-(-(n + max(c, 0)) // P) for n, c in zip(before, counts)) + 5
    order = torch.randperm(want, generator=gen, **dev).to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32, **dev)
    column = torch.arange(width, **dev)[None]
    first = torch.cumsum(used, 0) - used
    table = torch.where(column < used[:, None], order[(first[:, None] + column).clamp(max=want - 1)], table)
    s["pool_table"], s["lengths"], s["seqs"] = table.contiguous(), lengths.to(torch.int32), seqs.to(torch.int32)
    s["free_pages"] = torch.full((want,), -1, dtype=torch.int32, **dev)
    taken = int(used.sum())
    s["free_pages"][:want - taken] = order[taken:]
    s["free_count"] = torch.tensor([want - taken], dtype=torch.int32, **dev)
    s["new_tokens"] = torch.tensor(counts, dtype=torch.int32, **dev)
    T = sum(max(c, 0) for c in counts) + 13 if packed else B * new  # (a packed batch has room for a few more)
    s["positions"], s["slots"] = (torch.empty(T, dtype=torch.int32, **dev) for _ in range(2))
    s["starts"] = torch.empty(B + 1, dtype=torch.int32, **dev) if packed else None
    s["batch_table"] = torch.full((B, width), -1, dtype=torch.int32, **dev)
    s["batch_lengths"] = torch.empty(B, dtype=torch.int32, **dev)
    s["lengths_out"] = s["lengths"].clone()                      # (a program gives the books themselves: here a pass can be repeated)
    s["free_out"] = torch.empty(1, dtype=torch.int32, **dev)
    s["status"] = torch.empty(2, dtype=torch.int32, **dev)
    s["books"] = torch.empty(1 << 20, dtype=torch.uint8, **dev)


def _new_tokens(case, B, new, packed):
    """(new tokens, tokens before) of each sequence of the batch; a negative number of new tokens is one of tokens that go."""
    rng = random.Random(B * 1000003 + case["longest"])
    if packed:
        # prompts, most of them begun here, and sequences that end
        counts, before = [rng.randint(1, new) for _ in range(B)], [0 if rng.random() < 0.7 else rng.randint(1, case["longest"]) for _ in range(B)]
        ends = [rng.random() < 0.15 for _ in range(B)]
        return [-n if n and end else c for c, n, end in zip(counts, before, ends)], before
    # a step; with drafts not every sequence has as many, and some lose those that were refused
    before = [rng.randint(1, case["longest"]) for _ in range(B)]
    counts = [new if rng.random() < 0.8 else rng.randint(-min(new, n), new) for n in before] if new > 1 else [1] * B
    return counts, before


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) + 715689)
    s = {"case": case}
    dev = {"device": "cuda"}
    kind = case["kind"]
    if kind == "product":
        M, K, N = case["M"], case["K"], case["N"]
        _weights(s, gen, N, K, case["G"], case["streamed"])
        x = torch.randn((M, K), generator=gen, **dev)
        x[:, torch.randperm(K, generator=gen, **dev)[:max(1, K // 256)]] *= 10.0
        s["x"] = x.to(torch.bfloat16)
        s["bias"] = torch.randn(N, generator=gen, **dev) if case["bias"] else None
        s["y"] = torch.empty((M, N), dtype=torch.float32 if case["f32"] else torch.bfloat16, **dev)
    elif kind == "lookup":
        _weights(s, gen, case["N"], case["K"], case["G"], case["streamed"])
        s["ids"] = torch.randint(0, case["N"], (case["T"],), generator=gen, dtype=torch.int32, **dev)
        s["scale"] = math.sqrt(case["K"])
        s["rows"] = torch.empty((case["T"], case["K"]), dtype=torch.bfloat16, **dev)
    elif kind == "sample":
        s["logits"] = _logits(gen, case["B"], case["V"], case["f32"])
        _choices(s, gen, case["B"], case["filters"])
    elif kind == "tables":
        _places(s, gen, case, case["B"], case["new"], case["packed"])
    else:
        B, K, V = case["B"], case["K"], case["V"]
        _places(s, gen, case, B, 1, False)
        _weights(s, gen, V, K, case["G"], True)
        s["ids"] = torch.randint(0, V, (B,), generator=gen, dtype=torch.int32, **dev)
        s["scale"] = math.sqrt(K)
        s["rows"] = torch.empty((B, K), dtype=torch.bfloat16, **dev)
        s["x"] = (3.0 * torch.randn((B, K), generator=gen, **dev)).to(torch.bfloat16)
        s["bias"] = None
        s["y"] = torch.empty((B, V), **dev)
        # most requests greedy, some out of the eight likeliest
        _choices(s, gen, B, "greedy")
        some = torch.arange(B, **dev) % 4 == 1
        s["temperature"][some] = 0.7
        s["top_k"][some] = 8
    return s


# ---- the library's operators -----------------------------------------------------------------------

def _layout(case):
    from paper_2506_15689_amd import binding as B
    return B.BASQ_W_DECODE16 if case.get("streamed", True) else B.BASQ_W_CANONICAL


def _own_product(s):
    from paper_2506_15689_amd import binding as B
    B.basq_w4a16_gemm(s["x"], s["Wq"], s["w_scale"], s["w_zero"], s["y"], s["bias"], w_layout=_layout(s["case"]))
    return [s["y"]]


def _own_lookup(s):
    from paper_2506_15689_amd import binding as B
    B.basq_w4a16_lookup(s["ids"], s["Wq"], s["w_scale"], s["w_zero"], s["rows"], s["scale"], w_layout=_layout(s["case"]))
    return [s["rows"]]


def _own_sample(s, logits):
    from paper_2506_15689_amd import binding as B
    B.basq_sample(logits, s["u"], s["token"], s["workspace"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                  min_p=s["min_p"], logprob=s["logprob"], kept=s["kept"])
    return [s["token"], s["logprob"], s["kept"]]


def _own_tables(s):
    from paper_2506_15689_amd import binding as B
    c = s["case"]
    B.basq_kv_extend(s["lengths"], s["pool_table"], s["free_pages"], s["free_count"], s["new_tokens"], c["page"], s["positions"],
                     s["slots"], s["status"], s["books"], seqs=s["seqs"], q_len=0 if c.get("packed") else c.get("new", 1), starts=s["starts"],
                     batch_table=s["batch_table"], batch_lengths=s["batch_lengths"], lengths_out=s["lengths_out"], free_out=s["free_out"])
    return _places_of(s)


def _places_of(s):
    names = ["positions", "slots", "batch_table", "batch_lengths", "pool_table", "lengths_out", "free_pages", "free_out", "status"]
    return [s[n] for n in names] + ([s["starts"]] if s["starts"] is not None else [])


# ---- the same in elementary operations, 32 bits throughout (a draw's sums and exponentials in 64: its token is a whole number) -------

def _values(codes, w_scale, w_zero):
    N, K = codes.shape[0], 2 * codes.shape[1]
    q = torch.stack([codes & 15, codes >> 4], -1).view(N, w_scale.shape[1], -1).float()
    return (w_scale.float()[..., None] * (q - w_zero.float()[..., None])).view(N, K)


def _plain_product(s):
    x, rows = s["x"].float(), max(1, (1 << 28) // s["x"].shape[1])
    for n in range(0, s["codes"].shape[0], rows):                # (a quarter of 2^30 weights at a time)
        part = x @ _values(s["codes"][n:n + rows], s["w_scale"][n:n + rows], s["w_zero"][n:n + rows]).t()
        if s["bias"] is not None:
            part = part + s["bias"][n:n + rows]
        s["y"][:, n:n + rows] = part.to(s["y"].dtype)
    return [s["y"]]


def _plain_lookup(s):
    at = s["ids"].long()
    return [(_values(s["codes"][at], s["w_scale"][at], s["w_zero"][at]) * s["scale"]).to(torch.bfloat16)]


def _plain_sample(s, logits):
    z = logits.float()
    z = torch.where(z.isnan(), torch.full_like(z, -math.inf), z)
    V = z.shape[1]
    ordered, order = torch.sort(z, dim=1, descending=True, stable=True)
    there = ordered > -math.inf
    temperature = s["temperature"].double()[:, None]
    greedy = ~(temperature > 0)
    top = ordered[:, :1].double()
    w = torch.exp((ordered.double() - top) / torch.where(greedy, torch.ones_like(temperature), temperature))
    w = torch.where(ordered == ordered[:, :1], torch.ones_like(w), w)
    w = torch.where(there, w, torch.zeros_like(w))
    running = torch.cumsum(w, 1)
    count = there.sum(1, keepdim=True)
    k = s["top_k"].long()[:, None]
    n = torch.minimum(count, torch.where(k > 0, k, V))
    mass = running.gather(1, (n - 1).clamp(min=0))
    p, m = s["top_p"].double()[:, None], s["min_p"].double()[:, None]
    enough = (running < p * mass).sum(1, keepdim=True) + 1
    first_n = torch.minimum(n, torch.where(p < 1, enough, n))
    likely = (w >= m.clamp(max=1.0)).sum(1, keepdim=True)
    first_n = torch.minimum(first_n, torch.where(m > 0, likely, first_n))
    first_n = torch.minimum(first_n, torch.where(greedy, torch.ones_like(first_n), first_n))
    total = running.gather(1, first_n - 1 + (first_n == 0).long())
    place = (running <= s["u"][:, None] * total).sum(1, keepdim=True)
    place = torch.minimum(place, (torch.minimum(first_n, (w > 0).sum(1, keepdim=True)) - 1).clamp(min=0))
    token = order.gather(1, place)
    logprob = torch.log(w.gather(1, place) / total)
    empty = count == 0
    token = torch.where(empty, torch.full_like(token, -1), token)
    logprob = torch.where(empty, torch.full_like(logprob, -math.inf), logprob)
    return [token[:, 0].to(torch.int32), logprob[:, 0].float(), first_n[:, 0].to(torch.int32)]


def _plain_tables(s):
    c = s["case"]
    P, B, width = c["page"], s["seqs"].numel(), s["pool_table"].shape[1]
    dev = s["seqs"].device
    rows, new = s["seqs"].long(), s["new_tokens"].long()
    before = s["lengths"][rows].long()
    after = before + new
    had, need = (before + P - 1) // P, (after + P - 1) // P
    more, less = (need - had).clamp(min=0), (had - need).clamp(min=0)
    first, first_back = torch.cumsum(more, 0) - more, torch.cumsum(less, 0) - less
    column = torch.arange(width, device=dev)[None]
    old = s["pool_table"][rows]
    # pages that go back lie behind the free ones, in the order of the sequences, a sequence's from its first on
    back = (column >= need[:, None]) & (column < had[:, None])
    to = s["free_count"].long() + first_back[:, None] + column - need[:, None]
    free = torch.cat([s["free_pages"], s["free_pages"].new_zeros(1)])
    free[torch.where(back, to, free.numel() - 1)] = old
    s["free_pages"].copy_(free[:-1])
    # the page table: what there was, then pages from the end of the free ones
    fresh = (column >= had[:, None]) & (column < need[:, None])
    at = s["free_count"].long() + less.sum() - 1 - (first[:, None] + column - had[:, None])
    table = torch.where(fresh, s["free_pages"][at.clamp(0, s["free_pages"].numel() - 1)], old)
    s["pool_table"][rows] = table
    s["batch_table"].copy_(torch.where(column < need[:, None], table, s["batch_table"]))
    s["batch_lengths"].copy_(after)
    s["lengths_out"][rows] = after.to(torch.int32)
    s["free_out"].copy_(s["free_count"] + less.sum() - more.sum())
    s["status"].zero_()
    # tokens
    T = s["positions"].numel()
    t = torch.arange(T, device=dev)
    if s["starts"] is not None:
        new = new.clamp(min=0)
        ends = torch.cumsum(new, 0)
        s["starts"][0] = 0
        s["starts"][1:] = ends
        seq = torch.searchsorted(ends, t, right=True).clamp(max=B - 1)
        i = t - (ends - new)[seq]
        there = t < ends[-1]
    else:
        q_len = c.get("new", 1)
        seq = t // q_len
        i = t % q_len - (q_len - new.clamp(min=0)[seq])
        there = i >= 0
    position = before[seq] + i
    page = table[seq, (position // P).clamp(0, width - 1)].long()
    s["positions"].copy_(torch.where(there, position, -1))
    s["slots"].copy_(torch.where(there, page * P + position % P, -1))
    return _places_of(s)


def run(s):
    kind = s["case"]["kind"]
    product, lookup, sample, tables = ((_own_product, _own_lookup, _own_sample, _own_tables) if own else
                                       (_plain_product, _plain_lookup, _plain_sample, _plain_tables))
    if kind == "product":
        return product(s)
    if kind == "lookup":
        return lookup(s)
    if kind == "sample":
        return sample(s, s["logits"])
    if kind == "tables":
        return tables(s)
    places = tables(s)
    rows = lookup(s)
    logits = product(s)
    return places + rows + logits + sample(s, logits[0])


# ---- the same from its definition, in 64 bits ---------------------------------------------------------

def _exact_rows(s, at):
    """Rows `at` of the matrix, one group behind the other."""
    N, groups = s["w_scale"].shape
    codes = s["codes"][at]
    out = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    out[:, 0::2] = (codes % 16).double()
    out[:, 1::2] = (codes // 16).double()
    G = out.shape[1] // groups
    for g in range(groups):
        out[:, g * G:(g + 1) * G] -= s["w_zero"][at, g].double()[:, None]
        out[:, g * G:(g + 1) * G] *= s["w_scale"][at, g].double()[:, None]
    return out


def _exact_product(s):
    x = s["x"].double()
    N, rows = s["codes"].shape[0], max(1, (1 << 26) // x.shape[1])
    parts = [torch.matmul(x, _exact_rows(s, torch.arange(n, min(N, n + rows), device=x.device)).t().contiguous()) for n in range(0, N, rows)]
    y = torch.cat(parts, 1)
    return [y if s["bias"] is None else y + s["bias"].double()]


def _exact_sample(s, logits):
    """Row by row: the likeliest tokens one after the other, as the definition says it."""
    z = logits.double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).cpu().numpy()
    import numpy as np
    tokens, logprobs, counts = [], [], []
    for b in range(z.shape[0]):
        T, k, p, m, u = (float(s[n][b]) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        row = z[b]
        index = np.flatnonzero(row > -math.inf)
        if index.size == 0:
            tokens.append(-1), logprobs.append(-math.inf), counts.append(0)
            continue
        index = index[np.argsort(-row[index], kind="stable")]
        if not T > 0:
            index = index[:1]
            w = np.ones(1)
        else:
            w = np.where(row[index] == row[index[0]], 1.0, np.exp((row[index] - row[index[0]]) / T))
            if k > 0:
                index, w = index[:int(k)], w[:int(k)]
            n = w.size
            if p < 1:
                n = min(n, int(np.searchsorted(np.cumsum(w), p * w.sum(), side="left")) + 1)
            if m > 0:
                n = min(n, int((w >= min(m, 1.0)).sum()))
            index, w = index[:n], w[:n]
        running = np.cumsum(w)
        at = int(np.searchsorted(running, u * running[-1], side="right"))
        at = min(at, int(np.flatnonzero(w > 0)[-1]))
        tokens.append(int(index[at]))
        logprobs.append(math.log(w[at] / running[-1]))
        counts.append(index.size)
    dev = {"device": logits.device}
    return [torch.tensor(tokens, dtype=torch.int32, **dev), torch.tensor(logprobs, dtype=torch.float64, **dev),
            torch.tensor(counts, dtype=torch.int32, **dev)]


def _exact_tables(s):
    """Sequence by sequence, token by token, with a list of free pages."""
    c = s["case"]
    P, q_len = c["page"], 0 if c.get("packed") else c.get("new", 1)
    pool, lengths, batch = s["pool_table"].tolist(), s["lengths"].tolist(), s["batch_table"].tolist()
    seqs, new = s["seqs"].tolist(), s["new_tokens"].tolist()
    free, room = s["free_pages"].tolist(), s["free_pages"].numel()
    behind = free[int(s["free_count"]):]
    free = free[:int(s["free_count"])]
    for q, n in zip(seqs, new):
        if n < 0:
            free += pool[q][-(-(lengths[q] + n) // P):-(-lengths[q] // P)]
    behind = free + behind[len(free) + len(behind) - room:]
    positions, slots, starts, after = [], [], [0], []
    for b, (q, n) in enumerate(zip(seqs, new)):
        length, tokens = lengths[q], []
        for t in range(length, length + n):
            if t % P == 0:
                pool[q][t // P] = free.pop()
            tokens.append((t, pool[q][t // P] * P + t % P))
        lengths[q] = length + n
        after.append(length + n)
        used = -(-(length + n) // P)
        batch[b][:used] = pool[q][:used]
        tokens = [(-1, -1)] * (q_len - len(tokens)) + tokens if q_len else tokens
        positions += [t for t, _ in tokens]
        slots += [at for _, at in tokens]
        starts.append(len(positions))
    T = s["positions"].numel()
    positions += [-1] * (T - len(positions))
    slots += [-1] * (T - len(slots))
    out = [positions, slots, batch, after, pool, lengths, behind, [len(free)], [0, 0]] + ([starts] if not q_len else [])
    return [torch.tensor(v, dtype=torch.int32, device=s["seqs"].device) for v in out]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "product":
        return _exact_product(s)
    if kind == "lookup":
        return [_exact_rows(s, s["ids"].long()) * s["scale"]]
    if kind == "sample":
        return _exact_sample(s, s["logits"])
    if kind == "tables":
        return _exact_tables(s)
    # logits are stored in 32 bits, and the draw is from the stored ones
    logits = _exact_product(s)
    return _exact_tables(s) + [_exact_rows(s, s["ids"].long()) * s["scale"]] + logits + _exact_sample(s, logits[0].float())


# ---- what a pass cannot do without ------------------------------------------------------------------

def _weight_bytes(rows, K, G):
    return rows * (K // 2 + 4 * (K // G))


def _product_work(M, K, N, G, f32, bias):
    return _weight_bytes(N, K, G) + 2 * M * K + M * N * (4 if f32 else 2) + (4 * N if bias else 0), 2 * M * N * K


def _lookup_work(T, K, G):
    return _weight_bytes(T, K, G) + 4 * T + 2 * T * K, 3 * T * K


def _sample_work(B, V, f32):
    return B * (V * (4 if f32 else 2) + 4 * 4 + 8 + 3 * 4), 2 * B * V


def _tables_work(case, B, new, packed):
    counts, before = _new_tokens(case, B, new, packed)
    P = case["page"]
    pages = sum(-(-(n + c) // P) for n, c in zip(before, counts))
    moved = sum(abs(-(-(n + c) // P) - -(-n // P)) for n, c in zip(before, counts))
    T = sum(max(c, 0) for c in counts) + 13 if packed else B * new
    # the batch's table read and written, pages taken or given back, tokens' places, five numbers a sequence
    return 4 * (2 * pages + moved) + 8 * T + 20 * B, 4 * T + pages


def work(case):
    kind = case["kind"]
    if kind == "product":
        parts = [_product_work(case["M"], case["K"], case["N"], case["G"], case["f32"], case["bias"])]
    elif kind == "lookup":
        parts = [_lookup_work(case["T"], case["K"], case["G"])]
    elif kind == "sample":
        parts = [_sample_work(case["B"], case["V"], case["f32"])]
    elif kind == "tables":
        parts = [_tables_work(case, case["B"], case["new"], case["packed"])]
    else:
        B, K, V, G = case["B"], case["K"], case["V"], case["G"]
        parts = [_tables_work(case, B, 1, False), _lookup_work(B, K, G), _product_work(B, K, V, G, True, False), _sample_work(B, V, True)]
    return {"bytes": sum(p[0] for p in parts), "flops": sum(p[1] for p in parts)}

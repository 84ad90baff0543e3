"""The operators around the linear layer on the GPU, against their definitions (block_ref.py).  Tolerances are stated where they are
used, with what they follow from."""
import math

import pytest
import torch

from paper_2506_15689_amd import binding as B

import block_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16 = torch.bfloat16
UNTOUCHED = 0xA5


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def strided(t, pad):
    """The same values in rows that are `pad` elements further apart."""
    if pad == 0:
        return t.contiguous()
    M, width = t.shape[0], t[0].numel()
    wide = torch.full((M, width + pad), 7.0, dtype=torch.float32, device=t.device).to(t.dtype)
    view = wide[:, :width].unflatten(1, t.shape[1:]) if t.dim() == 3 else wide[:, :width]
    view.copy_(t)
    return view


def check_stored(got, want, slack):
    """bf16 values against fp64 ones that the arithmetic in front of the store may miss by `slack`: rounding is monotonic, so what is
    stored lies between the roundings of the ends."""
    got, low, high = ref.f64(got), (want - slack).to(BF16).double(), (want + slack).to(BF16).double()
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values; the furthest {float(((got - want).abs() / slack)[bad].max())} times the slack away"


# ---- norm ----------------------------------------------------------------------------------------

def check_norm(y, want):
    # fp32: a sum of squares in runs of up to 64 and a tree behind, three roundings and rsqrt: under 2^-16
    check_stored(y, want, want.abs() * 2.0 ** -16)


@pytest.mark.parametrize("M,K", [(1, 8), (3, 520), (2, 512), (5, 1016), (4, 2048), (3, 2056), (61, 4096), (1, 8192), (7, 11008), (5, 14336), (2, 16392), (2, 32768)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_norm(M, K, with_residual):
    g = gen(M * K)
    x, r = (randn(g, M, K) * 3).to(BF16), randn(g, M, K).to(BF16) if with_residual else None
    w = (1 + 0.2 * randn(g, K)).to(BF16)
    x = strided(x, 24)
    r = strided(r, 8) if with_residual else None
    y, h = strided(torch.zeros(M, K, dtype=BF16, device=DEV), 16), torch.zeros(M, K, dtype=BF16, device=DEV)
    y8, s8 = torch.zeros(M, K + 8, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)[:, :K], torch.zeros(M, device=DEV)
    B.basq_add_rms_norm(x, r, w, 1e-5, y, h, Y8=y8, y8_scale=s8)
    want_h, want = ref.add_rms_norm(x, r, w, 1e-5)
    assert torch.equal(h.cpu(), want_h)
    check_norm(y, want)
    if M > 1:
        assert (y._base[:, K:] == 7).all(), "the gaps between rows were written"
    top = want.abs().amax(1)
    assert ((ref.f64(s8) - top / 448).abs() <= top / 448 * 2.0 ** -16).all()
    # e4m3: half of a step, 2^-4 of a normal number, 2^-10 of the scale below; and fp32 in front
    got = ref.f64(y8.float()) * ref.f64(s8)[:, None]
    tol = torch.maximum(want.abs() * 2.0 ** -4, ref.f64(s8)[:, None] * 2.0 ** -10) * (1 + 2.0 ** -10)
    assert ((got - want).abs() <= tol).all()
    # either output alone, in place of the inputs
    x2 = x.contiguous().clone()
    r2 = None if r is None else r.contiguous().clone()
    B.basq_add_rms_norm(x2, r2, w, 1e-5, x2, r2)
    assert torch.equal(x2, y) and (r2 is None or torch.equal(r2, h))
    y8b, s8b = torch.zeros_like(y8.contiguous()), torch.zeros_like(s8)
    B.basq_add_rms_norm(x, r, w, 1e-5, None, Y8=y8b, y8_scale=s8b)
    assert torch.equal(y8b.view(torch.uint8), y8.contiguous().view(torch.uint8)) and torch.equal(s8b, s8)


def test_norm_of_unusual_rows():
    """Zeros, infinities and NaN stay in their rows; tiny and huge rows are normed like others as far as fp32 squares go."""
    g = gen(1)
    K = 4096
    x = randn(g, 8, K).to(BF16)
    clean = x.clone()
    x[1] = 0
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    x[4] *= 1e-15
    x[5] *= 1e15
    w = torch.ones(K, dtype=BF16, device=DEV)
    y, y8, s8 = torch.empty_like(x), torch.empty(8, K, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(8, device=DEV)
    B.basq_add_rms_norm(x, None, w, 0.0, y, Y8=y8, y8_scale=s8)
    y0 = torch.empty_like(x)
    B.basq_add_rms_norm(clean, None, w, 0.0, y0)
    for m in (0, 6, 7):
        assert torch.equal(y[m], y0[m])
    for m in (4, 5):
        check_norm(y[m:m + 1], ref.add_rms_norm(x[m:m + 1], None, w, 0.0)[1])
    assert torch.isnan(y[3]).all() and torch.isnan(y[2, 5])
    B.basq_add_rms_norm(x, None, w, 1e-5, y, Y8=y8, y8_scale=s8)
    assert (y[1] == 0).all() and (y8[1].float() == 0).all() and s8[1] == 1.0


# ---- rotary positions, rotation, cache -----------------------------------------------------------

@pytest.mark.parametrize("scaling,kw", [
    (B.ROPE_PLAIN, {}), (B.ROPE_LINEAR, dict(factor=4.0)), (B.ROPE_BANDS, dict(factor=8.0, low=1.0, high=4.0, original_len=8192.0)),
    (B.ROPE_YARN, dict(factor=16.0, low=1.0, high=32.0, original_len=4096.0)),
])
def test_rope_table(scaling, kw):
    for rot, base, n in [(128, 500000.0, 1000), (32, 10000.0, 77), (2, 10000.0, 1)]:
        t = torch.empty(n, rot, device=DEV)
        B.basq_rope_table(t, base, scaling=scaling, **kw)
        want = ref.rope_table(n, rot, base, scaling, **kw)
        # fp64 inside (positions of a thousand: angles to 2^-40), rounded to fp32 once
        assert ((ref.f64(t) - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -38).all()
    # far positions
    big = torch.empty(1 << 20, 16, device=DEV)
    B.basq_rope_table(big, 10000.0, scaling=scaling, **kw)
    want = ref.rope_table(1 << 20, 16, 10000.0, scaling, **kw)
    assert ((ref.f64(big) - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -30).all()


def append_case(seed, T, heads, kv_heads, D, P, rot, pages=None):
    g = gen(seed)
    x = randn(g, T, heads + 2 * kv_heads, D)
    x[:, :, :3] += 5
    x = x.to(BF16)
    rows = 50
    table = torch.empty(rows, rot, device=DEV) if rot else None
    if rot:
        B.basq_rope_table(table, 10000.0)
    pages = pages or -(-2 * T // P) + 1
    cache = torch.full((pages, max(kv_heads, 1), P * (D + 16)), UNTOUCHED, dtype=torch.uint8, device=DEV)
    slots = torch.randperm(pages * P, generator=g, device=DEV)[:T].to(torch.int32)
    positions = torch.randint(0, rows, (T,), generator=g, device=DEV, dtype=torch.int32)
    return x, table, cache, slots, positions


@pytest.mark.parametrize("T,heads,kv_heads,D,P,rot,interleaved,rotate", [
    (1, 32, 32, 128, 64, 128, False, True),
    (5, 8, 2, 128, 16, 64, True, True),
    (37, 7, 1, 64, 32, 64, False, True),
    (3, 71, 1, 64, 16, 16, True, False),
    (130, 28, 4, 128, 128, 32, False, False),
    (9, 5, 5, 64, 16, 0, False, True),
    (2, 3, 3, 128, 1024, 112, False, True),
    (11, 6, 6, 128, 16, 48, True, True),
    (700, 2, 1, 128, 64, 128, False, True),
    (4, 1, 9, 64, 16, 64, False, False),
])
def test_append_is_the_definition_bit_for_bit(T, heads, kv_heads, D, P, rot, interleaved, rotate):
    x, table, cache, slots, positions = append_case(T * heads + D, T, heads, kv_heads, D, P, rot)
    want_cache = cache.cpu().clone()
    slots[0] = -1 if T > 2 else slots[0]                            # not stored
    if T > 4:
        slots[1] = cache.shape[0] * P                               # nor this one
        positions[2], positions[3] = -1, 50                         # padding, if there are positions
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    q_out = torch.full((T, heads, D), 9.0, dtype=BF16, device=DEV)
    hats = [strided(torch.full((T, kv_heads, D), 9.0, dtype=BF16, device=DEV), 8) for _ in range(2)]
    B.basq_rope_append(q, k, v, positions if rot else None, table, slots, cache, 0.9, 0.8, q_out, *hats, interleaved=interleaved, rotate=rotate)

    skipped = torch.zeros(T, dtype=torch.bool)
    if rot:
        skipped = (positions.cpu() < 0) | (positions.cpu() >= 50)
    keep = (~skipped)[:, None, None]
    nine = torch.tensor(9.0, dtype=BF16)
    want_q = ref.turn(q, table, positions, interleaved, rotate)
    assert torch.equal(q_out.cpu(), torch.where(keep, want_q.to(BF16), nine))
    stored = torch.where(skipped, torch.tensor(-1, dtype=torch.int32), slots.cpu())
    for which, part in enumerate([ref.turn(k, table, positions, interleaved, rotate), v.cpu().float()]):
        codes, s, lo = ref.quantise(part, 0.9, 0.8)
        ref.put(want_cache, D, stored, which, codes, s, lo)
        assert torch.equal(hats[which].cpu(), torch.where(keep, ref.dequantise(codes, s, lo).to(BF16), nine))
    assert torch.equal(cache.cpu(), want_cache)
    # and in 64 bits: the transform's sums of up to D values lose 2^-24 a stage, of the vector's length
    exact = ref.turn(q, table, positions, interleaved, rotate, torch.float64)
    length = q.cpu().double().norm(dim=-1, keepdim=True)
    check_stored(q_out.cpu()[~skipped], exact[~skipped], (16 * 2.0 ** -24 * length + 0 * exact)[~skipped])


def test_append_parts_and_places():
    """q alone, keys and values alone, without a cache, in place: the same values as all together."""
    T, heads, kv_heads, D, P = 33, 8, 4, 128, 16
    x, table, cache, slots, positions = append_case(3, T, heads, kv_heads, D, P, 128)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    q_out = torch.empty(T, heads, D, dtype=BF16, device=DEV)
    hats = [torch.empty(T, kv_heads, D, dtype=BF16, device=DEV) for _ in range(2)]
    B.basq_rope_append(q, k, v, positions, table, slots, cache, 0.9, 0.9, q_out, *hats)
    q2 = torch.empty_like(q_out)
    B.basq_rope_append(q, None, None, positions, table, None, None, 0.9, 0.9, q2)
    assert torch.equal(q2, q_out)
    cache2 = torch.full_like(cache, UNTOUCHED)
    B.basq_rope_append(None, k, v, positions, table, slots, cache2, 0.9, 0.9, None)
    assert torch.equal(cache2, cache)
    inplace = x.clone()
    B.basq_rope_append(inplace[:, :heads], inplace[:, heads:heads + kv_heads], inplace[:, heads + kv_heads:], positions, table, None, None,
                       0.9, 0.9, inplace[:, :heads], inplace[:, heads:heads + kv_heads], inplace[:, heads + kv_heads:])
    assert torch.equal(inplace[:, :heads], q_out)
    assert torch.equal(inplace[:, heads:heads + kv_heads], hats[0]) and torch.equal(inplace[:, heads + kv_heads:], hats[1])


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_heads_whose_sums_cancel(D):
    """Heads of zeros, of one value, of alternating values and of one channel: the transform's zeros are positive, every bit of the
    cache as defined."""
    T, P = 5, 16
    x, _, cache, slots, _ = append_case(6, T, 2, 2, D, P, 0)
    x[:, :4:2] = 0
    x[1, :] = 1.5
    x[2, :, ::2], x[2, :, 1::2] = -3.0, 3.0
    x[3, 1:3] = 0
    x[3, 1, D - 1], x[3, 2, 9] = 7.0, -7.0
    want_cache = cache.cpu().clone()
    q, k, v = x[:, :2], x[:, 2:4], x[:, 4:]
    q_out = torch.empty(T, 2, D, dtype=BF16, device=DEV)
    B.basq_rope_append(q, k, v, None, None, slots, cache, 0.9, 0.8, q_out)
    bits = lambda y: y.cpu().to(BF16).contiguous().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(q_out), bits(ref.turn(q, None, None, False, True)))
    for which, part in enumerate([ref.turn(k, None, None, False, True), v.cpu().float()]):
        codes, s, lo = ref.quantise(part, 0.9, 0.8)
        ref.put(want_cache, D, slots.cpu(), which, codes, s, lo)
    assert torch.equal(cache.cpu(), want_cache)


def test_append_of_unusual_vectors():
    """Constant, zero, infinite and NaN vectors: the quantiser's rules for them, and no other vector changes."""
    T, D, P = 6, 64, 16
    x, _, cache, slots, _ = append_case(4, T, 1, 2, D, P, 0)
    k, v = x[:, 1:3], x[:, 3:5]
    k[0, 0], v[1, 1], v[2, 0], k[3, 1], v[4, 0, 5] = 0, 2.5, float("inf"), float("nan"), float("nan")
    clean = cache.clone()
    B.basq_rope_append(None, k, v, None, None, slots, cache, 0.9, 0.9, None, rotate=False)
    codes, ranges = ref.cache_views(cache.cpu(), D)
    place = [(s // P, s % P) for s in slots.tolist()]
    at = lambda t, h, which: ranges[place[t][0], h, which, place[t][1]]  # noqa: E731
    assert at(0, 0, 0).tolist() == [1.0, 0.0] and at(2, 0, 1)[0] == 1.0 and at(3, 1, 0)[0] == 1.0
    # (a constant: 0.9 of it at both ends)
    assert at(1, 1, 1).tolist() == [1.0, float(torch.tensor(0.9) * 2.5)]
    for t, h, which, part in [(5, 0, 0, k), (5, 1, 1, v), (0, 1, 0, k), (1, 0, 1, v), (4, 1, 1, v)]:
        want, s, lo = ref.quantise(part[t, h].cpu().float(), 0.9, 0.9)
        c = codes[place[t][0], h, which, place[t][1]]
        assert torch.equal(torch.stack([c & 15, c >> 4], -1).flatten().float(), want) and at(t, h, which).tolist() == [float(s), float(lo)]
    assert not torch.equal(clean, cache)


def test_append_agrees_with_the_per_head_quantiser():
    """k without rotary positions is what basq_rotate_quant with rot_size = group_size = 128 makes of it, but for the order of sums."""
    T, heads, D, P = 300, 4, 128, 64
    x, _, cache, slots, _ = append_case(5, T, 0, heads, D, P, 0)
    k, v = x[:, :heads].contiguous(), x[:, heads:]
    B.basq_rope_append(None, k, v, None, None, slots, cache, 0.9, 0.9, None)
    Aq = torch.empty(T, heads * D // 2, dtype=torch.uint8, device=DEV)
    meta = torch.empty(T * heads, 4, dtype=torch.int32, device=DEV)
    B.basq_rotate_quant(k.view(T, heads * D), D, None, None, 0.9, 0.9, Aq, meta, group_size=D)
    codes, ranges = ref.cache_views(cache, D)
    s = slots.long()
    mine, theirs = codes[s // P, :, 0, s % P], Aq.view(T, heads, D // 2)
    # another order of fp32 sums moves a code in some ten thousand at most
    assert (mine != theirs).float().mean() <= 1e-4
    r = meta.view(torch.float32).view(T, heads, 4)[..., :2]
    torch.testing.assert_close(ranges[s // P, :, 0, s % P], r, rtol=1e-5, atol=1e-5)


# ---- attention -----------------------------------------------------------------------------------

def attention_case(seed, lengths, heads, kv_heads, D, P, q_len, spare=2, holes=0, scale_of_values=0.36):
    """A cache whose pages are in random order, and whatever lies outside the contexts is 0xFF: codes of 15, ranges that are NaN."""
    g = gen(seed)
    Bn = len(lengths)
    used = [max(-(-n // P), 0) for n in lengths]
    pages = sum(used) + spare
    cache = torch.full((pages, kv_heads, P * (D + 16)), 0xFF, dtype=torch.uint8, device=DEV)
    codes, ranges = ref.cache_views(cache, D)
    order = torch.randperm(pages, generator=g, device=DEV)
    table = torch.full((Bn, max(used + [1]) + 1), -7, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(lengths):
        mine = order[at:at + used[b]]
        at += used[b]
        table[b, :used[b]] = mine.to(torch.int32)
        if n > 0:
            t = torch.arange(n, device=DEV)
            page, off = mine[t // P], t % P
            codes[page, :, :, off] = torch.randint(0, 256, (n, kv_heads, 2, D // 2), generator=g, device=DEV, dtype=torch.uint8)
            s = torch.exp(0.3 * randn(g, n, kv_heads, 2)) * 0.36
            s[..., 1] *= scale_of_values / 0.36
            ranges[page, :, :, off] = torch.stack([s, s * (-7.5 + 0.5 * randn(g, n, kv_heads, 2))], -1)
    for _ in range(holes):                                           # pages that are not there
        b = int(torch.randint(0, Bn, (1,), generator=g, device=DEV))
        if used[b] > 1:
            table[b, int(torch.randint(0, used[b], (1,), generator=g, device=DEV))] = pages if holes % 2 else -1
            holes -= 1
    q = (1.8 * randn(g, Bn * q_len, heads, D)).to(BF16)
    return q, cache, table, torch.tensor(lengths, dtype=torch.int32, device=DEV)


def attend(q, cache, table, lengths, max_len, q_len=1, softcap=0.0, window=0, scale=None, pad=0, guard=True):
    rows, heads, D = q.shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    need = B.basq_paged_attention_workspace_bytes(lengths.numel(), q_len, heads, cache.shape[1], D, max_len, window)
    # (the workspace is full of NaN, and one byte longer would be seen)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    out = strided(torch.full((rows, heads, D), 9.0, dtype=BF16, device=DEV), pad)
    lse = torch.full((rows, heads), 9.0, device=DEV)
    B.basq_paged_attention(q, cache, table, lengths, max_len, scale, out, ws[:need] if need else None, q_len=q_len, softcap=softcap, window=window, lse=lse)
    if guard:
        assert (ws[need:] == 0xFF).all()
    return out, lse


def check_attention(q, cache, table, lengths, max_len, q_len=1, softcap=0.0, window=0, scale=None, pad=0):
    out, lse = attend(q, cache, table, lengths, max_len, q_len, softcap, window, scale, pad)
    scale = 1 / math.sqrt(q.shape[2]) if scale is None else scale
    want, want_lse, slack, slack_lse = ref.paged_attention(q, cache, table, lengths, max_len, scale, q_len, softcap, window)
    got, got_lse = ref.f64(out), ref.f64(lse)
    empty = torch.isinf(want_lse)
    assert torch.equal(got_lse[empty], want_lse[empty]) and (got[empty] == 0).all()
    check_stored(out.cpu()[~empty], want[~empty], slack[~empty])
    err_lse = (got_lse - want_lse).abs()[~empty]
    assert (err_lse <= slack_lse[~empty]).all(), f"lse: {float((err_lse / slack_lse[~empty]).max())} of the tolerance"
    return out, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (16, 2), (9, 1), (16, 1), (35, 1), (14, 2)])
def test_attention_lengths(heads, kv_heads, D):
    """Lengths of zero, one, ends inside a block, a page, a unit and a step, and one behind; with one workgroup to a segment and with
    shared work (which the bound on the lengths decides)."""
    lengths = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 512]
    case = attention_case(heads + D, lengths, heads, kv_heads, D, 16, 1)
    a = check_attention(*case, 512, pad=8)
    table = torch.nn.functional.pad(case[2], (0, 100), value=-7)
    b = check_attention(case[0], case[1], table, case[3], 2000)
    # the same work in other shares: other orders of fp32 sums
    torch.testing.assert_close(a[1][2:], b[1][2:], rtol=0, atol=1e-5)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 1024])
def test_attention_pages(P):
    """Page sizes, long and ragged contexts, and pages that are not there."""
    check_attention(*attention_case(P, [5000, 1, 2777, 0, 901, 64], 8, 2, 128, P, 1, holes=3), 5000)
    check_attention(*attention_case(P + 1, [3001, 130], 4, 4, 64, P, 1, holes=1), 3001)


@pytest.mark.parametrize("q_len,heads,kv_heads", [(2, 8, 2), (4, 28, 4), (5, 3, 1), (16, 2, 2), (33, 4, 1), (8, 71, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_several_new_tokens(q_len, heads, kv_heads, D):
    """Each new token sees those before it; a sequence may hold fewer tokens than there are new ones."""
    case = attention_case(q_len + D, [q_len, 700, q_len - 1, 90, 1, 0], heads, kv_heads, D, 16, q_len)
    check_attention(*case, 700, q_len)


@pytest.mark.parametrize("window", [1, 15, 16, 17, 100, 128, 1000, 100000])
@pytest.mark.parametrize("q_len", [1, 3])
def test_attention_windows(window, q_len):
    case = attention_case(window, [3, 16, 129, 1500, 0, 2100], 8, 4, 128, 32, q_len)
    check_attention(*case, 2100, q_len, window=window)
    check_attention(*case, 2100, q_len, window=window, softcap=20.0)


def test_attention_with_many_new_tokens_in_a_window():
    """Row tiles with different windows: most units of a segment are outside a tile's."""
    check_attention(*attention_case(9, [900, 640], 4, 2, 64, 16, 300), 900, 300, window=70)


@pytest.mark.parametrize("softcap", [1e-3, 5.0, 50.0, 1e6])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_softcap(softcap, D):
    check_attention(*attention_case(7, [1, 40, 777], 12, 4, D, 16, 1), 777, softcap=softcap)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-6, 3.0])
def test_attention_scales(scale):
    """Score scales of zero, below zero, and so large that one token takes all."""
    check_attention(*attention_case(8, [1, 700, 33], 8, 2, 128, 16, 1), 700, scale=scale)


@pytest.mark.parametrize("size", [1e-12, 1e-4, 1e4, 1e12])
def test_attention_of_small_and_large_values(size):
    """Weights times scales are kept near the middle of fp16 whatever the values' scales are, also where they change on the way."""
    check_attention(*attention_case(11, [900, 64], 8, 2, 128, 16, 1, scale_of_values=size), 900)
    q, cache, table, lengths = attention_case(12, [900, 64], 8, 2, 128, 16, 1)
    _, ranges = ref.cache_views(cache, 128)
    ranges[::3, :, 1] *= size
    check_attention(q, cache, table, lengths, 900)


def test_attention_reference_moves():
    """Scores that grow all along the context, by hundreds: the reference moves on again and again."""
    q, cache, table, lengths = attention_case(13, [2000], 8, 1, 128, 16, 1)
    codes, ranges = ref.cache_views(cache, 128)
    P = 16
    for t in range(0, 2000):
        ranges[int(table[0, t // P]), :, 0, t % P] *= 1 + t / 50
    check_attention(q, cache, table, lengths, 2000)


def test_attention_of_zero_scales():
    """Vectors whose scale is 0 stand for their lower bound, also where a page of zeros is attended to."""
    q, cache, table, lengths = attention_case(14, [300, 40], 8, 2, 128, 16, 1)
    _, ranges = ref.cache_views(cache, 128)
    ranges[:, :, 1, 3::5, 0] = 0
    ranges[:, :, 0, 1::7, 0] = 0
    check_attention(q, cache, table, lengths, 300)
    cache.zero_()
    out, lse = attend(q, cache, table, lengths, 300)
    assert (out == 0).all() and torch.allclose(lse[0], torch.full_like(lse[0], math.log(300)), atol=1e-5)


def test_attention_clamps_lengths():
    """More than max_len counts as max_len, less than nothing as nothing."""
    q, cache, table, lengths = attention_case(15, [600, 600, 600], 8, 2, 64, 16, 1)
    lengths.copy_(torch.tensor([600, 1 << 30, -5]))
    check_attention(q, cache, table, lengths, 400)


def test_attention_nan_stays_in_its_row():
    """A NaN in a query, or in a range that is seen, reaches the rows that read it and no other."""
    q, cache, table, lengths = attention_case(16, [300, 200, 900], 8, 2, 128, 16, 1)
    good, good_lse = attend(q, cache, table, lengths, 900)
    q2 = q.clone()
    q2[1, 3, 7] = float("nan")
    out, lse = attend(q2, cache, table, lengths, 900)
    assert torch.isnan(out[1, 3]).all() and torch.isnan(lse[1, 3])
    rest = torch.ones(3, 8, dtype=torch.bool)
    rest[1, 3] = False
    assert torch.equal(out[rest], good[rest]) and torch.equal(lse[rest], good_lse[rest])
    _, ranges = ref.cache_views(cache, 128)
    ranges[int(table[0, 2]), 1, 1, 5, 1] = float("nan")
    out, _ = attend(q, cache, table, lengths, 900)
    assert torch.isnan(out[0, 4:]).all()
    assert torch.equal(out[0, :4], good[0, :4]) and torch.equal(out[1:], good[1:])


def test_attention_of_infinite_query():
    q, cache, table, lengths = attention_case(17, [40, 30], 4, 2, 64, 16, 1)
    good, _ = attend(q, cache, table, lengths, 40)
    q[0, 1, 0] = float("inf")
    out, _ = attend(q, cache, table, lengths, 40)
    assert torch.equal(out[0, 2:], good[0, 2:]) and torch.equal(out[1], good[1]) and torch.equal(out[0, 0], good[0, 0])


def test_attention_many_sequences():
    """More sequences than a wavefront has lanes, so that the shares are found in several rounds."""
    lengths = [(37 * i) % 257 for i in range(200)]
    check_attention(*attention_case(18, lengths, 4, 2, 64, 16, 1), 272)
    q, cache, table, lens = attention_case(19, lengths, 4, 2, 64, 16, 1)
    table = torch.nn.functional.pad(table, (0, 400), value=-1)
    check_attention(q, cache, table, lens, 5000)


@pytest.mark.parametrize("Bn,heads,kv_heads,D,longest", [(130, 16, 8, 128, 300), (40, 160, 16, 128, 150), (110, 8, 8, 64, 64), (100, 40, 8, 128, 700)])
def test_attention_of_more_segments_than_the_chip_holds(Bn, heads, kv_heads, D, longest):
    """Workgroups that take several short segments, and segments that wait for a place."""
    lengths = [(31 * i) % (longest + 1) for i in range(Bn)]
    check_attention(*attention_case(Bn, lengths, heads, kv_heads, D, 16, 1), longest)


@pytest.mark.parametrize("heads,kv_heads,D", [(4, 4, 64), (4, 4, 128), (12, 1, 64), (12, 1, 128)])
@pytest.mark.parametrize("longest", [513, 900, 1100])
def test_attention_of_few_segments(heads, kv_heads, D, longest):
    """Eight waves to a segment."""
    check_attention(*attention_case(longest + D, [longest, 257, 0, 33], heads, kv_heads, D, 16, 1), longest)
    check_attention(*attention_case(longest + D, [longest, 257, 0, 33], heads, kv_heads, D, 16, 2), longest, 2, softcap=30.0, window=longest // 2)


def test_attention_is_the_same_every_time_and_anywhere():
    """Bits do not depend on the run, on where pages lie, or on the batch's other rows' values."""
    q, cache, table, lengths = attention_case(20, [4000, 77, 1300], 16, 2, 128, 16, 1)
    a = attend(q, cache, table, lengths, 4000)
    for _ in range(3):
        b = attend(q, cache, table, lengths, 4000)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    perm = torch.randperm(cache.shape[0], device=DEV)
    moved = torch.empty_like(cache)
    moved[perm] = cache
    there = table >= 0
    new_table = torch.where(there, perm[table.clamp(min=0).long()].to(torch.int32), table)
    b = attend(q, moved, new_table, lengths, 4000)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_past_four_gigabytes():
    """Pages beyond the 32-bit range of byte offsets, and append to them."""
    P, kv_heads, D = 64, 8, 128
    page_bytes = B.basq_kv_page_bytes(kv_heads, D, P)
    pages = (9 << 30) // page_bytes
    cache = torch.empty((pages, kv_heads, P * (D + 16)), dtype=torch.uint8, device=DEV)
    g = gen(21)
    T = 200
    ids = torch.tensor([pages - 1, pages // 2, 3, pages - 2], dtype=torch.int32, device=DEV)
    cache[ids.long()] = 0xFF
    k, v = randn(g, T, kv_heads, D).to(BF16), randn(g, T, kv_heads, D).to(BF16)
    t = torch.arange(T, device=DEV)
    slots = (ids.long()[t // P] * P + t % P).to(torch.int32)
    B.basq_rope_append(None, k, v, None, None, slots, cache, 0.9, 0.9, None)
    q = randn(g, 1, 16, D).to(BF16)
    lengths = torch.tensor([T], dtype=torch.int32, device=DEV)
    small = cache[ids.long()].clone()
    here = torch.arange(4, dtype=torch.int32, device=DEV)[None]
    want = check_attention(q, small, here, lengths, T)
    for max_len in (T, 256):
        out, lse = attend(q, cache, ids[None].contiguous(), lengths, max_len)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_attention_output_may_be_the_query():
    q, cache, table, lengths = attention_case(22, [700, 50], 8, 2, 128, 16, 1)
    for max_len in (700, 512):
        lengths.clamp_(max=max_len)
        out, _ = attend(q, cache, table, lengths, max_len)
        q2 = q.clone()
        need = B.basq_paged_attention_workspace_bytes(2, 1, 8, 2, 128, max_len)
        ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
        B.basq_paged_attention(q2, cache, table, lengths, max_len, 1 / math.sqrt(128), q2, ws)
        assert torch.equal(q2, out)


def test_on_another_stream_and_in_a_graph():
    """A whole step -- norm, append, attention -- on a side stream, and replayed from a graph between eager work."""
    heads, kv_heads, D, P, Bn = 16, 4, 128, 16, 3
    lengths = [900, 17, 333]
    q0, cache, table, lens = attention_case(23, lengths, heads, kv_heads, D, P, 1)
    g = gen(24)
    x = randn(g, Bn, heads * D).to(BF16)
    w = torch.ones(heads * D, dtype=BF16, device=DEV)
    qkv = randn(g, Bn, heads + 2 * kv_heads, D).to(BF16)
    cos_sin = torch.empty(1000, D, device=DEV)
    B.basq_rope_table(cos_sin, 10000.0)
    positions = lens - 1
    slots = (table.long().gather(1, (positions // P).long()[:, None])[:, 0] * P + positions % P).to(torch.int32)
    need = B.basq_paged_attention_workspace_bytes(Bn, 1, heads, kv_heads, D, 900)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    bufs = [torch.empty_like(x), torch.empty_like(x), torch.empty(Bn, heads, D, dtype=BF16, device=DEV), torch.empty(Bn, heads, D, dtype=BF16, device=DEV)]

    def step():
        B.basq_add_rms_norm(x, x, w, 1e-5, bufs[0], bufs[1])
        B.basq_rope_append(qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], positions, cos_sin, slots, cache, 0.9, 0.9, bufs[2])
        B.basq_paged_attention(bufs[2], cache, table, lens, 900, 1 / math.sqrt(D), bufs[3], ws)

    step()
    torch.cuda.synchronize()
    want = [b.clone() for b in bufs]
    side = torch.cuda.Stream()
    for b in bufs:
        b.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, bufs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for b in bufs:
            b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, bufs))
        step()
        torch.cuda.synchronize()


def test_more_tokens_than_one_grid_dimension_has_threads():
    """2^26 and a few tokens, of which 64 threads each are 2^32: norm and append, the last tokens and those around 2^26."""
    M, K = 2 ** 26 + 3, 8
    picked = torch.tensor([0, 1, 2 ** 20 - 1, 2 ** 20, 2 ** 26 - 1, 2 ** 26, 2 ** 26 + 2], device=DEV)
    x, y = torch.zeros(M, K, dtype=BF16, device=DEV), torch.full((M, K), 9.0, dtype=BF16, device=DEV)
    x[picked] = randn(gen(20), len(picked), K).to(BF16)
    w = torch.ones(K, dtype=BF16, device=DEV)
    B.basq_add_rms_norm(x, None, w, 1e-5, y)
    check_norm(y[picked], ref.add_rms_norm(x[picked], None, w, 1e-5)[1])
    assert int((y != 0).any(1).sum()) == len(picked)
    del x, y
    q = torch.zeros(M, 1, 64, dtype=BF16, device=DEV)
    q[picked] = randn(gen(21), len(picked), 1, 64).to(BF16)
    want = ref.turn(q[picked], None, None, False, True).to(BF16)
    B.basq_rope_append(q, None, None, None, None, None, None, 0.9, 0.9, q)
    assert torch.equal(q[picked].cpu(), want)
    assert int((q.view(torch.int64) != 0).flatten(1).any(1).sum()) == len(picked)


@pytest.mark.parametrize("softcap", [1e-40, 1e-38])
def test_attention_of_the_smallest_caps(softcap):
    """1 / cap is past the end of fp32: all tokens count alike."""
    check_attention(*attention_case(22, [1, 40, 300], 8, 2, 128, 16, 1), 300, softcap=softcap)


def test_norm_in_8_bits_is_a_quotient():
    """y / s rounded to e4m3, code by code: h of 1 and -1 have rstd = 1, so that y is the weight; every 8-bit significand under every largest
    one, among them quotients that lie between two codes, where a product with 1 / s comes out beside them."""
    significands = torch.arange(128, 256).float()
    for top in range(128, 256):
        w = torch.cat([significands * 2.0 ** -k for k in range(9)])
        w = w[w <= top]
        w = torch.cat([w, w.new_zeros(-len(w) % 8)])
        x = torch.ones(2, len(w))
        x[1, ::2] = -1.0
        y8, s8 = torch.empty(2, len(w), dtype=torch.float8_e4m3fn, device=DEV), torch.empty(2, device=DEV)
        B.basq_add_rms_norm(x.to(DEV, BF16), None, w.to(DEV, BF16), 0.0, None, Y8=y8, y8_scale=s8)
        s = torch.tensor(float(top)) / torch.tensor(448.0)
        assert (s8.cpu() == s).all(), top
        want = (x * w / s).clamp(-448, 448).to(torch.float8_e4m3fn)
        assert torch.equal(y8.cpu().float(), want.float()), top


@pytest.mark.parametrize("size", [1e-30, 1e-35, 1e-36, 1e-37])
def test_norm_in_8_bits_of_tiny_rows(size):
    """Scales whose reciprocal is past the end of fp32, down to subnormal ones; some outputs are 0."""
    g = gen(25)
    M, K = 5, 1032
    x = randn(g, M, K).to(BF16)
    x[:, ::7] = 0
    w = (size * (1 + 0.2 * randn(g, K))).to(BF16)
    y8, s8 = torch.empty(M, K, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(M, device=DEV)
    B.basq_add_rms_norm(x, None, w, 1e-5, None, Y8=y8, y8_scale=s8)
    _, want = ref.add_rms_norm(x, None, w, 1e-5)
    # fp32: 2^-16 as in check_norm, and half of the smallest subnormal number for each of three roundings
    slack = want.abs() * 2.0 ** -16 + 2.0 ** -148
    top, s = want.abs().amax(1), ref.f64(s8)
    assert ((s - top / 448).abs() <= top / 448 * 2.0 ** -16 + 2.0 ** -148).all()
    # monotonic roundings: a code lies between those of the ends
    got = ref.f64(y8.float())
    low, high = (((want + d) / s[:, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn).double() for d in (-slack, slack))
    assert ((got >= low) & (got <= high)).all()


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_padding_that_has_no_memory(D):
    """Nothing of a padding token is read or written: rows that lie 128 GB apart, of which only the first is there."""
    heads, kv_heads, P, far = 9, 3, 16, 1 << 36
    x, table, cache, slots, _ = append_case(26, 3, heads, kv_heads, D, P, D)
    q, k, v = (t[:1].contiguous() for t in (x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]))
    cache2 = cache.clone()
    positions = torch.tensor([7, -1, 50], dtype=torch.int32, device=DEV)
    want = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
    B.basq_rope_append(q, k, v, positions[:1], table, slots[:1], cache2, 0.9, 0.8, *want)
    got = [torch.full_like(t, 9.0) for t in want]
    p = lambda t: t.data_ptr()  # noqa: E731
    B._check(B.load().basq_rope_append(p(q), far, p(k), far, p(v), far, 3, heads, kv_heads, D, p(positions), p(table), 50, D, 0, 1, 0.9, 0.8, 4,
                                       p(slots), p(cache), cache.shape[0], P, p(got[0]), far, p(got[1]), p(got[2]), far, B._stream(None)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(cache, cache2)


@pytest.mark.parametrize("D,kv_heads,group", [(64, 16, 1), (128, 8, 9)])
def test_attention_of_one_long_context_among_many_short_ones(D, kv_heads, group):
    lengths = [(29 * i) % 100 for i in range(130)]
    lengths[77] = 9000
    check_attention(*attention_case(27, lengths, kv_heads * group, kv_heads, D, 64, 1), 9000)


@pytest.mark.parametrize("D,heads,kv_heads", [(64, 2, 2), (64, 12, 1), (128, 16, 2), (128, 10, 1)])
@pytest.mark.parametrize("lead", [6.0, 14.0, 17.0, 25.0, 40.0])
def test_attention_of_zero_values_with_the_largest_scores(D, heads, kv_heads, lead):
    """Tokens whose values are all 0 and whose scores are `lead` above the others', as append stores them (a scale of 1, codes of 0): all
    that is in the output comes from the others, by weights of e^-lead, and is to be as exact as without them."""
    T, P = 400, 16
    g = gen(28)
    q = (randn(g, kv_heads, D)[None, :, None] + 0.02 * randn(g, 1, kv_heads, heads // kv_heads, D)).flatten(1, 2).to(BF16)
    k, v = 0.1 * randn(g, T, kv_heads, D), 0.15 * randn(g, T, kv_heads, D)
    base = q.float().unflatten(1, (kv_heads, -1)).mean(2)[0]
    for t in (0, 37, 130, 131, 250, 399):
        k[t] = lead * math.sqrt(D) * base / (base * base).sum(-1, keepdim=True)
        v[t] = 0
    cache = B.alloc_kv_cache(T // P, kv_heads, D, P)
    B.basq_rope_append(None, k.to(BF16), v.to(BF16), None, None, torch.arange(T, dtype=torch.int32, device=DEV), cache, 1.0, 1.0, None, rotate=False)
    table = torch.arange(T // P, dtype=torch.int32, device=DEV)[None]
    for first in (0, 1):                                             # with such a token at the start, and without
        lengths = torch.tensor([T - P * first], dtype=torch.int32, device=DEV)
        check_attention(q, cache, table[:, first:].contiguous(), lengths, T - P * first)
        wide = torch.nn.functional.pad(table[:, first:], (0, 1000), value=-1)
        check_attention(q, cache, wide, lengths, 8000)


def test_attention_of_zero_values_far_from_each_other():
    """Such tokens in every step, above others that become smaller and smaller: the reference stays where the sums are."""
    T, P, D = 1600, 16, 128
    g = gen(29)
    q, k, v = randn(g, 1, 4, D).to(BF16), 0.1 * randn(g, T, 4, D), 0.15 * randn(g, T, 4, D)
    along = q.float()[0] * math.sqrt(D) / q.float()[0].pow(2).sum(-1, keepdim=True)
    k += -0.15 * torch.arange(T, device=DEV)[:, None, None] * along
    k[::32], v[::32] = 20 * along, 0
    cache = B.alloc_kv_cache(T // P, 4, D, P)
    B.basq_rope_append(None, k.to(BF16), v.to(BF16), None, None, torch.arange(T, dtype=torch.int32, device=DEV), cache, 1.0, 1.0, None, rotate=False)
    check_attention(q, cache, torch.arange(T // P, dtype=torch.int32, device=DEV)[None], torch.tensor([T], dtype=torch.int32, device=DEV), T)


@pytest.mark.parametrize("heads,kv_heads,D", [(8, 1, 128), (14, 1, 128), (8, 1, 64), (15, 1, 64)])
def test_attention_of_a_row_does_not_depend_on_other_rows(heads, kv_heads, D):
    """Whatever the other heads' and sequences' queries hold -- huge, tiny, zero or infinite values -- a row's bits stay."""
    q, cache, table, lengths = attention_case(30, [600, 70], heads, kv_heads, D, 16, 1)
    # rows of small values next to far smaller ones, and ordinary rows
    q[:, ::2] = (0.15 * torch.sign(q[:, ::2].float()) * 2.0 ** -torch.randint(0, 24, q[:, ::2].shape, generator=gen(31), device=DEV)).to(BF16)
    good, good_lse = attend(q, cache, table, lengths, 600)
    for value in (1e6, 3e38, 1e-30, 0.0, float("inf")):
        q2 = q.clone()
        q2[0, 3], q2[1, 6] = value, value
        out, lse = attend(q2, cache, table, lengths, 600)
        rest = torch.ones(2, heads, dtype=torch.bool)
        rest[0, 3] = rest[1, 6] = False
        assert torch.equal(out[rest], good[rest]) and torch.equal(lse[rest], good_lse[rest]), value


# ---- attention whose work is shared among workgroups and joined by a second launch

def check_shared(q, cache, table, lengths, max_len, q_len=1, softcap=0.0, window=0, whole=False):
    """check_attention of a call that is seen to share its contexts (or not to): without a workspace it is refused (or not)."""
    table = torch.nn.functional.pad(table, (0, max(0, -(-max_len * (q.shape[2] + 16) // cache.shape[2]) - table.shape[1])), value=-1)
    call = lambda: B.basq_paged_attention(q, cache, table, lengths, max_len, 1.0, torch.empty_like(q), None, q_len=q_len, softcap=softcap, window=window)  # noqa: E731
    if whole:
        call()
    else:
        with pytest.raises(B.BasqError, match="workspace is null"):
            call()
    check_attention(q, cache, table, lengths, max_len, q_len, softcap, window)


@pytest.mark.parametrize("heads,kv_heads,D", [(8, 2, 128), (8, 2, 64), (24, 2, 128), (12, 1, 64)])
@pytest.mark.parametrize("window,q_len,softcap", [(1900, 1, 0.0), (2048, 1, 20.0), (3999, 1, 0.0), (2000, 4, 0.0), (3000, 5, 30.0), (0, 3, 25.0)])
def test_shared_attention_in_windows(heads, kv_heads, D, window, q_len, softcap):
    """Parts that begin where a window does; several new tokens, of one row tile and of several; caps."""
    check_shared(*attention_case(window + q_len + D, [5003, 0, 1, 2999, 130, q_len, 4100], heads, kv_heads, D, 16, q_len), 30000, q_len, softcap, window)


@pytest.mark.parametrize("q_len,heads,kv_heads,D", [(2, 8, 2, 128), (4, 28, 4, 64), (5, 3, 1, 128), (33, 4, 1, 64), (8, 71, 1, 128), (17, 2, 2, 64)])
def test_shared_attention_of_several_new_tokens(q_len, heads, kv_heads, D):
    check_shared(*attention_case(q_len + D, [q_len, 1700, q_len - 1, 90, 1, 0, 300], heads, kv_heads, D, 32, q_len), 9000, q_len)


@pytest.mark.parametrize("D,window", [(64, 70), (128, 600)])
def test_shared_attention_of_row_tiles_with_windows_of_their_own(D, window):
    """Many new tokens: most units of a segment are outside a tile's window, some parts have none of its tokens."""
    check_shared(*attention_case(32, [3500], 2, 1, D, 16, 3000), 4000, 3000, window=window)


@pytest.mark.parametrize("softcap", [1e-3, 5.0, 50.0, 1e6])
@pytest.mark.parametrize("heads,D", [(4, 64), (4, 128), (40, 64), (40, 128)])
def test_shared_attention_softcap(softcap, heads, D):
    check_shared(*attention_case(33, [1, 40, 3777], heads, 4, D, 16, 1), 9000, softcap=softcap)


@pytest.mark.parametrize("scale_of_values", [1e-12, 1e12])
def test_shared_attention_of_small_and_large_values(scale_of_values):
    check_shared(*attention_case(34, [3900, 64], 8, 2, 128, 16, 1, scale_of_values=scale_of_values), 9000)


@pytest.mark.parametrize("heads,kv_heads,D,q_len", [(8, 2, 128, 1), (20, 2, 64, 3)])
def test_shared_attention_in_place_and_in_a_graph(heads, kv_heads, D, q_len):
    """The output in the query's place across both launches, eager, on a side stream, and replayed between eager calls."""
    q, cache, table, lengths = attention_case(35, [9000, 50, 3000], heads, kv_heads, D, 16, q_len)
    need = B.basq_paged_attention_workspace_bytes(3, q_len, heads, kv_heads, D, 9000)
    with pytest.raises(B.BasqError, match="workspace is null"):
        B.basq_paged_attention(q, cache, table, lengths, 9000, 0.1, torch.empty_like(q), None, q_len=q_len)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    want, want_lse = torch.empty_like(q), torch.empty(3 * q_len, heads, device=DEV)
    B.basq_paged_attention(q, cache, table, lengths, 9000, 0.1, want, ws, q_len=q_len, lse=want_lse)
    q2, lse = q.clone(), torch.empty_like(want_lse)

    def step():
        q2.copy_(q)
        B.basq_paged_attention(q2, cache, table, lengths, 9000, 0.1, q2, ws, q_len=q_len, lse=lse)

    same = lambda: torch.equal(q2, want) and torch.equal(lse, want_lse)  # noqa: E731
    step()
    assert same()
    side = torch.cuda.Stream()
    lse.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        lse.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        step()
        torch.cuda.synchronize()
        assert same()


def test_shared_attention_of_parts_of_more_than_32_steps():
    """Workgroups whose share of one context is more than the 32 steps whose pages a wave holds at once: 64 sequences whose tables name the
    same pages, with three queries between them."""
    q, cache, table, _ = attention_case(36, [8192, 1, 1], 8, 8, 64, 64, 1)
    n = [8192, 8191, 5000]
    want, want_lse, slack, slack_lse = ref.paged_attention(q, cache, table[:1].expand(3, -1), torch.tensor(n), 8192, 0.125, 1, 0.0, 0)
    pick = torch.arange(64) % 3
    lengths = torch.tensor(n, dtype=torch.int32)[pick].to(DEV)
    q64, table64 = q[pick.to(DEV)].contiguous(), table[:1].expand(64, -1).contiguous()
    with pytest.raises(B.BasqError, match="workspace is null"):
        B.basq_paged_attention(q64, cache, table64, lengths, 8192, 0.125, torch.empty_like(q64), None)
    # (its shares: all units and two more for each segment, by 768 workgroups)
    units = sum(-(-x // 128) + 2 for x in lengths.tolist()) * 8
    assert units / 768 > 33
    out, lse = attend(q64, cache, table64, lengths, 8192, scale=0.125)
    check_stored(out.cpu(), want[pick], slack[pick])
    assert ((ref.f64(lse) - want_lse[pick]).abs() <= slack_lse[pick]).all()


@pytest.mark.parametrize("D,heads", [(64, 8), (128, 8), (128, 80)])
def test_whole_contexts_of_more_than_32_steps(D, heads):
    """One workgroup to a segment, of up to 64 steps of each wave."""
    lengths = [(29 * i) % 60 for i in range(192)]
    lengths[5], lengths[90], lengths[191] = 8192, 4097, 5000
    check_shared(*attention_case(37, lengths, heads, 8, D, 64, 1), 8192, whole=True)

"""The ends of a step on the GPU, against their definitions (step_ref.py).  Tolerances are stated where they are used, with what they
follow from."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2506_15689_amd import binding as B

import step_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16 = torch.bfloat16
I32 = torch.int32


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def strided(t, pad, fill=7.0):
    """The same values in rows that are `pad` elements further apart."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=torch.float32, device=t.device).to(t.dtype)
    view = wide[:, :t.shape[1]]
    view.copy_(t)
    return view


def check_stored(got, want, slack):
    """Stored values against fp64 ones that the arithmetic in front of the store may miss by `slack`: rounding is monotonic, so what is
    stored lies between the roundings of the ends."""
    low, high, got = (want - slack).to(got.dtype).double(), (want + slack).to(got.dtype).double(), got.cpu().double()
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values; the furthest {float(((got - want).abs() / slack.clamp(min=1e-300))[bad].max())} times the slack away"


# ---- product and lookup ----------------------------------------------------------------------------

def weights(g, N, K, G, exact=False):
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8, device=DEV)
    if exact:
        s = 2.0 ** torch.randint(-2, 3, (N, K // G), generator=g, device=DEV).float()
        z = torch.randint(0, 16, (N, K // G), generator=g, device=DEV).float()
    else:
        s = torch.exp(0.3 * torch.randn((N, K // G), generator=g, device=DEV)) / (3.3 * math.sqrt(K))
        z = 7.5 + 1.2 * torch.randn((N, K // G), generator=g, device=DEV)
    return codes, s.to(BF16), z.to(BF16)


def laid_out(codes, layout):
    if layout == B.BASQ_W_CANONICAL:
        return codes
    N, KB = codes.shape
    out = torch.empty(B.basq_decode_bytes(N, 2 * KB), dtype=torch.uint8, device=DEV)
    B.basq_pack_decode(codes, out)
    return out


CANONICAL, STREAMED = B.BASQ_W_CANONICAL, B.BASQ_W_DECODE16
SHAPES = [(1, 32, 1, 32), (3, 160, 17, 32), (1, 96, 40, 96), (2, 128, 16, 128), (5, 384, 33, 64), (16, 512, 100, 128), (17, 640, 47, 32), (31, 256, 64, 256),
          (33, 1024, 130, 64), (48, 4096, 80, 128), (64, 2048, 31, 2048), (65, 512, 48, 32), (150, 384, 70, 384), (4, 14336, 20, 512), (9, 4128, 19, 4128),
          (7, 960, 600, 320), (1, 8192, 50, 128), (13, 11008, 33, 32), (20, 1152, 1100, 192)]


@pytest.mark.parametrize("M,K,N,G", SHAPES)
@pytest.mark.parametrize("layout", [CANONICAL, STREAMED])
def test_product_of_whole_numbers(M, K, N, G, layout):
    """Scales that are powers of two, whole zero points and whole activations: every product and sum is exact in fp32."""
    if layout == STREAMED and K % 128 != 0:
        pytest.skip("the streaming layout needs K % 128 == 0")
    g = gen(M + K + N)
    codes, s, z = weights(g, N, K, G, exact=True)
    x = torch.randint(-3, 4, (M, K), generator=g, device=DEV).to(BF16)
    bias = torch.randint(-50, 50, (N,), generator=g, device=DEV).float()
    want, made_of = ref.product(x, codes, s, z, bias)
    assert made_of.max() < 2.0 ** 22                              # (quarters, in 24 bits)
    for out_type in (torch.float32, BF16):
        y = strided(torch.zeros(M, N, dtype=out_type, device=DEV), 5)
        B.basq_w4a16_gemm(strided(x, 24), laid_out(codes, layout), s, z, y, bias, w_layout=layout)
        assert torch.equal(y.cpu(), want.to(out_type)), (out_type, (y.cpu().double() - want).abs().max())
        assert M == 1 or (y._base[:, N:] == 7).all(), "the gaps between rows were written"


@pytest.mark.parametrize("M,K,N,G", SHAPES)
@pytest.mark.parametrize("layout", [CANONICAL, STREAMED])
def test_product(M, K, N, G, layout):
    if layout == STREAMED and K % 128 != 0:
        pytest.skip("the streaming layout needs K % 128 == 0")
    g = gen(2 * M + K + N)
    codes, s, z = weights(g, N, K, G)
    x = torch.randn((M, K), generator=g, device=DEV) + 0.3
    x[:, ::37] *= 20
    x = x.to(BF16)
    bias = torch.randn(N, generator=g, device=DEV)
    want, made_of = ref.product(x, codes, s, z, bias)
    # fp32: at most 128 additions one behind the other in a unit, one for each of up to K/32 units, 20 joins, each within 2^-23 of what
    # the sums are made of; their errors have either sign, so that their squares add: the square root of their number, six times
    slack = made_of * 2.0 ** -23 * 6 * math.sqrt(148 + K / 32) / math.sqrt(128)
    for out_type in (torch.float32, BF16):
        y = torch.zeros(M, N, dtype=out_type, device=DEV)
        B.basq_w4a16_gemm(x, laid_out(codes, layout), s, z, y, bias, w_layout=layout)
        check_stored(y, want, slack)
        again = torch.ones_like(y)
        B.basq_w4a16_gemm(x, laid_out(codes, layout), s, z, again, bias, w_layout=layout)
        assert torch.equal(y, again)


def test_product_of_the_quantisers_weights():
    """Groups by the library's own quantiser: N * K / G rows of G channels."""
    N, K, G = 48, 512, 64
    g = gen(3)
    W = (torch.randn((N, K), generator=g, device=DEV) * 0.05).to(BF16)
    codes, s, z, total = B.alloc_weight_buffers(N * K // G, G, DEV)
    B.basq_quantize_weights(W.view(-1, G), codes, s, z, total)
    x = torch.randn((5, K), generator=g, device=DEV).to(BF16)
    y = torch.empty((5, N), device=DEV)
    B.basq_w4a16_gemm(x, codes.view(N, K // 2), s.view(N, -1), z.view(N, -1), y)
    want, _ = ref.product(x, codes.view(N, -1), s.view(N, -1), z.view(N, -1))
    assert (y.cpu().double() - want).abs().max() < 1e-5
    # half a step of the widest group, of some 0.25 / 15, in each of 512 weights: the root of their number, six times
    assert (y.cpu().double() - x.cpu().double() @ W.cpu().double().t()).abs().max() < 6 * math.sqrt(512) * 0.5 * 0.4 / 15


def test_product_with_a_token_that_is_not_finite():
    M, K, N, G = 20, 512, 40, 64
    g = gen(4)
    codes, s, z = weights(g, N, K, G)
    x = torch.randn((M, K), generator=g, device=DEV).to(BF16)
    clean, y = torch.empty((M, N), device=DEV), torch.empty((M, N), device=DEV)
    B.basq_w4a16_gemm(x, codes, s, z, clean)
    x[3, 5], x[17, 100] = math.nan, math.inf
    B.basq_w4a16_gemm(x, codes, s, z, y)
    rest = [m for m in range(M) if m not in (3, 17)]
    assert torch.equal(y[rest], clean[rest]) and not y[[3, 17]].isfinite().any()


@pytest.mark.parametrize("T,K,N,G", [(1, 32, 1, 32), (5, 160, 17, 32), (33, 256, 40, 256), (16, 4096, 100, 64), (300, 1152, 50, 192), (3, 14336, 16, 128)])
@pytest.mark.parametrize("layout", [CANONICAL, STREAMED])
def test_lookup(T, K, N, G, layout):
    if layout == STREAMED and K % 128 != 0:
        pytest.skip("the streaming layout needs K % 128 == 0")
    g = gen(T + K)
    codes, s, z = weights(g, N, K, G)
    ids = torch.randint(0, N, (T,), generator=g, dtype=I32, device=DEV)
    if T > 2:
        ids[1], ids[2] = -1, N
    y = strided(torch.ones(T, K, dtype=BF16, device=DEV), 8)
    B.basq_w4a16_lookup(ids, laid_out(codes, layout), s, z, y, math.sqrt(K), w_layout=layout)
    want = ref.lookup(ids, codes, s, z, math.sqrt(K))
    check_stored(y, want, want.abs() * 2.0 ** -22)                # three roundings in fp32
    assert T == 1 or (y._base[:, K:] == 7).all()


def test_rows_behind_2_to_the_31_bytes():
    """A lookup and a product whose weights lie beyond 32-bit offsets."""
    K, N, G = 8192, 540000, 8192
    codes = torch.zeros((N, K // 2), dtype=torch.uint8, device=DEV)
    codes[-1] = 0x21
    s, z = torch.ones((N, 1), dtype=BF16, device=DEV), torch.zeros((N, 1), dtype=BF16, device=DEV)
    y = torch.empty((1, K), dtype=BF16, device=DEV)
    B.basq_w4a16_lookup(torch.tensor([N - 1], dtype=I32, device=DEV), codes, s, z, y)
    assert torch.equal(y[0, :4].cpu(), torch.tensor([1, 2, 1, 2], dtype=BF16))
    x, out = torch.ones((1, K), dtype=BF16, device=DEV), torch.empty((1, N), device=DEV)
    B.basq_w4a16_gemm(x, codes, s, z, out)
    assert out[0, -1] == 1.5 * K and out[0, :-1].abs().max() == 0


# ---- draw ------------------------------------------------------------------------------------------

def draw(logits, u, **choices):
    """(token, logprob, kept), from a workspace of just the bytes that are asked for"""
    Bn, V = logits.shape
    token, kept, logprob = torch.full((Bn,), 77, dtype=I32, device=DEV), torch.full((Bn,), 77, dtype=I32, device=DEV), torch.full((Bn,), 77.0, device=DEV)
    need = B.basq_sample_workspace_bytes(Bn, V)
    work = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV) if need else None
    as_tensor = lambda v, t: None if v is None else torch.tensor(v, dtype=t, device=DEV)  # noqa: E731
    B.basq_sample(logits, torch.tensor(u, dtype=torch.float64, device=DEV), token, work,
                  temperature=as_tensor(choices.get("temperature"), torch.float32), top_k=as_tensor(choices.get("top_k"), I32),
                  top_p=as_tensor(choices.get("top_p"), torch.float32), min_p=as_tensor(choices.get("min_p"), torch.float32), logprob=logprob, kept=kept)
    return token.tolist(), logprob.tolist(), kept.tolist()


def check_draw(logits, u, **choices):
    tokens, logprobs, kept = draw(logits, u, **choices)
    rows = logits.cpu().double().numpy()
    for b in range(len(u)):
        mine = {k: (float(np.float32(v[b])) if k != "top_k" else v[b]) for k, v in choices.items()}
        token, logprob, n = ref.sample_row(rows[b], u=u[b], **mine)
        assert (tokens[b], kept[b]) == (token, n), (b, mine, u[b], (tokens[b], token), (kept[b], n))
        # one rounding to fp32, and the weights' steps of 2^-42 in the sum
        assert logprobs[b] == logprob or abs(logprobs[b] - logprob) <= abs(logprob) * 2.0 ** -24 + 2.0 ** -30, (b, logprobs[b], logprob)


def bell(g, rows, V, dtype, sd=2.2):
    z = sd * torch.randn((rows, V), generator=g, device=DEV)
    up = torch.randint(0, V, (rows, max(1, min(32, V // 8))), generator=g, device=DEV)
    z.scatter_add_(1, up, 8 * torch.rand(up.shape, generator=g, device=DEV))
    z[:, V // 3:V // 3 + V // 50] = -math.inf
    return z.to(dtype)


ROWS = 12
CHOICES = {
    "free": dict(), "warm": dict(temperature=[1.7] * ROWS), "top_k": dict(top_k=[1, 2, 3, 10, 40, 200, 1000, 5000, 1 << 30, 0, -1, 7]),
    "top_p": dict(top_p=[0.01, 0.1, 0.3, 0.5, 0.7, 0.8, 0.9, 0.95, 0.99, 0.9999, 1.0, 0.0], temperature=[0.8] * ROWS),
    "min_p": dict(min_p=[0.5, 0.1, 0.05, 0.01, 1e-3, 1e-5, 1e-9, 1.0, 2.0, 0.0, -1.0, 0.2], temperature=[1.3] * ROWS),
    "greedy": dict(temperature=[0.0, -1.0, math.nan] * 4),
    "mixed": dict(temperature=[0.0, 0.7, 1.0, 1.3] * 3, top_k=[0, 50, 0, 3, 1000, 0, 20, 0, 7, 100, 0, 2], top_p=[1.0, 0.9, 0.5, 0.99] * 3,
                  min_p=[0.0, 0.0, 0.02, 0.0, 0.1, 0.3] * 2),
}


@pytest.mark.parametrize("choices", CHOICES)
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4099, 32000, 32771, 50257, 128000, 200003])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_draw(choices, V, dtype):
    g = gen(V)
    logits = strided(bell(g, ROWS, V, dtype), 3)
    rng = random.Random(V)
    u = [rng.random() for _ in range(ROWS)]
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -53
    check_draw(logits, u, **CHOICES[choices])


@pytest.mark.parametrize("rows", [1, 2, 3, 8, 33, 130, 300])
@pytest.mark.parametrize("V", [777, 40000, 70001])
def test_draw_of_batches(rows, V):
    g = gen(rows)
    rng = random.Random(rows)
    check_draw(bell(g, rows, V, torch.float32), [rng.random() for _ in range(rows)], temperature=[rng.choice([0.0, 0.6, 1.0]) for _ in range(rows)],
               top_k=[rng.choice([0, 0, 5, 50]) for _ in range(rows)], top_p=[rng.choice([1.0, 0.9, 0.5]) for _ in range(rows)],
               min_p=[rng.choice([0.0, 0.0, 0.05]) for _ in range(rows)])


@pytest.mark.parametrize("V", [5, 1000, 40000, 130000])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_rows_out_of_the_ordinary(V, dtype):
    """Equal logits, two values, no token, one token, infinities, NaN, both zeros, tiny and huge logits, a slope."""
    g = gen(V)
    n = lambda: torch.randn(V, generator=g, device=DEV)  # noqa: E731
    equal, two, none, one, up, nan, zeros, tiny, huge, slope, near, all_up = (torch.full((V,), 1.25, device=DEV) for _ in range(12))
    two[V // 2:] = 2.0
    none[:], one[:] = -math.inf, -math.inf
    one[V - 1] = -3.0
    up[V // 3], up[V // 2] = math.inf, math.inf
    nan[:] = n()
    nan[::2] = math.nan
    zeros[:] = 0.0
    zeros[::2] = -0.0
    tiny[:] = n() * 1e-39
    huge[:] = n() * 1e30
    slope[:] = torch.arange(V, device=DEV) * (20.0 / V)
    near[:] = 5 + 1e-4 * n()
    all_up[:] = math.inf
    logits = torch.stack([equal, two, none, one, up, nan, zeros, tiny, huge, slope, near, all_up]).to(dtype)
    for u in (0.0, 0.37, 0.9999):
        check_draw(logits, [u] * ROWS)
        check_draw(logits, [u] * ROWS, top_p=[0.6] * ROWS, temperature=[0.9] * ROWS)
        check_draw(logits, [u] * ROWS, top_k=[3] * ROWS)
        check_draw(logits, [u] * ROWS, min_p=[0.3] * ROWS, top_k=[V // 2 + 1] * ROWS, top_p=[0.9] * ROWS)


@pytest.mark.parametrize("V", [3001, 90001])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("shape", ["far up", "far down", "flat", "flatter", "masked by a number", "steep", "one above all"])
def test_logits_of_other_shapes(V, dtype, shape):
    """The grid of cells is the temperature's: rows that fill few of its cells, or many, lie anywhere on it or reach below it."""
    g = gen(V)
    z = torch.randn((ROWS, V), generator=g, device=DEV)
    z = {"far up": 2 * z + 300, "far down": 2 * z - 5000, "flat": 0.3 * z, "flatter": 0.003 * z, "steep": 40 * z,
         "masked by a number": torch.where(z > 0, 2 * z, torch.full_like(z, -1e9)), "one above all": z}[shape]
    if shape == "one above all":
        z[:, V // 7] = 25.0
    z = z.to(dtype)
    rng = random.Random(V)
    u = [rng.random() for _ in range(ROWS - 1)] + [1 - 2.0 ** -40]
    heat = [0.05, 0.5, 1.0, 3.0, 10.0, 100.0] * 2
    check_draw(z, u, temperature=heat)
    check_draw(z, u, temperature=heat, top_p=[0.5, 0.9, 0.999, 0.1] * 3)
    check_draw(z, u, temperature=heat, top_k=[1500, 2000, V // 2, V - 1] * 3, top_p=[0.7, 0.99, 1.0] * 4)
    check_draw(z, u, temperature=heat, top_k=[1500, 30, 0] * 4, min_p=[0.05, 1e-4, 1e-10, 1e-14] * 3)
    check_draw(z, u, temperature=heat, top_p=[0.99, 0.6, 1.0] * 4, min_p=[0.2, 1e-3, 1e-13, 0.9] * 3)


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_long_rows(dtype):
    g = gen(9)
    for V in ((1 << 20) - 3, (1 << 20) + 5):
        z = bell(g, 5, V, dtype)
        check_draw(z, [0.1, 0.9, 0.5, 0.99, 0.7], temperature=[1.0, 0.7, 0.0, 1.2, 1.0], top_p=[1.0, 0.9, 1.0, 0.95, 1.0], top_k=[0, 0, 0, 3000, 20],
                   min_p=[0.0, 0.0, 0.0, 0.0, 0.05])


def test_all_tokens_forbidden_but_nan():
    logits = torch.full((3, 500), math.nan, device=DEV)
    logits[1, 7] = -1e30
    assert draw(logits, [0.5] * 3) == ([-1, 7, -1], [-math.inf, 0.0, -math.inf], [0, 1, 0])


def test_numbers_outside_the_unit():
    logits = torch.tensor([[3.0, 1.0, 2.0, 0.0]] * 6, device=DEV)
    tokens, _, _ = draw(logits, [-1.0, math.nan, 0.0, 1.0, 5.0, math.inf])
    assert tokens == [0, 0, 0, 3, 3, 3]


def test_frequencies():
    """65536 evenly spaced numbers: each token as often as its share says, within one at either end."""
    n = 65536
    row = torch.tensor([0.3, -1.0, 2.0, -math.inf, 1.0, 0.3], device=DEV)
    tokens = torch.tensor(draw(row.expand(n, -1), [(i + 0.5) / n for i in range(n)])[0])
    share = torch.softmax(row.double().cpu(), 0) * n
    assert ((torch.bincount(tokens, minlength=6) - share).abs() <= 1.0).all()


def test_cuts_where_masses_are_equal():
    """Four equal logits and p of a half: exactly two are kept; p just above it: three."""
    logits = torch.full((3, 4), 0.7, device=DEV)
    tokens, _, kept = draw(logits, [0.5, 0.0, 0.5], top_p=[0.5, 0.25, 0.5000001])
    assert kept == [2, 1, 3] and tokens == [1, 0, 1]


@pytest.mark.parametrize("V", [2, 3, 500, 5000, 40000])
@pytest.mark.parametrize("heat", [57.0, 100.0, 1e4, 1e30, 3e38, math.inf])
def test_logits_just_below_zero(V, heat):
    """At temperatures of 57 and more the grid of cells is coarser than 1, and a logit's place on it rounds to -0 for the least negative ones:
    they lie beside 0, between tokens on both sides, where top-k cuts and where draws lead."""
    g = gen(V)
    spread = min(4 * heat, 1e38)
    z = (2 * torch.rand((ROWS, V), generator=g, device=DEV) - 1) * spread
    below = torch.tensor([-1e-45, -3e-45, -1e-44, -1e-40, -1e-38, -1e-30, -1e-17, -1e-10, -9e-10, 0.0], device=DEV)
    n = min(V - 1, 10)
    for r in range(ROWS):
        z[r, torch.randperm(V, generator=g, device=DEV)[:n]] = below[r % 3:][:n] if n < 7 else below[:n]
    z[0], z[0, V - 1] = -1.0, -1e-45                              # (alone on top)
    rows = z.cpu()
    assert (rows[0] > -1e-44).sum() == 1
    above = [int((row > 0).sum()) for row in rows]
    rng = random.Random(V)
    for more in (1, 2, n, n + 1):
        k = [a + more for a in above]
        for u in ([rng.random() for _ in range(ROWS)], [1.0] * ROWS, [0.0] * ROWS):
            check_draw(z, u, temperature=[heat] * ROWS, top_k=k)
    for u in ([rng.random() for _ in range(ROWS)], [1.0] * ROWS):
        check_draw(z, u, temperature=[heat] * ROWS)
        check_draw(z, u, temperature=[heat] * ROWS, min_p=[0.5, 0.2, 0.05] * 4, top_p=[1.0, 0.9, 0.6, 0.99] * 3)
    # numbers that lead to each of them
    logits = z[1:2].cpu().double().numpy()[0]
    w = np.sort(np.exp((logits - logits.max()) / float(np.float32(heat))))[::-1]
    running = np.cumsum(w) / w.sum()
    u = [float(running[min(above[1] + i, V - 1)] - w[0] / w.sum() * 1e-3) for i in range(-1, n + 1)]
    check_draw(z[1:2].expand(len(u), -1), [min(max(x, 0.0), 1.0) for x in u], temperature=[heat] * len(u))


def test_logits_that_all_lie_just_below_zero():
    """Two tokens and three, as few as can be: the cell of 0 has them all, by the temperature."""
    for row in ([0.0, -1e-45], [-1e-45, 0.0], [-1e-45, -1e-45], [-5e-10, 0.0], [0.5, 0.25, -1e-10], [-1e-30, -1e-20, -1e-40], [1.0, -1e-45, 2.0, -1.0]):
        logits = torch.tensor([row] * 4, device=DEV)
        for heat in (57.0, 100.0, 1e30, 3e38, math.inf):
            for k in range(len(row) + 1):
                check_draw(logits, [0.0, 0.3, 0.6, 0.99], temperature=[heat] * 4, top_k=[k] * 4)
                check_draw(logits, [0.0, 0.3, 0.6, 0.99], temperature=[heat] * 4, top_k=[k] * 4, top_p=[0.7] * 4, min_p=[0.5] * 4)


@pytest.mark.parametrize("V", [3, 900, 5000, 40000])
@pytest.mark.parametrize("heat", [1e-34, 2.5e-35, 2e-35, 1e-36, 1e-38, 1e-42])
def test_tiny_logits_at_tiny_temperatures(V, heat):
    """Where cells cannot be as narrow as the temperature, and where they just can."""
    g = gen(V)
    top = float(np.float32(heat)) * 30
    z = (bell(g, ROWS, V, torch.float32).clamp(max=9.0).double() * top / 30).float()
    rng = random.Random(V)
    u = [rng.random() for _ in range(ROWS)]
    check_draw(z, u, temperature=[heat] * ROWS)
    check_draw(z, u, temperature=[heat] * ROWS, top_p=[0.9, 0.5, 0.99] * 4, min_p=[0.0, 0.1, 0.01, 1e-4] * 3)
    check_draw(z, u, temperature=[heat] * ROWS, top_k=[1, 2, 10, 100, 1000, V // 2] * 2, top_p=[1.0, 0.8] * 6)


@pytest.mark.parametrize("V,dtype", [(1, torch.float32), (1000, torch.float32), (32768, torch.float32), (1000, BF16), (32769, BF16), (50000, BF16), (150000, BF16), ((1 << 20) + 1, BF16)])
def test_draws_without_a_workspace(V, dtype):
    g = gen(V)
    wide = bell(g, 3, V + 1, dtype)
    for logits in (wide[:, :V], wide[:, 1:]):                     # (a row in pieces, and what is in front of and behind them)
        token = torch.full((3,), 77, dtype=I32, device=DEV)
        B.basq_sample(logits, torch.tensor([0.2, 0.5, 0.9], dtype=torch.float64, device=DEV), token, None)
        assert token.tolist() == [ref.sample_row(row, u=u)[0] for row, u in zip(logits.cpu().double().numpy(), (0.2, 0.5, 0.9))]


def row_that_reaches_p_at_a_cells_end(V, p, tokens=4000):
    """fp32 logits, for a temperature of 1, of which one weighs 1 and `tokens` equal ones, on the grid of 1/32, together about a half, each of them a
    whole number of 2^-bits and 0.35 to 0.5 more; and as much behind them as makes p of all end in those parts."""
    one = np.longdouble(2) ** min(50, 62 - (V - 1).bit_length())
    weight = lambda z: np.exp(np.longdouble(z)) * one  # noqa: E731
    z = next(-k / 32 for k in range(int(32 * math.log(2 * tokens)) - 20, 10000) if 0.35 < float(weight(-k / 32) % 1) < 0.5)
    whole, parts = tokens * np.floor(weight(z)), np.rint(tokens * weight(z))
    rest = (one + (whole + parts) / 2) / np.longdouble(np.float32(p)) - one - parts
    low = z - 40 / 32
    row = [0.0] + [z] * tokens + [low] * int(rest / weight(low))
    assert rest > 0 and len(row) < V - 4
    rest -= np.rint((len(row) - 1 - tokens) * weight(low))
    while rest >= 1:
        last = np.float32(np.log(rest / one))
        last = last if weight(last) <= rest else np.nextafter(last, np.float32(-math.inf))
        assert last < z
        row.append(float(last))
        rest -= np.rint(weight(last))
    return torch.tensor(row + [-math.inf] * (V - len(row)), dtype=torch.float32, device=DEV)


@pytest.mark.parametrize("V", [8200, 40000, 300000, 1 << 20])
def test_top_p_between_a_cells_tokens_and_their_sum(V):
    """The tokens' masses, rounded one by one, come to 1500 steps less than their sum's, and p lies in between."""
    row = row_that_reaches_p_at_a_cells_end(V, 0.9)
    n = 6
    logits = torch.stack([row[torch.randperm(V, generator=gen(i), device=DEV)] for i in range(n)])
    u = [0.0, 0.3, 0.6, 0.8, 0.999, 1.0]
    check_draw(logits, u, top_p=[0.9] * n)
    check_draw(logits, u, top_p=[0.9] * n, min_p=[1e-4, 1e-5, 1e-6, 2.5e-4, 0.5, 2e-5])
    check_draw(logits, u, top_p=[0.9] * n, top_k=[1 << 30, 7000, 5000, 4001, 4000, 2])


# ---- books -----------------------------------------------------------------------------------------

def make_books(rng, rows, columns, P, spare, longest):
    lengths = [rng.randint(0, min(longest, columns * P)) for _ in range(rows)]
    used = sum(-(-n // P) for n in lengths)
    pages = list(range(used + spare))
    rng.shuffle(pages)
    table = [[rng.randint(-5, 1 << 20) for _ in range(columns)] for _ in range(rows)]       # (entries past a length may hold anything)
    for r, n in enumerate(lengths):
        for c in range(-(-n // P)):
            table[r][c] = pages.pop()
    return {"lengths": lengths, "table": table, "free": pages, "columns": columns, "capacity": used + spare}


def on_gpu(books):
    t = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    free = torch.full((books["capacity"],), -9, dtype=I32, device=DEV)
    free[:len(books["free"])] = t(books["free"])
    return dict(lengths=t(books["lengths"]), pool_table=strided(t(books["table"]), 2, -3), free_pages=free, free_count=t([len(books["free"])]))


def copy_of(books):
    return {"lengths": list(books["lengths"]), "table": [list(r) for r in books["table"]], "free": list(books["free"]),
            "columns": books["columns"], "capacity": books["capacity"]}


def check_extend(books, gpu, seqs, new, P, q_len, T, in_place=True):
    """One call on the GPU's books and one on the lists, which are updated where it is in place."""
    Bn, columns = len(seqs), books["columns"]
    t = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    positions, slots, status = torch.full((T,), 55, dtype=I32, device=DEV), torch.full((T,), 55, dtype=I32, device=DEV), t([9, 9])
    starts = torch.full((Bn + 1,), 55, dtype=I32, device=DEV) if not q_len else None
    batch, lengths = strided(torch.full((Bn, columns), -7, dtype=I32, device=DEV), 1, -3), torch.full((Bn,), 55, dtype=I32, device=DEV)
    work = torch.full((B.basq_kv_books_bytes(Bn),), 0xA5, dtype=torch.uint8, device=DEV)
    lists = books if in_place else copy_of(books)
    before = copy_of(lists)
    if not in_place:                                             # (the table and the free pages are, in any case)
        gpu = dict(gpu, pool_table=gpu["pool_table"]._base.clone()[:, :columns], free_pages=gpu["free_pages"].clone())
    out = {} if in_place else dict(lengths_out=gpu["lengths"].clone(), free_out=t([0]))
    B.basq_kv_extend(**gpu, new_tokens=t(new), page_size=P, positions=positions, slots=slots, status=status, books=work, seqs=t(seqs), q_len=q_len,
                     starts=starts, batch_table=batch, batch_lengths=lengths, **out)
    want = ref.extend(lists, list(seqs), list(new), P, q_len, T)
    assert status.tolist() == want["status"]
    assert positions.tolist() == want["positions"] and slots.tolist() == want["slots"] and lengths.tolist() == want["lengths"]
    if starts is not None:
        assert starts.tolist() == want["starts"]
    for b in range(Bn):
        pages = want["batch"][b] if want["batch"] is not None else []
        assert batch[b].tolist() == pages + [-7] * (columns - len(pages))
    assert (batch._base[:, columns:] == -3).all() and (gpu["pool_table"]._base[:, columns:] == -3).all()
    assert gpu["pool_table"].tolist() == lists["table"]
    assert out.get("lengths_out", gpu["lengths"]).tolist() == lists["lengths"]
    count = out.get("free_out", gpu["free_count"]).item()
    assert gpu["free_pages"][:count].tolist() == lists["free"]
    if want["status"] != [0, 0]:
        assert lists == before and gpu["free_pages"][count:].eq(-9).sum() >= 0
    return want


@pytest.mark.parametrize("Bn,P,longest,new,packed", [
    (1, 16, 40, 1, False), (1, 64, 100, 5, True), (3, 16, 33, 4, False), (7, 32, 200, 90, True), (64, 64, 500, 1, False), (64, 16, 100, 8, False),
    (129, 128, 300, 3, False), (40, 16, 64, 700, True), (200, 1024, 3000, 60, True), (512, 16, 50, 2, False), (1024, 16, 40, 3, True), (1, 16, 0, 9000, True),
])
def test_books(Bn, P, longest, new, packed):
    rng = random.Random(Bn * 31 + new)
    rows = Bn + rng.randint(0, 5)
    columns = -(-(longest + 4 * new) // P) + 1
    books = make_books(rng, rows, columns, P, Bn * (-(-4 * new // P) + 1), longest)
    gpu = on_gpu(books)
    for step in range(4):
        seqs = rng.sample(range(rows), Bn)
        counts = [rng.choice([new, rng.randint(0, new), 0, -rng.randint(0, books["lengths"][s])]) for s in seqs]
        T = sum(max(c, 0) for c in counts) + rng.choice([0, 1, 300]) if packed else Bn * new
        want = check_extend(books, gpu, seqs, counts, P, 0 if packed else new, T, in_place=step != 1)
        assert want["status"] == [0, 0]


def test_without_the_optional():
    books = make_books(random.Random(5), 4, 6, 16, 8, 30)
    gpu = on_gpu(books)
    positions, slots, status = (torch.zeros(n, dtype=I32, device=DEV) for n in (6, 6, 2))
    work = torch.empty(256, dtype=torch.uint8, device=DEV)
    seqs = torch.tensor([2, 0, 3], dtype=I32, device=DEV)
    B.basq_kv_extend(**gpu, new_tokens=None, page_size=16, positions=positions, slots=slots, status=status, books=work, seqs=seqs, q_len=2)
    want = ref.extend(books, [2, 0, 3], [2, 2, 2], 16, 2, 6)
    assert positions.tolist() == want["positions"] and slots.tolist() == want["slots"]
    B.basq_kv_extend(**gpu, new_tokens=torch.ones(3, dtype=I32, device=DEV), page_size=16, positions=positions[:3], slots=slots[:3], status=status, books=work)
    want = ref.extend(books, [0, 1, 2], [1, 1, 1], 16, 1, 3)
    assert positions[:3].tolist() == want["positions"] and gpu["lengths"].tolist() == books["lengths"]


@pytest.mark.parametrize("q_len,T", [(4, 12), (0, 12), (0, 5000)])
@pytest.mark.parametrize("fault", ["row", "negative row", "twice", "longer than a row", "shorter than nothing", "pages", "count", "room", "tokens", "length"])
def test_refused_books_stay_as_they_were(fault, q_len, T):
    rng = random.Random(8)
    books = make_books(rng, 5, 8, 16, 3, 60)
    books["lengths"][1], books["lengths"][4] = 40, 17
    seqs, new = [1, 4, 2], [2, 1, 3]
    if fault == "row":
        seqs[1] = 5
    elif fault == "negative row":
        seqs[2] = -1
    elif fault == "twice":
        seqs[2] = 1
    elif fault == "longer than a row":
        books["lengths"][4] = 128
    elif fault == "shorter than nothing":
        new[1] = -18
    elif fault == "pages":
        books["free"] = []
        books["lengths"][1] = 32
    elif fault == "length":
        books["lengths"][4] = -2
    elif fault == "tokens":
        new = [4, 5, 4]
        if T > 13:
            pytest.skip("they fit")
    gpu = on_gpu(books)
    if fault == "count":
        gpu["free_count"].fill_(books["capacity"] + 1)
    elif fault == "room":
        new[0] = -30
        gpu["free_count"].fill_(books["capacity"])
        books["free"] = gpu["free_pages"].tolist()
    want_status = {"row": [1, 1], "negative row": [1, 2], "twice": [1, 2], "longer than a row": [2, 1], "shorter than nothing": [2, 1], "length": [2, 1],
                   "count": [3, books["capacity"] + 1], "room": [3, books["capacity"]]}.get(fault)
    if fault == "tokens" and q_len:
        want_status = [2, 1]
    if fault == "count":
        books["free"] = gpu["free_pages"].tolist() + [-9]
        saved = {k: v.clone() for k, v in gpu.items()}
        Bn = 3
        out = [torch.full((n,), 5, dtype=I32, device=DEV) for n in (T, T, 2)]
        B.basq_kv_extend(**gpu, new_tokens=torch.tensor(new, dtype=I32, device=DEV), page_size=16, positions=out[0], slots=out[1], status=out[2],
                         books=torch.empty(B.basq_kv_books_bytes(Bn), dtype=torch.uint8, device=DEV), seqs=torch.tensor(seqs, dtype=I32, device=DEV), q_len=q_len)
        assert out[2].tolist() == want_status and (out[0] == -1).all() and (out[1] == -1).all()
        assert all(torch.equal(gpu[k], saved[k]) for k in gpu)
        return
    want = check_extend(books, gpu, seqs, new, 16, q_len, T)
    assert want["status"][0] != 0 and (want_status is None or want["status"] == want_status)


def test_no_sequences():
    books = make_books(random.Random(1), 2, 4, 16, 3, 20)
    gpu = on_gpu(books)
    starts, status = torch.full((1,), 5, dtype=I32, device=DEV), torch.full((2,), 5, dtype=I32, device=DEV)
    places = torch.full((2, 7), 5, dtype=I32, device=DEV)
    empty = torch.empty(0, dtype=I32, device=DEV)
    B.basq_kv_extend(**gpu, new_tokens=empty, page_size=16, positions=places[0], slots=places[1], status=status,
                     books=torch.empty(64, dtype=torch.uint8, device=DEV), q_len=0, starts=starts)
    assert (places == -1).all() and starts.tolist() == [0] and status.tolist() == [0, 0] and gpu["free_count"].item() == len(books["free"])


# ---- streams and graphs ----------------------------------------------------------------------------

class Step:
    """A step's ends on state of their own: places, embeddings, logits and tokens; the tokens are the next step's."""

    def __init__(self, seed, Bn=6, K=256, V=1200, P=16, columns=6):
        g = gen(seed)
        self.P, self.V = P, V
        self.lists = make_books(random.Random(seed), Bn + 2, columns, P, 40, 50)
        self.gpu = on_gpu(self.lists)
        self.codes, self.scale, self.zero = weights(g, V, K, 64)
        self.Wq = laid_out(self.codes, STREAMED)
        ints = lambda *n: torch.zeros(n, dtype=I32, device=DEV)  # noqa: E731
        self.seqs = torch.tensor(random.Random(seed).sample(range(Bn + 2), Bn), dtype=I32, device=DEV)
        self.positions, self.slots, self.status, self.lengths, self.table = ints(Bn), ints(Bn), ints(2), ints(Bn), ints(Bn, columns)
        self.token, self.kept, self.logprob = torch.randint(0, V, (Bn,), generator=g, dtype=I32, device=DEV), ints(Bn), torch.zeros(Bn, device=DEV)
        self.x, self.y = torch.empty((Bn, K), dtype=BF16, device=DEV), torch.empty((Bn, V), device=DEV)
        self.u = torch.rand(Bn, generator=g, dtype=torch.float64, device=DEV)
        self.heat, self.top_p = torch.tensor([0.0, 1.0, 0.7] * 2, device=DEV)[:Bn], torch.full((Bn,), 0.9, device=DEV)
        self.books = torch.empty(B.basq_kv_books_bytes(Bn), dtype=torch.uint8, device=DEV)
        need = B.basq_sample_workspace_bytes(Bn, V)
        self.work = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None

    def __call__(self, stream=None):
        B.basq_kv_extend(**self.gpu, new_tokens=None, page_size=self.P, positions=self.positions, slots=self.slots, status=self.status, books=self.books,
                         seqs=self.seqs, batch_table=self.table, batch_lengths=self.lengths, stream=stream)
        B.basq_w4a16_lookup(self.token, self.Wq, self.scale, self.zero, self.x, 16.0, w_layout=STREAMED, stream=stream)
        B.basq_w4a16_gemm(self.x, self.Wq, self.scale, self.zero, self.y, w_layout=STREAMED, stream=stream)
        B.basq_sample(self.y, self.u, self.token, self.work, temperature=self.heat, top_p=self.top_p, logprob=self.logprob, kept=self.kept, stream=stream)

    def check(self, before):
        """What one step made of the tokens `before` it, the books on the lists with it."""
        seqs = self.seqs.tolist()
        want = ref.extend(self.lists, seqs, [1] * len(seqs), self.P, 1, len(seqs))
        assert self.status.tolist() == want["status"] == [0, 0]
        assert self.positions.tolist() == want["positions"] and self.slots.tolist() == want["slots"]
        assert self.gpu["lengths"].tolist() == self.lists["lengths"] and self.gpu["free_count"].item() == len(self.lists["free"])
        x = ref.lookup(before, self.codes, self.scale, self.zero, 16.0)
        check_stored(self.x, x, x.abs() * 2.0 ** -22)
        y, made_of = ref.product(self.x, self.codes, self.scale, self.zero)
        check_stored(self.y, y, made_of * 2.0 ** -20)
        rows, u, heat = self.y.cpu().double().numpy(), self.u.tolist(), self.heat.tolist()
        for b, (token, kept) in enumerate(zip(self.token.tolist(), self.kept.tolist())):
            got = ref.sample_row(rows[b], temperature=heat[b], top_p=float(np.float32(0.9)), u=u[b])
            assert (token, kept) == (got[0], got[2])


def test_a_step_again_and_again():
    step = Step(1)
    for _ in range(20):
        before = step.token.clone()
        step()
        step.check(before)
        step.u.uniform_()


def test_two_captured_steps():
    """Two graphs of steps with state of their own, and eager steps, in turn."""
    one, two, eager = Step(2), Step(3), Step(4)
    for s in (one, two, eager):
        before = s.token.clone()
        s()
        s.check(before)
    graphs = []
    for s in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s()
        graphs.append(graph)
    for i in range(6):
        for s, graph in ((one, graphs[0]), (two, graphs[1]), (eager, None)):
            before = s.token.clone()
            if graph is None:
                s()
            else:
                graph.replay()
            if i % 2:
                torch.cuda.synchronize()
            s.check(before)
            s.u.uniform_()


def test_on_another_stream():
    step = Step(5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    before = step.token.clone()
    torch.cuda.synchronize()
    step(stream)
    stream.synchronize()
    step.check(before)


# ---- calls that documentation allows and that are rarer ---------------------------------------------

@pytest.mark.parametrize("M,K,N,G,layout", [(2, 1 << 20, 17, 128, CANONICAL), (17, 1 << 20, 16, 1 << 19, STREAMED), (1, 1 << 20, 1, 32, CANONICAL), (70, 256, 13000, 64, STREAMED),
                                            (3, 128, 100000, 128, STREAMED), (40, 512, 100000, 128, STREAMED), (1100, 160, 33, 160, CANONICAL)])
def test_products_that_are_long_or_wide(M, K, N, G, layout):
    test_product(M, K, N, G, layout)


WIDE = [(N, K, G, M) for i, N in enumerate([4200, 8300, 12400, 96100]) for j, K in enumerate([512, 1024, 1536, 2560]) for k, G in enumerate([32, 64, 128, 256])
        for M in [[1, 16, 45], [5, 30], [13, 60], [3, 16]][(i + j + k) % 4]]


@pytest.mark.parametrize("N,K,G,M", WIDE)
@pytest.mark.parametrize("layout", [CANONICAL, STREAMED])
def test_wide_products_of_whole_numbers(N, K, G, M, layout):
    """As above, exactly; of matrices of 263 to 6007 tiles, whose rows are looked at in three places."""
    g = gen(N + K + G + M)
    codes, s, z = weights(g, N, K, G, exact=True)
    x = torch.randint(-3, 4, (M, K), generator=g, device=DEV).to(BF16)
    y = torch.full((M, N), math.nan, device=DEV)
    B.basq_w4a16_gemm(x, laid_out(codes, layout), s, z, y, w_layout=layout)
    assert y.isfinite().all()
    rows = torch.cat([torch.arange(130), torch.arange(N // 2, N // 2 + 130), torch.arange(N - 130, N)]).to(DEV)
    want, made_of = ref.product(x, codes[rows], s[rows], z[rows])
    assert made_of.max() < 2.0 ** 22
    assert torch.equal(y[:, rows].cpu(), want.float())


@pytest.mark.parametrize("M,K,layout", [(1, 32, CANONICAL), (17, 32, CANONICAL), (2, 128, STREAMED)])
def test_products_of_more_rows_than_a_launch_has(M, K, layout):
    """2^27 rows and some, which go in parts of 2^26, exactly; looked at beside the parts' ends."""
    N = (1 << 27) + 33
    g = gen(M)
    room = (N + 15) // 16 * 16
    Wq = torch.randint(0, 256, (room * K // 2,), generator=g, dtype=torch.uint8, device=DEV)
    s = torch.randint(-2, 3, (N, 1), generator=g, dtype=torch.int8, device=DEV).to(BF16).exp2()
    z = torch.randint(0, 16, (N, 1), generator=g, dtype=torch.uint8, device=DEV).to(BF16)
    x = torch.randint(-3, 4, (M, K), generator=g, device=DEV).to(BF16)
    bias = torch.randint(-50, 50, (N,), generator=g, dtype=torch.int8, device=DEV).float()
    y = torch.full((M, N), math.nan, device=DEV)
    B.basq_w4a16_gemm(x, Wq if layout == STREAMED else Wq[:N * K // 2], s, z, y, bias, w_layout=layout)
    assert all(row.isfinite().all() for row in y)
    for at in (0, (1 << 26) - 64, (1 << 27) - 64, N - 33):        # 64 rows and more: four blocks, or what is left
        end = min(at + 128, N)
        rows = Wq[at * K // 2:(end + 15) // 16 * 16 * K // 2]
        if layout == STREAMED:
            rows = rows.view(-1, K // 128, 4, 16, 16).permute(0, 3, 1, 2, 4).contiguous()
        codes = rows.reshape(-1, K // 2)[:end - at]
        want, _ = ref.product(x, codes, s[at:end], z[at:end], bias[at:end])
        assert torch.equal(y[:, at:end].cpu(), want.float()), at


def test_lookup_of_many_tokens():
    """More of them than one dimension of a launch has."""
    T, K, N = 70001, 32, 50
    g = gen(11)
    codes, s, z = weights(g, N, K, 32)
    ids = torch.randint(-2, N + 2, (T,), generator=g, dtype=I32, device=DEV)
    y = torch.full((T, K), 7.0, dtype=BF16, device=DEV)
    B.basq_w4a16_lookup(ids, codes, s, z, y, 3.0)
    x = ref.lookup(ids, codes, s, z, 3.0)
    check_stored(y, x, x.abs() * 2.0 ** -22)


def test_draws_in_parts():
    """1100 rows in two slices each: more than the workspace holds at once.  Some rows against the definition, all against calls of few."""
    rows, V = 1100, 40000
    g = gen(12)
    logits = bell(g, rows, V, torch.float32)
    rng = random.Random(12)
    u, heat = [rng.random() for _ in range(rows)], [rng.choice([0.0, 0.7, 1.0, 1.4]) for _ in range(rows)]
    k, p = [rng.choice([0, 0, 5, 300]) for _ in range(rows)], [rng.choice([1.0, 0.9, 0.3]) for _ in range(rows)]
    whole = draw(logits, u, temperature=heat, top_k=k, top_p=p)
    for at in range(0, rows, 220):
        part = slice(at, at + 220)
        some = draw(logits[part], u[part], temperature=heat[part], top_k=k[part], top_p=p[part])
        assert all(a[part] == b for a, b in zip(whole, some))
    pick = [0, 1, 511, 512, 1022, 1023, 1024, 1025, 1099]
    check_draw(logits[pick], [u[i] for i in pick], temperature=[heat[i] for i in pick], top_k=[k[i] for i in pick], top_p=[p[i] for i in pick])


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_draws_of_more_rows_than_a_launch_has(dtype):
    """2^22 and some from one row: 2^32 threads and more, so they go in parts."""
    n = (1 << 22) + 5
    row = torch.tensor([0.5, -1.0, -math.inf, 2.0, 1.0], device=DEV).to(dtype)
    u = torch.arange(n, dtype=torch.float64, device=DEV) / n
    token, kept, logprob = torch.full((n,), 77, dtype=I32, device=DEV), torch.full((n,), 77, dtype=I32, device=DEV), torch.full((n,), 77.0, device=DEV)
    need = B.basq_sample_workspace_bytes(n, 5)
    B.basq_sample(row.expand(n, -1), u, token, torch.empty(need, dtype=torch.uint8, device=DEV) if need else None, kept=kept, logprob=logprob)
    assert (kept == 4).all()
    # the order is that of the logits, so the tokens come in four runs, of their shares
    share = torch.softmax(row.double(), 0)
    order = [3, 4, 0, 1]
    ends = (torch.cumsum(share[order], 0) * n).cpu()
    want = torch.tensor(order, dtype=I32, device=DEV)[torch.searchsorted(ends[:3].to(DEV), torch.arange(n, dtype=torch.float64, device=DEV), right=True)]
    assert (ends[:3] - ends[:3].round()).abs().min() > 1e-6        # (no number lies on an end)
    assert torch.equal(token, want)
    ln = torch.log(share)[token.long()]
    assert ((logprob.double() - ln).abs() <= ln.abs() * 2.0 ** -23).all()


@pytest.mark.parametrize("V", [900, 50000])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_temperatures_at_the_ends(V, dtype):
    heat = [math.inf, 3e38, 1e30, 1e4, 1e-4, 1e-20, 1e-37, 1e-42, -0.0, -math.inf]
    rng = random.Random(13)
    check_draw(bell(gen(13), len(heat), V, dtype), [rng.random() for _ in heat], temperature=heat, top_p=[0.9, 1.0] * 5)


def test_two_captured_draws_share_a_workspace():
    """One behind the other, with different rows, temperatures and numbers of rows."""
    g = gen(14)
    V, calls = 40000, []
    work = torch.full((B.basq_sample_workspace_bytes(5, V),), 0xA5, dtype=torch.uint8, device=DEV)
    for rows, heat in ((5, 0.8), (3, 1.5)):
        c = dict(logits=bell(g, rows, V, torch.float32), u=torch.rand(rows, generator=g, dtype=torch.float64, device=DEV), token=torch.zeros(rows, dtype=I32, device=DEV),
                 heat=torch.full((rows,), heat, device=DEV), top_p=torch.full((rows,), 0.95, device=DEV))
        calls.append(c)

    def run(c):
        B.basq_sample(c["logits"], c["u"], c["token"], work, temperature=c["heat"], top_p=c["top_p"])

    graphs = []
    for c in calls:
        run(c)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(c)
        graphs.append(graph)
    for _ in range(4):
        for c in calls:
            c["u"].uniform_()
            c["logits"][:, ::7] += 0.5                            # (tokens of the step before would be found out)
        graphs[0].replay()
        graphs[1].replay()
        for c in calls:
            rows, u = c["logits"].cpu().double().numpy(), c["u"].tolist()
            want = [ref.sample_row(r, temperature=float(np.float32(h)), top_p=float(np.float32(0.95)), u=x)[0] for r, h, x in zip(rows, c["heat"].tolist(), u)]
            assert c["token"].tolist() == want


@pytest.mark.parametrize("T", [8, 5000])
def test_pages_that_are_none(T):
    """A negative page, in the table or among the free ones: its tokens have places, but no slots."""
    ints = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    table, free = ints([[4, -1, 9], [-2, 0, 0]]), ints([-5, 7])
    lengths, count, status = ints([18, 15]), ints([2]), ints([9, 9])
    positions, slots = torch.full((T,), 55, dtype=I32, device=DEV), torch.full((T,), 55, dtype=I32, device=DEV)
    work = torch.zeros(B.basq_kv_books_bytes(2), dtype=torch.uint8, device=DEV)
    B.basq_kv_extend(lengths, table, free, count, ints([2, 4]), 16, positions, slots, status, work, q_len=0)
    assert status.tolist() == [0, 0] and lengths.tolist() == [20, 19] and count.tolist() == [1]
    assert positions.tolist() == [18, 19, 15, 16, 17, 18] + [-1] * (T - 6)
    assert slots.tolist() == [-1, -1, -1, 112, 113, 114] + [-1] * (T - 6)
    assert table.tolist() == [[4, -1, 9], [-2, 7, 0]]


@pytest.mark.parametrize("Bn,packed", [(3, True), (200, True), (130, False)])
def test_sequences_that_only_lose_tokens(Bn, packed):
    """Every one of them to nothing, and from nothing on again."""
    rng = random.Random(Bn)
    books = make_books(rng, Bn, 6, 16, 2, 90)
    gpu = on_gpu(books)
    seqs = list(range(Bn))
    had = list(books["lengths"])
    check_extend(books, gpu, seqs, [-n for n in had], 16, 0 if packed else 90, 5 if packed else 90 * Bn)
    assert books["lengths"] == [0] * Bn and len(books["free"]) == books["capacity"]
    check_extend(books, gpu, seqs[::-1], had, 16, 0 if packed else 90, sum(had) if packed else 90 * Bn)


@pytest.mark.parametrize("q_len,T", [(40, 160), (0, 40), (0, 5000)])
@pytest.mark.parametrize("why", ["pages", "tokens", "room", "later sequence"])
def test_refused_books_where_pages_would_go_back(q_len, T, why):
    """One sequence gives pages back, another is refused: not a value of the books changes, behind the free pages' count neither."""
    books = make_books(random.Random(3), 4, 8, 16, 4, 100)
    books["lengths"] = [90, 20, 33, 5]
    need = [-(-n // 16) for n in books["lengths"]]
    books["capacity"] = sum(need) + 4
    pages = list(range(100, 100 + books["capacity"]))
    for r, n in enumerate(need):
        books["table"][r][:n] = [pages.pop() for _ in range(n)]
    books["free"] = pages
    seqs, new = [0, 1, 2, 3], [-70, 3, 2, 1]                      # (four pages back)
    if why == "pages":
        new[1:] = [40, 40, 40]                                    # (six wanted)
        books["free"] = []
    elif why == "tokens":
        if q_len or T > 100:
            pytest.skip("they fit")
        new[1:] = [38, 3, 0]
    elif why == "room":
        books["capacity"] = 7
    else:
        seqs[3] = 4
    gpu = on_gpu(books)
    before = {k: v.clone() for k, v in gpu.items()}
    want = check_extend(books, gpu, seqs, new, 16, q_len, T)
    assert want["status"][0] == {"pages": 4, "tokens": 5, "room": 3, "later sequence": 1}[why]
    assert all(torch.equal(gpu[k], before[k]) for k in gpu)


@pytest.mark.parametrize("heads,kv_heads,D,P", [(4, 2, 64, 16), (8, 1, 128, 32)])
def test_attention_on_these_books(heads, kv_heads, D, P):
    """Places for tokens, their keys and values into the cache, attention over it: packed prompts, then captured steps of up to three tokens of
    each sequence, some of which lose tokens.  The same tokens on a cache where every sequence has pages of its own side by side give the same."""
    rng, g = random.Random(D), gen(D)
    Bn, rows, columns, q_len = 3, 5, 12, 3
    books = make_books(rng, rows, columns, P, 40, 0)
    gpu = on_gpu(books)
    seqs = rng.sample(range(rows), Bn)
    ints = lambda *n: torch.zeros(n, dtype=I32, device=DEV)  # noqa: E731
    t = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    which, status, table, lengths = t(seqs), ints(2), torch.full((Bn, columns), -1, dtype=I32, device=DEV), ints(Bn)
    work = torch.empty(B.basq_kv_books_bytes(Bn), dtype=torch.uint8, device=DEV)
    cos_sin = torch.empty((columns * P, D), device=DEV)
    B.basq_rope_table(cos_sin, 10000.0)
    cache, own = (B.alloc_kv_cache(n, kv_heads, D, P, DEV) for n in (books["capacity"], rows * columns))
    at_home = torch.arange(rows * columns, dtype=I32, device=DEV).view(rows, columns)[which.long()]
    room = B.basq_paged_attention_workspace_bytes(Bn, q_len, heads, kv_heads, D, columns * P)
    parts = torch.empty(room, dtype=torch.uint8, device=DEV) if room else None
    randn = lambda *n: torch.randn(n, generator=g, device=DEV).to(BF16)  # noqa: E731

    def append(x, positions, slots, cache):
        q = x[:, :heads].clone()
        B.basq_rope_append(q, x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], positions, cos_sin, slots, cache, 0.9, 0.9, q)
        return q

    def attend(q, cache, table, lengths):
        out = torch.empty_like(q)
        B.basq_paged_attention(q, cache, table, lengths, columns * P, 1 / math.sqrt(D), out, parts, q_len=q_len)
        return out

    def places_at_home(have, new, T):
        """Positions and slots of a sequence's own pages."""
        positions, slots = [], []
        for s, n, m in zip(seqs, have, new):
            run = [(p, s * columns * P + p) for p in range(n, n + m)]
            run = [(-1, -1)] * (0 if T else q_len - len(run)) + run
            positions += [p for p, _ in run]
            slots += [at for _, at in run]
        rest = [-1] * (T - len(positions))
        return t(positions + rest), t(slots + rest)

    # prompts, packed, with room to spare
    have, new = [0] * Bn, [5 * P + 3, 1, 2 * P]
    T = sum(new) + 7
    positions, slots = ints(T), ints(T)
    B.basq_kv_extend(**gpu, new_tokens=t(new), page_size=P, positions=positions, slots=slots, status=status, books=work, seqs=which, q_len=0,
                     batch_table=table, batch_lengths=lengths)
    x = randn(T, heads + 2 * kv_heads, D)
    here, there = append(x, positions, slots, cache), append(x, *places_at_home(have, new, T), own)
    assert status.tolist() == [0, 0] and torch.equal(here[:sum(new)], there[:sum(new)])
    have = [n + m for n, m in zip(have, new)]

    # steps; the captured one reads its tokens and their numbers from the same places each time
    counts, x = ints(Bn), randn(Bn * q_len, heads + 2 * kv_heads, D)
    positions, slots, out = ints(Bn * q_len), ints(Bn * q_len), torch.empty((Bn * q_len, heads, D), dtype=BF16, device=DEV)

    def step():
        B.basq_kv_extend(**gpu, new_tokens=counts, page_size=P, positions=positions, slots=slots, status=status, books=work, seqs=which, q_len=q_len,
                         batch_table=table, batch_lengths=lengths)
        out.copy_(attend(append(x, positions, slots, cache), cache, table, lengths))

    graph = None
    for i, new in enumerate([[3, 3, 3], [1, 2, 3], [-2 * P, 3, -5], [3, -1, 0], [2, 3, 3], [-3, 1, 3], [3, 3, 1], [0, 0, 2]]):
        counts.copy_(t(new))
        x.copy_(randn(*x.shape))
        if i == 1:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is None:
            step()
        else:
            graph.replay()
        q = append(x, *places_at_home(have, [max(n, 0) for n in new], 0), own)
        have = [n + m for n, m in zip(have, new)]
        want = attend(q, own, at_home, t(have))
        assert status.tolist() == [0, 0] and lengths.tolist() == have, i
        assert torch.equal(out, want) and out.isfinite().all() and out.abs().max() > 0, i
    assert gpu["free_count"].item() == books["capacity"] - sum(-(-n // P) for n in have)

"""The ends of a step without a GPU: what they refuse, before anything would be launched."""
import ctypes
import os

import pytest
import torch

from paper_2506_15689_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1008)
OFF = ctypes.c_void_p(0x1002)
BYTE = ctypes.c_void_p(0x1001)
BF16 = torch.bfloat16
I32 = torch.int32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2506_15689_amd import build
        build.build_lib(verbose=False)
    return B.load()


def product(lib, **kw):
    a = dict(X=FAKE, M=4, K=256, ldx=256, Wq=FAKE, N=48, w_layout=0, w_scale=FAKE, w_zero=FAKE, group_size=64, bias=None, Y=FAKE, ldy=48, y_f32=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_w4a16_gemm(*a.values(), None)


MATRIX = [
    (dict(N=0), B.BASQ_EINVAL), (dict(K=0), B.BASQ_EINVAL), (dict(K=48), B.BASQ_EINVAL), (dict(K=(1 << 20) + 32), B.BASQ_EUNSUPPORTED),
    (dict(w_layout=2), B.BASQ_EINVAL), (dict(w_layout=1, K=160, group_size=32), B.BASQ_EINVAL), (dict(group_size=16), B.BASQ_EINVAL),
    (dict(group_size=48), B.BASQ_EINVAL), (dict(group_size=96), B.BASQ_EINVAL), (dict(group_size=-32), B.BASQ_EINVAL), (dict(Wq=None), B.BASQ_EINVAL),
    (dict(Wq=ODD), B.BASQ_EINVAL), (dict(w_scale=None), B.BASQ_EINVAL), (dict(w_zero=None), B.BASQ_EINVAL), (dict(w_scale=BYTE), B.BASQ_EINVAL),
    (dict(w_zero=BYTE), B.BASQ_EINVAL), (dict(Y=None), B.BASQ_EINVAL), (dict(N=(1 << 28) + 1), B.BASQ_EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", MATRIX + [
    (dict(M=-1), B.BASQ_EINVAL), (dict(M=16 * 65535 + 1), B.BASQ_EUNSUPPORTED), (dict(X=None), B.BASQ_EINVAL), (dict(X=ODD), B.BASQ_EINVAL),
    (dict(ldx=248), B.BASQ_EINVAL), (dict(ldx=260), B.BASQ_EINVAL), (dict(ldx=(1 << 23) + 8), B.BASQ_EUNSUPPORTED), (dict(bias=OFF), B.BASQ_EINVAL), (dict(Y=BYTE), B.BASQ_EINVAL),
    (dict(Y=OFF, y_f32=1), B.BASQ_EINVAL), (dict(ldy=47), B.BASQ_EINVAL),
])
def test_product_refuses(lib, kw, code):
    assert product(lib, **kw) == code and B.basq_last_error()


def lookup(lib, **kw):
    a = dict(ids=FAKE, T=4, Wq=FAKE, N=48, K=256, w_layout=0, w_scale=FAKE, w_zero=FAKE, group_size=64, scale=2.0, Y=FAKE, ldy=256)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_w4a16_lookup(*a.values(), None)


@pytest.mark.parametrize("kw,code", MATRIX + [
    (dict(T=-1), B.BASQ_EINVAL), (dict(T=1 << 31), B.BASQ_EINVAL), (dict(T=(1 << 30) + 1), B.BASQ_EUNSUPPORTED), (dict(ids=None), B.BASQ_EINVAL), (dict(ids=OFF), B.BASQ_EINVAL),
    (dict(Y=ODD), B.BASQ_EINVAL), (dict(ldy=248), B.BASQ_EINVAL), (dict(ldy=260), B.BASQ_EINVAL), (dict(scale=float("inf")), B.BASQ_EINVAL),
])
def test_lookup_refuses(lib, kw, code):
    assert lookup(lib, **kw) == code and B.basq_last_error()


def sample(lib, **kw):
    a = dict(logits=FAKE, ldl=1000, B=2, V=1000, f32=1, temperature=FAKE, top_k=FAKE, top_p=FAKE, min_p=FAKE, u=FAKE, token=FAKE, logprob=FAKE,
             kept=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_sample(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), B.BASQ_EINVAL), (dict(V=0), B.BASQ_EINVAL), (dict(V=(1 << 22) + 1, ldl=1 << 23), B.BASQ_EUNSUPPORTED), (dict(logits=None), B.BASQ_EINVAL),
    (dict(logits=OFF), B.BASQ_EINVAL), (dict(logits=BYTE, f32=0), B.BASQ_EINVAL), (dict(ldl=999), B.BASQ_EINVAL), (dict(temperature=OFF), B.BASQ_EINVAL),
    (dict(top_k=OFF), B.BASQ_EINVAL), (dict(top_p=OFF), B.BASQ_EINVAL), (dict(min_p=OFF), B.BASQ_EINVAL), (dict(u=None), B.BASQ_EINVAL),
    (dict(u=ctypes.c_void_p(0x1004)), B.BASQ_EINVAL), (dict(token=None), B.BASQ_EINVAL), (dict(token=OFF), B.BASQ_EINVAL), (dict(logprob=OFF), B.BASQ_EINVAL),
    (dict(kept=OFF), B.BASQ_EINVAL),
])
def test_sample_refuses(lib, kw, code):
    assert sample(lib, **kw) == code and B.basq_last_error()


def test_sample_workspace(lib):
    for shape in ((0, 1000), (-1, 1000), (4, 0), (4, (1 << 22) + 1)):
        assert B.basq_sample_workspace_bytes(*shape) == 0
    sizes = {(b, v): B.basq_sample_workspace_bytes(b, v) for b in (1, 2, 7, 64, 256, 300, 5000) for v in (1, 1000, 32000, 32769, 128000, 1 << 22)}
    for (b, v), n in sizes.items():
        for (b2, v2), n2 in sizes.items():
            assert not (b2 <= b and v2 <= v) or n2 <= n, "a workspace does for smaller calls"
        if n > 0:
            assert sample(lib, B=b, V=v, ldl=v, workspace=None) == B.BASQ_EINVAL
            assert sample(lib, B=b, V=v, ldl=v, workspace=ctypes.c_void_p(0x1010)) == B.BASQ_EINVAL
            assert sample(lib, B=b, V=v, ldl=v, workspace_bytes=n - 1) == B.BASQ_EWORKSPACE


def test_rows_that_a_workgroup_holds_need_no_workspace(lib):
    for b in (1, 64, 5000, 1 << 22):
        assert [B.basq_sample_workspace_bytes(b, v) for v in (1, 1000, 32768)] == [0] * 3
        assert B.basq_sample_workspace_bytes(b, 32769) > 0


def extend(lib, **kw):
    a = dict(lengths=FAKE, pool_table=FAKE, pool_stride=8, rows=6, columns=8, page_size=16, free_pages=FAKE, capacity=48, free_count=FAKE, seqs=FAKE,
             new_tokens=FAKE, B=3, q_len=2, positions=FAKE, slots=FAKE, T=6, starts=None, batch_table=FAKE, batch_stride=8, batch_lengths=FAKE,
             lengths_out=FAKE, free_out=FAKE, status=FAKE, books=FAKE, books_bytes=1 << 20)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_kv_extend(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), B.BASQ_EINVAL), (dict(q_len=-1), B.BASQ_EINVAL), (dict(rows=-1), B.BASQ_EINVAL), (dict(columns=-1), B.BASQ_EINVAL),
    (dict(capacity=-1), B.BASQ_EINVAL), (dict(page_size=8), B.BASQ_EUNSUPPORTED), (dict(page_size=48), B.BASQ_EUNSUPPORTED),
    (dict(page_size=2048), B.BASQ_EUNSUPPORTED), (dict(B=1025, T=2050), B.BASQ_EUNSUPPORTED),
    (dict(columns=1 << 30, pool_stride=1 << 30), B.BASQ_EUNSUPPORTED), (dict(columns=1 << 27, pool_stride=1 << 27), B.BASQ_EUNSUPPORTED),
    (dict(T=-1, q_len=0), B.BASQ_EINVAL), (dict(T=5), B.BASQ_EINVAL), (dict(starts=FAKE), B.BASQ_EINVAL), (dict(q_len=0, new_tokens=None), B.BASQ_EINVAL),
    (dict(seqs=None, rows=2), B.BASQ_EINVAL), (dict(pool_stride=7), B.BASQ_EINVAL), (dict(batch_stride=7), B.BASQ_EINVAL), (dict(books=None), B.BASQ_EINVAL),
    (dict(books=ODD), B.BASQ_EINVAL), (dict(books_bytes=64 + 32 * 3 - 1), B.BASQ_EWORKSPACE),
] + [({name: bad}, B.BASQ_EINVAL) for name in ("lengths", "pool_table", "free_pages", "free_count", "positions", "slots", "lengths_out", "free_out", "status")
     for bad in (None, OFF)] + [({name: OFF}, B.BASQ_EINVAL) for name in ("seqs", "new_tokens", "batch_table", "batch_lengths")]
    + [(dict(starts=OFF, q_len=0), B.BASQ_EINVAL)])
def test_extend_refuses(lib, kw, code):
    assert extend(lib, **kw) == code and B.basq_last_error()


def test_empty_calls_do_nothing(lib):
    assert product(lib, M=0, X=None, Y=None) == B.BASQ_OK
    assert lookup(lib, T=0, ids=None, Y=None) == B.BASQ_OK
    assert sample(lib, B=0, logits=None, u=None, token=None, workspace=None) == B.BASQ_OK
    assert B.basq_kv_books_bytes(3) == 64 + 96 and B.basq_kv_books_bytes(1025) == B.basq_kv_books_bytes(-1) == 0


# ---- the binding: shapes, types, places ------------------------------------------------------------

def zeros(*shape, dtype=I32):
    return torch.zeros(shape, dtype=dtype)


def test_binding_of_the_product():
    x, Wq, s, z, y = zeros(4, 256, dtype=BF16), zeros(48, 128, dtype=torch.uint8), zeros(48, 4, dtype=BF16), zeros(48, 4, dtype=BF16), zeros(4, 48, dtype=BF16)
    for args, what in (((x.float(), Wq, s, z, y), "x must be"), ((x[0], Wq, s, z, y), "x must be"), ((x[:, ::2], Wq, s, z, y), "side by side"),
                       ((x, Wq[1:], s, z, y), "Wq must be"), ((x, Wq, s.float(), z, y), "w_scale must be"), ((x, Wq, s, z[:, :2], y), "w_zero must be"),
                       ((x, Wq, s[:, :3].contiguous(), z, y), "w_zero must be"), ((x, Wq, zeros(48, 5, dtype=BF16), zeros(48, 5, dtype=BF16), y), "not 5 groups"),
                       ((x, Wq, s, z, y.half()), "y must be"), ((x, Wq, s, z, y[:3]), "y must be"), ((x, Wq, s, z, y, zeros(48)), "bias must be"),
                       ((x, Wq, s, z, None), "y must be given"), ((x, Wq, s, z, y), "not on the GPU")):
        with pytest.raises(ValueError, match=what):
            B.basq_w4a16_gemm(*args)
    with pytest.raises(ValueError, match="Wq must be"):
        B.basq_w4a16_gemm(x, zeros(47, 128, dtype=torch.uint8), zeros(47, 4, dtype=BF16), zeros(47, 4, dtype=BF16), zeros(4, 47, dtype=BF16),
                          w_layout=B.BASQ_W_DECODE16)


def test_binding_of_the_lookup():
    ids, Wq, s, z, y = zeros(4), zeros(48, 128, dtype=torch.uint8), zeros(48, 4, dtype=BF16), zeros(48, 4, dtype=BF16), zeros(4, 256, dtype=BF16)
    for args, what in (((ids.long(), Wq, s, z, y), "ids must be"), ((ids[:3], Wq, s, z, y), "ids must be"), ((ids, Wq, s, z, y.float()), "y must be"),
                       ((ids, Wq, s, z, y[:, :128].contiguous()), "Wq must be"), ((ids, Wq, s, z, y), "not on the GPU")):
        with pytest.raises(ValueError, match=what):
            B.basq_w4a16_lookup(*args)


def test_binding_of_the_draw():
    logits, u, token = zeros(3, 50, dtype=torch.float32), zeros(3, dtype=torch.float64), zeros(3)
    w = zeros(64, dtype=torch.uint8)
    for args, kw, what in (((logits.half(), u, token, w), {}, "logits must be"), ((logits[0], u, token, w), {}, "logits must be"),
                           ((logits, u.float(), token, w), {}, "u must be"), ((logits, u, token.long(), w), {}, "token must be"),
                           ((logits, u, token, w), dict(temperature=u), "temperature must be"), ((logits, u, token, w), dict(top_k=u), "top_k must be"),
                           ((logits, u, token, w), dict(top_p=token), "top_p must be"), ((logits, u, token, w), dict(min_p=token), "min_p must be"),
                           ((logits, u, token, w), dict(logprob=token), "logprob must be"), ((logits, u, token, w), dict(kept=u), "kept must be"),
                           ((logits, u, token, w), {}, "not on the GPU")):
        with pytest.raises(ValueError, match=what):
            B.basq_sample(*args, **kw)


def test_binding_of_the_books():
    a = dict(lengths=zeros(6), pool_table=zeros(6, 8), free_pages=zeros(48), free_count=zeros(1), new_tokens=zeros(3), page_size=16, positions=zeros(3),
             slots=zeros(3), status=zeros(2), books=zeros(1024, dtype=torch.uint8))
    opt = dict(seqs=zeros(3), batch_table=zeros(3, 8), batch_lengths=zeros(3))
    for kw, what in ((dict(lengths=zeros(5)), "lengths must be"), (dict(pool_table=zeros(48)), "pool_table must be"), (dict(free_pages=zeros(48).long()), "free_pages must be"),
                     (dict(free_count=zeros(2)), "free_count must be"), (dict(new_tokens=zeros(4)), "new_tokens must be"), (dict(slots=zeros(4)), "slots must be"),
                     (dict(status=zeros(1)), "status must be"), (dict(seqs=zeros(3).long()), "seqs must be"), (dict(batch_table=zeros(3, 7)), "batch_table must be"),
                     (dict(batch_lengths=zeros(4)), "batch_lengths must be"), (dict(starts=zeros(3), q_len=0), "starts must be"), (dict(lengths_out=zeros(5)), "lengths_out must be"),
                     (dict(free_out=zeros(2)), "free_out must be"), (dict(seqs=None, new_tokens=None), "seqs or new_tokens"), ({}, "not on the GPU")):
        all_ = {**a, **opt, **kw}
        with pytest.raises(ValueError, match=what):
            B.basq_kv_extend(**all_)

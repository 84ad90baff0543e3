"""The operators around the linear layer without a GPU: what they refuse, before anything would be launched."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2506_15689_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1008)
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2506_15689_amd import build
        build.build_lib(verbose=False)
    return B.load()


def norm(lib, **kw):
    a = dict(X=FAKE, residual=FAKE, weight=FAKE, M=4, K=64, ldx=64, ldr=64, eps=1e-5, res_out=FAKE, ldro=64, Y=FAKE, ldy=64, Y8=None,
             ldy8=0, y8_scale=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_add_rms_norm(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), B.BASQ_EINVAL), (dict(M=1 << 31), B.BASQ_EINVAL), (dict(K=0), B.BASQ_EINVAL), (dict(K=60), B.BASQ_EINVAL),
    (dict(K=32776, ldx=32776), B.BASQ_EUNSUPPORTED), (dict(eps=-1.0), B.BASQ_EINVAL), (dict(eps=float("nan")), B.BASQ_EINVAL),
    (dict(X=None), B.BASQ_EINVAL), (dict(X=ODD), B.BASQ_EINVAL), (dict(ldx=56), B.BASQ_EINVAL), (dict(ldx=68), B.BASQ_EINVAL),
    (dict(residual=ODD), B.BASQ_EINVAL), (dict(ldr=60), B.BASQ_EINVAL), (dict(weight=None), B.BASQ_EINVAL),
    (dict(res_out=ODD), B.BASQ_EINVAL), (dict(ldro=0), B.BASQ_EINVAL), (dict(Y=None), B.BASQ_EINVAL), (dict(Y=ODD), B.BASQ_EINVAL),
    (dict(ldy=63), B.BASQ_EINVAL), (dict(Y8=FAKE, ldy8=64), B.BASQ_EINVAL), (dict(Y8=FAKE, ldy8=60, y8_scale=FAKE), B.BASQ_EINVAL),
    (dict(Y8=ctypes.c_void_p(0x1004), ldy8=64, y8_scale=FAKE), B.BASQ_EINVAL),
    (dict(Y8=FAKE, ldy8=64, y8_scale=ctypes.c_void_p(0x1002)), B.BASQ_EINVAL),
])
def test_norm_refuses(lib, kw, code):
    assert norm(lib, **kw) == code and B.basq_last_error()


def test_empty_calls_do_nothing(lib):
    assert norm(lib, M=0, X=None, Y=None) == B.BASQ_OK
    assert append(lib, T=0, q=None, k=None, v=None, q_out=None, positions=None, slots=None) == B.BASQ_OK
    assert attention(lib, B=0, q=None, out=None, page_table=None, lengths=None) == B.BASQ_OK
    assert lib.basq_rope_table(64, 0, 10000.0, 0, 1.0, 1.0, 2.0, 1.0, None, None) == B.BASQ_OK


def append(lib, **kw):
    a = dict(q=FAKE, ldq=512, k=FAKE, ldk=256, v=FAKE, ldv=256, T=4, heads=4, kv_heads=2, head_dim=128, positions=FAKE, cos_sin=FAKE,
             table_rows=16, rot_dim=128, interleaved=0, rotate=1, clip_lo=0.9, clip_hi=0.9, bits=4, slots=FAKE, cache=FAKE, num_pages=4,
             page_size=16, q_out=FAKE, ldqo=512, k_hat=None, v_hat=None, ldh=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_rope_append(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), B.BASQ_EINVAL), (dict(head_dim=96), B.BASQ_EUNSUPPORTED), (dict(heads=-1), B.BASQ_EINVAL),
    (dict(heads=0, kv_heads=0), B.BASQ_EINVAL), (dict(bits=8), B.BASQ_EUNSUPPORTED), (dict(q=None), B.BASQ_EINVAL),
    (dict(q=ODD), B.BASQ_EINVAL), (dict(ldq=504), B.BASQ_EINVAL), (dict(ldq=516), B.BASQ_EINVAL), (dict(k=None), B.BASQ_EINVAL),
    (dict(v=None), B.BASQ_EINVAL), (dict(ldv=128), B.BASQ_EINVAL), (dict(q_out=None), B.BASQ_EINVAL), (dict(ldqo=0), B.BASQ_EINVAL),
    (dict(positions=None), B.BASQ_EINVAL), (dict(slots=None), B.BASQ_EINVAL), (dict(cos_sin=ODD), B.BASQ_EINVAL),
    (dict(table_rows=0), B.BASQ_EINVAL), (dict(rot_dim=0), B.BASQ_EUNSUPPORTED), (dict(rot_dim=24), B.BASQ_EUNSUPPORTED),
    (dict(rot_dim=144), B.BASQ_EUNSUPPORTED), (dict(clip_lo=0.0), B.BASQ_EINVAL), (dict(clip_hi=1.5), B.BASQ_EINVAL),
    (dict(cache=None), B.BASQ_EINVAL), (dict(cache=ODD), B.BASQ_EINVAL), (dict(num_pages=0), B.BASQ_EINVAL),
    (dict(num_pages=1 << 27), B.BASQ_EINVAL), (dict(page_size=8), B.BASQ_EUNSUPPORTED), (dict(page_size=48), B.BASQ_EUNSUPPORTED),
    (dict(page_size=2048), B.BASQ_EUNSUPPORTED), (dict(k_hat=FAKE, ldh=128), B.BASQ_EINVAL), (dict(v_hat=ODD, ldh=256), B.BASQ_EINVAL),
    (dict(positions=ctypes.c_void_p(0x1002)), B.BASQ_EINVAL),
])
def test_append_refuses(lib, kw, code):
    assert append(lib, **kw) == code and B.basq_last_error()


@pytest.mark.parametrize("args", [
    (0, 4, 1e4, 0, 1.0, 1.0, 2.0, 1.0), (63, 4, 1e4, 0, 1.0, 1.0, 2.0, 1.0), (64, -1, 1e4, 0, 1.0, 1.0, 2.0, 1.0),
    (64, 4, 1.0, 0, 1.0, 1.0, 2.0, 1.0), (64, 4, 1e4, 1, 0.0, 1.0, 2.0, 1.0), (64, 4, 1e4, 2, 8.0, 4.0, 1.0, 8192.0),
    (64, 4, 1e4, 3, 8.0, 1.0, 32.0, 0.0), (64, 4, float("inf"), 0, 1.0, 1.0, 2.0, 1.0),
])
def test_table_refuses(lib, args):
    assert lib.basq_rope_table(*args, FAKE, None) == B.BASQ_EINVAL
    assert lib.basq_rope_table(64, 4, 1e4, 4, 1.0, 1.0, 2.0, 1.0, FAKE, None) == B.BASQ_EUNSUPPORTED
    assert lib.basq_rope_table(64, 4, 1e4, 0, 1.0, 1.0, 2.0, 1.0, None, None) == B.BASQ_EINVAL


def attention(lib, **kw):
    a = dict(q=FAKE, ldq=512, B=2, q_len=1, heads=4, kv_heads=2, head_dim=128, bits=4, cache=FAKE, num_pages=64, page_size=16,
             page_table=FAKE, table_stride=32, lengths=FAKE, max_len=512, scale=0.1, softcap=0.0, window=0, out=FAKE, ldo=512, lse=None,
             workspace=None, workspace_bytes=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.basq_paged_attention(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), B.BASQ_EINVAL), (dict(q_len=0), B.BASQ_EINVAL), (dict(heads=0), B.BASQ_EINVAL), (dict(kv_heads=0), B.BASQ_EINVAL),
    (dict(heads=5), B.BASQ_EINVAL), (dict(head_dim=256), B.BASQ_EUNSUPPORTED), (dict(bits=8), B.BASQ_EUNSUPPORTED),
    (dict(q_len=32769), B.BASQ_EUNSUPPORTED), (dict(q_len=32768, heads=32768, kv_heads=32768, ldq=1 << 22), B.BASQ_EUNSUPPORTED),
    (dict(max_len=0x7FFF0001, table_stride=1 << 28), B.BASQ_EUNSUPPORTED),
    (dict(max_len=-1), B.BASQ_EINVAL), (dict(max_len=513), B.BASQ_EINVAL), (dict(table_stride=-1), B.BASQ_EINVAL),
    (dict(scale=float("inf")), B.BASQ_EINVAL), (dict(softcap=-1.0), B.BASQ_EINVAL), (dict(softcap=float("nan")), B.BASQ_EINVAL),
    (dict(window=-1), B.BASQ_EINVAL), (dict(cache=None), B.BASQ_EINVAL), (dict(cache=ODD), B.BASQ_EINVAL), (dict(num_pages=0), B.BASQ_EINVAL),
    (dict(page_size=24), B.BASQ_EUNSUPPORTED), (dict(q=None), B.BASQ_EINVAL), (dict(ldq=511), B.BASQ_EINVAL), (dict(out=None), B.BASQ_EINVAL),
    (dict(ldo=256), B.BASQ_EINVAL), (dict(page_table=None), B.BASQ_EINVAL), (dict(lengths=None), B.BASQ_EINVAL),
    (dict(lse=ctypes.c_void_p(0x1002)), B.BASQ_EINVAL),
    (dict(B=1 << 20, max_len=1 << 19, table_stride=1 << 15), B.BASQ_EUNSUPPORTED),
    # a call that splits its contexts needs a workspace
    (dict(max_len=8192, table_stride=512), B.BASQ_EINVAL), (dict(max_len=8192, table_stride=512, workspace=ctypes.c_void_p(0x1010)), B.BASQ_EINVAL),
    (dict(max_len=8192, table_stride=512, workspace=FAKE, workspace_bytes=64), B.BASQ_EWORKSPACE),
])
def test_attention_refuses(lib, kw, code):
    assert attention(lib, **kw) == code and B.basq_last_error()


def test_sizes(lib):
    assert B.basq_kv_page_bytes(8, 128, 64) == 8 * 64 * 144 and B.basq_kv_page_bytes(1, 64, 16) == 16 * 80
    assert [B.basq_kv_page_bytes(*s) for s in [(0, 128, 64), (8, 96, 64), (8, 128, 8), (8, 128, 48), (8, 128, 2048)]] == [0] * 5
    W = B.basq_paged_attention_workspace_bytes
    # short contexts (a window shortens them too) need none; longer ones no more than the workgroups' parts, whatever the batch
    assert W(4, 1, 32, 8, 128, 512) == 0 and W(4, 1, 32, 8, 128, 100000, 300) == 0 and W(4, 1, 32, 8, 128, 100000, 3000) > 0
    assert 0 < W(1, 1, 64, 8, 128, 131072) <= W(64, 1, 64, 8, 128, 131072) < 16 << 20
    assert W(0, 1, 32, 8, 128, 512) == W(4, 0, 32, 8, 128, 512) == W(4, 1, 30, 8, 128, 512) == W(1 << 20, 1, 4, 2, 128, 1 << 19) == 0


def test_binding_refuses_tensors_that_do_not_fit(lib):
    """Shapes, types and layouts are checked before a raw pointer is passed."""
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype)  # noqa: E731
    x, w = z(4, 64), z(64)
    bad = [
        lambda: B.basq_add_rms_norm(x, z(4, 56), w, 1e-5, z(4, 64)),
        lambda: B.basq_add_rms_norm(x, None, z(56), 1e-5, z(4, 64)),
        lambda: B.basq_add_rms_norm(x, None, w.float(), 1e-5, z(4, 64)),
        lambda: B.basq_add_rms_norm(x, None, w, 1e-5, z(64, 4).t()),
        lambda: B.basq_add_rms_norm(x, None, w, 1e-5, z(3, 64)),
        lambda: B.basq_add_rms_norm(x, None, w, 1e-5, None, Y8=z(4, 64, dtype=torch.uint8), y8_scale=z(4, dtype=torch.float32)),
        lambda: B.basq_add_rms_norm(x, None, w, 1e-5, None, Y8=z(4, 64, dtype=torch.float8_e4m3fn), y8_scale=z(3, dtype=torch.float32)),
    ]
    q, k, cache = z(3, 4, 64), z(3, 2, 64), z(5, 2, 16 * 80, dtype=torch.uint8)
    i32 = lambda n: z(n, dtype=torch.int32)  # noqa: E731
    table = z(8, 64, dtype=torch.float32)
    good = dict(q=q, k=k, v=k, positions=i32(3), cos_sin=table, slots=i32(3), cache=cache, clip_lo=0.9, clip_hi=0.9, q_out=z(3, 4, 64))
    for change in [dict(q_out=None), dict(q_out=z(3, 4, 32)), dict(v=None), dict(v=z(3, 4, 64)), dict(positions=z(3, dtype=torch.int64)),
                   dict(positions=i32(2)), dict(slots=None), dict(slots=z(3, dtype=torch.int64)), dict(positions=None),
                   dict(cache=z(5, 4, 16 * 80, dtype=torch.uint8)), dict(cache=z(5, 2, 1000, dtype=torch.uint8)), dict(cache=z(5, 2, 16 * 80)),
                   dict(cos_sin=z(8, 64)), dict(q=z(3, 64, 4).transpose(1, 2)), dict(k_hat=z(3, 2, 32)),
                   dict(k_hat=z(3, 2, 64), v_hat=z(3, 4, 64)[:, :2]), dict(q=None, k=None, v=None)]:
        bad.append(lambda change=change: B.basq_rope_append(**{**good, **change}))
    attend = dict(q=q, cache=cache, page_table=z(3, 4, dtype=torch.int32), lengths=i32(3), max_len=64, scale=0.1, out=z(3, 4, 64), workspace=None)
    for change in [dict(max_len=65), dict(q_len=2), dict(lengths=z(3, dtype=torch.int64)), dict(page_table=z(3, 4, dtype=torch.int64)),
                   dict(page_table=z(2, 4, dtype=torch.int32)), dict(out=z(3, 4, 32)), dict(lse=z(3, 4)), dict(lse=z(2, 4, dtype=torch.float32)),
                   dict(cache=cache[:, :, :-16])]:
        bad.append(lambda change=change: B.basq_paged_attention(**{**attend, **change}))
    bad.append(lambda: B.basq_rope_table(z(8, 64), 1e4))
    bad.append(lambda: B.alloc_kv_cache(4, 2, 96, 16, device="cpu"))
    for n, call in enumerate(bad):
        with pytest.raises(ValueError) as refused:
            call()
            pytest.fail(f"call {n} was not refused")
        # by its own fault, not because all of this is on the CPU
        assert "on the GPU of" not in str(refused.value), n
    for call in [lambda: B.basq_add_rms_norm(x, None, w, 1e-5, z(4, 64)), lambda: B.basq_rope_append(**good), lambda: B.basq_paged_attention(**attend)]:
        with pytest.raises(ValueError, match="is not on the GPU"):
            call()
    with pytest.raises(TypeError):
        B.basq_add_rms_norm(x, None, w, "small", z(4, 64))
    with pytest.raises(ValueError, match="must be a tensor"):
        B.basq_add_rms_norm(x, None, w.tolist(), 1e-5, z(4, 64))


WRAPPED = """
import types
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2506_15689_amd import binding as B

handle = types.SimpleNamespace(cuda_stream=0)
bf16 = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
i32 = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
refused = 0
with FakeTensorMode():
    x, w, q, k = bf16(2, 3, 64), bf16(64), bf16(2, 3, 4, 64), bf16(3, 2, 64)
    cache = torch.empty((5, 2, 16 * 80), dtype=torch.uint8, device="cuda")

    def norm(x):
        B.basq_add_rms_norm(x, None, w, 1e-5, x, stream=handle)
        return x

    def append(q):
        B.basq_rope_append(q, k, k, None, None, i32(3), cache, 0.9, 0.9, q, stream=handle)
        return q

    def attend(q):
        B.basq_paged_attention(q, cache, i32(3, 4), i32(3), 64, 0.1, q, None, stream=handle)
        return q

    for call, t in [(norm, x), (append, q), (attend, q)]:
        for wrapped in [lambda: torch.vmap(call)(t), lambda: torch.func.jvp(call, (t[0],), (t[0],))]:
            try:
                wrapped()
            except RuntimeError as e:
                refused += "storage" in str(e)
print("refused", refused)
"""


def test_tensors_without_storage_are_an_error(lib):
    """Tensors that stand for others (under torch.vmap, with a tangent) have no values of their own to point to: an exception, not the end
    of the process."""
    done = subprocess.run([sys.executable, "-c", WRAPPED], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.split()[-2:] == ["refused", "6"], done.stdout[-2000:]


COUNTS = """
import ctypes
from paper_2506_15689_amd import binding as B

lib, there = B.load(), ctypes.c_void_p(0x1000)
codes = []
for T in [1 << 31, 1 << 61, (1 << 63) - 8192, (1 << 63) - 1]:
    codes.append(lib.basq_rope_append(there, 512, there, 256, there, 256, T, 4, 2, 128, there, there, 16, 128, 0, 1, 0.9, 0.9, 4, there, there, 4, 16,
                                      there, 512, None, None, 0, None))
for rot, positions in [(1024, 1 << 31), (64, 1 << 59), (64, 1 << 62), (1024, (1 << 63) - 1), (2, (1 << 63) - 1)]:
    codes.append(lib.basq_rope_table(rot, positions, 1e4, 0, 1.0, 1.0, 2.0, 1.0, there, None))
print("codes", *codes)
"""


def test_counts_past_what_a_grid_holds(lib):
    """Tokens and positions up to the end of 64 bits are refused, not divided by what has wrapped to 0 (in a process of its own)."""
    done = subprocess.run([sys.executable, "-c", COUNTS], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.split()[-10:] == ["codes"] + [str(B.BASQ_EUNSUPPORTED)] * 9, done.stdout[-2000:]


@pytest.mark.parametrize("Bn", [1, 16, 64, 191, 192, 193, 1000])
def test_long_contexts_are_shared_whatever_the_batch(lib, Bn):
    """One sequence may be far longer than the others, which the host does not know: its workgroups must not be left with it."""
    long_call = dict(B=Bn, heads=64, kv_heads=8, ldq=8192, ldo=8192, max_len=131072, table_stride=8192)
    assert B.basq_paged_attention_workspace_bytes(Bn, 1, 64, 8, 128, 131072) > 0
    assert attention(lib, **long_call) == B.BASQ_EINVAL and "workspace" in B.basq_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that are not refused would be launched, on places that are not there")
def test_a_workspace_for_the_largest_call_does_for_smaller_ones(lib):
    """A program asks for its largest batch and context once; batches shrink and contexts end."""
    W = B.basq_paged_attention_workspace_bytes
    shared = 0
    for heads, kv_heads, D in [(32, 8, 128), (64, 8, 128), (32, 32, 128), (28, 4, 64), (71, 1, 128)]:
        for most_B, most_new, most_len, window in [(64, 1, 4096, 0), (64, 4, 8192, 0), (300, 1, 2048, 0), (16, 8, 40000, 3000), (1, 1, 100000, 0)]:
            room = W(most_B, most_new, heads, kv_heads, D, most_len, window)
            assert room % 8 == 0 and room <= 768 * 2 * 16 * (4 * D + 8) + 8 * most_B * kv_heads * -(-(heads // kv_heads) * most_new // 16)
            for Bn in {1, 2, 3, most_B // 4 + 1, most_B // 2 + 1, most_B}:
                for q_len in {1, most_new}:
                    for max_len in {1, 500, 513, 1000, 2049, most_len // 2, most_len}:
                        for w in {0, 600, window} if window == 0 else {600, window}:
                            if Bn > most_B or max_len > most_len:
                                continue
                            for cap in (0.0, 30.0):
                                call = dict(B=Bn, q_len=q_len, heads=heads, kv_heads=kv_heads, head_dim=D, ldq=heads * D, ldo=heads * D, max_len=max_len,
                                            table_stride=1 << 16, window=w, softcap=cap, workspace=FAKE)
                                need = 0
                                if attention(lib, **call, workspace_bytes=0) == B.BASQ_EWORKSPACE:
                                    need = int(B.basq_last_error().split()[-2])
                                    shared += 1
                                assert need <= W(Bn, q_len, heads, kv_heads, D, max_len, w) <= room
    assert shared > 100
    # what the call refuses needs none
    assert W(4, 32769, 32, 8, 128, 8192) == W(4, 1, 32, 8, 128, 0x7FFF0001) == W(4, 1, 65536, 1, 128, 8192) == W(4, 1, 32, 8, 128, 8192, -1) == 0
    assert W(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 1, 128, 2 ** 31 - 1) == 0


def test_calls_go_to_the_gpu_of_their_tensors(lib, monkeypatch):
    """Which is not always the current one: its current stream is asked for, a stream of another GPU is refused."""
    from torch._subclasses.fake_tensor import FakeTensorMode

    class Asked(Exception):
        pass

    def handle_of(stream, device):
        raise Asked(stream, device)

    monkeypatch.setattr(B, "_stream_on", handle_of)
    with FakeTensorMode():
        new = lambda dtype, *s: torch.empty(s, dtype=dtype, device="cuda:1")  # noqa: E731
        x, q, k = new(BF16, 3, 64), new(BF16, 3, 4, 64), new(BF16, 3, 2, 64)
        cache, i32 = new(torch.uint8, 5, 2, 16 * 80), lambda *s: new(torch.int32, *s)  # noqa: E731
        for call in [lambda **kw: B.basq_add_rms_norm(x, None, new(BF16, 64), 1e-5, x, **kw),
                     lambda **kw: B.basq_rope_append(q, k, k, None, None, i32(3), cache, 0.9, 0.9, q, **kw),
                     lambda **kw: B.basq_paged_attention(q, cache, i32(3, 4), i32(3), 64, 0.1, q, None, **kw),
                     lambda **kw: B.basq_rope_table(new(torch.float32, 8, 64), 1e4, **kw)]:
            with pytest.raises(Asked) as asked:
                call()
            assert asked.value.args == (None, 1)
            with pytest.raises(Asked) as asked:
                call(stream="a stream")
            assert asked.value.args == ("a stream", 1)
        with pytest.raises(ValueError, match="is not on the GPU of the other tensors"):
            B.basq_add_rms_norm(x, torch.empty((3, 64), dtype=BF16, device="cuda:0"), new(BF16, 64), 1e-5, x)


@pytest.mark.parametrize("documented", [False, True])
def test_the_stream_of_a_gpu(monkeypatch, documented):
    class Stream:
        cuda_stream = 0x5678
        device_index = 1

    monkeypatch.setattr(B, "_raw_stream", None if documented else lambda device: 0x1000 + device)
    monkeypatch.setattr(B.torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(B.torch.cuda, "current_stream", lambda device: type("S", (), {"cuda_stream": 0x1000 + device}))
    assert B._stream_on(None, 3) == 0x1003
    assert B._stream_on(Stream, 1) == 0x5678
    with pytest.raises(ValueError, match="the stream is on GPU 1, the tensors are on GPU 0"):
        B._stream_on(Stream, 0)

"""The attention block's entry points without a GPU: sizes, and what they refuse
on the host before anything is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

import block_ref as ref
import paper_1705_01462_amd as fgq

no_device = pytest.mark.skipif(fgq.lib().fgq_device_count() > 0,
                               reason="placeholder pointers are only passed on a host without a GPU")
P = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)
N = None
NULL, SHAPE, GROUP, BITS, HIP, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 6, 7, 8


def test_sizes():
    L = fgq.lib()
    for D, page, bits, G in [(64, 16, 4, 32), (128, 64, 4, 128), (256, 1024, 8, 32), (96, 32, 8, 32)]:
        assert L.fgq_kv_page_bytes(3, D, page, bits, G) == 3 * ref.head_bytes(page, D, bits, G)
    for bad in [(3, 64, 16, 5, 32), (3, 64, 16, 4, 48), (3, 80, 16, 4, 32), (3, 64, 24, 4, 32), (3, 64, 8, 4, 32),
                (3, 64, 2048, 4, 32), (0, 64, 16, 4, 32), (3, 4096, 16, 4, 32), (40000, 2048, 1024, 8, 32)]:
        assert L.fgq_kv_page_bytes(*bad) == 0
    # few rows are quantized in the product itself: no workspace
    assert L.fgq_linear_i8_ws_bytes(1, 4096, 4096) == 0 and L.fgq_linear_i8_ws_bytes(8, 4096, 100) == 0
    assert L.fgq_linear_i8_ws_bytes(9, 4000, 100) == 9 * (4096 + 4)
    assert L.fgq_linear_i8_ws_bytes(0, 64, 64) == 0
    # no device here: 256 compute units assumed; one long sequence is split, a prompt is not
    assert L.fgq_attn_kv_ws_bytes(1, 8, 8, 128, 1, 1, 65536) > 0
    assert L.fgq_attn_kv_ws_bytes(4096, 8, 8, 128, 1, 4096, 65536) == 0
    assert L.fgq_attn_kv_ws_bytes(0, 8, 8, 128, 1, 1, 65536) == 0


@no_device
def test_products_refuse():
    L = fgq.lib()
    rows = lambda x=P, t=0, M=4, K=100, ldx=100, q=P, ldq=128, s=P: L.fgq_quantize_rows(x, t, M, K, ldx, q, ldq, s, N)
    assert rows(x=N) == NULL and rows(q=N) == NULL and rows(s=N) == NULL
    assert rows(t=3) == SHAPE and rows(M=-1) == SHAPE and rows(K=0) == SHAPE and rows(ldx=99) == SHAPE
    assert rows(ldq=127) == SHAPE and rows(ldq=136) == SHAPE and rows(q=ODD) == SHAPE and rows(x=ODD) == SHAPE
    assert rows(M=0, x=N) == 0

    gemm = lambda q=P, ldq=128, sx=P, M=4, K=100, w=P, ldw=128, sw=P, O=8, b=N, t=2, y=P, ldy=8: \
        L.fgq_gemm_i8(q, ldq, sx, M, K, w, ldw, sw, O, b, t, y, ldy, N)
    assert gemm(q=N) == NULL and gemm(sx=N) == NULL and gemm(w=N) == NULL and gemm(sw=N) == NULL and gemm(y=N) == NULL
    assert gemm(ldq=112) == SHAPE and gemm(ldw=100) == SHAPE and gemm(ldy=7) == SHAPE and gemm(t=-1) == SHAPE
    assert gemm(O=0) == SHAPE and gemm(M=-1) == SHAPE and gemm(q=ODD) == SHAPE and gemm(w=ODD) == SHAPE
    assert gemm(K=131072, ldq=131072, ldw=131072) == UNSUPPORTED
    assert gemm(M=0, q=N) == 0

    lin = lambda x=P, t=0, ldx=100, M=40, K=100, w=P, ldw=128, sw=P, O=8, y=P, ws=P, nb=1 << 20: \
        L.fgq_linear_i8(x, t, ldx, M, K, w, ldw, sw, O, N, t, y, 8, ws, nb, N)
    assert lin(x=N) == NULL and lin(y=N) == NULL and lin(ldx=99) == SHAPE and lin(t=9) == SHAPE
    assert lin(ws=N) == WORKSPACE and lin(nb=40 * 132 - 1) == WORKSPACE and lin(ws=ODD) == WORKSPACE
    assert lin(M=0, x=N) == 0


@no_device
def test_cache_refuses():
    L = fgq.lib()
    write = lambda k=P, v=P, t=0, T=5, s=P, c=P, n=4, H=2, D=64, p=16, b=4, G=32: \
        L.fgq_kv_write(k, v, t, T, H * D, D, H * D, D, s, c, n, H, D, p, b, G, N)
    read = lambda s=P, T=5, c=P, n=4, H=2, D=64, p=16, b=4, G=32, t=0, k=P, v=P: \
        L.fgq_kv_read(s, T, c, n, H, D, p, b, G, t, k, v, N)
    for f in (write, read):
        assert f(k=N) == NULL and f(v=N) == NULL and f(s=N) == NULL and f(c=N) == NULL
        assert f(b=6) == BITS and f(G=16) == GROUP and f(D=80) == GROUP and f(n=0) == SHAPE and f(H=0) == SHAPE
        assert f(T=-1) == SHAPE and f(t=5) == SHAPE and f(c=ODD) == SHAPE and f(k=ODD) == SHAPE
        assert f(p=48) == UNSUPPORTED and f(p=8) == UNSUPPORTED and f(D=4096) == UNSUPPORTED
        assert f(T=0, k=N, s=N) == 0


@no_device
def test_attention_refuses():
    L = fgq.lib()

    def attn(q=P, t=1, T=5, Hq=4, cu=P, B=2, mq=3, c=P, n=4, H=2, D=64, p=16, b=4, G=32, pg=P, mp=2, ln=P, sc=0.1,
             causal=1, w=0, o=P, ws=P, nb=1 << 30):
        return L.fgq_attn_kv(q, t, T, Hq, Hq * D, D, cu, B, mq, c, n, H, D, p, b, G, pg, mp, ln, sc, causal, w, o, N,
                             ws, nb, N)
    for name in ("q", "cu", "c", "pg", "ln", "o"):
        assert attn(**{name: N}) == NULL
    assert attn(b=2) == BITS and attn(G=48) == GROUP and attn(D=96, G=32) == UNSUPPORTED and attn(p=100) == UNSUPPORTED
    assert attn(t=0) == UNSUPPORTED and attn(t=7) == SHAPE and attn(Hq=3) == SHAPE and attn(Hq=1) == SHAPE
    assert attn(mq=6) == SHAPE and attn(w=-1) == SHAPE and attn(w=4, causal=0) == UNSUPPORTED
    assert attn(sc=0.0) == SHAPE and attn(sc=float("inf")) == SHAPE and attn(sc=float("nan")) == SHAPE
    assert attn(mp=1 << 30) == SHAPE and attn(c=ODD) == SHAPE and attn(q=ODD) == SHAPE
    assert attn(T=1, B=1, mq=1, mp=1 << 12, ws=N) == WORKSPACE
    assert attn(T=1, B=1, mq=1, mp=1 << 12, nb=16) == WORKSPACE
    assert attn(T=0, mq=0, q=N) == 0 and attn(B=0, cu=N) == 0


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x = torch.zeros(2, 128)
    with pytest.raises(ValueError):
        fgq.fgq_quantize_rows(x)
    with pytest.raises(TypeError):
        fgq.fgq_quantize_rows(np.zeros((2, 128)))
    with pytest.raises(ValueError):
        fgq.fgq_kv_cache(2, 2, 64, 20, 4, 32, device="cpu")
    cache = fgq.fgq_kv_cache(2, 2, 64, 16, 4, 32, device="cpu")
    assert cache.shape == (2, 2, ref.head_bytes(16, 64, 4, 32)) and cache.dtype is torch.uint8
    with pytest.raises(ValueError):
        fgq.fgq_kv_read(torch.zeros(1, dtype=torch.int64), cache, 16, 64, 4, 32, torch.float32)


def test_reference_rows_and_groups():
    """The tests' own definitions on hand-made values."""
    q, s = ref.rows(np.array([[2.0, -1.0, 0.0, 1.5], [0, 0, 0, 0]], np.float32))
    assert q.tolist() == [[127, -64, 0, 95], [0, 0, 0, 0]] and s[1] == 1 and s[0] == np.float32(2) / np.float32(127)
    x = np.zeros((1, 32), np.float32)
    x[0, 0], x[0, 1] = -1.0, 2.0                # lo -1, step 3 / 15 = 0.2 up to bf16
    c, lo, st = ref.groups(x, 4, 32)
    assert lo[0, 0] == -1 and 0.2 <= st[0, 0] <= 0.2 * (1 + 2.0 ** -7) and (st.view(np.uint32) & 0xFFFF == 0).all()
    assert c[0, 0] == 0 and c[0, 1] == 15 and (c[0, 2:] == 5).all()
    assert np.abs(ref.values(c, lo, st, 32) - x).max() <= st[0, 0] / 2 * (1 + 2.0 ** -20)

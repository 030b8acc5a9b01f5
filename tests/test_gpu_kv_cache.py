"""GPU: the quantized key/value cache (fgq_kv_write, fgq_kv_read) against its
definition: every byte of the pages, and the values read back rounded once."""
import numpy as np
import pytest
import torch

import block_ref as ref

fgq = pytest.importorskip("paper_1705_01462_amd")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def tokens(T, H, D, dtype, seed):
    r = np.random.default_rng(seed)
    x = r.standard_normal((2, T, H, D)) * np.exp(2 * r.standard_normal((2, T, H, 1)))
    x = torch.from_numpy(x.astype(np.float32)).to(dtype)
    return x[0], x[1]


def ref_pages(k, v, slots, pages, P, bits, G, fill):
    """What the cache's bytes have to be after the write, from bytes `fill`."""
    T, H, D = k.shape
    ck, lk, sk = ref.groups(k.float().numpy(), bits, G)
    cv, lv, sv = ref.groups(v.float().numpy(), bits, G)
    out = fill.copy()
    row, ng = D * bits // 8, D // G
    for t, s in enumerate(slots):
        if s < 0 or s >= pages * P:
            continue
        page, at = s // P, s % P
        for z, (c, lo, st) in enumerate(((ck, lk, sk), (cv, lv, sv))):
            b = c[t] if bits == 8 else c[t][:, 0::2] | c[t][:, 1::2] << 4
            o = (z * P + at) * row
            out[page, :, o:o + row] = b.astype(np.uint8)
            w = (lo[t].view(np.uint32) >> 16) | (st[t].view(np.uint32) & 0xFFFF0000)
            for g in range(ng):
                o = 2 * P * row + 4 * ((z * ng + g) * P + at)
                out[page, :, o:o + 4] = np.ascontiguousarray(w[:, g]).view(np.uint8).reshape(H, 4)
    return out


CASES = [(1, 1, 64, 16, 4, 64), (1, 8, 128, 16, 4, 128), (3, 2, 128, 32, 8, 64), (17, 5, 64, 16, 8, 32),
         (40, 3, 256, 64, 4, 32), (100, 8, 128, 64, 4, 64), (130, 1, 96, 128, 4, 32), (33, 2, 256, 16, 8, 128),
         (50, 12, 32, 1024, 4, 32), (7, 3, 640, 16, 4, 128)]


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("T,H,D,P,bits,G", CASES)
def test_write_and_read(T, H, D, P, bits, G, dtype):
    r = np.random.default_rng(T + D)
    pages = -(-T // P) + 2
    k, v = tokens(T, H, D, dtype, T)
    slots = r.permutation(pages * P)[:T]
    slots[r.random(T) < 0.1] = -1
    if T > 10:
        slots[3] = pages * P       # outside: skipped
    fill = r.integers(0, 256, (pages, H, ref.head_bytes(P, D, bits, G)), dtype=np.uint8)
    cache = torch.from_numpy(fill.copy()).cuda()
    assert fgq.fgq_kv_page_bytes(H, D, P, bits, G) == H * ref.head_bytes(P, D, bits, G)
    sl = torch.from_numpy(slots).cuda()
    fgq.fgq_kv_write(k.cuda(), v.cuda(), sl, cache, P, bits, G)
    want = ref_pages(k, v, slots, pages, P, bits, G, fill)
    assert np.array_equal(cache.cpu().numpy(), want)
    ko, vo = fgq.fgq_kv_read(sl, cache, P, D, bits, G, dtype)
    live = (slots >= 0) & (slots < pages * P)
    for x, o in ((k, ko), (v, vo)):
        val = ref.values(*ref.groups(x.float().numpy(), bits, G), G)
        val[~live] = 0
        # lo + step * code needs at most 8 + 8 bits beside lo's 8: one rounding to fp32, one to the type
        u, tiny = ref.ROUND[dtype]
        got = o.double().cpu().numpy()
        assert (np.abs(got - val) <= (u + 2.0 ** -24) * np.abs(val) * (1 + u) + tiny).all()


@pytest.mark.parametrize("bits,G", [(4, 32), (8, 64)])
def test_values_are_within_half_a_step(bits, G):
    k, v = tokens(64, 2, 128, torch.float32, 9)
    cache = fgq.fgq_kv_cache(4, 2, 128, 16, bits, G)
    sl = torch.arange(64, device="cuda")
    fgq.fgq_kv_write(k.cuda(), v.cuda(), sl, cache, 16, bits, G)
    ko, _ = fgq.fgq_kv_read(sl, cache, 16, 128, bits, G, torch.float32)
    _, _, s = ref.groups(k.numpy(), bits, G)
    half = np.repeat(s.astype(np.float64), G, -1) * (0.5 + 2.0 ** -12)
    assert (np.abs(ko.cpu().numpy().astype(np.float64) - k.numpy()) <= half + 2.0 ** -23 * np.abs(k.numpy())).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_strided_tokens(bits):
    """k and v as parts of one projection's rows, at an odd offset."""
    T, H, D, P, G = 21, 3, 64, 16, 32
    r = np.random.default_rng(2)
    x = torch.from_numpy(r.standard_normal((T, 2 * H * D + 3)).astype(np.float32)).to(torch.bfloat16)
    xd = x.cuda()
    part = lambda t, z: t[:, 1 + z * H * D:1 + (z + 1) * H * D].unflatten(1, (H, D))
    cache = torch.zeros((2, H, ref.head_bytes(P, D, bits, G)), dtype=torch.uint8, device="cuda")
    sl = np.arange(T)
    fgq.fgq_kv_write(part(xd, 0), part(xd, 1), torch.from_numpy(sl).cuda(), cache, P, bits, G)
    want = ref_pages(part(x, 0), part(x, 1), sl, 2, P, bits, G, np.zeros(cache.shape, np.uint8))
    assert np.array_equal(cache.cpu().numpy(), want)


def test_extreme_groups():
    """Constant, tiny, huge and non-finite groups."""
    D, G, P = 128, 32, 16
    x = np.zeros((10, 1, D), np.float32)
    x[0] = 3.14159                                   # constant: step 0 or one rounding of lo
    x[1] = 1e-38 * np.linspace(-1, 1, D)             # step below 2^-120: lo alone
    x[2] = np.where(np.arange(D) % 2, 3.3e38, -3.3e38)  # the range overflows fp32
    x[3, 0, 5] = np.nan
    x[4, 0, 40] = np.inf
    x[5, 0, 70] = -np.inf
    x[6] = -3.4e38                                   # rounds down to minus infinity in bf16
    x[7] = np.linspace(1000, 1001, D)
    x[8] = -np.linspace(1000, 1001, D)
    x[9] = np.where(np.arange(D) % 32 == 3, 500.0, 0.01)
    for bits in (4, 8):
        cache = fgq.fgq_kv_cache(1, 1, D, P, bits, G)
        sl = torch.arange(10, device="cuda")
        t = torch.from_numpy(x).cuda()
        fgq.fgq_kv_write(t, t, sl, cache, P, bits, G)
        k, v = fgq.fgq_kv_read(sl, cache, P, D, bits, G, torch.float32)
        assert torch.equal(k.view(torch.int32), v.view(torch.int32))
        k = k.cpu().numpy().astype(np.float64)
        bad = np.zeros((10, 4), bool)
        bad[3, 0] = bad[4, 1] = bad[5, 2] = True
        bad[6] = True
        assert np.array_equal(np.isnan(k).reshape(10, 4, 32).all(-1), bad) and np.isnan(k).sum() == bad.sum() * 32
        fine = [0, 1, 2, 7, 8, 9]
        want = ref.values(*ref.groups(x[fine], bits, G), G)
        assert (np.abs(k[fine] - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -149).all()


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GB: tokens in its last pages."""
    H, D, P, bits, G = 8, 128, 64, 4, 128
    pages = (5 << 30) // fgq.fgq_kv_page_bytes(H, D, P, bits, G)
    cache = fgq.fgq_kv_cache(pages, H, D, P, bits, G)
    k, v = tokens(100, H, D, torch.bfloat16, 1)
    slots = torch.arange(pages * P - 100, pages * P, device="cuda")
    fgq.fgq_kv_write(k.cuda(), v.cuda(), slots, cache, P, bits, G)
    ko, vo = fgq.fgq_kv_read(slots, cache, P, D, bits, G, torch.float32)
    for x, o in ((k, ko), (v, vo)):
        want = ref.values(*ref.groups(x.float().numpy(), bits, G), G)
        assert (np.abs(o.double().cpu().numpy() - want) <= 2.0 ** -23 * np.abs(want) + 2.0 ** -149).all()


def test_refusals():
    H, D, P, bits, G = 2, 64, 16, 4, 32
    cache = fgq.fgq_kv_cache(2, H, D, P, bits, G)
    k = torch.zeros((3, H, D), device="cuda")
    sl = torch.arange(3, device="cuda")
    assert fgq.fgq_kv_page_bytes(H, D, 24, bits, G) == 0 and fgq.fgq_kv_page_bytes(H, D, P, 5, G) == 0
    assert fgq.fgq_kv_page_bytes(H, D, P, bits, 48) == 0 and fgq.fgq_kv_page_bytes(H, 80, P, bits, 32) == 0
    for call, err in [
            (lambda: fgq.fgq_kv_write(k, k[:, :1], sl, cache, P, bits, G), ValueError),
            (lambda: fgq.fgq_kv_write(k, k.half(), sl, cache, P, bits, G), ValueError),
            (lambda: fgq.fgq_kv_write(k.double(), k.double(), sl, cache, P, bits, G), TypeError),
            (lambda: fgq.fgq_kv_write(k, k, sl.int(), cache, P, bits, G), TypeError),
            (lambda: fgq.fgq_kv_write(k, k, sl[:2], cache, P, bits, G), ValueError),
            (lambda: fgq.fgq_kv_write(k.transpose(1, 2), k.transpose(1, 2), sl, cache, P, bits, G), ValueError),
            (lambda: fgq.fgq_kv_write(k, k, sl, cache, 32, bits, G), ValueError),       # another cache's P
            (lambda: fgq.fgq_kv_write(k, k, sl, cache, P, 6, G), (ValueError, fgq.FgqError)),
            (lambda: fgq.fgq_kv_read(sl, cache, P, 128, bits, G, torch.float32), ValueError),
            (lambda: fgq.fgq_kv_read(sl, cache, P, D, bits, G, torch.float64), TypeError),
            (lambda: fgq.fgq_kv_cache(2, H, D, 20, bits, G), ValueError)]:
        with pytest.raises(err):
            call()
    empty = torch.empty((0, H, D), device="cuda")
    fgq.fgq_kv_write(empty, empty, sl[:0], cache, P, bits, G)
    assert fgq.fgq_kv_read(sl[:0], cache, P, D, bits, G, torch.float32)[0].shape == (0, H, D)

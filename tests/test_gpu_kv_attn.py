"""GPU: attention over the quantized cache (fgq_attn_kv) against the definition
in 64 bits on the values the cache's codes stand for.

Bound of an output's error, with p the exact probabilities and S = sum_j p_j
step_j mid (mid the middle code), V = sum_j p_j |v_j|:
  the probabilities' products with the steps are rounded to fp16: 2^-11 S (twice
  that is allowed: the running maximum may scale them once more);
  a score is off by at most d = scale * 2^-24 * 16 * (1264 max step + max |lo|)
  * sum |q| (fp32 sums of 1024 + 16 c, their corrections, two products), and a
  shift of all scores by up to d changes an output by at most 2 d V;
  fp32 sums over the keys: 2^-19 V; the output's own rounding.
"""
import numpy as np
import pytest
import torch

import block_ref as ref

fgq = pytest.importorskip("paper_1705_01462_amd")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


class Case:
    """Sequences (keys, queries) over a cache of random tokens in scattered pages."""

    def __init__(self, seqs, Hq, Hkv, D, P, bits, G, dtype, seed=0, spread=1.0, extra=1):
        r = np.random.default_rng(seed)
        self.seqs, self.Hq, self.Hkv, self.D, self.P, self.bits, self.G, self.dtype = seqs, Hq, Hkv, D, P, bits, G, dtype
        maxp = max(-(-n // P) for n, _ in seqs)
        total = sum(-(-n // P) for n, _ in seqs)
        pages = total + 2
        ids = r.permutation(pages)[:total]
        k = (r.standard_normal((pages * P, Hkv, D)) * np.exp(0.7 * r.standard_normal((1, Hkv, D)))).astype(np.float32)
        v = (r.standard_normal((pages * P, Hkv, D)) * np.exp(0.7 * r.standard_normal((pages * P, Hkv, 1))) + 0.3)
        v = v.astype(np.float32)
        self.par = [ref.groups(x, bits, G) for x in (k, v)]
        self.pool = ref.pack_pages(*self.par[0], *self.par[1], P, bits, G)
        self.val = [ref.values(*p, G) for p in self.par]
        # entries past a sequence's pages name no page at all
        self.table = np.full((len(seqs), maxp + extra), 1 << 30, np.int32)
        at = 0
        for b, (n, _) in enumerate(seqs):
            m = -(-n // P)
            self.table[b, :m] = ids[at:at + m]
            at += m
        T = sum(q for _, q in seqs)
        self.q = torch.from_numpy((spread * r.standard_normal((T, Hq, D))).astype(np.float32)).to(dtype)
        self.cu = np.concatenate([[0], np.cumsum([q for _, q in seqs])]).astype(np.int32)
        self.lens = np.array([n for n, _ in seqs], np.int32)

    def device(self):
        d = lambda x: torch.from_numpy(x).cuda()
        return dict(q=self.q.cuda(), cu_q=d(self.cu), max_q=max(q for _, q in self.seqs), cache=d(self.pool.copy()),
                    pages=d(self.table), kv_lens=d(self.lens), P=self.P, bits=self.bits, G=self.G)

    def slots(self, b):
        n = self.seqs[b][0]
        j = np.arange(n)
        return self.table[b, j // self.P].astype(np.int64) * self.P + j % self.P

    def check(self, o, lse, causal=True, window=0, scale=None):
        scale = self.D ** -0.5 if scale is None else scale
        u, tiny = ref.ROUND[self.dtype]
        got, gl = o.double().cpu().numpy(), lse.double().cpu().numpy()
        mid = 8 if self.bits == 4 else 128
        ratio = self.Hq // self.Hkv
        worst = 0.0
        for b, (n, nq) in enumerate(self.seqs):
            sl, rows = self.slots(b), slice(self.cu[b], self.cu[b + 1])
            for h in range(self.Hq):
                hk = h // ratio
                k, v = (x[sl, hk] for x in self.val)
                q = self.q[rows, h].double().numpy()
                want, wl, p = ref.attention(q, k, v, n, causal, window, scale)
                lo, st = (np.abs(x[sl, hk]).max(initial=0) for x in self.par[0][1:])
                d = scale * 2.0 ** -24 * 16 * (1264 * st + lo) * np.abs(q).sum(1)
                S = p @ np.repeat(self.par[1][2][sl, hk].astype(np.float64), self.G, -1) * mid
                V = p @ np.abs(v)
                tol = 2 * 2.0 ** -11 * S + (2 * d[:, None] + 2.0 ** -19) * (V + S) + u * np.abs(want) + tiny
                err = np.abs(got[rows, h] - want)
                assert (err <= tol).all(), (b, h, float((err / np.maximum(tol, 1e-300)).max()))
                worst = max(worst, float((err / np.maximum(tol, 1e-300)).max(initial=0)))
                e = np.isneginf(wl)
                assert np.array_equal(np.isneginf(gl[rows, h]), e)
                assert (np.abs(gl[rows, h][~e] - wl[~e]) <= d[~e] + 2.0 ** -19 * (1 + np.abs(wl[~e]))).all(), (b, h)
                assert not got[rows, h][e].any()
        return worst

    def run(self, **kw):
        lse = torch.full((self.q.shape[0], self.Hq), 7.0, dtype=torch.float32, device="cuda")
        return fgq.fgq_attn_kv(**self.device(), lse=lse, **kw), lse


LAYOUTS = [(64, 4, 64), (64, 4, 32), (64, 8, 32), (64, 8, 64), (128, 4, 128), (128, 4, 64), (128, 4, 32),
           (128, 8, 128), (128, 8, 64), (128, 8, 32), (256, 4, 128), (256, 4, 64), (256, 4, 32), (256, 8, 128),
           (256, 8, 64), (256, 8, 32)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,bits,G", LAYOUTS)
def test_single_tokens(D, bits, G, dtype):
    """One query a sequence; lengths from one key to several tiles, and none."""
    c = Case([(1, 1), (0, 1), (16, 1), (17, 1), (300, 1), (1111, 1)], 8, 2, D, 16, bits, G, dtype, seed=D + G)
    c.check(*c.run())


@pytest.mark.parametrize("D,bits,G", LAYOUTS)
def test_many_queries(D, bits, G):
    """Prompts: more rows than a workgroup has, ragged, and more queries than keys (rows that see nothing)."""
    c = Case([(200, 77), (33, 33), (20, 50), (100, 1)], 6, 2, D, 32, bits, G, torch.float16, seed=D + G)
    c.check(*c.run())


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (5, 1), (12, 4), (16, 1), (20, 1), (40, 2)])
@pytest.mark.parametrize("nq", [1, 2, 5, 40])
def test_head_layouts(Hq, Hkv, nq):
    c = Case([(nq + 61, nq), (nq, nq), (500, nq)], Hq, Hkv, 128, 16, 4, 64, torch.bfloat16, seed=nq)
    c.check(*c.run())


@pytest.mark.parametrize("P", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("nq", [1, 70])
def test_page_sizes(P, nq):
    c = Case([(P, min(nq, P)), (P + 1, min(nq, P)), (3 * P - 1, 1), (777, nq)], 4, 2, 128, P, 4, 128, torch.float16,
             seed=P)
    c.check(*c.run())


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 33, 100, 4000])
@pytest.mark.parametrize("nq", [1, 7, 90])
def test_windows(window, nq):
    c = Case([(500, nq), (nq, nq), (40, nq), (131, nq)], 4, 2, 64, 16, 8, 32, torch.float16, seed=window)
    c.check(*c.run(window=window), window=window)


@pytest.mark.parametrize("nq", [1, 9, 80])
def test_without_causal(nq):
    c = Case([(300, nq), (5, nq), (0, nq), (64, nq)], 4, 4, 128, 16, 4, 64, torch.bfloat16, seed=nq)
    c.check(*c.run(causal=False), causal=False)


@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("scale,spread", [(1.0, 4.0), (0.001, 1.0), (0.088, 1e-3), (0.088, 300.0)])
def test_score_ranges(scale, spread, nq):
    """Probabilities from all alike to a single one."""
    c = Case([(600, nq), (70, nq)], 4, 2, 128, 16, 4, 64, torch.bfloat16, seed=3, spread=spread)
    c.check(*c.run(scale=scale), scale=scale)


def test_long_contexts():
    """Keys divided among workgroups, uneven lengths."""
    c = Case([(20000, 1), (700, 1), (1, 1), (5000, 1)], 8, 2, 128, 64, 4, 128, torch.float16, seed=8)
    c.check(*c.run())
    c = Case([(9000, 3), (4097, 5)], 6, 1, 64, 32, 8, 64, torch.bfloat16, seed=9)
    c.check(*c.run())


@pytest.mark.parametrize("nq", [1, 3, 50])
@pytest.mark.parametrize("bits", [4, 8])
def test_what_hidden_places_hold_does_not_matter(bits, nq):
    """Places past the keys, pages of nobody and keys outside windows hold NaN and infinite parameters."""
    D, G, P = 128, 64, 16
    c = Case([(163, nq), (70, nq), (nq, nq)], 4, 2, D, P, bits, G, torch.float16, seed=5)
    want, wl = c.run(window=50)
    seen = np.zeros(c.pool.shape[0] * P, bool)
    for b, (n, q) in enumerate(c.seqs):
        seen[c.slots(b)[max(0, n - q - 50 + 1):]] = True
    row, ng = D * bits // 8, D // G
    par = c.pool[..., 2 * P * row:].view(np.uint32).reshape(-1, 2, 2, ng, P)  # [page][head][k, v][group][place]
    bad = np.array([0x7FC07FC0, 0x7F80FF80, 0xFF807F80, 0x7F7F7F7F], np.uint32)
    hidden = ~seen.reshape(-1, P)
    for p, at in zip(*np.nonzero(hidden)):
        par[p, ..., at] = bad[(p + at) % 4]
    got, gl = c.run(window=50)
    assert torch.equal(got, want) and torch.equal(gl, wl)
    c.check(got, gl, window=50)


@pytest.mark.parametrize("nq", [1, 40])
def test_a_key_that_is_nan_reaches_the_rows_that_see_it_only(nq):
    D, G, P, bits, n = 64, 32, 16, 4, 100
    c = Case([(n, nq)], 2, 2, D, P, bits, G, torch.float16, seed=6)
    clean, cl = c.run()
    bad = n - nq + nq // 2  # seen by the queries from nq / 2 on
    par = c.pool[..., 2 * P * D * bits // 8:].view(np.uint32).reshape(-1, 2, 2, D // G, P)
    par[c.table[0, bad // P], 0, 0, 1, bad % P] = 0x7FC07FC0  # a key of head 0
    got, gl = c.run()
    assert torch.isnan(got[nq // 2:, 0]).all()
    assert torch.equal(got[:nq // 2], clean[:nq // 2]) and torch.equal(got[:, 1], clean[:, 1])
    assert torch.equal(gl[:, 1], cl[:, 1])
    q = c.q.clone()
    c.q[0, 1, 3] = float("inf")  # a query that is not finite: its own row alone
    got, _ = c.run()
    assert torch.isnan(got[0, 1]).all() and torch.equal(got[1:, 1], clean[1:, 1])
    c.q = q


@pytest.mark.parametrize("bits,G", [(4, 128), (8, 32)])
def test_steps_of_all_magnitudes(bits, G):
    """Values whose steps grow by orders of magnitude along the sequence, and fall again."""
    D, P, n = 128, 16, 400
    c = Case([(n, 1), (n, 30)], 4, 2, D, P, bits, G, torch.bfloat16, seed=12)
    r = np.random.default_rng(1)
    v = r.standard_normal((c.pool.shape[0] * P, 2, D)).astype(np.float32)
    for b in range(2):
        for j, s in enumerate(c.slots(b)):
            v[s] *= np.float32(10.0 ** (30 * np.sin(j / 40)))
    c.par[1] = ref.groups(v, bits, G)
    c.pool = ref.pack_pages(*c.par[0], *c.par[1], P, bits, G)
    c.val[1] = ref.values(*c.par[1], G)
    c.check(*c.run())


def test_strided_queries_and_other_streams():
    """q as a part of a projection's rows; a stream of one's own."""
    c = Case([(90, 5), (33, 1)], 6, 2, 64, 16, 4, 32, torch.bfloat16, seed=2)
    want, wl = c.run()
    d = c.device()
    T = c.q.shape[0]
    wide = torch.zeros((T, 6 * 64 + 77), dtype=torch.bfloat16, device="cuda")
    wide[:, 11:11 + 6 * 64] = d["q"].flatten(1)
    d["q"] = wide[:, 11:11 + 6 * 64].unflatten(1, (6, 64))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = fgq.fgq_attn_kv(**d)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(got, want)


def test_written_then_attended():
    """Through the cache's own write, against the values it reads back."""
    H, D, P, bits, G, n = 2, 128, 32, 4, 64, 150
    r = np.random.default_rng(4)
    k, v = (torch.from_numpy(r.standard_normal((n, H, D)).astype(np.float32)).to(torch.bfloat16).cuda() for _ in "kv")
    cache = fgq.fgq_kv_cache(8, H, D, P, bits, G)
    table = torch.tensor([[5, 0, 7, 2, 1]], dtype=torch.int32, device="cuda")
    j = torch.arange(n, device="cuda")
    slots = table[0, j // P].long() * P + j % P
    fgq.fgq_kv_write(k, v, slots, cache, P, bits, G)
    kr, vr = fgq.fgq_kv_read(slots, cache, P, D, bits, G, torch.float32)
    q = torch.from_numpy(r.standard_normal((n, 4, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    o = fgq.fgq_attn_kv(q, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, cache, table,
                        torch.tensor([n], dtype=torch.int32, device="cuda"), P, bits, G)
    for h in range(4):
        want, _, _ = ref.attention(*(t[:, i].double().cpu().numpy() for t, i in ((q, h), (kr, h // 2), (vr, h // 2))),
                                   n, True, 0, D ** -0.5)
        assert np.abs(o[:, h].double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max()


def test_offsets_beyond_32_bits():
    H, D, P, bits, G = 8, 128, 64, 4, 128
    c = Case([(130, 1), (90, 20)], 16, H, D, P, bits, G, torch.float16, seed=7)
    pages = (5 << 30) // fgq.fgq_kv_page_bytes(H, D, P, bits, G)
    want, wl = c.run()
    d = c.device()
    m = c.pool.shape[0]
    big = torch.empty((pages,) + c.pool.shape[1:], dtype=torch.uint8, device="cuda")
    big[pages - m:] = d["cache"]
    d["cache"] = big
    d["pages"] = torch.where(d["pages"] < m, d["pages"] + (pages - m), d["pages"])
    assert torch.equal(fgq.fgq_attn_kv(**d), want)


def test_runs_are_identical_and_replay_from_a_graph():
    c = Case([(3000, 1), (100, 1), (1700, 1)], 8, 2, 128, 16, 4, 64, torch.bfloat16, seed=10)
    d = c.device()
    a = fgq.fgq_attn_kv(**d)
    assert torch.equal(a, fgq.fgq_attn_kv(**d))
    nb = fgq.fgq_attn_kv_ws_bytes(3, 8, 2, 128, 3, 1, d["pages"].shape[1] * 16)
    ws = torch.empty(max(nb, 4), dtype=torch.uint8, device="cuda")
    o = torch.empty_like(d["q"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fgq.fgq_attn_kv(**d, o=o, ws=ws)
    for k in range(3):
        d["q"].copy_(torch.randn(d["q"].shape, generator=torch.Generator().manual_seed(k)))
        d["kv_lens"].copy_(torch.tensor([3000 - 500 * k, 100 + k, 1700], dtype=torch.int32))
        want = fgq.fgq_attn_kv(**d).clone()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), k


def test_refusals():
    c = Case([(40, 2)], 4, 2, 64, 16, 4, 32, torch.float16)
    d = c.device()
    for change, err in [
            (dict(q=d["q"].float()), fgq.FgqError), (dict(q=d["q"].double()), TypeError),
            (dict(q=d["q"][:, :3]), fgq.FgqError),                   # 3 query heads over 2 key heads
            (dict(q=d["q"].cpu()), ValueError), (dict(q=d["q"].transpose(1, 2)), ValueError),
            (dict(cu_q=d["cu_q"].long()), TypeError), (dict(cu_q=d["cu_q"][:1]), ValueError),
            (dict(max_q=3), fgq.FgqError),                          # more than there are tokens
            (dict(window=-1), fgq.FgqError), (dict(window=5, causal=False), fgq.FgqError),
            (dict(scale=float("nan")), fgq.FgqError), (dict(scale=0.0), fgq.FgqError),
            (dict(P=32), ValueError), (dict(G=64), ValueError), (dict(bits=8), ValueError),
            (dict(pages=d["pages"].long()), TypeError), (dict(pages=d["pages"][0]), ValueError),
            (dict(o=torch.empty(3, device="cuda", dtype=torch.float16)), ValueError),
            (dict(lse=torch.empty(3, device="cuda")), ValueError)]:
        with pytest.raises(err):
            fgq.fgq_attn_kv(**dict(d, **change))
    with pytest.raises(fgq.FgqError):  # 32 channels a head: written and read back, not attended
        c3 = Case([(40, 2)], 4, 2, 32, 16, 4, 32, torch.float16)
        c3.run()
    e = dict(d, q=d["q"][:0], cu_q=torch.zeros(2, dtype=torch.int32, device="cuda"), max_q=0)
    assert fgq.fgq_attn_kv(**e).shape == (0, 4, 64)

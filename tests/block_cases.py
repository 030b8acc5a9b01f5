"""Calls of the attention block's operators over their kernels' forms, for the
checking build (run as a script with FGQ_LIBRARY=check: writes every output and
the number of violations into a folder) and the run-twice test."""
import os
import sys

import numpy as np

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__))]


def run_cases(fgq, torch):
    out = {}
    r = np.random.default_rng(11)
    t = lambda a, dt=torch.float32: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()

    def keep(name, *xs):
        for i, x in enumerate(xs):
            v = x.contiguous()
            out[f"{name}_{i}"] = (v.view(torch.int16) if v.dtype is torch.bfloat16 else v).cpu().numpy()

    types = [torch.float32, torch.float16, torch.bfloat16]
    # every tile of the products, and the few-row forms with 1 to 4 row blocks (and two channel blocks), ragged
    for i, (M, K, O) in enumerate([(1, 333, 37), (7, 4100, 33), (13, 700, 65), (30, 1001, 77), (48, 512, 100),
                                   (61, 2049, 16), (70, 300, 1000), (300, 260, 2000), (700, 130, 1900),
                                   (1030, 200, 2100), (900, 3300, 700), (2100, 513, 3000), (3000, 300, 5000),
                                   (40, 260, 8200), (60, 1300, 9001)]):
        x, w, b = t(r.standard_normal((M, K)), types[i % 3]), t(r.standard_normal((O, K))), t(r.standard_normal(O))
        wq, sw = fgq.fgq_quantize_rows(w)
        keep(f"linear{i}", fgq.fgq_linear_i8(x, wq, sw, bias=b, dtype=types[(i + 1) % 3]))
        q, s = fgq.fgq_quantize_rows(x)
        keep(f"rows{i}", q, s, fgq.fgq_gemm_i8(q, s, K, wq, sw))
    # cache and attention
    layouts = [(64, 4, 32), (64, 8, 64), (128, 4, 128), (128, 4, 64), (128, 8, 32), (256, 4, 64), (256, 8, 128)]
    seqs = [[(700, 1), (0, 1), (33, 1)], [(100, 40), (20, 33)], [(300, 3), (5, 5)], [(3000, 1), (40, 1)],
            [(500, 140), (1, 1)], [(200, 90), (33, 70)] + [(b % 5, b % 2) for b in range(260)]]
    for i, (D, bits, G) in enumerate(layouts):
        for j, sq in enumerate(seqs):
            Hkv, ratio, P = 1 + (i + j) % 3, (1, 4, 3)[j % 3], (16, 32, 64, 128)[(i + j) % 4]
            maxp = max(1, max(-(-n // P) for n, _ in sq))
            pages = len(sq) * maxp + 1
            cache = fgq.fgq_kv_cache(pages, Hkv, D, P, bits, G)
            cache.zero_()
            table = r.permutation(pages)[:len(sq) * maxp].reshape(len(sq), maxp).astype(np.int32)
            slots = np.concatenate([table[b, np.arange(n) // P].astype(np.int64) * P + np.arange(n) % P
                                    for b, (n, _) in enumerate(sq)])
            kv = r.standard_normal((2, len(slots), Hkv, D))
            dt = types[(i + j) % 3]
            fgq.fgq_kv_write(t(kv[0], dt), t(kv[1], dt), t(slots, torch.int64), cache, P, bits, G)
            keep(f"cache{i}_{j}", cache, *fgq.fgq_kv_read(t(slots, torch.int64), cache, P, D, bits, G, dt))
            cu = np.concatenate([[0], np.cumsum([q for _, q in sq])])
            q = t(r.standard_normal((cu[-1], Hkv * ratio, D)), types[1 + (i + j) % 2])
            lse = torch.empty((cu[-1], Hkv * ratio), dtype=torch.float32, device="cuda")
            o = fgq.fgq_attn_kv(q, t(cu, torch.int32), max(n for _, n in sq), cache, t(table, torch.int32),
                                t([n for n, _ in sq], torch.int32), P, bits, G, window=(0, 50)[j % 2], lse=lse)
            keep(f"attn{i}_{j}", o, lse)
    torch.cuda.synchronize()
    return out


if __name__ == "__main__":
    import torch

    import paper_1705_01462_amd as lib
    print(lib.LIB_PATH, flush=True)
    lib.fgq_check_violations()
    got = run_cases(lib, torch)
    for k, v in got.items():
        np.save(os.path.join(sys.argv[1], k + ".npy"), v)
    with open(os.path.join(sys.argv[1], "violations.txt"), "w") as f:
        f.write(" ".join(str(v) for v in lib.fgq_check_violations()))

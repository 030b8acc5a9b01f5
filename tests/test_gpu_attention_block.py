"""GPU: the operators of a quantized attention block together, as
examples/attention_block.py runs them."""
import importlib.util
import os

import pytest
import torch

fgq = pytest.importorskip("paper_1705_01462_amd")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits,G,D", [(4, 64, 128), (8, 32, 64)])
def test_tokens_one_by_one_are_the_prompt(ex, bits, G, D):
    """Quantization is per token and group, so a sequence's cache is the same
    bytes whether its tokens come at once or one by one; the attention's outputs
    differ by the order of their sums alone: the fp16 rounding of a probability
    (2^-11 of an output's terms, which are of the order of the largest value)
    and the output's own rounding (2^-8), on both sides."""
    Hq, Hkv, E, P, counts = 8, 2, 256, 16, [37, 5, 18]
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    wqkv, wo = rnd((Hq + 2 * Hkv) * D, E) / 16, rnd(E, Hq * D) / 32
    x = [rnd(n, E).to(torch.bfloat16) for n in counts]
    caches, outs = [], []
    for chunks in ([counts], [[1 if s < n else 0 for n in counts] for s in range(max(counts))]):
        block = ex.AttentionBlock(wqkv, wo, Hq, Hkv, D, 8, P, bits, G)
        block.cache.zero_()
        pages = ex.Pages(8, len(counts), max(counts), P)
        # both runs own the same pages
        for b, n in enumerate(counts):
            for p in range(-(-n // P)):
                pages.table[b, p] = pages.free.pop()
        pages.free = None
        pages.extend = lambda c, pages=pages: _extend(pages, c)
        rows = [[] for _ in counts]
        for c in chunks:
            slots = pages.extend(c)
            cu, mq, pos, lens = ex.batch(c, pages.lens)
            xs = torch.cat([t[n - k:n] for t, k, n in zip(x, c, pages.lens)])
            o = block.attend(xs, pos, slots, cu, mq, pages.table, lens)
            for b, r in enumerate(o.split(c)):
                rows[b].append(r)
        caches.append(block.cache.clone())
        outs.append(torch.cat([torch.cat(r) for r in rows]).float())
    assert torch.equal(caches[0], caches[1])
    assert (outs[0] - outs[1]).abs().max() <= (2 * 2.0 ** -8 + 2 * 2.0 ** -11) * outs[0].abs().max() * 2


def _extend(pages, counts):
    slots = []
    owned = pages.table.tolist()
    for b, n in enumerate(counts):
        slots += [owned[b][t // pages.P] * pages.P + t % pages.P for t in range(pages.lens[b], pages.lens[b] + n)]
        pages.lens[b] += n
    return torch.tensor(slots, dtype=torch.int64, device="cuda")


def test_example_runs(ex):
    """8-bit products and a 4-bit cache in groups of 64: a code is off by half a
    step, a twelfth of a step's square on average; a group's range of 64 normal
    values is about 4.7 of their deviations, so keys and values are off by 0.09 of
    theirs, the output by that and, through the scores, by as much again."""
    assert ex.main() < 0.25

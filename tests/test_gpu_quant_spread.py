"""Decode over a cache in 8 bits in each of the ways its rows are spread over the blocks: which way a case takes is looked at by
test_paged_launches_host.py, without a GPU."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2502_01068_amd import binding as fk
from test_gpu_append import bits, dev, make_table
from test_gpu_quant import full_pools, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(max_total_tokens=4096, max_seqs=64)
    yield c
    c.close()


# tokens of the entries, heads, page, scale block, the kernel <rows cut apart, waves>, tiles of its longest block
UNEVEN = [
    ([400] * 15 + [16000] + [400] * 16, 32, 8, 16, 16, "<true, 8>", 32), ([0] * 11 + [300] * 20 + [9001], 8, 8, 64, 32, "<true, 8>", 16),
    ([500] * 40 + [20000] + [500] * 23, 32, 8, 16, 16, "<true, 4>", 29), ([7000, 0] + [515, 33] * 30, 16, 8, 32, 32, "<true, 4>", 17),
]
# rows of equal length that are not cut, entries of the same few sequences: a wave asks for its page entries three times, 32 tiles at a time
REFILL = [
    ([20000 - 3 * i for i in range(32)], 8, 8, 16, 16, "<true, 8>", 625), ([9000 - i for i in range(64)], 8, 8, 16, 16, "<true, 4>", 282),
    ([17000 - i for i in range(32)], 16, 8, 64, 64, "<true, 8>", 532),
]
# equal shares of the line of all tiles: blocks that go through several rows, rows that several blocks share, empty ones among them
SHARES = [
    ([4000 - 7 * i for i in range(20)], 32, 8, 16, 16, "<false, 8>", 78), ([60000] * 3 + [100, 0, 33] * 5 + [0, 1], 8, 4, 64, 32, "<false, 8>", 89),
    ([0, 2500, 50, 9000] * 12, 32, 8, 16, 16, "<false, 4>", 69), ([3000 - i for i in range(40)], 16, 8, 128, 64, "<false, 4>", 59),
    ([14000 - i for i in range(20)] + [0, 1], 8, 8, 16, 16, "<false, 8>", 274), ([0] + [12000 - i for i in range(40)], 8, 8, 32, 16, "<false, 4>", 235),
]


def check(ctx, ns, hq, hkv, page, block, distinct=None):
    """Entry b attends over the first ns[b] tokens of sequence b % distinct (its own one unless given).  Checked: the first entries, the last, the longest
    and shortest, each against 64 bits."""
    B, rng = len(ns), np.random.default_rng(sum(ns) + hq + page)
    lengths = [max(ns[b::distinct]) for b in range(distinct)] if distinct else ns
    table, n_pages = make_table(rng, lengths, page)
    table = table[np.arange(B) % len(lengths)]
    codes, scales = full_pools(rng, n_pages, hkv, page, block, powers=False)
    q = bits(rng, B, hq, 128)
    shape = fk.make_shape([8] * B, n_q_heads=hq, n_kv_heads=hkv)
    args = (shape, dev(q), *up((codes, scales)), torch.from_numpy(table).cuda(), ns)
    out = ctx.fkv_decode_attention_paged_quant(*args)
    assert torch.equal(out, ctx.fkv_decode_attention_paged_quant(*args))
    o = out.cpu().numpy()
    assert np.isfinite(o).all() and not o[np.array(ns) == 0].any()
    off = lambda b, row: np.abs(o[b] - (ref := paged.attend(paged.bf16_to_f64(q[b]), *(paged.dequant(c, s, row, ns[b]) for c, s in zip(codes, scales)),
                                                            128 ** -0.5))[0]) - ref[1]
    for b in sorted({0, 1, B - 1, int(np.argmax(ns)), int(np.argmin(ns))}):
        assert (off(b, table[b]) <= 0).all(), (b, ns[b])
    return off, table


@pytest.mark.parametrize("ns,hq,hkv,page,block,kernel,tiles", UNEVEN)
def test_a_long_sequence_among_short_ones(ctx, ns, hq, hkv, page, block, kernel, tiles):
    print("case: quant decode uneven %d x %d, heads=%d/%d page=%d block=%d" % (len(ns), max(ns), hq, hkv, page, block), flush=True)
    check(ctx, ns, hq, hkv, page, block)


@pytest.mark.parametrize("ns,hq,hkv,page,block,kernel,tiles", REFILL)
def test_many_tiles_of_a_wave(ctx, ns, hq, hkv, page, block, kernel, tiles):
    """A page read in place of another, in tiles behind a wave's first 32 or 64, would be seen: the oracle's result with it is out of bounds."""
    print("case: quant decode long rows %d x %d, heads=%d/%d page=%d block=%d" % (len(ns), max(ns), hq, hkv, page, block), flush=True)
    off, table = check(ctx, ns, hq, hkv, page, block, distinct=3)
    waves = int(kernel[-2])
    for first in (32, 64):  # tokens of the wave's tile with that number
        wrong, at = table[0].copy(), first * waves * 32 // page
        wrong[at] = wrong[at + 1]
        assert at + 1 < ns[0] // page and (off(0, wrong) > 0).any(), first


@pytest.mark.parametrize("ns,hq,hkv,page,block,kernel,tiles", SHARES)
def test_equal_shares(ctx, ns, hq, hkv, page, block, kernel, tiles):
    print("case: quant decode equal shares %d x %d, heads=%d/%d page=%d block=%d" % (len(ns), max(ns), hq, hkv, page, block), flush=True)
    check(ctx, ns, hq, hkv, page, block, distinct=2)


@pytest.mark.parametrize("k_exp,v_exp", [(-8, -80), (-8, 79), (-126, 0), (-4, 0)])
def test_scales_at_the_edges(ctx, k_exp, v_exp):
    """Scales of either sign, not powers of two, as small and as large as they may be: within the bound of fp32 sums."""
    print("case: quant decode, scales about 2^%d (K), 2^%d (V)" % (k_exp, v_exp), flush=True)
    rng, ns = np.random.default_rng(abs(v_exp - k_exp)), [700, 40]
    table, n_pages = make_table(rng, ns, 16)
    codes, scales = full_pools(rng, n_pages, 8, 16, 16)
    scales = [(np.ldexp(rng.uniform(1, 2, s.shape), e) * rng.choice([-1, 1], s.shape)).astype(np.float32) for s, e in zip(scales, (k_exp, v_exp))]
    q = bits(rng, 2, 32, 128)
    out = ctx.fkv_decode_attention_paged_quant(fk.make_shape([8, 8]), dev(q), *up((codes, scales)), torch.from_numpy(table).cuda(), ns).cpu().numpy()
    for b, n in enumerate(ns):
        want, bound = paged.attend(paged.bf16_to_f64(q[b]), *(paged.dequant(c, s, table[b], n) for c, s in zip(codes, scales)), 128 ** -0.5)
        assert (np.abs(out[b] - want) <= bound).all(), (b, (np.abs(out[b] - want) / bound).max())


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_scales_that_are_not_finite(ctx, which, value):
    """NaN in the outputs of the block's head, and nowhere else."""
    rng, ns = np.random.default_rng(50), [70, 300]
    shape = fk.make_shape([8, 8], n_q_heads=8, n_kv_heads=4)
    table, n_pages = make_table(rng, ns, 16)
    codes, scales = full_pools(rng, n_pages, 4, 16, 16)
    q, tab = dev(bits(rng, 2, 8, 128)), torch.from_numpy(table).cuda()
    clean = ctx.fkv_decode_attention_paged_quant(shape, q, *up((codes, scales)), tab, ns)
    scales[which][table[1][18], 3, 0] = value  # tokens 288 .. 299 of sequence 1, head 3
    out = ctx.fkv_decode_attention_paged_quant(shape, q, *up((codes, scales)), tab, ns)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[1, 6:8] = True
    assert torch.equal(out.isnan(), bad) and torch.equal(out[~bad], clean[~bad])

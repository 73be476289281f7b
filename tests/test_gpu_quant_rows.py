"""What the calls that fill a cache in 8 bits store: keys turned in every form of the embedding, K gathered alone, blocks that a gather puts
nothing into.  Against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2502_01068_amd import binding as fk
from parity import host_bits
from test_gpu_append import bits, dev, make_table, turned_close
from test_gpu_quant import keys_close, noise_pools, same, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(max_total_tokens=8192, max_seqs=8)
    yield c
    c.close()


def pair_sizes(x, rotary, inter):
    """|a| + |b| of a column's pair, 0 where nothing is turned."""
    size = np.zeros_like(x)
    one, two = (slice(0, rotary, 2), slice(1, rotary, 2)) if inter else (slice(0, rotary // 2), slice(rotary // 2, rotary))
    size[..., one] = size[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    return size


@pytest.mark.parametrize("rotary", [16, 64, 96, 128])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("page,block,hq,hkv", [(16, 16, 32, 8), (64, 32, 12, 4), (64, 64, 2, 2)])
def test_turned_keys(ctx, rotary, inter, page, block, hq, hkv):
    """The second call joins a block that tokens are in, of rows that are four times as large."""
    print("case: quant append rotary=%d %s page=%d block=%d heads=%d/%d" % (rotary, inter, page, block, hq, hkv), flush=True)
    rng = np.random.default_rng(rotary + block + inter)
    shape = fk.make_shape([8, 8], n_q_heads=hq, n_kv_heads=hkv)
    table, n_pages = make_table(rng, [95, 40], page)
    codes, scales = noise_pools(rng, n_pages, hkv, page, block)
    got, tab = up((codes, scales)), torch.from_numpy(table).cuda()
    freq = 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    rope = fk.make_rope(rotary, inv_freq=freq, interleaved=inter)
    for start, new, size in (([0, 0], [83, 5], 1.0), ([83, 5], [12, 35], 4.0)):
        total = sum(new)
        rows = dev(bits(rng, total, hq + 2 * hkv, 128)) * size
        x, positions = paged.bf16_to_f64(host_bits(rows)), rng.integers(-(1 << 20), 1 << 20, total).astype(np.int32)
        k, v = x[:, hq:hq + hkv], x[:, hq + hkv:]
        q = ctx.fkv_append_kv_paged_quant(shape, rows[:, hq:hq + hkv], rows[:, hq + hkv:], start, new, tab, *got, rope=rope,
                                          positions=torch.from_numpy(positions).cuda(), q=rows[:, :hq])
        turned_close(host_bits(q).reshape(total, hq, 128), x[:, :hq], positions, freq, inter)
        turned, at, where = paged.rope(k, positions, freq, inter), 0, []
        for b, n in enumerate(new):
            for i, rows64 in enumerate((turned, v)):
                paged.append_quant(codes[i], scales[i], rows64[at:at + n], start[b], table[b])
            where += [(table[b][(start[b] + j) // page], (start[b] + j) % page) for j in range(n)]
            at += n
        keys_close(got, codes[0], scales[0], (turned, pair_sizes(k, rotary, inter)), where, block)
        same([got[1], got[3]], [codes[1]], [scales[1]])
        codes[0][:] = got[0].cpu().numpy()


def gather64(codes, scales, x, idx, lengths, budget, table):
    row = at = 0
    for b, n in enumerate(lengths):
        own = idx[:, at:at + budget[b]].T
        rows = paged.bf16_to_f64(x[row:row + n])[np.maximum(own, 0), np.arange(x.shape[1])]
        paged.append_quant(codes, scales, rows, 0, table[b], own >= 0)
        row, at = row + n, at + budget[b]


@pytest.mark.parametrize("lengths,budget,hkv,page,block", [([700], [100], 8, 16, 16), ([300, 2000], [9, 513], 4, 64, 32), ([90, 90], [16, 90], 3, 128, 64)])
def test_keys_gathered_alone(ctx, lengths, budget, hkv, page, block):
    """Codes with their signs, scales, and what has to stay as it was."""
    print("case: quant gather of K, lengths=%s budget=%s hkv=%d page=%d block=%d" % (lengths, budget, hkv, page, block), flush=True)
    rng = np.random.default_rng(sum(budget) + page)
    shape, k = fk.make_shape(lengths, n_q_heads=hkv, n_kv_heads=hkv), bits(rng, sum(lengths), hkv, 128)
    table, n_pages = make_table(rng, budget, page)
    (codes, _), (scales, _) = noise_pools(rng, n_pages, hkv, page, block)
    idx = np.concatenate([np.stack([np.sort(rng.choice(n, b, replace=False)) for _ in range(hkv)]) for n, b in zip(lengths, budget)], 1).astype(np.int32)
    idx[0, 2:4] = -1
    pools = [torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()]
    res = ctx.fkv_gather_kv_paged_quant(shape, dev(k), None, torch.from_numpy(idx).cuda(), budget, torch.from_numpy(table).cuda(), pools[0], None,
                                        pools[1], None)
    assert res[1] is None and res[3] is None
    gather64(codes, scales, k, idx, lengths, budget, table)
    same(pools, [codes], [scales])


@pytest.mark.parametrize("page,block", [(16, 16), (64, 32), (64, 64)])
def test_appending_behind_rows_that_are_not_there(ctx, page, block):
    """A head's block of nothing but negative indices counts as filled, so what is appended behind must not meet the scale that memory held."""
    print("case: quant gather of no rows, append behind, page=%d block=%d" % (page, block), flush=True)
    rng = np.random.default_rng(page + block)
    lengths, budget, hkv = [200, 100], [2 * block + 5, 9], 4
    shape = fk.make_shape(lengths, n_q_heads=hkv, n_kv_heads=hkv)
    k, v = bits(rng, 300, hkv, 128), bits(rng, 300, hkv, 128)
    table, n_pages = make_table(rng, [b + 8 for b in budget], page)
    codes, _ = noise_pools(rng, n_pages, hkv, page, block)
    scales = [np.full((n_pages, hkv, page // block), 1e30, np.float32) for _ in range(2)]
    got, tab = up((codes, scales)), torch.from_numpy(table).cuda()
    idx = np.concatenate([np.stack([np.sort(rng.choice(n, b, replace=False)) for _ in range(hkv)]) for n, b in zip(lengths, budget)], 1).astype(np.int32)
    idx[1] = -1                               # all of a head
    idx[2, block:sum(budget)] = -1            # of the first sequence all but its first block, the second sequence
    ctx.fkv_gather_kv_paged_quant(shape, dev(k), dev(v), torch.from_numpy(idx).cuda(), budget, tab, *got)
    for i, x in enumerate((k, v)):
        gather64(codes[i], scales[i], x, idx, lengths, budget, table)
    assert scales[0][table[0][0], 1, 0] == 2.0 ** -126
    same(got, codes, scales)
    new = bits(rng, 9, 2 * hkv, 128)
    ctx.fkv_append_kv_paged_quant(shape, dev(new)[:, :hkv], dev(new)[:, hkv:], budget, [8, 1], tab, *got)
    x = paged.bf16_to_f64(new)
    for i, rows in enumerate((x[:, :hkv], x[:, hkv:])):
        paged.append_quant(codes[i], scales[i], rows[:8], budget[0], table[0])
        paged.append_quant(codes[i], scales[i], rows[8:], budget[1], table[1])
    same(got, codes, scales)
    for at, row in ((budget[0], 0), (budget[1], 8)):  # the tokens are there, within half a step of a scale that is theirs
        p, s = table[0 if row < 8 else 1][at // page], at % page
        v64 = paged.e4m3_decode(got[0].cpu().numpy()[p, :, s]) * got[2].cpu().numpy()[p, :, s // block][:, None].astype(np.float64)
        assert (np.abs(v64 - x[row, :hkv]) <= np.abs(x[row, :hkv]) * 2.0 ** -4 + got[2].cpu().numpy()[p, :, s // block][:, None] * 2.0 ** -10).all()

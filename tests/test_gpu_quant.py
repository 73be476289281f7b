"""The paged cache in 8 bits: what the writing calls store and what decoding over it gives, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2502_01068_amd import binding as fk
from parity import host_bits
from test_gpu_append import bits, dev, make_table, turned_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(max_total_tokens=40000, max_seqs=64)
    yield c
    c.close()


def noise_pools(rng, n_pages, hkv, page, block):
    """Pools as memory comes: every code, NaN among them, and scales of any kind."""
    codes = [rng.integers(0, 256, (n_pages, hkv, page, 128)).astype(np.uint8) for _ in range(2)]
    scales = [rng.choice([np.nan, 1.0, -3.0, 1e30], (n_pages, hkv, page // block)).astype(np.float32) for _ in range(2)]
    return codes, scales


def up(pools):
    codes, scales = pools
    return [torch.from_numpy(c).cuda() for c in codes] + [torch.from_numpy(s).cuda() for s in scales]


def same(got, codes, scales):
    for g, want in zip(got, codes + scales):
        g = g.cpu().numpy()
        if want.dtype == np.uint8:  # the two NaN codes say the same
            g, want = np.where(g & 127 == 127, 127, g), np.where(want & 127 == 127, 127, want)
        np.testing.assert_array_equal(g, want)


def keys_close(got, want_codes, want_scale, exact, where, block):
    """Turned keys: the scale is the oracle's (the largest values are not within 2^-20 of a border), and a code stands for the exact
    value within half a step (2^-4 of it, or half of the smallest step) and what fp32 and the angles make of it (2^-20 of the pair)."""
    codes, scales = got[0].cpu().numpy(), got[2].cpu().numpy()
    np.testing.assert_array_equal(scales, want_scale)
    touched = np.zeros(codes.shape[:3], bool)
    for (page, slot), x, size in zip(where, exact[0], exact[1]):
        s = scales[page, :, slot // block][:, None].astype(np.float64)
        off = size * 2.0 ** -20
        v = paged.e4m3_decode(codes[page, :, slot]) * s
        assert (np.abs(v - x) <= (np.abs(x) + off) * 2.0 ** -4 + s * 2.0 ** -10 + off).all()
        touched[page, :, slot] = True
    np.testing.assert_array_equal(np.where(touched[..., None], 0, codes), np.where(touched[..., None], 0, want_codes))


@pytest.mark.parametrize("steps,hq,hkv,page,block", [
    ([[(0, 1)], [(1, 1)], [(2, 15)], [(17, 1)]], 32, 8, 16, 16),
    ([[(0, 100), (0, 0), (0, 5)], [(100, 29), (0, 64), (5, 1)], [(129, 1), (64, 1), (6, 70)]], 28, 4, 64, 32),
    ([[(0, 63)], [(63, 1)], [(64, 200)], [(264, 1)]], 8, 1, 128, 64),
    ([[(0, 17), (0, 16)], [(17, 1), (16, 3)]], 64, 8, 32, 16),
])
@pytest.mark.parametrize("turn", [False, True])
def test_appending_in_steps(ctx, steps, hq, hkv, page, block, turn):
    print("case: quant append %s heads=%d/%d page=%d block=%d turn=%s" % (steps, hq, hkv, page, block, turn), flush=True)
    rng = np.random.default_rng(page + block + len(steps) + hq)
    B = len(steps[0])
    shape = fk.make_shape([8] * B, n_q_heads=hq, n_kv_heads=hkv)
    table, n_pages = make_table(rng, [s + n for s, n in steps[-1]], page)
    codes, scales = noise_pools(rng, n_pages, hkv, page, block)
    got, tab = up((codes, scales)), torch.from_numpy(table).cuda()
    freq = 10000.0 ** (-np.arange(0, 64, 2) / 64)
    for i, step in enumerate(steps):
        start, new = [s for s, _ in step], [n for _, n in step]
        total = sum(new)
        # sizes that differ from step to step and head to head: scales grow, by much and not at all; a whole block of zeros is among them
        rows = paged.bf16_to_f64(bits(rng, total, hq + 2 * hkv, 128)) * 4.0 ** ((i * 5) % 3) * np.ldexp(1.0, rng.integers(-3, 4, (1, hq + 2 * hkv, 1)))
        rows[:, hq] *= 0.0 if i == 0 else 1.0
        t = torch.from_numpy(rows.astype(np.float32)).to(torch.bfloat16).cuda()
        x = paged.bf16_to_f64(host_bits(t))
        positions = rng.integers(0, 1 << 20, total).astype(np.int32)
        kw = dict(rope=fk.make_rope(64, inv_freq=freq), positions=torch.from_numpy(positions).cuda(), q=t[:, :hq]) if turn else {}
        before = [g.clone() for g in got]
        out = ctx.fkv_append_kv_paged_quant(shape, t[:, hq:hq + hkv], t[:, hq + hkv:], start, new, tab, *got, **kw)
        k, v = x[:, hq:hq + hkv], x[:, hq + hkv:]
        if turn:
            turned_close(host_bits(out).reshape(total, hq, 128), x[:, :hq], positions, freq, False)
            k = paged.rope(k, positions, freq)
            size = np.abs(x[:, hq:hq + hkv])
            size = np.concatenate([np.tile(size[..., :32] + size[..., 32:64], 2), np.zeros_like(size[..., 64:])], -1)
        at, where = 0, []
        for b in range(B):
            for xs, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
                paged.append_quant(c, s, xs[at:at + new[b]], start[b], table[b])
            where += [(table[b][(start[b] + j) // page], (start[b] + j) % page) for j in range(new[b])]
            at += new[b]
        if turn:
            keys_close(got, codes[0], scales[0], (k, size), where, block)
            codes[0][:] = got[0].cpu().numpy()  # the next step begins from what the call stored
            same([got[1], got[3]], [codes[1]], [scales[1]])
        else:
            same(got, codes, scales)
        # a second call of the same tokens changes nothing more
        again = [g.clone() for g in got]
        ctx.fkv_append_kv_paged_quant(shape, t[:, hq:hq + hkv], t[:, hq + hkv:], start, new, tab, *got, **kw)
        assert all(torch.equal(a.view(torch.uint8), g.view(torch.uint8)) for a, g in zip(again, got))
        assert not all(torch.equal(a.view(torch.uint8), g.view(torch.uint8)) for a, g in zip(before, got)) or total == 0


def test_what_is_not_finite_poisons_itself_only(ctx):
    rng = np.random.default_rng(20)
    shape = fk.make_shape(8, n_q_heads=2, n_kv_heads=2)
    x = paged.bf16_to_f64(bits(rng, 40, 2, 128))
    x[3, 0, 5], x[7, 1, 100], x[20, 0, 0], x[33, :, :] = np.inf, np.nan, -np.inf, np.inf
    x[25, 0, 9] = 3.38e38  # finite, and the block's other values vanish beside it
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()
    x = paged.bf16_to_f64(host_bits(t))
    table = np.array([[0, 2, 1]], np.int32)
    codes, scales = noise_pools(rng, 3, 2, 16, 16)
    got = up((codes, scales))
    ctx.fkv_append_kv_paged_quant(shape, t, t, 0, 40, torch.from_numpy(table).cuda(), *got)
    for c, s in zip(codes, scales):
        paged.append_quant(c, s, x, 0, table[0])
    same(got, codes, scales)
    assert np.isfinite(scales[0][:, :, 0]).all()


@pytest.mark.parametrize("lengths,budget,hkv,page,block", [
    ([700], [100], 8, 16, 16), ([300, 2000, 64], [9, 513, 64], 4, 64, 32), ([1500], [1000], 1, 128, 64), ([90, 90], [16, 90], 3, 32, 32),
])
def test_gather(ctx, lengths, budget, hkv, page, block):
    print("case: quant gather lengths=%s budget=%s hkv=%d page=%d block=%d" % (lengths, budget, hkv, page, block), flush=True)
    rng = np.random.default_rng(sum(lengths) + page)
    shape = fk.make_shape(lengths, n_q_heads=hkv, n_kv_heads=hkv)
    k, v = bits(rng, sum(lengths), hkv, 128), bits(rng, sum(lengths), hkv, 128)
    table, n_pages = make_table(rng, budget, page)
    codes, scales = noise_pools(rng, n_pages, hkv, page, block)
    idx = np.concatenate([np.stack([np.sort(rng.choice(n, b, replace=False)) for _ in range(hkv)]) for n, b in zip(lengths, budget)], 1).astype(np.int32)
    idx[0, 3:5] = -1   # the mark of a failed selection: nothing is written
    idx[-1, 0:8] = -1
    got = up((codes, scales))
    ctx.fkv_gather_kv_paged_quant(shape, dev(k), dev(v), torch.from_numpy(idx).cuda(), budget, torch.from_numpy(table).cuda(), *got)
    row, at = 0, 0
    for b, n in enumerate(lengths):
        own = idx[:, at:at + budget[b]].T
        for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
            rows = paged.bf16_to_f64(x[row:row + n])[np.maximum(own, 0), np.arange(hkv)]
            paged.append_quant(c, s, rows, 0, table[b], own >= 0)
        row, at = row + n, at + budget[b]
    same(got, codes, scales)
    fresh = up(noise_pools(rng, n_pages, hkv, page, block))  # K alone
    keep = fresh[1].clone()
    ctx.fkv_gather_kv_paged_quant(shape, dev(k), None, torch.from_numpy(idx).cuda(), budget, torch.from_numpy(table).cuda(), fresh[0], None, fresh[2], None)
    assert torch.equal(fresh[1], keep)
    put = codes[0].copy()
    for b in range(len(lengths)):  # rows that hold kept tokens
        for t in range(budget[b]):
            p = table[b][t // page]
            sel = idx[:, sum(budget[:b]) + t] >= 0
            assert (np.where(sel[:, None], fresh[0].cpu().numpy()[p, :, t % page], put[p, :, t % page]) & 127 == put[p, :, t % page] & 127).all()


def test_gather_indices_repeat_and_run_over(ctx):
    """An index twice is a row twice; one beyond its sequence is clamped into it, as by the other gathers."""
    rng = np.random.default_rng(31)
    shape = fk.make_shape([40, 30], n_q_heads=2, n_kv_heads=2)
    k = bits(rng, 70, 2, 128)
    idx = np.stack([[3, 3, 3, 39, 40, 1000, 0, 7, 2 ** 31 - 1, 29, 30, 0, 0, 5, 6, 6]] * 2).astype(np.int32)
    table = np.array([[0], [1]], np.int32)
    codes, scales = noise_pools(rng, 2, 2, 16, 16)
    got = up((codes, scales))
    ctx.fkv_gather_kv_paged_quant(shape, dev(k), dev(k), torch.from_numpy(idx).cuda(), 8, torch.from_numpy(table).cuda(), *got)
    for c, s in zip(codes, scales):
        for b, (row, n) in enumerate(((0, 40), (40, 30))):
            own = np.minimum(idx[:, 8 * b:8 * b + 8].T, n - 1)
            paged.append_quant(c, s, paged.bf16_to_f64(k[row:row + n])[own, np.arange(2)], 0, table[b])
    same(got, codes, scales)


def test_pages_outside_the_pool(ctx):
    rng = np.random.default_rng(30)
    shape = fk.make_shape(64, n_q_heads=2, n_kv_heads=2)
    k = bits(rng, 64, 2, 128)
    table = np.array([[1, -5, 3, 0]], np.int32)
    codes, scales = noise_pools(rng, 3, 2, 16, 16)
    got = up((codes, scales))
    tab, x = torch.from_numpy(table).cuda(), paged.bf16_to_f64(k)
    ctx.fkv_append_kv_paged_quant(shape, dev(k)[:48], dev(k)[:48], 16, 48, tab, *got)
    for c, s in zip(codes, scales):
        paged.append_quant(c, s, x[:48], 16, table[0])
    same(got, codes, scales)
    idx = torch.arange(64, dtype=torch.int32, device="cuda").repeat(2, 1)
    ctx.fkv_gather_kv_paged_quant(shape, dev(k), dev(k), idx, 64, tab, *got)
    for c, s in zip(codes, scales):
        paged.append_quant(c, s, x, 0, table[0])
    same(got, codes, scales)


def full_pools(rng, n_pages, hkv, page, block, powers=True):
    codes = [rng.integers(0, 254, (n_pages, hkv, page, 128)).astype(np.uint8) for _ in range(2)]
    codes = [np.where(c & 127 >= 120, c & 0x87, c).astype(np.uint8) for c in codes]  # no NaN, no value over 240
    size = np.ldexp(1.0, rng.integers(-9, -5, (2, n_pages, hkv, page // block)))
    return codes, list((size if powers else size * rng.uniform(0.6, 1.7, size.shape)).astype(np.float32))


def check_decode(ctx, rng, ns, hq, hkv, page, block, scale=0.0, powers=True, poison=True):
    B = len(ns)
    shape = fk.make_shape([8] * B, n_q_heads=hq, n_kv_heads=hkv, softmax_scale=scale)
    table, n_pages = make_table(rng, ns, page)
    codes, scales = full_pools(rng, n_pages, hkv, page, block, powers)
    if poison:  # whatever lies behind a sequence's end, its codes' NaN and its scales' too, has no part in the result
        used = np.zeros((n_pages, page), bool)
        for b, n in enumerate(ns):
            t = np.arange(n)
            used[table[b][t // page], t % page] = True
        for c in codes:
            c[np.broadcast_to(~used[:, None, :, None], c.shape)] = 0x7F
        for s in scales:
            s[np.broadcast_to(~used.reshape(n_pages, 1, -1, block).any(-1), s.shape)] = np.nan
    q = bits(rng, B, hq, 128)
    got = up((codes, scales))
    out = ctx.fkv_decode_attention_paged_quant(shape, dev(q), *got, torch.from_numpy(table).cuda(), ns)
    assert out.dtype == torch.float32
    o = out.cpu().numpy()
    for b, n in enumerate(ns):
        k, v = (paged.dequant(c, s, table[b], n) for c, s in zip(codes, scales))
        want, bound = paged.attend(paged.bf16_to_f64(q[b]), k, v, scale or 128 ** -0.5)
        assert (np.abs(o[b] - want) <= bound).all(), (b, n, np.abs(o[b] - want).max(), bound.min())
    return got, table, q, out, shape


@pytest.mark.parametrize("ns,hq,hkv,page,block,scale", [
    ([1], 32, 8, 16, 16, 0.0), ([0], 32, 8, 16, 16, 0.0), ([15, 0, 16, 17], 32, 8, 16, 16, 0.0), ([31, 32, 33], 64, 8, 32, 16, 0.0),
    ([63, 64, 65, 1], 28, 4, 64, 64, 0.0), ([127, 129, 128], 8, 8, 128, 32, 0.25), ([1000], 7, 1, 256, 64, 0.0), ([2048], 32, 8, 16, 16, 0.0),
    ([500, 3, 2049], 12, 4, 16, 16, 0.0), ([12000], 32, 8, 64, 32, 0.0), ([9001, 300], 64, 8, 16, 16, 0.01), ([333] * 7, 15, 5, 32, 32, 0.0),
])
def test_decode(ctx, ns, hq, hkv, page, block, scale):
    print("case: quant decode n=%s heads=%d/%d page=%d block=%d scale=%g" % (ns, hq, hkv, page, block, scale), flush=True)
    check_decode(ctx, np.random.default_rng(sum(ns) + hq + page), ns, hq, hkv, page, block, scale, powers=page != 32)


@pytest.mark.parametrize("seed", range(4))
def test_decode_batches(ctx, seed):
    """Every way of spreading rows over the blocks: many short rows, a long one among them, empty ones, few."""
    rng = np.random.default_rng(100 + seed)
    ns = [[0, 700, 0, 90] * 16, list(rng.integers(0, 400, 40)) + [9000], [5000] + [0] * 3, list(rng.integers(600, 1200, 33))][seed]
    ns = [int(n) for n in ns]
    print("case: quant decode batch n=%s" % ns, flush=True)
    check_decode(ctx, rng, ns, 32, 8, 16, 16)


def test_decode_entries_may_share_pages(ctx):
    """Several queries of one sequence, each with the tokens that it sees: entries with the same table row; as one by one."""
    rng = np.random.default_rng(40)
    table, n_pages = make_table(rng, [900], 32)
    codes, scales = full_pools(rng, n_pages, 8, 32, 32)
    pools, q = up((codes, scales)), bits(rng, 5, 32, 128)
    ns = [896, 897, 1, 899, 900]
    out = ctx.fkv_decode_attention_paged_quant(fk.make_shape([8] * 5), dev(q), *pools, torch.from_numpy(np.repeat(table, 5, 0)).cuda(), ns)
    for i, n in enumerate(ns):
        k, v = (paged.dequant(c, s, table[0], n) for c, s in zip(codes, scales))
        want, bound = paged.attend(paged.bf16_to_f64(q[i]), k, v, 128 ** -0.5)
        assert (np.abs(out[i].cpu().numpy() - want) <= bound).all()


def test_decode_poison_stays_in_its_head(ctx):
    """NaN in a valid token's key or value: NaN in the outputs that it enters, and nowhere else."""
    rng = np.random.default_rng(41)
    ns, hkv = [70, 300], 4
    shape = fk.make_shape([8, 8], n_q_heads=8, n_kv_heads=hkv)
    table, n_pages = make_table(rng, ns, 16)
    codes, scales = full_pools(rng, n_pages, hkv, 16, 16)
    q, tab = dev(bits(rng, 2, 8, 128)), torch.from_numpy(table).cuda()
    clean = ctx.fkv_decode_attention_paged_quant(shape, q, *up((codes, scales)), tab, ns)
    codes[0][table[0][4], 2, 5, 77] = 0xFF   # key of token 69 of sequence 0, head 2
    codes[1][table[1][18], 1, 11, 3] = 0x7F  # value of token 299 of sequence 1, head 1, column 3
    out = ctx.fkv_decode_attention_paged_quant(shape, q, *up((codes, scales)), tab, ns)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 4:6] = True
    bad[1, 2:4, 3] = True
    assert torch.equal(out.isnan(), bad) and torch.equal(out[~bad], clean[~bad])


def test_decode_entries_outside_the_pool_are_clamped(ctx):
    rng = np.random.default_rng(42)
    shape = fk.make_shape(8, n_q_heads=4, n_kv_heads=2)
    pools = up(full_pools(rng, 3, 2, 16, 16))
    q = dev(bits(rng, 1, 4, 128))
    a = ctx.fkv_decode_attention_paged_quant(shape, q, *pools, torch.tensor([[1, -9, 77]], dtype=torch.int32, device="cuda"), 40)
    b = ctx.fkv_decode_attention_paged_quant(shape, q, *pools, torch.tensor([[1, 0, 2]], dtype=torch.int32, device="cuda"), 40)
    assert torch.equal(a, b)


def test_float8_tensors_and_a_given_output(ctx):
    rng = np.random.default_rng(43)
    got, table, q, out, shape = check_decode(ctx, rng, [90, 200], 32, 8, 16, 16, poison=False)
    given = torch.full((2, 32, 128), 7.0, device="cuda")
    k, v, ks, vs = got
    res = ctx.fkv_decode_attention_paged_quant(shape, dev(q), k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs,
                                               torch.from_numpy(table).cuda(), [90, 200], out=given)
    assert res is given and torch.equal(res, out)

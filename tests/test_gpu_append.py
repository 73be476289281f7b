"""New tokens into a bf16 paged cache, keys and queries turned on the way, against the 64-bit oracle."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2502_01068_amd import binding as fk
from parity import host_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(max_total_tokens=4096, max_seqs=8)
    yield c
    c.close()


def make_table(rng, counts, page, spare=3):
    need = [-(-c // page) for c in counts]
    n_pages = sum(need) + spare
    perm = rng.permutation(n_pages)
    table = np.full((len(counts), max(max(need), 1) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, n_pages


def bits(rng, *shape):
    return (torch.from_numpy(rng.normal(size=shape).astype(np.float32)).to(torch.bfloat16)).view(torch.int16).numpy().view(np.uint16)


def dev(b):
    return torch.from_numpy(b.view(np.int16)).cuda().view(torch.bfloat16)


def turned_close(got_bits, x, positions, freq, inter):
    """A stored value is the turned one, off by sine and cosine (2^-22 each) and fp32 products (2^-23 of the row pair's size), rounded
    once to bf16 (2^-8 of the value)."""
    want = paged.rope(x, positions, freq, inter)
    got = paged.bf16_to_f64(got_bits)
    r = 2 * len(freq)
    size = np.abs(x).copy()
    one, two = (slice(0, r, 2), slice(1, r, 2)) if inter else (slice(0, r // 2), slice(r // 2, r))
    size[..., one] = size[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    off = size * 2.0 ** -20
    off[..., r:] = 0
    assert (np.abs(got - want) <= (np.abs(want) + off) * 2.0 ** -8 * (np.arange(x.shape[-1]) < r) + off).all()


@pytest.mark.parametrize("start,new,hq,hkv,page,rotary,inter,span", [
    ([5], [1], 32, 8, 16, 128, False, 100), ([0], [1], 8, 1, 1, 128, True, 10), ([16], [33], 28, 4, 16, 64, False, 2000000000),
    ([3, 0, 40, 7], [0, 5, 1, 17], 32, 8, 32, 128, True, 1 << 20), ([100, 9], [300, 251], 64, 8, 64, 96, False, 131072),
    ([2], [129], 12, 3, 8, 16, True, 5000), ([31, 1, 0], [2, 0, 0], 5, 5, 256, 48, False, 77),
])
@pytest.mark.parametrize("fused", [True, False])
def test_append_turns_and_places(ctx, start, new, hq, hkv, page, rotary, inter, span, fused):
    print("case: append start=%s new=%s heads=%d/%d page=%d rotary=%d %s fused=%s" % (start, new, hq, hkv, page, rotary, inter, fused), flush=True)
    rng = np.random.default_rng(sum(start) + 7 * sum(new) + page)
    total, B = sum(new), len(start)
    shape = fk.make_shape([8] * B, n_q_heads=hq, n_kv_heads=hkv)
    rows = bits(rng, total, hq + 2 * hkv, 128)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    f = dev(rows)
    fq, fk_, fv = f[:, :hq], f[:, hq:hq + hkv], f[:, hq + hkv:]
    if not fused:
        fq, fk_, fv = fq.contiguous(), fk_.contiguous(), fv.contiguous()
    table, n_pages = make_table(rng, [s + n for s, n in zip(start, new)], page)
    kp, vp = bits(rng, n_pages, page, hkv, 128), bits(rng, n_pages, page, hkv, 128)
    dkp, dvp, tab = dev(kp), dev(vp), torch.from_numpy(table).cuda()
    positions = rng.integers(-span, span, total).astype(np.int32)
    freq = 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    rope = fk.make_rope(rotary, inv_freq=freq, interleaved=inter)
    out = ctx.fkv_append_kv_paged(shape, fk_, fv, start, new, tab, dkp, dvp, rope=rope, positions=torch.from_numpy(positions).cuda(), q=fq)
    assert out.shape == (total, hq, 128) and out.is_contiguous()
    turned_close(host_bits(out).reshape(total, hq, 128), paged.bf16_to_f64(q), positions, freq, inter)
    # slots: V bit for bit, K turned, all others as they were
    got_k, got_v, want_v, mark = host_bits(dkp), host_bits(dvp), vp.copy(), kp.copy()
    at = 0
    for b in range(B):
        paged.append_pages(want_v, v[at:at + new[b]], start[b], table[b])
        paged.append_pages(mark, np.zeros((new[b], hkv, 128), np.uint16), start[b], table[b])
        for i in range(new[b]):
            t = start[b] + i
            page_no, slot = table[b][t // page], t % page
            turned_close(got_k[page_no, slot][None], paged.bf16_to_f64(k[at + i])[None], positions[at + i:at + i + 1], freq, inter)
            got_k[page_no, slot] = 0
        at += new[b]
    np.testing.assert_array_equal(got_v, want_v)
    np.testing.assert_array_equal(got_k, mark)
    # without a rope the keys are copied
    ctx.fkv_append_kv_paged(shape, fk_, fv, start, new, tab, dkp, dvp)
    at = 0
    for b in range(B):
        paged.append_pages(mark, k[at:at + new[b]], start[b], table[b])
        at += new[b]
    np.testing.assert_array_equal(host_bits(dkp), mark)


def test_queries_in_place_and_at_a_stride(ctx):
    rng = np.random.default_rng(8)
    shape = fk.make_shape(8)
    rows, pos = dev(bits(rng, 6, 48, 128)), torch.arange(100, 106, dtype=torch.int32, device="cuda")
    tab, rope = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), fk.make_rope()
    pools = [torch.zeros((1, 16, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    before = rows.clone()
    call = lambda q, **kw: ctx.fkv_append_kv_paged(shape, before[:, 32:40], before[:, 40:], 3, 6, tab, *pools, rope=rope, positions=pos, q=q, **kw)
    want = call(before[:, :32])
    q = rows[:, :32]
    assert call(q, q_out=q) is q
    assert torch.equal(q, want) and torch.equal(rows[:, 32:], before[:, 32:])
    wide = torch.zeros((6, 40, 128), dtype=torch.bfloat16, device="cuda")
    call(before[:, :32], q_out=wide[:, 4:36])
    assert torch.equal(wide[:, 4:36], want) and not wide[:, :4].any() and not wide[:, 36:].any()


def test_entries_outside_the_pool_write_nothing(ctx):
    rng = np.random.default_rng(9)
    shape = fk.make_shape(8, n_q_heads=4, n_kv_heads=2)
    k, v = bits(rng, 50, 2, 128), bits(rng, 50, 2, 128)
    table = np.array([[1, -1, 4, 0]], np.int32)  # pages 1 and 2 of the sequence lie outside a pool of 4
    pools = [bits(rng, 4, 16, 2, 128) for _ in range(2)]
    d = [dev(p) for p in pools]
    ctx.fkv_append_kv_paged(shape, dev(k), dev(v), 4, 50, torch.from_numpy(table).cuda(), *d)
    for p, x, got in zip(pools, (k, v), d):
        paged.append_pages(p, x, 4, table[0])
        np.testing.assert_array_equal(host_bits(got), p)


def test_no_new_token_is_no_call(ctx):
    shape = fk.make_shape([8, 8], n_q_heads=4, n_kv_heads=2)
    none = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    pools = [torch.ones((4, 16, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tab = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    out = ctx.fkv_append_kv_paged(shape, none, none, [3, 16], [0, 0], tab, *pools, rope=fk.make_rope(), positions=torch.empty(0, dtype=torch.int32, device="cuda"),
                                  q=torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda"))
    assert out.shape == (0, 4, 128) and all((p == 1).all() for p in pools)


def test_the_largest_frequencies_and_positions(ctx):
    """Angles of up to 2^39 radians.  Rows are (1, 0) per pair, so what is stored is bf16(cos), bf16(sin): off by 2^-22 and one rounding, 2^-8 of the
    value; the angle itself is reduced here in exact arithmetic."""
    turn = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
    rng = np.random.default_rng(11)
    positions = np.concatenate([[2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, -1, 0, 1], rng.integers(-2 ** 31, 2 ** 31, 122)]).astype(np.int32)
    freq = np.concatenate([[256.0, -256.0, np.nextafter(256.0, 0), 2.0 ** -60, 1e-300, 0.0, 1 / 3, -1e-7], rng.uniform(-256, 256, 56)])
    x = np.zeros((128, 1, 128), np.uint16)
    x[..., :64] = 0x3F80
    shape, tab = fk.make_shape(8, n_q_heads=1, n_kv_heads=1), torch.arange(2, dtype=torch.int32, device="cuda")[None]
    pools = [torch.zeros((2, 64, 1, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx.fkv_append_kv_paged(shape, dev(x), dev(x), 0, 128, tab, *pools, rope=fk.make_rope(inv_freq=freq), positions=torch.from_numpy(positions).cuda())
    angle = np.array([[float((Fraction(int(p)) * Fraction(float(f))) % turn) for f in freq] for p in positions])
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    got = paged.bf16_to_f64(host_bits(pools[0])).reshape(128, 128)
    assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -8 + 2.0 ** -22 * (1 + 2.0 ** -8)).all()

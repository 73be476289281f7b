"""The paged calls as a serving program strings them together, in graphs, on other streams, by either call path, over large pools."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2502_01068_amd import binding as fk
from parity import host_bits
from test_gpu_append import bits, dev, make_table, turned_close
from test_gpu_decode_split import _Ctx
from test_gpu_quant import full_pools, noise_pools, same, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(max_total_tokens=8192, max_seqs=8)
    yield c
    c.close()


@pytest.mark.parametrize("page,block", [(16, 16), (64, 32)])
def test_prefill_then_tokens(ctx, page, block):
    """KVCompress into the cache in 8 bits, then tokens one and several at a time, each step attended over: pools code by code, outputs
    within their bound; and the same over the bf16 pools."""
    print("case: compress, append, decode; page %d block %d" % (page, block), flush=True)
    rng = np.random.default_rng(page)
    lengths, budget, hq, hkv = [900, 300], [100, 37], 32, 8
    shape = fk.make_shape(lengths)
    qw, k, v = (bits(rng, *s) for s in ((2, 8, hq, 128), (1200, hkv, 128), (1200, hkv, 128)))
    steps = [[1, 1], [1, 0], [5, 33], [1, 1]]
    total = [b + sum(s[i] for s in steps) for i, b in enumerate(budget)]
    table, n_pages = make_table(rng, total, page)
    tab, (codes, scales) = torch.from_numpy(table).cuda(), noise_pools(rng, n_pages, hkv, page, block)
    pools = up((codes, scales))
    idx = ctx.fkv_compress_kv_paged_quant(shape, dev(qw), dev(k), dev(v), budget, tab, *pools)
    plain = [torch.zeros((n_pages, page, hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert torch.equal(idx, ctx.fkv_compress_kv_paged(shape, dev(qw), dev(k), dev(v), budget, tab, *plain))
    apart = up(noise_pools(rng, n_pages, hkv, page, block))
    ctx.fkv_gather_kv_paged_quant(shape, dev(k), dev(v), idx, budget, tab, *apart)
    picked, row, at = idx.cpu().numpy(), 0, 0
    for b, n in enumerate(lengths):
        own = picked[:, at:at + budget[b]].T
        for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
            paged.append_quant(c, s, paged.bf16_to_f64(x[row:row + n])[own, np.arange(hkv)], 0, table[b])
        row, at = row + n, at + budget[b]
    same(pools, codes, scales)
    for b in range(2):  # the one call and the two leave the same rows
        for t in range(budget[b]):
            p, s = table[b][t // page], t % page
            assert torch.equal(apart[0][p, :, s], pools[0][p, :, s]) and torch.equal(apart[1][p, :, s], pools[1][p, :, s])
            assert torch.equal(apart[2][p, :, s // block], pools[2][p, :, s // block])
    cached = list(budget)
    freq = 10000.0 ** (-np.arange(0, 128, 2) / 128)
    rope = fk.make_rope(inv_freq=freq)
    for new in steps:
        n = sum(new)
        rows = bits(rng, n, hq + 2 * hkv, 128)
        f, pos = dev(rows), np.concatenate([np.arange(lengths[b], lengths[b] + new[b]) for b in range(2)]).astype(np.int32)
        kw = dict(rope=rope, positions=torch.from_numpy(pos).cuda(), q=f[:, :hq])
        q = ctx.fkv_append_kv_paged_quant(shape, f[:, hq:hq + hkv], f[:, hq + hkv:], cached, new, tab, *pools, **kw)
        q2 = ctx.fkv_append_kv_paged(shape, f[:, hq:hq + hkv], f[:, hq + hkv:], cached, new, tab, *plain, **kw)
        assert torch.equal(q, q2)
        turned_close(host_bits(q).reshape(n, hq, 128), paged.bf16_to_f64(rows[:, :hq]), pos, freq, False)
        cached = [a + b for a, b in zip(cached, new)]
        last = torch.stack([q[sum(new[:b]) + max(new[b] - 1, 0)] if sum(new[:b]) + max(new[b] - 1, 0) < n else q[0] for b in range(2)])
        out = ctx.fkv_decode_attention_paged_quant(shape, last, *pools, tab, cached).cpu().numpy()
        ref = ctx.fkv_decode_attention_paged(shape, last, *plain, tab, cached).cpu().numpy()
        c, s = [p.cpu().numpy() for p in pools[:2]], [p.cpu().numpy() for p in pools[2:]]
        for b in range(2):
            kk, vv = (paged.dequant(c[i], s[i], table[b], cached[b]) for i in range(2))
            want, bound = paged.attend(paged.bf16_to_f64(host_bits(last))[b], kk, vv, 128 ** -0.5)
            assert (np.abs(out[b] - want) <= bound).all()
        # e4m3 keeps 4 significant bits: the rounding of V alone leaves 2^-4 of a weighted mean of |v| <= 5, that of K some as much again
        assert np.abs(out - ref).max() < 0.5


def _steps(ctx, shape, rope, tab, cached, new, s, out):
    kw = dict(rope=rope, positions=s["pos"], q=s["rows"][:, :32], q_out=out["q"])
    k, v = s["rows"][:, 32:40], s["rows"][:, 40:]
    ctx.fkv_append_kv_paged_quant(shape, k, v, cached, new, tab, *s["pools"], **kw)
    total = [a + b for a, b in zip(cached, new)]
    last = out["q"][:2]
    ctx.fkv_decode_attention_paged_quant(shape, last, *s["pools"], tab, total, out=out["o8"])
    ctx.fkv_append_kv_paged(shape, k, v, cached, new, tab, *s["plain"], **kw)
    ctx.fkv_decode_attention_paged(shape, last, *s["plain"], tab, total, out=out["o16"])
    ctx.fkv_gather_kv_paged_quant(shape, s["ctx_k"], s["ctx_v"], s["idx"], [20, 9], tab, *s["fresh"])
    ctx.fkv_compress_kv_paged_quant(shape, s["qw"], s["ctx_k"], s["ctx_v"], [20, 9], tab, *s["fresh2"], idx_kv=out["idx"])


def _copy(dst, src):
    for name, t in src.items():
        for a, b in zip(dst[name], t) if isinstance(t, list) else [(dst[name], t)]:
            a.copy_(b)


def test_graph_replays_match_eager(ctx):
    print("case: graph of the paged calls", flush=True)
    rng = np.random.default_rng(5)
    shape, rope = fk.make_shape([600, 40]), fk.make_rope()
    cached, new = [2100, 30], [3, 1]
    table, n_pages = make_table(rng, [2103, 31], 16)
    tab = torch.from_numpy(table).cuda()

    def state():
        return {"rows": dev(bits(rng, 4, 48, 128)), "pos": torch.from_numpy(rng.integers(0, 1 << 20, 4).astype(np.int32)).cuda(),
                "pools": up(full_pools(rng, n_pages, 8, 16, 16)), "plain": [dev(bits(rng, n_pages, 16, 8, 128)) for _ in range(2)],
                "ctx_k": dev(bits(rng, 640, 8, 128)), "ctx_v": dev(bits(rng, 640, 8, 128)), "qw": dev(bits(rng, 2, 8, 32, 128)),
                "idx": torch.from_numpy(np.sort(rng.integers(0, 40, (8, 29)), axis=1).astype(np.int32)).cuda(),
                "fresh": up(full_pools(rng, n_pages, 8, 16, 16)), "fresh2": up(full_pools(rng, n_pages, 8, 16, 16))}

    def outputs():
        return {"q": torch.zeros((4, 32, 128), dtype=torch.bfloat16, device="cuda"), "o8": torch.zeros((2, 32, 128), device="cuda"),
                "o16": torch.zeros((2, 32, 128), device="cuda"), "idx": torch.zeros((8, 29), dtype=torch.int32, device="cuda")}

    def snapshot(s, o):
        return [t.clone().view(torch.uint8) for t in list(o.values()) + s["pools"] + s["plain"] + s["fresh"] + s["fresh2"]]

    clone = lambda s: {n: [t.clone() for t in x] if isinstance(x, list) else x.clone() for n, x in s.items()}
    fresh = [state() for _ in range(2)]
    eager = []
    for f in fresh:
        s, o = clone(f), outputs()
        _steps(ctx, shape, rope, tab, cached, new, s, o)
        torch.cuda.synchronize()
        eager.append(snapshot(s, o))
    buf, out = clone(fresh[0]), outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        _steps(ctx, shape, rope, tab, cached, new, buf, out)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            _steps(ctx, shape, rope, tab, cached, new, buf, out)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        which = rep % 2
        _copy(buf, fresh[which])
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i, (got, want) in enumerate(zip(snapshot(buf, out), eager[which])):
            assert torch.equal(got, want), (rep, i)
        s, o = clone(fresh[1 - which]), outputs()   # eager work between replays
        _steps(ctx, shape, rope, tab, cached, new, s, o)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(snapshot(s, o), eager[1 - which]))
    # on another stream, behind the same inputs
    s, o = clone(fresh[0]), outputs()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _steps(ctx, shape, rope, tab, cached, new, s, o)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(snapshot(s, o), eager[0]))
    assert ctx.fkv_query_error() == 0


class _Watched:
    def __init__(self, native):
        self.native, self.taken = native, []

    def __getattr__(self, name):
        def fn(*args):
            out = getattr(self.native, name)(*args)
            self.taken.append((name, out is not None))
            return out
        return fn


def test_both_call_paths_agree(ctx, monkeypatch):
    """Lists of counts go the native way, numpy's counts the ctypes way: the same results; and what either refuses."""
    watch = _Watched(fk._native)
    monkeypatch.setattr(fk, "_native", watch)
    rng = np.random.default_rng(6)
    shape, rope = fk.make_shape([300, 300]), fk.make_rope(64, interleaved=True)
    table, n_pages = make_table(rng, [60, 60], 16)
    tab = torch.from_numpy(table).cuda()
    rows, pos = dev(bits(rng, 12, 48, 128)), torch.arange(12, dtype=torch.int32, device="cuda")
    q, k, v = rows[:, :32], rows[:, 32:40], rows[:, 40:]
    start = up(full_pools(rng, n_pages, 8, 16, 16))
    plain0 = [dev(bits(rng, n_pages, 16, 8, 128)) for _ in range(2)]
    ck, cv, qw, qd = (dev(bits(rng, *s)) for s in ((600, 8, 128), (600, 8, 128), (2, 8, 32, 128), (2, 32, 128)))
    idx = torch.from_numpy(np.sort(rng.integers(0, 300, (8, 60)), axis=1).astype(np.int32)).cuda()
    n64 = lambda *n: [np.int64(x) for x in n]
    e4m3 = lambda p: [p[0].view(torch.float8_e4m3fn), p[1].view(torch.float8_e4m3fn), p[2], p[3]]

    def results(count, pools, plain):
        return [ctx.fkv_append_kv_paged_quant(shape, k, v, count(20, 7), count(5, 7), tab, *pools, rope=rope, positions=pos, q=q),
                ctx.fkv_append_kv_paged_quant(shape, k, v, count(30, 17), count(5, 7), tab, *e4m3(pools)),
                ctx.fkv_append_kv_paged(shape, k, v, count(20, 7), count(5, 7), tab, *plain, rope=rope, positions=pos, q=q),
                ctx.fkv_append_kv_paged(shape, k, v, count(20, 17), count(5, 7), tab, *plain, rope=rope, positions=pos),
                ctx.fkv_decode_attention_paged_quant(shape, qd, *pools, tab, count(40, 0)),
                ctx.fkv_compress_kv_paged_quant(shape, qw, ck, cv, count(20, 9), tab, *pools),
                *ctx.fkv_gather_kv_paged_quant(shape, ck, cv, idx, count(20, 40), tab, *pools),
                *ctx.fkv_gather_kv_paged_quant(shape, ck, None, idx, count(20, 40), tab, pools[0], None, pools[2], None), *pools, *plain]

    got = []
    for count in (lambda *n: list(n), n64):
        watch.taken.clear()
        pools, plain = [p.clone() for p in start], [p.clone() for p in plain0]
        r = results(count, pools, plain)
        torch.cuda.synchronize()
        got.append([None if t is None else t.clone().view(torch.uint8) for t in r])
        names = [n for n, _ in watch.taken]
        assert names == ["append_kv_paged"] * 4 + ["decode_attention_paged_quant", "compress_kv_paged_quant"] + ["gather_kv_paged_quant"] * 2
        assert all(ok == (count is not n64) for _, ok in watch.taken), watch.taken
    for a, b in zip(*got):
        assert (a is None and b is None) or torch.equal(a, b)
    pools, plain = [p.clone() for p in start], plain0
    bad = [lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 6], tab, *plain),                       # 11 of 12 rows
           lambda: ctx.fkv_append_kv_paged(shape, k[:, :, :64], v, [0, 0], [5, 7], tab, *plain),
           lambda: ctx.fkv_append_kv_paged(shape, k.expand(12, 8, 128)[:1].expand(12, 8, 128), v, [0, 0], [5, 7], tab, *plain),
           lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 7], tab, *plain, q=q),                    # no rope
           lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 7], tab, *plain, rope=rope, q=q),         # no positions
           lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 7], tab, *plain, rope=rope, positions=pos[:11], q=q),
           lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 7], tab, *plain, rope=shape, positions=pos),
           lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 7], tab, *plain, rope=rope, positions=pos, q_out=torch.empty_like(q)),
           lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 0], [5, 7], tab, *pools[:2]),                     # pools in 8 bits
           lambda: ctx.fkv_append_kv_paged_quant(shape, k, v, [0, 0], [5, 7], tab, *plain, *pools[2:]),
           lambda: ctx.fkv_append_kv_paged_quant(shape, k, v, [0, 0], [5, 7], tab, pools[0], pools[1], pools[2], pools[3][:1]),
           lambda: ctx.fkv_append_kv_paged_quant(shape, k, v, [0, 0], [5, 7], tab[:1], *pools),
           lambda: ctx.fkv_decode_attention_paged_quant(shape, qd.float(), *pools, tab, 5),
           lambda: ctx.fkv_decode_attention_paged_quant(shape, qd, pools[0], pools[1], None, pools[3], tab, 5),
           lambda: ctx.fkv_gather_kv_paged_quant(shape, ck, None, idx, 20, tab, *pools),
           lambda: ctx.fkv_gather_kv_paged_quant(shape, ck[1:], cv, idx, 20, tab, *pools)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    for call in (lambda: ctx.fkv_append_kv_paged(shape, k, v, [0, 75], [5, 7], tab, *plain), lambda: ctx.fkv_decode_attention_paged_quant(shape, qd, *pools, tab, 81),
                 lambda: ctx.fkv_append_kv_paged(shape, k, v, [-1, 0], [5, 7], tab, *plain)):
        with pytest.raises(fk.FkvError):
            call()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        ctx.fkv_decode_attention_paged_quant(shape, qd, *pools, tab, n64(5, 5))
    with pytest.raises(ValueError, match="current device"):
        ctx.fkv_append_kv_paged(shape, k, v, n64(0, 0), n64(5, 7), tab, *plain)


def test_pools_and_strides_past_32_bits(ctx):
    """Pages whose bytes lie past 2^32, rows that lie 2^31 bytes apart: the same as in a small pool."""
    rng = np.random.default_rng(7)
    shape, rope = fk.make_shape(8), fk.make_rope()
    n_pages, used = (1 << 32) // (8 * 256 * 128) + 9, 5  # 256-token pages of 256 KiB: 4.6 GB
    rows, pos = dev(bits(rng, 700, 48, 128)), torch.arange(700, dtype=torch.int32, device="cuda")
    q = dev(bits(rng, 1, 32, 128))
    far = torch.tensor([[n_pages - 1 - i for i in range(used)]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[used - 1 - i for i in range(used)]], dtype=torch.int32, device="cuda")
    res = []
    for pages, tab in ((used, near), (n_pages, far)):
        pools = fk.quant_pages(pages, 256, scale_block=64)
        for p in (pools[0][-used:], pools[1][-used:], pools[2][-used:], pools[3][-used:]):
            p.view(torch.uint8).zero_()
        out = ctx.fkv_append_kv_paged_quant(shape, rows[:, 32:40], rows[:, 40:], 100, 700, tab, *pools, rope=rope, positions=pos, q=rows[:, :32])
        o = ctx.fkv_decode_attention_paged_quant(shape, q, *pools, tab, 800)
        res.append([out, o] + [p[-used:].clone() for p in pools])
        del pools, out, o
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*res))
    res = []
    for pages, tab in ((used, near), (n_pages // 2, far - n_pages + n_pages // 2)):
        pools = [torch.empty((pages, 256, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for p in pools:
            p[-used:].zero_()
        ctx.fkv_append_kv_paged(shape, rows[:, 32:40], rows[:, 40:], 100, 700, tab, *pools, rope=rope, positions=pos)
        res.append([p[-used:].clone() for p in pools])
        del pools
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(*res))
    stride = 1 << 30
    flat = torch.empty(2 * stride + 48 * 128, dtype=torch.bfloat16, device="cuda")
    wide = flat.as_strided((3, 48, 128), (stride, 128, 1))
    wide.copy_(rows[:3])
    got = []
    for r in (rows[:3], wide):
        pools = [torch.zeros((1, 16, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        tab = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
        got.append([ctx.fkv_append_kv_paged(shape, r[:, 32:40], r[:, 40:], 2, 3, tab, *pools, rope=rope, positions=pos[:3], q=r[:, :32])] + pools)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(*got))


def test_timing_and_counts(ctx):
    """Launches appear under the gather's and the decode's name; counts of pieces that a cut launch left are reset with the error."""
    rng = np.random.default_rng(8)
    c = fk.Context(max_total_tokens=8192, max_seqs=2)
    shape = fk.make_shape([8, 8])
    table, n_pages = make_table(rng, [4000, 4000], 16)
    tab, pools = torch.from_numpy(table).cuda(), up(full_pools(rng, n_pages, 8, 16, 16))
    q, rows = dev(bits(rng, 2, 32, 128)), dev(bits(rng, 2, 16, 128))
    want = c.fkv_decode_attention_paged_quant(shape, q, *pools, tab, [4000, 3990])
    c.fkv_profile_enable(True)
    assert torch.equal(c.fkv_decode_attention_paged_quant(shape, q, *pools, tab, [4000, 3990]), want)
    c.fkv_append_kv_paged_quant(shape, rows[:, :8], rows[:, 8:], [3990, 3995], 1, tab, *[p.clone() for p in pools])
    seen = {n: k for n, (ms, k) in c.fkv_profile_read().items() if k}
    assert seen == {"k_decode": 1, "k_gather": 1}
    c.fkv_profile_enable(False)
    raw = _Ctx.from_address(c.handle.value)
    off = (ctypes.c_uint32 * ((raw.lay.wout_o - raw.lay.dec_count) // 4))()
    assert len(off) >= 2 * 8
    for i in range(len(off)):
        off[i] = i % 7 + 1
    torch.cuda.synchronize()
    copy = fk.load().hipMemcpy
    copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
    assert copy(raw.ws + raw.lay.dec_count, ctypes.addressof(off), ctypes.sizeof(off), 1) == 0
    c.fkv_clear_error()
    for _ in range(2):
        assert torch.equal(c.fkv_decode_attention_paged_quant(shape, q, *pools, tab, [4000, 3990]), want)
    c.close()

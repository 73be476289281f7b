"""Performance cases of the operators that fill a paged cache and read it in 8 bits.

A serving program keeps the tokens that the selection path left in pages, appends each new token behind them and attends over the
lot.  The operators, all of them on scattered pages through a block table:

``append``      new tokens' keys and values into a bf16 paged cache, with the rotary position embedding applied to the keys on
                the way and to the new tokens' queries in the same call; q, k and v are slices of one fused projection
``append_fp8``  the same into a cache held in e4m3, with a power-of-two scale for each block of tokens and head; a block that the
                tokens begin in the middle of grows its scale, and its earlier tokens are rounded again, where they need it
``gather_fp8``  the rows that the selection kept, per KV head, into such a cache (the cache of Algorithm 1 in 8 bits)
``decode_fp8``  one new query per sequence against such a cache

Sizes are those of the repository's benchmark and tests: 32 query / 8 KV heads (64 / 8 and 28 / 4 besides), head size 128, up to 64
sequences and 131072 tokens a call.  ``lo`` and ``hi`` bound the cached (decode, append), or source (gather), tokens of the sequences
of a call; ``new_lo`` and ``new_hi`` the tokens appended, ``budget`` the rows kept.

The 8-bit rule, for a block with new values x: p(a) is the smallest power of two not below 2^-126 with a <= 448 p(a); s' = p(max |x|) over
the finite x, or the larger of that and the block's scale s where earlier tokens of the sequence lie in it; codes are
e4m3(x / s'), earlier ones e4m3(code * s / s').
"""
import random

import torch

own = False

HEAD_DIM = 128
MAX_TOKENS, MAX_SEQS = 131072, 64
E4M3_MAX = 448.0
TINY = 2.0 ** -126
_SEED_STRIDE = 1_000_003

_context = None


def _ctx():
    """The one context of the program: a server makes it once, for its longest input."""
    global _context
    if _context is None:
        from paper_2502_01068_amd import binding as fk
        _context = fk.Context(max_total_tokens=MAX_TOKENS, max_seqs=MAX_SEQS)
    return _context


# ---- cases ---------------------------------------------------------------------------------
def _append(name, lo, new_lo, hi=None, new_hi=None, n_seq=1, hq=32, hkv=8, page=16, block=0, rotary=HEAD_DIM, interleaved=False):
    c = {"op": "append_fp8" if block else "append", "n_seq": n_seq, "lo": lo, "hi": lo if hi is None else hi, "new_lo": new_lo,
         "new_hi": new_lo if new_hi is None else new_hi, "hq": hq, "hkv": hkv, "page": page, "block": block, "rotary": rotary,
         "interleaved": interleaved}
    return dict(c, name=name) if name else c


def _gather(name, lo, budget, hi=None, n_seq=1, hkv=8, page=16, block=16):
    c = {"op": "gather_fp8", "n_seq": n_seq, "lo": lo, "hi": hi or lo, "budget": budget, "hq": 4 * hkv, "hkv": hkv, "page": page, "block": block}
    return dict(c, name=name) if name else c


def _decode(name, lo, hi=None, n_seq=1, hq=32, hkv=8, page=16, block=16):
    c = {"op": "decode_fp8", "n_seq": n_seq, "lo": lo, "hi": hi or lo, "hq": hq, "hkv": hkv, "page": page, "block": block}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the next token of one request behind its compacted cache: the smallest call, made once per layer and token
        _append("append_1", 2048, 1),
        # a serving batch: one token for each of 64 requests of different lengths
        _append("append_64x1", 300, 1, hi=1000, n_seq=64),
        # a prompt whose tokens all go into the cache before anything is dropped; odd length, larger pages
        _append("append_prompt_8191", 0, 8191, page=64),
        # the next token of one request, into the cache in 8 bits
        _append("append_fp8_1", 2048, 1, block=16),
        # requests that take several tokens at once (accepted drafts, the tail of a prompt): blocks are begun, filled and joined
        _append("append_fp8_32x", 300, 1, hi=2000, new_hi=24, n_seq=32, block=16),
        # three prompts in chunks behind what is cached, the largest append; interleaved pairs, half of the columns rotated
        _append("append_fp8_chunk", 1000, 3001, hi=5000, new_hi=4099, n_seq=3, page=64, block=32, rotary=64, interleaved=True),
        # a layer of the benchmark: 2048 rows of 32768 tokens kept per KV head
        _gather("gather_fp8_2048", 32768, 2048),
        # a long context at a tenth
        _gather("gather_fp8_13107", 131072, 13107, page=128, block=64),
        # eight prompts of different lengths in one call, odd budget
        _gather("gather_fp8_8x", 8192, 1021, hi=16384, n_seq=8, page=32, block=32),
        # one new token of one request over the compacted cache of one layer: the call made most often
        _decode("decode_fp8_2048", 2048),
        # the same step over a long cache that nothing was dropped from
        _decode("decode_fp8_32768", 32768, page=64, block=64),
        # a serving batch: requests at different points of their generation
        _decode("decode_fp8_32x", 2048, hi=2560, n_seq=32),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def _spread(rng, lo, hi, most_total):
    """(n_seq, shortest, longest) of a call of at most `most_total` tokens; some calls hold one sequence."""
    n_seq = 1 if rng.random() < 0.4 else _log_uniform(rng, 2, MAX_SEQS)
    longest = _log_uniform(rng, lo, max(lo, min(hi, most_total // n_seq)))
    return n_seq, (longest if n_seq == 1 else max(1, round(longest * rng.uniform(0.5, 1.0)))), longest


def draw(rng):
    hq, hkv = rng.choice(((32, 8),) * 4 + ((64, 8), (28, 4)))
    page = rng.choice((16, 16, 32, 64, 128))
    block = rng.choice([b for b in (16, 32, 64) if b <= page])
    op = rng.choice(("append", "append_fp8", "append_fp8", "gather_fp8", "decode_fp8", "decode_fp8"))
    if op == "gather_fp8":
        n_seq, lo, hi = _spread(rng, 200, MAX_TOKENS, MAX_TOKENS)
        return _gather(None, lo, _log_uniform(rng, 8, max(8, lo // 8)), hi, n_seq, hkv, page, block)
    if op == "decode_fp8":
        n_seq, lo, hi = _spread(rng, 1, 60000, 80000)
        return _decode(None, lo, hi, n_seq, hq, hkv, page, block)
    n_seq, lo, hi = _spread(rng, 1, 30000, 30000)
    if rng.random() < 0.5:  # decoding: a token each, or a few
        new_lo, new_hi = 1, rng.choice((1, 1, 2, 7))
    else:
        new_hi = _log_uniform(rng, 1, 8191 // n_seq if hq == 32 else 4000 // n_seq)
        new_lo = new_hi if n_seq == 1 else max(1, new_hi // 2)
    return _append(None, rng.choice((0, lo)) if n_seq == 1 else lo, new_lo, hi if n_seq > 1 else None, new_hi, n_seq, hq, hkv, page,
                   block if op == "append_fp8" else 0, rng.choice((HEAD_DIM, HEAD_DIM, 64)), rng.random() < 0.3)


def _lengths(case, lo="lo", hi="hi", salt=0):
    """Tokens of each sequence: spread over [lo, hi], in an order that is not sorted, the largest among them."""
    if case["n_seq"] == 1:
        return [case[hi]]
    rng = random.Random(case["n_seq"] * _SEED_STRIDE + case[hi] + salt)
    rest = [rng.randint(case[lo], case[hi]) for _ in range(case["n_seq"] - 1)]
    rest.insert(rng.randrange(case["n_seq"]), case[hi])
    return rest


# ---- what a program has in hand before the call ----------------------------------------------
def _keys(gen, tokens, hkv):
    """Keys of a trained layer in outline: channels of unequal size, a few of them several times the others'."""
    size = torch.exp(0.5 * torch.randn((hkv, HEAD_DIM), device="cuda", generator=gen))
    return (torch.randn((tokens, hkv, HEAD_DIM), device="cuda", generator=gen) * size).to(torch.bfloat16)


def _table(gen, counts, page):
    """A table that scatters every sequence's pages over a pool with room to spare."""
    need = [-(-c // page) for c in counts]
    n_pages = sum(need) + 8
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(counts), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _pow2_scale(a):
    """p(a): 448 is 0.875 * 2^9, so the power follows from the mantissa and exponent of a, exactly."""
    mant, exp = torch.frexp(a)
    return torch.ldexp((a > 0).to(a.dtype), exp - 9 + (mant > 0.875).to(exp.dtype)).clamp_min(TINY)


def _fp8_pool(gen, n_pages, hkv, page, block, std):
    """A pool of e4m3 pages full of tokens: (codes [n_pages, Hkv, page, d], scales [n_pages, Hkv, page / block])."""
    shape = (n_pages, hkv, page // block, block, HEAD_DIM)
    size = std * torch.exp(0.5 * torch.randn((hkv, 1, 1, HEAD_DIM), device="cuda", generator=gen))
    x = (torch.randn(shape, device="cuda", generator=gen) * size).to(torch.bfloat16).float()
    scale = _pow2_scale(x.abs().amax((3, 4)))
    codes = (x / scale[..., None, None]).to(torch.float8_e4m3fn)
    return codes.reshape(n_pages, hkv, page, HEAD_DIM), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * _SEED_STRIDE + 29)
    op, n_seq, hq, hkv, page, block = (case[k] for k in ("op", "n_seq", "hq", "hkv", "page", "block"))
    lengths = _lengths(case)
    s = {"op": op, "case": case, "n": lengths}
    if own:
        from paper_2502_01068_amd import binding as fk
        s["ctx"], s["shape"] = _ctx(), fk.make_shape([max(n, 8) for n in lengths], n_q_heads=hq, n_kv_heads=hkv)
    if op == "decode_fp8":
        s["table"], n_pages = _table(gen, lengths, page)
        s["q"] = torch.randn((n_seq, hq, HEAD_DIM), device="cuda", generator=gen).to(torch.bfloat16)
        s["k"], s["k_scale"] = _fp8_pool(gen, n_pages, hkv, page, block, 1.5)
        s["v"], s["v_scale"] = _fp8_pool(gen, n_pages, hkv, page, block, 1.0)
        return s
    if op == "gather_fp8":
        s["budget"] = [min(case["budget"], n) for n in lengths]
        s["table"], n_pages = _table(gen, s["budget"], page)
        s["k_new"] = _keys(gen, sum(lengths), hkv)
        s["v_new"] = torch.randn((sum(lengths), hkv, HEAD_DIM), device="cuda", generator=gen, dtype=torch.bfloat16)
        rows = [torch.rand((hkv, n), device="cuda", generator=gen).topk(b).indices.sort().values for n, b in zip(lengths, s["budget"])]
        s["idx"] = torch.cat(rows, dim=1).to(torch.int32)
        for x in ("k", "v"):
            s[x], s[x + "_scale"] = _fp8_pool(gen, n_pages, hkv, page, block, 1.0)
        return s
    new = _lengths(case, "new_lo", "new_hi", salt=5)
    total, r = sum(new), case["rotary"]
    s["new"] = new
    s["table"], n_pages = _table(gen, [a + b for a, b in zip(lengths, new)], page)
    # one fused projection [tokens, (Hq + 2 Hkv) d]; q, k and v are views of it
    fused = torch.empty((total, hq + 2 * hkv, HEAD_DIM), dtype=torch.bfloat16, device="cuda")
    fused[:, :hq] = torch.randn((total, hq, HEAD_DIM), device="cuda", generator=gen)
    fused[:, hq:hq + hkv] = _keys(gen, total, hkv)
    fused[:, hq + hkv:] = torch.randn((total, hkv, HEAD_DIM), device="cuda", generator=gen)
    s["q"], s["k_new"], s["v_new"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    # a compacted cache holds fewer tokens than the context had: positions run ahead of the slots, here by up to a million
    ahead = torch.randint(0, 1 << 20, (n_seq,), device="cuda", generator=gen)
    first = torch.tensor(lengths, device="cuda") + ahead
    before = torch.tensor([sum(new[:b]) for b in range(n_seq)], device="cuda")
    seq = torch.repeat_interleave(torch.arange(n_seq, device="cuda"), torch.tensor(new, device="cuda"))
    s["positions"] = (torch.arange(total, device="cuda") - before[seq] + first[seq]).to(torch.int32)
    s["inv_freq"] = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if own:
        s["rope"] = fk.make_rope(r, inv_freq=s["inv_freq"].tolist(), interleaved=case["interleaved"])
    for x, std in (("k", 1.5), ("v", 1.0)):
        if block:
            s[x], s[x + "_scale"] = _fp8_pool(gen, n_pages, hkv, page, block, std)
        else:
            s[x] = std * torch.randn((n_pages, page, hkv, HEAD_DIM), device="cuda", generator=gen, dtype=torch.bfloat16)
    return s


# ---- one pass ------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    ctx, shape, op = s["ctx"], s["shape"], s["op"]
    if op == "decode_fp8":
        return ctx.fkv_decode_attention_paged_quant(shape, s["q"], s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["n"])
    if op == "gather_fp8":
        ctx.fkv_gather_kv_paged_quant(shape, s["k_new"], s["v_new"], s["idx"], s["budget"], s["table"], s["k"], s["v"], s["k_scale"], s["v_scale"])
        return s["k"], s["v"], s["k_scale"], s["v_scale"]
    if op == "append":
        q = ctx.fkv_append_kv_paged(shape, s["k_new"], s["v_new"], s["n"], s["new"], s["table"], s["k"], s["v"], rope=s["rope"],
                                    positions=s["positions"], q=s["q"])
        return q, s["k"], s["v"]
    q = ctx.fkv_append_kv_paged_quant(shape, s["k_new"], s["v_new"], s["n"], s["new"], s["table"], s["k"], s["v"], s["k_scale"], s["v_scale"],
                                    rope=s["rope"], positions=s["positions"], q=s["q"])
    return q, s["k"], s["v"], s["k_scale"], s["v_scale"]


def _rotate(x, positions, inv_freq, interleaved):
    """x [T, H, d] -> fp32, rotated; angles in 64 bits (positions run to a million radians)."""
    angle = positions.double()[:, None, None] * inv_freq.to(x.device)
    cos, sin = angle.cos().float(), angle.sin().float()
    r = 2 * inv_freq.numel()
    x = x.float()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _owners(counts, device):
    """For a packed batch of `counts` entries per sequence: each entry's sequence, and its place there."""
    n = torch.tensor(counts, device=device)
    seq = torch.repeat_interleave(torch.arange(len(counts), device=device), n)
    return seq, torch.arange(seq.numel(), device=device) - (n.cumsum(0) - n)[seq]


def _store_blocks(x, start, new, table, pages, scales):
    """x [T, Hkv, d] fp32: the packed new tokens, start_b + 0, 1, .. of each sequence, into e4m3 pages."""
    dev, (page, block) = x.device, (pages.shape[2], pages.shape[2] // scales.shape[2])
    first = [a // block for a in start]
    seq, at = _owners([(a + n + block - 1) // block - f if n else 0 for a, n, f in zip(start, new, first)], dev)
    start_t, new_t = torch.tensor(start, device=dev)[seq], torch.tensor(new, device=dev)
    token = (torch.tensor(first, device=dev)[seq] + at)[:, None] * block + torch.arange(block, device=dev)  # [blocks, block]
    is_old = token < start_t[:, None]
    is_new = ~is_old & (token < (start_t + new_t[seq])[:, None])
    where = table[seq, token[:, 0] // page].long()
    place = token[:, 0] % page // block
    source = ((new_t.cumsum(0) - new_t)[seq][:, None] + token - start_t[:, None]).clamp(0, x.shape[0] - 1)
    val = x[source].transpose(1, 2)  # [blocks, Hkv, block, d]
    old, fresh = is_old[:, None, :, None], is_new[:, None, :, None]
    amax = torch.where(fresh & val.isfinite(), val.abs(), 0.0).amax((2, 3))
    had = torch.where(is_old[:, :1], scales[where, :, place], 0.0)
    scale = torch.maximum(_pow2_scale(amax), had)
    view = pages.view(pages.shape[0], pages.shape[1], -1, block, HEAD_DIM)
    codes = view[where, :, place].float()
    codes = torch.where(old, codes * (had / scale)[..., None, None], codes)
    view[where, :, place] = torch.where(fresh, val / scale[..., None, None], codes).to(torch.float8_e4m3fn)
    scales[where, :, place] = scale


def _store_kept(x, idx, lengths, budget, table, pages, scales):
    """Row idx[h][t] of sequence b for its kept token t of head h, as new tokens from slot 0 on."""
    begin = torch.tensor(lengths, device=x.device).cumsum(0) - torch.tensor(lengths, device=x.device)
    seq, _ = _owners(budget, x.device)
    rows = (begin[seq] + idx.long()).t()  # [T, Hkv]
    kept = x.gather(0, rows[..., None].expand(-1, -1, HEAD_DIM)).float()
    _store_blocks(kept, [0] * len(budget), budget, table, pages, scales)


def _logical(pages, scales, table, n):
    """The tokens of every sequence, dequantised and padded to the longest: [B, Hkv, tokens, d] fp32."""
    block = pages.shape[2] // scales.shape[2]
    page = table[:, :-(-n // pages.shape[2])].long().clamp(min=0)
    x = pages[page].float() * scales[page].repeat_interleave(block, dim=3)[..., None]
    return x.transpose(1, 2).flatten(2, 3)[:, :, :n]


def _run_plain(s):
    op = s["op"]
    if op == "decode_fp8":
        b, hq, _ = s["q"].shape
        hkv, longest = s["k"].shape[1], max(s["n"])
        q = s["q"].float().view(b, hkv, hq // hkv, HEAD_DIM)
        k = _logical(s["k"], s["k_scale"], s["table"], longest)
        z = (q @ k.transpose(2, 3)) * HEAD_DIM ** -0.5
        beyond = torch.arange(longest, device=z.device) >= torch.tensor(s["n"], device=z.device)[:, None, None, None]
        z = z.masked_fill(beyond, -torch.inf)
        p = (z - z.amax(-1, keepdim=True)).exp()
        v = _logical(s["v"], s["v_scale"], s["table"], longest)
        return ((p / p.sum(-1, keepdim=True)) @ v).view(b, hq, HEAD_DIM)
    if op == "gather_fp8":
        for x in ("k", "v"):
            _store_kept(s[x + "_new"], s["idx"], s["n"], s["budget"], s["table"], s[x], s[x + "_scale"])
        return s["k"], s["v"], s["k_scale"], s["v_scale"]
    turn = (s["positions"], s["inv_freq"], s["case"]["interleaved"])
    q, k = _rotate(s["q"], *turn).to(torch.bfloat16), _rotate(s["k_new"], *turn)
    if op == "append":
        seq, at = _owners(s["new"], k.device)
        token, page = torch.tensor(s["n"], device=k.device)[seq] + at, s["k"].shape[1]
        where = s["table"][seq, token // page].long()
        s["k"][where, token % page] = k.to(torch.bfloat16)
        s["v"][where, token % page] = s["v_new"]
        return q, s["k"], s["v"]
    _store_blocks(k, s["n"], s["new"], s["table"], s["k"], s["k_scale"])
    _store_blocks(s["v_new"].float(), s["n"], s["new"], s["table"], s["v"], s["v_scale"])
    return q, s["k"], s["v"], s["k_scale"], s["v_scale"]


def work(case):
    """Every input and output once; the rows of a cache that a call neither reads nor writes do not count."""
    hq, hkv, lengths = case["hq"], case["hkv"], _lengths(case)
    row, total = 2 * HEAD_DIM, sum(lengths)
    if case["op"] == "decode_fp8":
        scales = sum(-(-n // case["block"]) for n in lengths) * hkv * 4
        return {"bytes": 2 * (total * hkv * HEAD_DIM + scales) + case["n_seq"] * hq * HEAD_DIM * (2 + 4), "flops": 4 * total * hq * HEAD_DIM}
    if case["op"] == "gather_fp8":
        kept = sum(min(case["budget"], n) for n in lengths) * hkv
        return {"bytes": kept * (2 * (row + HEAD_DIM) + 4), "flops": 2 * 2 * kept * HEAD_DIM}
    new = sum(_lengths(case, "new_lo", "new_hi", salt=5))
    stored = row // 2 if case["block"] else row
    return {"bytes": new * (2 * hq * row + 2 * hkv * (row + stored) + 4), "flops": 3 * new * (hq + hkv) * case["rotary"]}


# ---- the definition in 64 bits, sequence by sequence -------------------------------------------
def _turn64(x, positions, inv_freq, interleaved):
    z = x.double().clone()
    for i, f in enumerate(inv_freq.tolist()):
        one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + len(inv_freq))
        c, w = torch.cos(positions.double() * f)[:, None], torch.sin(positions.double() * f)[:, None]
        z[..., one], z[..., two] = x[..., one].double() * c - x[..., two].double() * w, x[..., one].double() * w + x[..., two].double() * c
    return z


def _scale64(a):
    return torch.exp2(torch.ceil(torch.log2((a / E4M3_MAX).clamp_min(TINY))))


def _fill64(pool, scales, x, start, table):
    """Tokens start, start + 1, .. of one sequence; x [n, Hkv, d]; pool in units of the scales, both changed in place."""
    page, block = pool.shape[2], pool.shape[2] // scales.shape[2]
    at, n = 0, x.shape[0]
    if n and start % block:  # the block that earlier tokens are in
        m = min(n, block - start % block)
        p, o = int(table[start // page]), start % page
        new = torch.maximum(scales[p, :, o // block], _scale64(x[:m].abs().amax((0, 2))))
        pool[p, :, o - start % block:o] *= (scales[p, :, o // block] / new)[:, None, None]
        pool[p, :, o:o + m] = x[:m].transpose(0, 1) / new[:, None, None]
        scales[p, :, o // block] = new
        at = m
    whole = torch.zeros((-(-(n - at) // block), block) + x.shape[1:], dtype=torch.float64, device=x.device)
    if not whole.numel():
        return
    whole.view((-1,) + x.shape[1:])[:n - at] = x[at:]
    scale = _scale64(whole.abs().amax((1, 3)))  # [blocks, Hkv]
    whole /= scale[:, None, :, None]
    token = start + at + torch.arange(n - at, device=x.device)
    pool[table[token // page].long(), :, token % page] = whole.view((-1,) + x.shape[1:])[:n - at]
    head = token[::block]
    scales[table[head // page].long(), :, head % page // block] = scale


def exact(case, seed):
    s = prepare(case, seed)
    tables = s["table"].clone()
    if case["op"] == "decode_fp8":
        out = []
        for b, n in enumerate(s["n"]):
            at = torch.arange(n, device="cuda")
            page, slot = tables[b][at // case["page"]].long(), at % case["page"]
            k, v = (s[x][page, :, slot].double() * s[x + "_scale"][page, :, slot // case["block"]].double()[..., None] for x in ("k", "v"))
            q = s["q"][b].double().view(case["hkv"], -1, HEAD_DIM)
            rows = [torch.softmax(k[:, h] @ q[h].t() / HEAD_DIM ** 0.5, 0).t().contiguous() @ v[:, h] for h in range(case["hkv"])]
            out.append(torch.cat(rows))
        return torch.stack(out)
    pools, scales = {x: s[x].double() for x in ("k", "v")}, {x: s[x + "_scale"].double() for x in ("k", "v") if case["block"]}
    at = 0
    if case["op"] == "gather_fp8":
        out = 0
        for b, (n, kept) in enumerate(zip(s["n"], s["budget"])):
            for x in ("k", "v"):
                rows = s[x + "_new"][at:at + n].double()
                picked = torch.stack([rows[s["idx"][h, out:out + kept].long(), h] for h in range(case["hkv"])], 1)
                _fill64(pools[x], scales[x], picked, 0, tables[b])
            at, out = at + n, out + kept
        return pools["k"], pools["v"], scales["k"], scales["v"]
    turned = {x: _turn64(s[n], s["positions"], s["inv_freq"], case["interleaved"]) for x, n in (("q", "q"), ("k", "k_new"))}
    turned["v"] = s["v_new"].double()
    for b, (start, n) in enumerate(zip(s["n"], s["new"])):
        for x in ("k", "v"):
            rows = turned[x][at:at + n]
            if case["block"]:
                _fill64(pools[x], scales[x], rows, start, tables[b])
            else:
                token = start + torch.arange(n, device="cuda")
                pools[x][tables[b][token // case["page"]].long(), token % case["page"]] = rows
        at += n
    return (turned["q"], pools["k"], pools["v"]) + ((scales["k"], scales["v"]) if case["block"] else ())

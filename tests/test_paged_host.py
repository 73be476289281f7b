"""Refusals of the calls that append to a paged cache and of those on the cache in 8 bits, before any launch (no GPU)."""
import ctypes
import os

import pytest
import torch

from paper_2502_01068_amd import binding as fk
from test_binding_host import FakeGpuTensor

P, ODD = 4096, 4104  # made-up device pointers, on 16 bytes and not


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fk.LIB_PATH):
        from paper_2502_01068_amd import build
        build.build()
    return fk.load()


def i32(*values):
    return (ctypes.c_int32 * len(values))(*values)


def tokens(n_cached=(5, 0), n_new=(3, 1), **kw):
    t = fk.FkvNewTokens(k=P, v=P, q=P, q_out=P, positions=P)
    for name, value in kw.items():
        setattr(t, name, value)
    t._keep = (i32(*n_cached), i32(*n_new))
    t.n_cached, t.n_new = (ctypes.cast(a, ctypes.POINTER(ctypes.c_int32)) for a in t._keep)
    return t


def pages(**kw):
    p = fk.FkvQuantPages(k_pages=P, v_pages=P, k_scale=P, v_scale=P, block_table=P, max_pages_per_seq=8, page_size=32, scale_block=16, n_pages=100)
    for name, value in kw.items():
        setattr(p, name, value)
    return p


def append(lib, t, rope=fk.make_rope(), quant=False, shape=None, **paging):
    s = shape or fk.make_shape([8, 8])
    r = rope and ctypes.byref(rope)
    if quant:
        return lib.fkv_append_kv_paged_quant(None, ctypes.byref(s), r, t and ctypes.byref(t), ctypes.byref(pages(**paging)), None)
    p = dict(block_table=P, max_pages_per_seq=8, page_size=32, n_pages=100, k_pages=P, v_pages=P)
    p.update(paging)
    return lib.fkv_append_kv_paged(None, ctypes.byref(s), r, t and ctypes.byref(t), p["block_table"], p["max_pages_per_seq"], p["page_size"], p["n_pages"],
                                   p["k_pages"], p["v_pages"], None)


def bad_rope(**kw):
    r = fk.make_rope()
    for name, value in kw.items():
        setattr(r, name, value)
    return r


@pytest.mark.parametrize("quant", [False, True])
def test_append_refuses(lib, quant):
    call = lambda t, rope=fk.make_rope(), **kw: append(lib, t, rope, quant, **kw)
    assert call(tokens()) == fk.FKV_ENULL  # everything in order but for the context
    assert call(tokens(), shape=fk.make_shape([8, 8], n_q_heads=30)) == fk.FKV_EINVAL
    assert call(None) == fk.FKV_ENULL
    for name in ("k", "v", "positions", "q", "q_out"):
        assert call(tokens(**{name: None})) == fk.FKV_ENULL, name
    for name in ("k", "v", "q", "q_out"):
        assert call(tokens(**{name: ODD})) == fk.FKV_EALIGN, name
    t = tokens()
    t.n_new = None
    assert call(t) == fk.FKV_ENULL
    for cached, new in (((-1, 0), (1, 1)), ((0, 0), (1, -1)), ((250, 0), (7, 1)), ((0, 0), (1 << 30, 1))):
        assert call(tokens(cached, new)) == fk.FKV_EINVAL
    assert call(tokens((249, 0), (7, 1))) == fk.FKV_ENULL  # the last slot of the table: fits
    big = dict(max_pages_per_seq=1 << 26)
    assert call(tokens(((1 << 30) - 3, 0), (3, 1)), **big) == fk.FKV_ENULL and call(tokens(((1 << 30) - 2, 0), (3, 1)), **big) == fk.FKV_EUNSUPPORTED
    assert call(tokens((0, 5), ((1 << 22) - 1, 1)), **big) == fk.FKV_ENULL and call(tokens((0, 5), (1 << 22, 1)), **big) == fk.FKV_EUNSUPPORTED
    assert call(tokens(k_stride=1016)) == fk.FKV_EINVAL and call(tokens(k_stride=1028)) == fk.FKV_EALIGN and call(tokens(k_stride=-1024)) == fk.FKV_EINVAL
    assert call(tokens(q_stride=4088)) == fk.FKV_EINVAL and call(tokens(v_stride=1 << 40)) == fk.FKV_EINVAL
    assert call(tokens(q_out_stride=8192)) == fk.FKV_EINVAL      # in place at another stride
    assert call(tokens(q_out_stride=8192, q_stride=8192)) == fk.FKV_ENULL
    assert call(tokens(), rope=None) == fk.FKV_EINVAL            # queries that nothing turns
    assert call(tokens(q=None, q_out=None, positions=None), rope=None) == fk.FKV_ENULL
    for kw, code in ((dict(rotary_dim=0), -1), (dict(rotary_dim=24), -1), (dict(rotary_dim=144), -1), (dict(rotary_dim=-16), -1), (dict(interleaved=2), -1),
                     (dict(inv_freq=None), -2)):
        assert call(tokens(), rope=bad_rope(**kw)) == code, kw
    assert call(tokens(), rope=fk.make_rope(16, inv_freq=[1.0] * 7 + [float("inf")])) == fk.FKV_EINVAL
    assert call(tokens(), rope=fk.make_rope(16, inv_freq=[1.0] * 7 + [float("nan")])) == fk.FKV_EINVAL
    assert call(tokens(), block_table=None) == fk.FKV_ENULL and call(tokens(), k_pages=None) == fk.FKV_ENULL
    assert call(tokens(), v_pages=ODD) == fk.FKV_EALIGN and call(tokens(), page_size=48) == fk.FKV_EINVAL and call(tokens(), n_pages=0) == fk.FKV_EINVAL
    assert call(tokens(), n_pages=1 << 27) == fk.FKV_EINVAL
    # nothing to append: pointers of empty tensors are NULL
    assert call(tokens((3, 4), (0, 0), k=None, v=None, q=None, q_out=None, positions=None)) == fk.FKV_ENULL  # the context


def test_quant_calls_refuse(lib):
    s = fk.make_shape([300, 100])
    budget, n = i32(100, 20), i32(200, 0)
    gather = lambda k=P, v=P, idx=P, b=budget, **kw: lib.fkv_gather_kv_paged_quant(None, ctypes.byref(s), k, v, idx, b, ctypes.byref(pages(**kw)), None)
    compress = lambda q=P, k=P, v=P, idx=P, b=budget, **kw: lib.fkv_compress_kv_paged_quant(None, ctypes.byref(s), q, k, v, b, ctypes.byref(pages(**kw)), idx, None)
    decode = lambda q=P, out=P, n=n, **kw: lib.fkv_decode_attention_paged_quant(None, ctypes.byref(s), q, ctypes.byref(pages(**kw)), n, out, None)
    for call in (gather, compress, decode):
        assert call() == fk.FKV_ENULL  # the context
        for name in ("k_pages", "k_scale", "v_scale", "v_pages", "block_table"):
            assert call(**{name: None}) == fk.FKV_ENULL, name
        for name in ("k_pages", "k_scale", "v_scale", "v_pages"):
            assert call(**{name: ODD}) == fk.FKV_EALIGN, name
        for kw in (dict(page_size=8), dict(page_size=48), dict(scale_block=8), dict(scale_block=64), dict(scale_block=24), dict(scale_block=0), dict(n_pages=0),
                   dict(n_pages=1 << 24), dict(max_pages_per_seq=0), dict(max_pages_per_seq=3, page_size=32)):
            assert call(**kw) == fk.FKV_EINVAL, kw
        assert call(scale_block=32) == fk.FKV_ENULL
    assert gather(k=None) == fk.FKV_ENULL and gather(idx=None) == fk.FKV_ENULL and gather(v=None) == fk.FKV_ENULL
    assert gather(v=None, v_pages=None, v_scale=None) == fk.FKV_ENULL and gather(b=i32(7, 20)) == fk.FKV_EINVAL
    assert gather(idx=ODD) == fk.FKV_EALIGN and compress(q=ODD) == fk.FKV_EALIGN and compress(v=None) == fk.FKV_ENULL and compress(b=i32(100, 101)) == fk.FKV_EINVAL
    assert decode(n=None) == fk.FKV_ENULL and decode(n=i32(-1, 0)) == fk.FKV_EINVAL and decode(n=i32(257, 0)) == fk.FKV_EINVAL
    assert decode(n=i32(1 << 30, 0), max_pages_per_seq=1 << 26) == fk.FKV_ENULL and decode(n=i32((1 << 30) + 1, 0), max_pages_per_seq=1 << 26) == fk.FKV_EUNSUPPORTED
    assert decode(out=ODD) == fk.FKV_EALIGN
    assert lib.fkv_decode_attention_paged_quant(None, ctypes.byref(s), P, None, n, P, None) == fk.FKV_ENULL


def test_structs_match_the_header():
    assert ctypes.sizeof(fk.FkvRope) == 16 and ctypes.sizeof(fk.FkvNewTokens) == 88 and ctypes.sizeof(fk.FkvQuantPages) == 64
    assert fk.FkvNewTokens.positions.offset == 64 and fk.FkvQuantPages.n_pages.offset == 56


def test_rope_helper():
    r = fk.make_rope(64, theta=500.0, interleaved=True)
    assert (r.rotary_dim, r.interleaved) == (64, 1) and [r.inv_freq[i] for i in range(32)] == [500.0 ** (-2.0 * i / 64) for i in range(32)]
    with pytest.raises(ValueError, match="frequencies"):
        fk.make_rope(64, inv_freq=[1.0] * 31)


class Rows(FakeGpuTensor):
    def __init__(self, shape, strides=None, **kw):
        n = 1
        for s in shape:
            n *= s
        super().__init__(n, **kw)
        self.shape = torch.Size(shape)
        self._strides = strides or (shape[1] * shape[2], shape[2], 1)

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]


@pytest.mark.parametrize("rows,match", [
    (Rows((3, 8, 128)), "must be"), (Rows((4, 8, 64)), "must be"), (Rows((4, 8, 128), dtype=torch.float32), "dtype"), (Rows((4, 8, 128), index=1), "context"),
    (Rows((4, 8, 128), (8, 128, 1)), "overlap"), (Rows((4, 8, 128), (0, 128, 1)), "overlap"), (Rows((4, 8, 128), (2048, 256, 1)), "side by side"),
    (Rows((4, 8, 128), (1024, 1, 8)), "side by side"), (torch.zeros((4, 8, 128), dtype=torch.bfloat16), "GPU tensor"),
])
def test_token_rows_refuse(rows, match):
    with pytest.raises(ValueError, match=match):
        fk._token_rows(rows, "k", 4, 8, 128, 0)


def test_token_rows_take_slices():
    assert fk._token_rows(Rows((4, 8, 128), (6144, 128, 1)), "k", 4, 8, 128, 0) == (0x1000, 6144)
    assert fk._token_rows(Rows((1, 8, 128), (5, 128, 1)), "k", 1, 8, 128, 0) == (0x1000, 0)  # one token has no next one
    assert fk._token_rows(Rows((4, 1, 128), (128, 7, 1)), "k", 4, 1, 128, 0) == (0x1000, 128)
    assert fk._token_rows(Rows((0, 8, 128)), "k", 0, 8, 128, 0) == (None, 0)


def test_quant_pages_helper():
    with pytest.raises(ValueError, match="multiple"):
        fk.quant_pages(4, 16, scale_block=32)
    k, v, ks, vs = fk.quant_pages(4, 64, n_kv_heads=2, scale_block=32, device="cpu")
    assert k.shape == v.shape == (4, 2, 64, 128) and ks.shape == vs.shape == (4, 2, 2) and k.dtype == torch.float8_e4m3fn and ks.dtype == torch.float32


def test_frequencies_that_the_angles_cannot_hold_are_refused(lib):
    for f, code in ((256.0, fk.FKV_ENULL), (-256.0, fk.FKV_ENULL), (0.0, fk.FKV_ENULL), (5e-324, fk.FKV_ENULL), (256.0 * (1 + 2.0 ** -52), fk.FKV_EUNSUPPORTED),
                    (-1e6, fk.FKV_EUNSUPPORTED), (2.0 ** 118, fk.FKV_EUNSUPPORTED)):  # ENULL: only the context is missing
        for quant in (False, True):
            assert append(lib, tokens(), fk.make_rope(16, inv_freq=[1.0] * 7 + [f]), quant) == code, f

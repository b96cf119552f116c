"""Host-side checks (no GPU) of the group quantizer, the products with a step per group, rotary positions, the 4-bit cache
and its attention: refusals, sizes, and the table of frequencies."""
import os

import numpy as np
import pytest

import operators_util as ou
import paper_2511_22316_amd as sq
from paper_2511_22316_amd import binding

FAKE = 0x1000          # 16-byte aligned, never dereferenced: validation fails first
OK, NULL, SHAPE, ALIGN = 0, 1, 2, 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sq.library_path()):
        from paper_2511_22316_amd import build
        build.build()
    return binding._load()


def test_quantize_grouped_refusals(lib):
    def call(X=FAKE, T=4, K=256, ldx=256, group=64, Q=FAKE, s=FAKE):
        return lib.sq_quantize_grouped(X, T, K, ldx, group, Q, s, None)
    assert call(T=0) == OK
    assert call(T=0, X=None, Q=None, s=None) == OK
    for group in (0, 16, 48, 512, -32):
        assert call(group=group) == SHAPE
    assert call(K=96) == SHAPE and call(K=0) == SHAPE and call(K=131072 + 256, ldx=1 << 20) == SHAPE
    assert call(T=-1) == SHAPE and call(T=(1 << 30) + 1) == SHAPE and call(ldx=248) == SHAPE
    assert call(T=1 << 30, K=131072, ldx=131072) == SHAPE
    assert call(X=None) == NULL and call(Q=None) == NULL and call(s=None) == NULL
    assert call(X=FAKE + 2) == ALIGN and call(ldx=260) == ALIGN and call(Q=FAKE + 8) == ALIGN and call(s=FAKE + 1) == ALIGN


def test_w4a16_gemm_grouped_refusals(lib):
    def call(X=FAKE, T=4, K=256, ldx=256, Q=FAKE, s=FAKE, group=64, N=8, Y=FAKE, ldy=8):
        return lib.sq_w4a16_gemm_grouped(X, T, K, ldx, Q, s, group, N, Y, ldy, None)
    assert call(T=0) == OK and call(N=0, ldy=0) == OK
    for group in (0, 16, 96, 512):
        assert call(group=group) == SHAPE
    assert call(K=96, group=32) == SHAPE and call(K=320, ldx=320, group=128) == SHAPE and call(K=0) == SHAPE
    assert call(K=131072 + 256, ldx=1 << 20) == SHAPE
    assert call(T=-1) == SHAPE and call(N=-1) == SHAPE and call(T=(1 << 24) + 1) == SHAPE
    assert call(ldx=248) == SHAPE and call(ldy=7) == SHAPE
    for name in ("X", "Q", "s", "Y"):
        assert call(**{name: None}) == NULL
    assert call(X=FAKE + 8) == ALIGN and call(ldx=260) == ALIGN and call(Q=FAKE + 8) == ALIGN
    assert call(Y=FAKE + 1) == ALIGN and call(s=FAKE + 1) == ALIGN


def test_rotary_refusals(lib):
    def call(X=FAKE, T=2, H=3, D=64, ldx=192, ldh=64, p=FAKE, t=FAKE, rot=32, half=0, Y=2 * FAKE, ldy=192, ldyh=64):
        return lib.sq_rotary_fp16(X, T, H, D, ldx, ldh, p, t, rot, half, 1.0, Y, ldy, ldyh, None)
    assert call(T=0) == OK and call(H=0) == OK
    assert call(rot=0, Y=FAKE) == OK                        # in place and nothing to turn
    assert call(rot=31) == SHAPE and call(rot=66) == SHAPE and call(rot=-2) == SHAPE and call(D=2048, ldh=2048, ldyh=2048, ldx=6144, ldy=6144, rot=1026) == SHAPE
    assert call(half=2) == SHAPE and call(T=-1) == SHAPE and call(H=-1) == SHAPE and call(D=0) == SHAPE
    assert call(ldh=63) == SHAPE and call(ldx=191) == SHAPE and call(ldyh=63) == SHAPE and call(ldy=191) == SHAPE
    assert call(Y=FAKE, ldy=200) == SHAPE                   # in place with other strides
    for name in ("X", "Y", "p", "t"):
        assert call(**{name: None}) == NULL
    assert call(X=FAKE + 1) == ALIGN and call(Y=FAKE + 1) == ALIGN and call(p=FAKE + 2) == ALIGN and call(t=FAKE + 4) == ALIGN


@pytest.mark.parametrize("rot", [2, 4, 20, 64, 128, 1024])
def test_rotary_table(lib, rot):
    for kind in (dict(), dict(base=500000.0), dict(scaling=sq.SQ_ROTARY_LINEAR, factor=4.0), dict(scaling=sq.SQ_ROTARY_BASE, factor=3.0),
                 dict(scaling=sq.SQ_ROTARY_PARTS, factor=8.0, trained=8192.0, low=1.0, high=4.0),
                 dict(scaling=sq.SQ_ROTARY_PARTS, factor=1.0, trained=4096.0, low=0.0, high=32.0)):
        if rot == 2 and kind.get("scaling") == sq.SQ_ROTARY_BASE:
            continue
        turns = sq.sq_rotary_table(rot, **kind).numpy().view(np.uint64).astype(np.float64) / 2.0 ** 64
        f = ou.frequencies(rot, **kind)
        assert np.abs(turns * 2 * np.pi / f - 1).max() < 1e-13, kind      # a few roundings in 64 bits


def test_rotary_table_refusals(lib):
    for bad in (dict(rot=3), dict(rot=0), dict(rot=-2), dict(rot=1026), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")),
                dict(rot=2, scaling=2, factor=2.0), dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, trained=8.0, low=2.0, high=2.0),
                dict(scaling=3, factor=2.0, trained=8.0, low=-1.0, high=2.0)):
        with pytest.raises(sq.SQError) as e:
            sq.sq_rotary_table(**{"rot": 64, **bad})
        assert e.value.code == SHAPE, bad
    assert lib.sq_rotary_table(64, 10000.0, 0, 1.0, 0.0, 0.0, 0.0, None) == NULL


def test_cache_page_bytes(lib):
    assert sq.sq_cache_page_bytes(8, 128, 64) == 8 * 64 * 132
    assert sq.sq_cache_page_bytes(1, 64, 16) == (16 * 68 + 255) // 256 * 256
    for bad in ((0, 128, 64), (257, 128, 64), (8, 96, 64), (8, 512, 64), (8, 128, 8), (8, 128, 48), (8, 128, 2048), (8, 128, 0)):
        assert sq.sq_cache_page_bytes(*bad) == 0, bad


def test_cache_refusals(lib):
    def append(K=FAKE, ldk=256, V=FAKE, ldv=256, T=4, Hk=2, D=128, start=FAKE, cached=FAKE, B=2, table=FAKE, per=3, page=16, cache=FAKE, pages=9):
        a = lib.sq_cache_append(K, ldk, V, ldv, T, Hk, D, start, cached, B, table, per, page, cache, pages, None)
        b = lib.sq_cache_read(cache, pages, Hk, D, start, cached, B, table, per, page, K, ldk, V, ldv, T, None)
        assert a == b
        return a
    for name in ("T", "B", "per", "pages"):
        assert append(**{name: 0}) == OK                    # nothing to do, nothing enqueued
    for name in ("T", "B", "per", "pages", "Hk", "page", "D"):
        assert append(**{name: -1}) == SHAPE
    assert append(Hk=257, ldk=1 << 20, ldv=1 << 20) == SHAPE and append(D=96) == SHAPE and append(page=24) == SHAPE
    assert append(B=65536) == SHAPE and append(per=1 << 27, page=16) == SHAPE and append(ldk=248) == SHAPE and append(ldv=248) == SHAPE
    for name in ("K", "V", "start", "cached", "table", "cache"):
        assert append(**{name: None}) == NULL
    assert append(K=FAKE + 2) == ALIGN and append(V=FAKE + 8) == ALIGN and append(ldk=260) == ALIGN and append(ldv=260) == ALIGN
    assert append(cache=FAKE + 8) == ALIGN and append(start=FAKE + 2) == ALIGN and append(cached=FAKE + 1) == ALIGN and append(table=FAKE + 2) == ALIGN


def test_tree_attention_refusals(lib):
    def call(Q=FAKE, ldq=512, T=4, Hq=4, Hk=2, D=128, start=FAKE, cached=FAKE, B=2, mask=FAKE, max_rows=4, max_keys=100, table=FAKE,
             per=3, page=16, cache=FAKE, pages=9, scale=0.1, O=FAKE, ldo=512, ws=FAKE, bytes_=64):
        return lib.sq_tree_attention(Q, ldq, T, Hq, Hk, D, start, cached, B, mask, max_rows, max_keys, table, per, page, cache, pages,
                                     scale, O, ldo, ws, bytes_, None)
    assert call(T=0) == OK and call(B=0) == OK and call(max_rows=0) == OK
    for name in ("T", "B", "per", "pages", "Hk", "Hq", "page", "D", "max_rows", "max_keys", "bytes_"):
        assert call(**{name: -1}) == SHAPE, name
    assert call(Hq=3, ldq=512) == SHAPE and call(D=96) == SHAPE and call(page=40) == SHAPE and call(ldq=504) == SHAPE and call(ldo=504) == SHAPE
    assert call(max_rows=65) == SHAPE                       # a word of the mask has 64 bits
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == SHAPE
    for name in ("Q", "O", "start", "cached", "table", "cache", "ws"):
        assert call(**{name: None}) == NULL, name
    assert call(Q=FAKE + 2) == ALIGN and call(O=FAKE + 8) == ALIGN and call(ldq=516) == ALIGN and call(ldo=516) == ALIGN
    assert call(mask=FAKE + 4) == ALIGN and call(cache=FAKE + 8) == ALIGN and call(ws=FAKE + 8) == ALIGN and call(table=FAKE + 2) == ALIGN
    assert sq.sq_tree_attention_workspace_bytes(-1, 4, 128) == -1 and sq.sq_tree_attention_workspace_bytes(4, 0, 128) == -1
    assert sq.sq_tree_attention_workspace_bytes(4, 4, 96) == -1 and sq.sq_tree_attention_workspace_bytes(0, 4, 128) >= 0


def test_bindings_refuse_wrong_types_and_shapes(lib):
    import torch
    h = lambda *s: torch.zeros(s, dtype=torch.float16)      # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)        # noqa: E731
    u = lambda *s: torch.zeros(s, dtype=torch.uint8)        # noqa: E731
    with pytest.raises(ValueError):
        sq.sq_quantize_grouped(h(2, 64), 32, u(2, 32), torch.zeros(2, 2))
    with pytest.raises(ValueError):
        sq.sq_quantize_grouped(h(2, 64), 32, u(2, 16), h(2, 2))
    with pytest.raises(ValueError):
        sq.sq_quantize_grouped(h(64, 2).t(), 32, u(2, 32), h(2, 2))
    with pytest.raises(ValueError):
        sq.sq_w4a16_gemm_grouped(h(2, 64), u(5, 32), torch.zeros(5, 2), h(2, 5))
    with pytest.raises(ValueError):
        sq.sq_w4a16_gemm_grouped(h(2, 64), u(5, 32), h(5, 2), h(2, 4))
    with pytest.raises(ValueError):
        sq.sq_w4a16_gemm_grouped(h(2, 64).float(), u(5, 32), h(5, 2), h(2, 5))
    x = h(2, 3, 64)
    turns = sq.sq_rotary_table(32)
    with pytest.raises(ValueError):
        sq.sq_rotary_fp16(x, torch.zeros(2, dtype=torch.int64), turns, True, x)
    with pytest.raises(ValueError):
        sq.sq_rotary_fp16(x, i(3), turns, True, x)
    with pytest.raises(ValueError):
        sq.sq_rotary_fp16(x, i(2), turns.float(), True, x)
    with pytest.raises(ValueError):
        sq.sq_rotary_fp16(x.transpose(1, 2), i(2), turns, True, x.transpose(1, 2))
    cache = u(4 * sq.sq_cache_page_bytes(3, 64, 16))
    good = dict(row_start=i(3), cached=i(2), table=i(2, 2), page=16, cache=cache)
    for bad in (dict(row_start=i(2)), dict(cached=i(3)), dict(table=torch.zeros(2, 2, dtype=torch.int64)), dict(cache=cache[:-1]),
                dict(table=i(4, 2)[::2])):
        with pytest.raises(ValueError):
            sq.sq_cache_append(x, x, **{**good, **bad})
    with pytest.raises(ValueError):
        sq.sq_cache_append(x, h(2, 2, 64), **good)
    with pytest.raises(ValueError):
        sq.sq_cache_append(h(2, 6, 64)[:, ::2], x, **good)  # heads that do not lie side by side
    with pytest.raises(ValueError):
        sq.sq_tree_attention(x, i(3), i(2), torch.zeros(2, dtype=torch.int32), i(2, 2), 16, cache, 3, 0.1, x.clone())
    with pytest.raises(ValueError):
        sq.sq_tree_attention(x, i(3), i(2), torch.zeros(1, dtype=torch.int64), i(2, 2), 16, cache, 3, 0.1, x.clone())


def test_host_tensors_are_refused(lib):
    """A kernel that follows a host pointer would take the process down."""
    import torch
    h = lambda *n: torch.zeros(n, dtype=torch.float16)      # noqa: E731
    u = lambda *n: torch.zeros(n, dtype=torch.uint8)        # noqa: E731
    i = lambda *n: torch.zeros(n, dtype=torch.int32)        # noqa: E731
    x, cache = h(2, 3, 64), u(4 * sq.sq_cache_page_bytes(3, 64, 16))
    for call in (lambda: sq.sq_quantize_grouped(h(2, 64), 32, u(2, 32), h(2, 2)),
                 lambda: sq.sq_w4a16_gemm_grouped(h(2, 64), u(5, 32), h(5, 2), h(2, 5)),
                 lambda: sq.sq_rotary_fp16(x, i(2), sq.sq_rotary_table(32), True, x),
                 lambda: sq.sq_cache_append(x, x, i(3), i(2), i(2, 2), 16, cache),
                 lambda: sq.sq_cache_read(cache, i(3), i(2), i(2, 2), 16, x, x),
                 lambda: sq.sq_tree_attention(x, i(3), i(2), None, i(2, 2), 16, cache, 3, 0.1, x.clone())):
        with pytest.raises(ValueError, match="device"):
            call()


def test_attention_workspace_is_bounded(lib):
    size = sq.sq_tree_attention_workspace_bytes
    assert size(1, 32, 128) == 64 * 32 * 130 * 4            # every split of the only row
    assert size(256, 1, 64) == size(2048, 32, 64) == 16384 * 66 * 4
    assert [size(T, 8, 256) for T in (1, 31, 32)] == [64 * T * 8 * 258 * 4 for T in (1, 31, 32)]


def test_grouped_steps_of_groups_of_32_are_read_in_pairs(lib):
    call = lambda group, s: lib.sq_w4a16_gemm_grouped(FAKE, 4, 256, 256, FAKE, s, group, 8, FAKE, 8, None)       # noqa: E731
    assert call(32, FAKE + 2) == ALIGN and call(32, FAKE + 1) == ALIGN and call(64, FAKE + 1) == ALIGN

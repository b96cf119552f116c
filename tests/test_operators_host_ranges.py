"""Host-side checks (no GPU) of the group, rotary, cache and attention calls at the ends of their ranges."""
import decimal
import os

import numpy as np
import pytest

import paper_2511_22316_amd as sq
from paper_2511_22316_amd import binding


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sq.library_path()):
        from paper_2511_22316_amd import build
        build.build()
    return binding._load()


def turns_exact(rot, base=10000.0, scaling=0, factor=1.0, trained=0.0, low=0.0, high=0.0):
    """The frequencies in units of 2^-64 of a turn, to 60 digits."""
    with decimal.localcontext() as c:
        c.prec = 60
        D = decimal.Decimal
        two_pi = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459")
        base, factor, trained, low, high = (D(v) for v in (base, factor, trained, low, high))
        if scaling == sq.SQ_ROTARY_BASE:
            base *= (factor.ln() * rot / (rot - 2)).exp()
        out = []
        for i in range(rot // 2):
            f = (base.ln() * (-2 * i) / rot).exp()
            if scaling == sq.SQ_ROTARY_LINEAR:
                f /= factor
            if scaling == sq.SQ_ROTARY_PARTS:
                keep = min(max((trained * f / two_pi - low) / (high - low), D(0)), D(1))
                f = f * keep + f / factor * (1 - keep)
            out.append(f / two_pi * 2 ** 64)
        return out


@pytest.mark.parametrize("rot", [2, 6, 128, 1024])
@pytest.mark.parametrize("kind", [dict(), dict(base=500000.0), dict(base=1.0000001), dict(base=1e18), dict(scaling=sq.SQ_ROTARY_LINEAR, factor=3.0),
                                  dict(scaling=sq.SQ_ROTARY_BASE, factor=2.7), dict(scaling=sq.SQ_ROTARY_BASE, factor=1e9),
                                  dict(scaling=sq.SQ_ROTARY_PARTS, factor=8.0, trained=8192.0, low=1.0, high=32.0)])
def test_rotary_table_to_the_last_units(lib, rot, kind):
    """A frequency is a 64-bit fraction of a turn, and an angle is position * frequency modulo a turn: at position 2^31 an entry off by 2^10
    units would be an angle off by 2^-23 of a turn.  The logarithm, power, quotients and sums are 64-bit significands: of a number below
    2^61.4 units a few roundings are a few units."""
    if rot == 2 and kind.get("scaling") == sq.SQ_ROTARY_BASE:
        return
    got = [int(v) for v in sq.sq_rotary_table(rot, **kind).numpy().view(np.uint64)]
    off = [abs(g - w) for g, w in zip(got, turns_exact(rot, **kind))]
    assert max(off) <= 4, (rot, kind, [int(o) for o in off[:8]])


def test_grouped_product_refuses_more_channels_than_it_numbers(lib):
    """Channel numbers are 32-bit and are padded to a tile's end."""
    FAKE, SHAPE = 0x1000, 2                                 # never dereferenced: validation fails first
    for T in (1, 16, 32, 33, 64, 1000):
        for N in ((1 << 28) + 1, 2 ** 31 - 1):
            for group in (32, 256):
                assert lib.sq_w4a16_gemm_grouped(FAKE, T, 256, 256, FAKE, FAKE, group, N, FAKE, N, None) == SHAPE, (T, N, group)
    assert lib.sq_w4a16_gemm_grouped(FAKE, 1 << 24, 256, 256, FAKE, FAKE, 64, 1 << 28, FAKE, 1 << 28, None) == SHAPE     # 2^37 tiles


def test_attention_plan(lib):
    """What the rules of a call's sizes say, without a GPU: refusals, and workgroups that a launch can count."""
    import ctypes
    out = [ctypes.c_int32(0) for _ in range(3)]
    def plan(T=64, Hq=32, Hk=8, D=128, B=64, max_rows=1, max_keys=4096, workspace=64 << 20):
        splits = lib.sq_debug_tree_attention_plan(T, Hq, Hk, D, B, max_rows, max_keys, workspace, *[ctypes.byref(o) for o in out])
        return (splits, *[o.value for o in out])
    for bad in (dict(T=0), dict(T=-1), dict(Hq=31), dict(Hk=0), dict(D=96), dict(B=0), dict(max_rows=0), dict(max_keys=-1), dict(workspace=-1)):
        assert plan(**bad)[0] == -1, bad
    assert plan()[:3] == (2, 16, 0) and plan(max_keys=2000)[:3] == (1, 16, 0)        # 512 workgroups for the sequences, twice for long ones
    assert plan(T=1, B=1, max_keys=16384)[:3] == (32, 16, 0) and plan(T=1, B=1, max_keys=16384, workspace=0)[0] == 1
    assert plan(T=61, B=1, max_rows=61, max_keys=16384)[:3] == (8, 32, 0)
    assert plan(T=16 * 61, B=16, max_rows=61)[:3] == (1, 32, 0)
    assert plan(T=2111, B=64, max_rows=2048, max_keys=32768)[:3] == (1, 32, 1)
    assert plan(T=8192, B=1024, max_rows=8192, D=256)[:3] == (1, 16, 1)
    # keys of a split times splits hold max_keys, whatever it is
    for keys in (0, 1, 127, 129, 1000, 4097, 70000, 2 ** 31 - 1):
        for T in (1, 3, 40):
            splits, _, _, each = plan(T=T, B=T, max_keys=keys)
            assert 1 <= splits <= 64 and splits * each >= keys and each % 128 == 0


def test_grouped_plan(lib):
    """Which kernel a product takes: the shapes that the GPU tests mean for each of them."""
    from test_gpu_operators_ranges import KERNELS
    for kernel, shapes in KERNELS.items():
        for T, K, N in shapes:
            for group in (32, 64, 128, 256):
                assert lib.sq_debug_grouped_plan(T, K, group, N) == kernel, (T, K, N, group)
    for bad in ((0, 256, 32, 8), (4, 256, 32, 0), (-1, 256, 32, 8), (4, 96, 32, 8), (4, 256, 48, 8), (4, 320, 128, 8), (4, 256, 32, (1 << 28) + 1)):
        assert lib.sq_debug_grouped_plan(*bad) == 0, bad


def test_library_loads_without_torch_names_of_its_own_gpu_build(lib, monkeypatch):
    """Host-only calls need no more of torch than its tensors; a torch without GPU has no device and stream calls of its own."""
    import torch
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    for name in ("_lib", "_raw_stream", "_raw_device"):
        monkeypatch.setattr(binding, name, None)
    assert sq.sq_kron_factor(4096) == (64, 64)
    assert sq.sq_status_string(0) == "ok" and sq.sq_cache_page_bytes(8, 128, 64) == 8 * 64 * 132
    x = torch.zeros(2, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="device"):
        sq.sq_quantize_grouped(x, 32, torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.float16))
    assert binding._raw_device is torch.cuda.current_device and callable(binding._raw_stream)


def test_bindings_refuse_numbers_beyond_32_bits(lib):
    """ctypes would pass on the lower 32 bits: 2^32 + 1 rows at most would be one."""
    import torch
    i = lambda *n: torch.zeros(n, dtype=torch.int32)        # noqa: E731
    x, cache = torch.zeros(2, 3, 64, dtype=torch.float16), torch.zeros(4 * sq.sq_cache_page_bytes(3, 64, 16), dtype=torch.uint8)
    def attention(**kw):
        sq.sq_tree_attention(x, i(3), i(2), None, i(2, 2), kw.pop("page", 16), cache, kw.pop("Hk", 3), 0.1, x.clone(), **kw)
    for bad in (dict(max_rows=2 ** 32 + 1), dict(max_keys=2 ** 32), dict(page=2 ** 32 + 16), dict(Hk=2 ** 32 + 3)):
        with pytest.raises(ValueError, match="32 bits"):
            attention(**bad)
    with pytest.raises(ValueError, match="32 bits"):
        sq.sq_cache_append(x, x, i(3), i(2), i(2, 2), 2 ** 32 + 16, cache)
    assert sq.sq_cache_page_bytes(2 ** 32 + 3, 64, 16) == 0
    for rot in (2 ** 32 + 64, 2 ** 40):
        with pytest.raises(sq.SQError):
            sq.sq_rotary_table(rot)

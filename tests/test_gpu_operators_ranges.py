"""GPU parity of the group, rotary, cache and attention calls at the ends of their ranges, and on every kernel that a call may take,
against the plain 64-bit forms and bounds of operators_util."""
import numpy as np
import pytest

import operators_util as ou
from parity_util import dev, host
from test_gpu_operators import Setting, rng, rows, run_product, weights

pytestmark = pytest.mark.gpu


# ---- products --------------------------------------------------------------------------------------


@pytest.mark.parametrize("T,K,N,group", [(1, 256, 40, 32), (32, 512, 200, 128),           # a few tokens
                                         (64, 256, 8300, 32), (40, 512, 16500, 128),      # tiles of 64 x 128, K in two halves
                                         (300, 256, 8200, 64), (260, 512, 8200, 256),     # 128 x 128
                                         (100, 320, 8300, 32), (65, 192, 16400, 64),      # 128 x 256
                                         (3300, 192, 3900, 64)])                          # 256 x 256
def test_product_of_large_steps(T, K, N, group):
    """Steps up to the largest fp16, whose codes times the step are none, beside ordinary ones: a token's result does not depend on how
    many others there are.  Half the tokens are zero where the steps are large, so that what the ordinary ones give counts."""
    print(f"case product large steps {T} {K} {N} {group}", flush=True)
    g = rng(30, T, K, N, group)
    codes, steps = weights(g, N, K, group)
    large = g.random(steps.shape) < 0.3
    large[g.random(N) < 0.5] = False                        # half the channels have ordinary steps only
    steps[large] = g.choice([8184.0, 8192.0, -8192.0, 9000.0, 30000.0, -65504.0, 65504.0], int(large.sum())).astype(np.float16)
    X = (g.standard_normal((T, K)) * 2.0 ** -8).astype(np.float16)
    some = large.any(0)                                     # groups with a large step in any channel
    X.reshape(T, K // group, group)[1::2, some] = 0
    # the bound adds 16 |x| |step| over the channels; ou.product takes steps above 0, so the signs go to the codes: the same numbers
    want, bound = ou.product(X, codes * np.sign(steps).astype(int).repeat(group, 1), np.abs(steps), group, T > 32)
    if T > 32:
        # such a channel's codes * step / 8 are rounded to fp16 (below its normal range by 2^-25, so 2^-22) in place of codes * step
        beyond = (np.abs(steps.astype(np.float64)) >= 8192).any(1)
        bound = bound + (1 + ou.HALF) * (2.0 ** -22 - ou.TINY) * np.abs(X.astype(np.float64)).sum(1, keepdims=True) * beyond
    inside = np.abs(want) + bound < 65504.0
    assert inside.mean() > 0.9
    got = run_product(X, codes, steps, 8 * (T % 3), T % 2)
    ou.held(np.where(inside, got, 0), np.where(inside, want, 0), bound, f"{T} {K} {N} {group}")


def test_product_of_steps_that_are_not_finite():
    """A channel with an infinite step is not finite, and the others are what they are without it."""
    print("case product infinite steps", flush=True)
    for T, N in ((16, 100), (64, 8300)):
        g = rng(31, T)
        X = rows(g, T, 256)
        codes, steps = weights(g, N, 256, 64)
        want, bound = ou.product(X, codes, steps, 64, T > 32)
        steps[7, 1], steps[70, 3] = np.inf, np.nan
        got = run_product(X, codes, steps)
        there = np.isin(np.arange(N), (7, 70))
        assert not np.isfinite(got[:, there]).any()
        ou.held(got[:, ~there], want[:, ~there], bound[:, ~there], f"{T} {N}")


KERNELS = {  # what sq_debug_grouped_plan says: shapes (T, K, N), K an odd multiple of 256 (a half of it begins inside a group)
    1: [(5, 768, 1000), (33, 256, 500)], 2: [(1, 1280, 6000)], 3: [(3, 768, 9000)], 4: [(30, 768, 9000), (250, 768, 2040)],
    5: [(5, 4864, 7200)], 6: [(20, 1280, 16600), (15, 5376, 9000)], 7: [(20, 2304, 5000), (12, 8448, 5000)],
    8: [(64, 768, 8300)], 9: [(300, 768, 8200)], 10: [(600, 768, 9000)], 11: [(1000, 768, 9000)]}


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("kernel", sorted(KERNELS))
def test_product_on_every_kernel(kernel, group):
    """Every kernel with every group, and the shape that is meant to take it takes it."""
    from paper_2511_22316_amd import binding
    for T, K, N in KERNELS[kernel]:
        print(f"case product kernel {kernel} {T} {K} {N} {group}", flush=True)
        assert binding._load().sq_debug_grouped_plan(T, K, group, N) == kernel
        g = rng(32, T, K, N, group)
        X, (codes, steps) = rows(g, T, K), weights(g, N, K, group)
        want, bound = ou.product(X, codes, steps, group, T > 32)
        ou.held(run_product(X, codes, steps, 8, 3), want, bound, f"{kernel} {T} {K} {N} {group}")


@pytest.mark.parametrize("T,K,N,group", [(4, 512, 100, 64), (40, 512, 300, 32), (64, 512, 8300, 128), (100, 320, 8300, 32)])
def test_product_of_small_steps(T, K, N, group):
    """Steps below the normal range of fp16, whose codes times the step are below it too."""
    print(f"case product small steps {T} {K} {N} {group}", flush=True)
    g = rng(33, T, K, N, group)
    X = rows(g, T, K)
    codes = g.integers(-8, 8, (N, K))
    steps = (np.floor(2.0 ** g.uniform(0, 11, (N, K // group))) * 2.0 ** -24).astype(np.float16)
    want, bound = ou.product(X, codes, steps, group, T > 32)
    assert (bound < 0.2 * np.abs(want)).mean() > 0.7        # a number flushed to zero would be seen
    ou.held(run_product(X, codes, steps), want, bound, f"{T} {K} {N} {group}")


@pytest.mark.parametrize("T,group", [(1, 32), (20, 64), (300, 128), (40, 256)])
def test_layer_by_rotation_group_quantizer_and_product(T, group):
    """X W = (X R)(R^T W): rows of W^T and of X through the layer's own rotation, W to codes with steps per group, and the product of
    both.  R1 and R2 are Hadamard matrices / 4 and the rotated weights whole multiples -7 .. 7 of a power of two per group (7 among
    them), so every stage is exact: the weights before are multiples of 2^-4 of it below 2^11, the rotated X multiples of 2^-4 below 2^7,
    and the result is the fp16 next to X W."""
    import torch
    import paper_2511_22316_amd as sq
    print(f"case layer {T} {group}", flush=True)
    g = rng(34, T, group)
    K, N, n = 256, 300, 16
    H = np.array([[1.0]])
    while len(H) < n:
        H = np.block([[H, H], [H, -H]])
    R = np.kron(H / 4, H / 4)                               # x' = R1^T X_mat R2, row-major
    codes = g.integers(-7, 8, (N, K // group, group))
    codes[:, :, 5] = 7
    steps = 2.0 ** -g.integers(3, 5, (N, K // group)).astype(np.float64)
    rotated = (codes * steps[..., None]).reshape(N, K)
    Wt, X = rotated @ R.T, g.integers(-7, 8, (T, K)).astype(np.float64)
    assert np.array_equal(Wt, Wt.astype(np.float16)) and np.array_equal(X @ R, (X @ R).astype(np.float16))
    dR = dev((H / 4).astype(np.float16))
    out = []
    for x in (Wt, X):
        y = torch.empty(*x.shape, dtype=torch.float16, device="cuda")
        sq.sq_rotate_fp16(dev(x.astype(np.float16)), np.zeros(0, np.int32), np.zeros(0, np.int32), np.zeros(0, np.float32), dR, dR, y)
        out.append(y)
    Qw = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda")
    sw = torch.empty(N, K // group, dtype=torch.float16, device="cuda")
    Y = torch.empty(T, N, dtype=torch.float16, device="cuda")
    sq.sq_quantize_grouped(out[0], group, Qw, sw)
    sq.sq_w4a16_gemm_grouped(out[1], Qw, sw, Y)
    assert np.array_equal(host(sw), steps) and np.array_equal(host(Qw), ou.pack(codes.reshape(N, K)))
    assert np.array_equal(host(Y), (X @ Wt.T).astype(np.float16))


# ---- more threads than a launch counts along x -------------------------------------------------------


def test_rotary_of_more_pairs_than_32_bits():
    """2^32 pairs and a token more, in a place that allows one pair per lane, against the same tokens by themselves."""
    import torch
    import paper_2511_22316_amd as sq
    print("case rotary 2^32 pairs", flush=True)
    T, H, D = (1 << 22) + 1, 1024, 2
    base = dev(rows(rng(40), 1, H * D))[0]
    buf = torch.empty(1 + T * H * D, dtype=torch.float16, device="cuda")
    x = buf[1:].view(T, H, D)
    x[:] = base.view(H, D)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    turns = sq.sq_rotary_table(D, base=3.0).cuda()
    sq.sq_rotary_fp16(x, pos, turns, False, x)
    for first in (0, (1 << 21) - 5, T - 300):
        few = base.view(1, H, D).repeat(300, 1, 1)
        sq.sq_rotary_fp16(few, pos[first: first + 300].contiguous(), turns, False, few)
        assert torch.equal(x[first: first + 300], few), first
    del buf, x
    torch.cuda.empty_cache()


def test_cache_of_more_rows_than_a_row_of_workgroups():
    import torch
    import paper_2511_22316_amd as sq
    print("case cache 2^26 rows", flush=True)
    T, D, page, n = (1 << 26) + 5, 64, 1024, 1 << 16
    base = dev(rows(rng(41), n, D))
    few = [torch.empty(n, 1, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")       # noqa: E731
    pages = -(-T // page)
    cache = torch.empty(pages, sq.sq_cache_page_bytes(1, D, page), dtype=torch.uint8, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    k, v = base.view(n, 1, D), base.flip(0).view(n, 1, D).contiguous()
    sq.sq_cache_append(k, v, i32(0, n), i32(0), table, page, cache)
    sq.sq_cache_read(cache, i32(0, n), i32(0), table, page, *few)
    cache.zero_()
    many = [torch.empty(T, 1, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    for t, x in zip(many, (k, v)):
        t[: T - 5].view(-1, n, D)[:] = x.view(1, n, D)
        t[T - 5:] = x[:5]
    sq.sq_cache_append(*many, i32(0, T), i32(0), table, page, cache)
    for t in many:
        t.fill_(3.0)
    sq.sq_cache_read(cache, i32(0, T), i32(0), table, page, *many)
    for t, x in zip(many, few):
        assert torch.equal(t[T - 5:], x[:5])
        for part in t[: T - 5].view(-1, n, 1, D):
            assert torch.equal(part, x)
    del many, cache
    torch.cuda.empty_cache()


# ---- attention: sequences of very different numbers of rows ------------------------------------------


RAGGED = [  # past, new, Hq, Hk, D, page, tree
    ([3] * 30 + [40], [1] * 30 + [100], 8, 2, 64, 16, False), ([0, 5] * 20 + [17, 100], [0, 1] * 20 + [160, 0], 4, 4, 128, 64, False),
    ([30] * 20 + [2500, 9], [1] * 20 + [60, 2], 8, 1, 128, 32, True), ([200] * 33 + [1], [1] * 33 + [70], 16, 2, 256, 16, False),
    ([11] * 70, [1] * 69 + [64], 4, 2, 64, 16, True)]


@pytest.mark.parametrize("case", range(len(RAGGED)))
@pytest.mark.parametrize("max_keys", [None, 2 ** 31 - 1])
def test_attention_of_one_prompt_among_single_rows(case, max_keys):
    past, new, Hq, Hk, D, page, tree = RAGGED[case]
    print(f"case attention ragged {case} {max_keys}", flush=True)
    s = Setting(1300 + case, past, new, Hk, D, page)
    Q, scale = s.queries(Hq, 2.0), D ** -0.5
    words = s.trees() if tree else None
    want, bound = s.expect(Q, Hq // Hk, s.by_mask(words) if tree else s.causal, scale)
    for workspace in (0, 8 << 20):
        ou.held(s.run(Q, words, scale, workspace, max_keys=max_keys), want, bound, f"{case} {workspace}")
    # fewer rows than a sequence has: the others keep what they held
    most = max(new) - 7
    over = np.concatenate([np.arange(n) >= most for n in new])
    got = s.run(Q, words, scale, max_rows=most, max_keys=max_keys)
    assert (got[over] == 3.0).all()
    ou.held(got[~over], want[~over], bound[~over], f"{case} max_rows")


def test_attention_of_thousands_of_sequences_and_a_prompt():
    print("case attention 5000 sequences", flush=True)
    g = rng(42)
    new = g.integers(0, 2, 5000)
    new[3210], new[:7], new[-9:] = 90, 0, 0
    s = Setting(1400, list(g.integers(0, 3, 5000)), list(new), 1, 64, 16)
    Q = s.queries(2)
    want, bound = s.expect(Q, 2, s.causal, 0.2)
    ou.held(s.run(Q, None, 0.2, max_rows=90, max_keys=64), want, bound, "prompt among 5000")


def test_attention_of_rows_far_below_their_bound():
    """2^24 workgroups, were every sequence given row blocks for max_rows, and a launch has fewer."""
    print("case attention far below max_rows", flush=True)
    new = [0] * 1024
    new[0], new[500], new[1023] = 1, 40, 3
    s = Setting(1500, [2] * 1024, new, 8, 256, 16)
    import torch
    import paper_2511_22316_amd as sq
    Q = s.queries(32)
    want, bound = s.expect(Q, 4, s.causal, 0.1)
    T = 8192                                                # rows behind the last sequence
    q, o = (torch.full((T, 32, 256), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    q[: s.T] = dev(Q)
    sq.sq_tree_attention(q, s.dstart, s.dcached, None, s.dtable, 16, s.cache, 8, 0.1, o, max_rows=8192)
    torch.cuda.synchronize()
    ou.held(host(o[: s.T]), want, bound, "far below")
    assert (o[s.T:] == 3.0).all()


# ---- attention: long sequences, split and shared out in every way ------------------------------------


def plan(T, Hq, Hk, D, B, max_rows, max_keys, workspace):
    """Splits, query rows of a workgroup, whether row blocks are packed, and neighbouring keys of a split."""
    import ctypes
    from paper_2511_22316_amd import binding
    out = [ctypes.c_int32(0) for _ in range(3)]
    splits = binding._load().sq_debug_tree_attention_plan(T, Hq, Hk, D, B, max_rows, max_keys, workspace, *[ctypes.byref(o) for o in out])
    return (splits, out[0].value, out[1].value, out[2].value)


def held_long(s, got, Q, G, sees_of, scale, what):
    """As Setting.expect and held, with the term of products below the normal range of fp16 as the kernel's offset has it: where the offset
    moves, a row's largest product of weight and step is 2^5.9 or more, and it never falls afterwards; a product below the normal range
    is off by 2^-25 at most, times codes up to 8: n keys by n 2^-22 where the sum of products is 2^5.9 or more, n 2^-27.9 of it.
    operators_util.attention has n 2^-21, for a largest product of 2^-1."""
    want, bound = s.expect(Q, G, sees_of, scale)
    for b in range(s.B):
        L, rows_ = int(s.past[b] + s.new[b]), slice(s.start[b], s.start[b + 1])
        if L == 0 or s.new[b] == 0:
            continue
        (k, sk), (v, sv) = (s.numbers.values(b, w, L) for w in (0, 1))
        sees = sees_of(b, L)
        for h in range(Q.shape[1]):
            x = np.where(sees, (Q[rows_, h].astype(np.float64) @ k[:, h // G].T) * scale, -np.inf)
            some = sees.any(1)
            p = np.zeros(x.shape)
            p[some] = np.exp(x[some] - x[some].max(1, keepdims=True))
            p[some] /= p[some].sum(1, keepdims=True)
            n = sees.sum(1, keepdims=True)
            bound[rows_, h] -= (1 + ou.HALF) * n * (2.0 ** -21 - 2.0 ** -27.9) * (p @ sv[:, h // G])[:, None]
    ou.held(got, want, bound, what)


LONG = [  # past, new, Hq, Hk, D, page, tree, max_keys: splits, rows, packed of the plan with a workspace
    ([9000], [61], 8, 2, 64, 16, True, 40000, (32, 32, 0)),                          # 32 rows, eight splits of 1280 keys with something in them
    ([9000], [61], 8, 2, 128, 64, True, 40000, (32, 32, 0)),
    ([300, 12000, 0, 50, 900, 31, 2, 40], [61, 60, 64, 1, 7, 33, 50, 12], 8, 2, 64, 32, True, 4200, (4, 32, 0)),     # the next chunk, three times
    ([7000, 20], [64, 64], 16, 4, 128, 16, True, 8300, (8, 32, 0)),
    ([3000, 900, 0, 2500], [1, 1, 1, 1], 8, 2, 64, 16, False, 1024, (8, 16, 0)),     # 16 rows, the next chunk
    ([3000, 900, 0, 2500], [1, 1, 0, 1], 8, 2, 256, 64, False, 1024, (8, 16, 0)),
    ([2100, 5], [9, 3], 8, 1, 128, 32, True, 1024, (8, 16, 0)),
    ([40] * 9 + [6000, 0], [1] * 9 + [50, 1], 4, 1, 64, 16, True, 45000, (28, 32, 1)),      # packed and split
    ([16383], [1], 4, 1, 128, 64, False, None, (64, 16, 0)), ([20000], [1], 2, 2, 64, 16, False, 20001, (64, 16, 0)),
    ([100], [2048], 4, 1, 64, 64, False, None, (2, 32, 0)), ([0, 700], [2100, 513], 2, 1, 128, 16, False, None, (1, 32, 0)),
    ([0], [4100], 2, 1, 128, 32, False, None, (1, 32, 0)), ([50], [1100], 2, 1, 256, 16, False, None, (1, 16, 0))]


@pytest.mark.parametrize("case", range(len(LONG)))
def test_attention_of_long_sequences(case):
    past, new, Hq, Hk, D, page, tree, max_keys, how = LONG[case]
    print(f"case attention long {LONG[case]}", flush=True)
    s = Setting(1600 + case, past, new, Hk, D, page)
    hint, workspace = s.per * page if max_keys is None else max_keys, 64 << 20
    assert plan(s.T, Hq, Hk, D, s.B, max(new), hint, workspace)[:3] == how
    if max_keys is not None and how[0] > 1:
        splits, _, _, keys = plan(s.T, Hq, Hk, D, s.B, max(new), hint, workspace)
        assert max(past) > 2 * keys                         # several splits have keys of their own
    Q, scale = s.queries(Hq, 2.0), D ** -0.5
    words = s.trees() if tree else None
    sees = s.by_mask(words) if tree else s.causal
    for ws in (workspace, 0):
        held_long(s, s.run(Q, words, scale, ws, max_keys=max_keys), Q, Hq // Hk, sees, scale, f"{case} {ws}")


def test_a_sequence_that_begins_below_zero_is_left_out():
    """By all three calls alike, also where row blocks are numbered by row_start."""
    import torch
    import paper_2511_22316_amd as sq
    print("case row_start below zero", flush=True)
    Hk, D, page = 1, 64, 16
    for B in (2, 40):
        start = np.minimum(np.array([-2, 1] + [3 + b for b in range(B - 1)]), 41).astype(np.int32)
        T = int(start[-1]) + 60
        x = rows(rng(43, B), T, Hk * D).reshape(T, Hk, D)
        args = dev(start), dev(np.zeros(B, np.int32)), dev(np.arange(B, dtype=np.int32)[:, None]), page
        cache = torch.full((B, sq.sq_cache_page_bytes(Hk, D, page)), 0x77, dtype=torch.uint8, device="cuda")
        sq.sq_cache_append(dev(x), dev(x), *args, cache)
        assert (cache[0] == 0x77).all()
        k, v, o = (torch.full((T, Hk, D), 3.0, dtype=torch.float16, device="cuda") for _ in range(3))
        sq.sq_cache_read(cache, *args, k, v)
        sq.sq_tree_attention(dev(x), *args[:2], None, *args[2:], cache, Hk, 0.1, o, max_rows=T)
        codes, steps = ou.quantize(x)
        want = (codes * steps.astype(np.float64)[..., None]).astype(np.float16)
        own = np.arange(T) >= 1
        own[start[-1]:] = False
        for got in (k, v):
            assert np.array_equal(host(got)[own], want[own]) and (host(got)[~own] == 3.0).all()
        assert (host(o)[~own] == 3.0).all() and not (host(o)[own] == 3.0).all()


def test_a_stream_of_another_device_is_refused():
    """The work would be enqueued on a device that the tensors are not on."""
    import types

    import torch
    import paper_2511_22316_amd as sq
    print("case stream of another device", flush=True)
    x = torch.ones(2, 64, dtype=torch.float16, device="cuda")
    Q, steps = torch.zeros(2, 32, dtype=torch.uint8, device="cuda"), torch.zeros(2, 2, dtype=torch.float16, device="cuda")
    own = torch.cuda.Stream()
    other = types.SimpleNamespace(cuda_stream=own.cuda_stream, device_index=torch.cuda.current_device() + 1)
    torch.cuda.synchronize()
    with pytest.raises(ValueError, match="stream"):
        sq.sq_quantize_grouped(x, 32, Q, steps, stream=other)
    sq.sq_quantize_grouped(x, 32, Q, steps, stream=own)
    torch.cuda.synchronize()
    assert np.array_equal(host(Q), ou.pack(ou.quantize(np.ones((2, 2, 32)))[0].reshape(2, 64)))


def test_ragged_batches_captured():
    """A graph of a call whose row blocks are numbered by row_start, and whose sequences are split, replayed as the arrays' contents change:
    which sequence has the prompt, how many rows there are, how long the cache is."""
    import torch
    import paper_2511_22316_amd as sq
    print("case ragged captured", flush=True)
    B, Hq, Hk, D, page, T = 12, 4, 1, 64, 16, 80            # T: the most rows of a step, those behind the last sequence padding
    g = rng(44)
    sets = []
    for i in range(5):
        new = [1] * B
        new[(5 * i) % B], new[(5 * i + 3) % B] = 50 + 3 * i, i
        past = list(g.integers(0, 40, B))
        past[(5 * i) % B] = [3000, 10, 700, 0, 5000][i]
        s = Setting(1700 + i, past, new, Hk, D, page)
        Q = s.queries(Hq, 2.0)
        sets.append((s, Q, *s.expect(Q, Hq // Hk, s.causal, 0.2)))
    hint, workspace = 50000, 8 << 20
    how = plan(T, Hq, Hk, D, B, 64, hint, workspace)
    assert how[0] > 1 and how[2] == 1
    per, pages = max(s.per for s, *_ in sets), max(s.cache.shape[0] for s, *_ in sets)
    q, o = (torch.zeros(T, Hq, D, dtype=torch.float16, device="cuda") for _ in range(2))
    start, cached, table = (torch.zeros(*n, dtype=torch.int32, device="cuda") for n in ((B + 1,), (B,), (B, per)))
    cache = torch.zeros(pages, sets[0][0].size, dtype=torch.uint8, device="cuda")
    ws = torch.empty(workspace, dtype=torch.uint8, device="cuda")

    def load(s, Q):
        q.zero_()
        q[: s.T] = dev(Q)
        o.fill_(3.0)
        start.copy_(s.dstart)
        cached.copy_(s.dcached)
        table.fill_(-1)
        table[:, : s.per] = s.dtable
        cache[: s.cache.shape[0]] = s.cache
        torch.cuda.synchronize()

    def call():
        sq.sq_tree_attention(q, start, cached, None, table, page, cache, Hk, 0.2, o, ws, max_rows=64, max_keys=hint)

    load(*sets[0][:2])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for s, Q, want, bound in sets + sets[:2]:
        load(s, Q)
        graph.replay()
        torch.cuda.synchronize()
        replayed = o.clone()
        ou.held(host(o[: s.T]), want, bound, "replayed")
        assert (o[s.T:] == 3.0).all()
        o.fill_(3.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(o, replayed)

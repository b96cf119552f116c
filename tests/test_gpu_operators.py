"""GPU parity of the group quantizer, the products with a step per group, rotary positions, the paged 4-bit cache and its
attention, against plain 64-bit forms on the host (operators_util, where the bounds are derived)."""
import numpy as np
import pytest

import operators_util as ou
from parity_util import dev, host

pytestmark = pytest.mark.gpu


def rng(*seed):
    return np.random.default_rng(list(seed))


def rows(g, T, K):
    x = g.standard_normal((T, K)) * np.where(g.random((T, K)) < 0.01, 20.0, 1.0)
    x[:, g.integers(0, K, 2)] *= 30.0
    return x.astype(np.float16)


# ---- group quantizer -------------------------------------------------------------------------------


def run_quantize(X, group, pad=0):
    import torch
    import paper_2511_22316_amd as sq
    T, K = X.shape
    full = torch.full((T, K + pad), float("nan"), dtype=torch.float16, device="cuda")
    full[:, :K] = dev(X)
    Q = torch.full((T, K // 2), 0xA5, dtype=torch.uint8, device="cuda")
    steps = torch.full((T, K // group), 9.0, dtype=torch.float16, device="cuda")
    sq.sq_quantize_grouped(full[:, :K], group, Q, steps)
    torch.cuda.synchronize()
    return host(Q), host(steps)


@pytest.mark.parametrize("T,K,group,pad", [(1, 32, 32, 0), (1, 256, 256, 0), (3, 96, 32, 8), (5, 320, 64, 0), (257, 4096, 128, 0),
                                           (64, 11008, 128, 16), (130, 768, 256, 8), (1000, 64, 64, 0), (2, 131072, 32, 0)])
def test_quantize_grouped(T, K, group, pad):
    print(f"case quantize_grouped {T} {K} {group} {pad}", flush=True)
    X = rows(rng(1, T, K, group), T, K)
    Q, steps = run_quantize(X, group, pad)
    codes, want = ou.quantize(X.reshape(T, K // group, group))
    assert np.array_equal(steps, want)
    assert np.array_equal(Q, ou.pack(codes.reshape(T, K)))


def test_quantize_grouped_halves_zeros_and_the_ends_of_fp16():
    print("case quantize_grouped edges", flush=True)
    K = 128
    X = np.zeros((9, K), np.float16)
    X[0, :15] = np.arange(-7, 8)                             # step 1
    X[0, 32:47] = np.arange(-7, 8) - 0.5                     # max 7.5: step 1.0712890625
    X[0, 64:79], X[0, 80] = np.arange(-7, 8) - 0.5, 7.0      # every half-integer at step 15/14 rounded
    X[1, :14], X[1, 14] = np.arange(-7, 7) + 0.5, 7.0        # halves at step 1 go up
    X[2] = 65504.0
    X[3] = -65504.0
    X[4, ::3] = np.float16(2.0 ** -24)                       # below seven halves of the smallest step: step 1, codes 0
    X[5, ::5] = np.float16(5 * 2.0 ** -24)                   # the step is the smallest number
    X[6, ::7] = np.float16(10 * 2.0 ** -24)                  # the step rounds down: codes beyond the end are cut
    X[7] = np.linspace(-1e-4, 1e-4, K)
    X[8] = rng(5).standard_normal(K) * 6e-5
    Q, steps = run_quantize(X, 32)
    codes, want = ou.quantize(X.reshape(9, 4, 32))
    assert np.array_equal(steps, want)
    assert np.array_equal(Q, ou.pack(codes.reshape(9, K)))
    # every fp16 number up to the maximum of its group, against steps of all sizes
    g = rng(6)
    top = np.concatenate([np.float16(2.0) ** g.integers(-24, 16, 500), g.uniform(0, 60000, 524)]).astype(np.float16)
    top[top == 0] = 1
    X = (top[:, None].astype(np.float64) * g.uniform(-1, 1, (1024, 64))).astype(np.float16)
    X[:, 0] = top
    half = (np.floor(g.uniform(-7, 7, (1024, 20))) + 0.5) * (X[:, :1] / np.float32(7)).astype(np.float16).astype(np.float64)
    X[:, 1:21] = np.clip(half, -top[:, None].astype(np.float64), top[:, None].astype(np.float64)).astype(np.float16)
    Q, steps = run_quantize(X, 64)
    codes, want = ou.quantize(X.reshape(1024, 1, 64))
    assert np.array_equal(steps, want)
    assert np.array_equal(Q, ou.pack(codes.reshape(1024, 64)))


# ---- products --------------------------------------------------------------------------------------


def run_product(X, codes, steps, pad_x=0, pad_y=0):
    import torch
    import paper_2511_22316_amd as sq
    T, K = X.shape
    N = codes.shape[0]
    full = torch.full((T, K + pad_x), float("nan"), dtype=torch.float16, device="cuda")
    full[:, :K] = dev(X)
    Y = torch.full((T, N + pad_y), 7.0, dtype=torch.float16, device="cuda")
    sq.sq_w4a16_gemm_grouped(full[:, :K], dev(ou.pack(codes)), dev(steps), Y[:, :N])
    torch.cuda.synchronize()
    Y = host(Y)
    assert (Y[:, N:] == 7.0).all()
    return Y[:, :N]


def weights(g, N, K, group):
    steps = (g.uniform(0.2, 1.0, (N, K // group)) * np.where(g.random((N, K // group)) < 0.05, 8.0, 1.0) * 0.01).astype(np.float16)
    return g.integers(-8, 8, (N, K)), steps


FEW = [(1, 64, 1, 32), (1, 64, 17, 64), (1, 256, 100, 256), (2, 320, 33, 64), (3, 384, 50, 128), (1, 4096, 256, 128),
       (16, 4096, 130, 32), (15, 2048, 16, 64), (5, 11008, 48, 128), (17, 512, 96, 32), (32, 1024, 80, 256), (31, 4160, 40, 32),
       (8, 8192, 4100, 128), (1, 8192, 4112, 32), (4, 1024, 16500, 64), (1, 28672, 64, 64), (7, 192, 20000, 32), (1, 131072, 20, 256)]
MANY = [(33, 64, 40, 32), (64, 4096, 256, 128), (100, 320, 130, 64), (333, 512, 200, 32), (129, 2048, 97, 256), (257, 1088, 64, 64),
        (600, 4096, 300, 32), (1000, 256, 1111, 128), (2048, 128, 512, 64),
        (3300, 192, 3900, 64), (3300, 256, 3850, 32)]


@pytest.mark.parametrize("T,K,N,group", FEW + MANY)
def test_product(T, K, N, group):
    print(f"case product {T} {K} {N} {group}", flush=True)
    g = rng(2, T, K, N, group)
    X = rows(g, T, K)
    codes, steps = weights(g, N, K, group)
    Y, bound = ou.product(X, codes, steps, group, T > 32)
    ou.held(run_product(X, codes, steps, 8 * (T % 3), T % 2), Y, bound, f"{T} {K} {N} {group}")


@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
def test_product_finds_every_place(T, group):
    """Rows with one channel set, codes and steps all different: every product must be the one code times the one step."""
    K, N = 512, 70
    print(f"case product places {T} {group}", flush=True)
    g = rng(3, T, group)
    codes = g.integers(-8, 8, (N, K))
    steps = (2.0 ** g.integers(-8, 3, (N, K // group))).astype(np.float16)
    for k in (list(range(0, K, 37)) + [K - 1])[:: 1 if T == 1 else 4]:
        X = np.zeros((T, K), np.float16)
        at = (k + 5 * np.arange(T)) % K
        X[np.arange(T), at] = 1 + np.arange(T)
        want = (codes[:, at] * steps[:, at // group].astype(np.float64)).T * (1 + np.arange(T))[:, None]
        assert np.array_equal(run_product(X, codes, steps).astype(np.float64), want), k


def test_product_small_and_large_activations():
    print("case product range", flush=True)
    g = rng(4)
    for T in (1, 12, 50):
        for factor in (2.0 ** -12, 1.0, 500.0):
            X = (g.standard_normal((T, 512)) * factor).astype(np.float16)
            codes, steps = weights(g, 64, 512, 64)
            Y, bound = ou.product(X, codes, steps, 64, T > 32)
            ou.held(run_product(X, codes, steps), Y, bound, f"{T} {factor}")
    # beyond fp16: infinite, as any rounding to it; a row of infinities stays in its row
    X = np.full((2, 64), 1000.0, np.float16)
    X[1] = 1.0
    got = run_product(X, np.full((3, 64), 7), np.full((3, 2), 100.0, np.float16))
    assert np.isposinf(got[0]).all() and (got[1] == 44800.0).all()


# ---- rotary ----------------------------------------------------------------------------------------


ROTARY = [(1, 1, 2, 2), (1, 40, 128, 128), (3, 5, 64, 32), (7, 3, 80, 80), (5, 2, 80, 20), (9, 4, 96, 48), (2, 3, 7, 4),
          (300, 12, 128, 64), (17, 1, 256, 256), (2, 2, 24, 16), (4, 3, 40, 0), (1000, 40, 64, 64)]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("T,H,D,rot", ROTARY)
def test_rotary(T, H, D, rot, half):
    import torch
    import paper_2511_22316_amd as sq
    print(f"case rotary {T} {H} {D} {rot} {half}", flush=True)
    g = rng(7, T, H, D, rot)
    X = rows(g, T, (H + 2) * D).reshape(T, H + 2, D)
    pos = g.integers(0, 2 ** 20, T).astype(np.int32)
    pos[0] = 2 ** 31 - 1 if T % 2 else -5
    kinds = [dict(), dict(scaling=1, factor=4.0), dict(scaling=3, factor=8.0, trained=8192.0, low=1.0, high=32.0, base=500000.0)]
    if rot > 2:
        kinds.append(dict(scaling=2, factor=2.5))
    kind = kinds[T % len(kinds)]
    magnitude = 1.2079 if T % 2 else 1.0
    turns = sq.sq_rotary_table(rot, **kind) if rot else torch.zeros(0, dtype=torch.int64)
    want, bound = ou.rotary(X[:, :H], pos, ou.frequencies(rot, **kind), half, np.float32(magnitude).astype(np.float64))
    # part of a wider row into a tensor of its own
    dX = dev(X)
    Y = torch.full((T, H, D), 5.0, dtype=torch.float16, device="cuda")
    sq.sq_rotary_fp16(dX[:, :H], dev(pos), turns.cuda(), half, Y, magnitude=magnitude)
    ou.held(host(Y), want, bound, "own tensor")
    assert np.array_equal(host(dX), X)
    # in place: the heads behind and the channels behind `rot` stay
    sq.sq_rotary_fp16(dX[:, :H], dev(pos), turns.cuda(), half, dX[:, :H], magnitude=magnitude)
    got = host(dX)
    assert np.array_equal(got[:, :H], host(Y)) and np.array_equal(got[:, H:], X[:, H:])


def test_rotary_strides_and_alignment():
    import torch
    import paper_2511_22316_amd as sq
    print("case rotary strides", flush=True)
    g = rng(8)
    T, H, D, rot = 11, 3, 64, 32
    X = rows(g, T, H * D).reshape(T, H, D)
    pos = np.arange(T, dtype=np.int32) * 1000
    turns = sq.sq_rotary_table(rot)
    want, bound = ou.rotary(X, pos, ou.frequencies(rot), True)
    for shift, head, extra in ((0, D, 0), (1, D, 0), (8, D + 8, 16), (0, D + 1, 3), (4, D, 4)):
        buf = torch.zeros(shift + T * (H * head + extra), dtype=torch.float16, device="cuda")
        view = buf[shift:].as_strided((T, H, D), (H * head + extra, head, 1), shift)
        view.copy_(dev(X))
        Y = torch.empty(T, H, D, dtype=torch.float16, device="cuda")
        sq.sq_rotary_fp16(view, dev(pos), turns.cuda(), True, Y)
        ou.held(host(Y), want, bound, f"strides {shift} {head} {extra}")
        sq.sq_rotary_fp16(dev(X), dev(pos), turns.cuda(), True, view)
        ou.held(host(view.contiguous()), want, bound, f"strides out {shift} {head} {extra}")


# ---- cache and attention ---------------------------------------------------------------------------


class Setting:
    """Sequences of given lengths in a cache of scattered pages, appended in two calls; what the numbers are, on the host."""

    def __init__(self, seed, past, new, Hk, D, page, spare=3, scale_v=1.0, fill=0xFF, pages_more=0):
        import torch
        import paper_2511_22316_amd as sq
        self.g = g = rng(9, seed)
        self.past, self.new = np.asarray(past), np.asarray(new)
        self.Hk, self.D, self.page, self.B = Hk, D, page, len(past)
        total = self.past + self.new
        self.per = max(1, int(-(-total.max() // page)))
        count = self.B * self.per + spare
        self.size = sq.sq_cache_page_bytes(Hk, D, page)
        # never-written slots hold bytes that are NaN as steps
        self.cache = torch.full((count + pages_more, self.size), fill, dtype=torch.uint8, device="cuda")
        self.table = (pages_more + g.permutation(count)[: self.B * self.per]).reshape(self.B, self.per).astype(np.int32)
        self.dtable = dev(self.table)
        self.numbers = ou.Cache(self.B)
        ends = np.concatenate([[0], np.cumsum(self.past)]).astype(np.int32)
        self._append(ends, np.zeros(self.B, np.int32), scale_v)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self._append(self.start, self.past.astype(np.int32), scale_v)
        self.T = int(self.start[-1])
        self.dstart, self.dcached = dev(self.start), dev(self.past.astype(np.int32))

    def _append(self, start, cached, scale_v):
        import paper_2511_22316_amd as sq
        T, W = int(start[-1]), self.Hk * self.D
        if T == 0:
            return
        kv = rows(self.g, T, 2 * W + 8)
        kv[:, W: 2 * W] = (kv[:, W: 2 * W].astype(np.float64) * scale_v).astype(np.float16)
        if T > 2:
            kv[T // 2] = 0
        d = dev(kv)
        k, v = (d[:, i * W: (i + 1) * W].unflatten(1, (self.Hk, self.D)) for i in range(2))
        sq.sq_cache_append(k, v, dev(start), dev(cached), self.dtable, self.page, self.cache)
        for b in range(self.B):
            for r in range(start[b], start[b + 1]):
                self.numbers.append(b, kv[r, :W].reshape(self.Hk, self.D), kv[r, W: 2 * W].reshape(self.Hk, self.D))

    def expect(self, Q, G, sees_of, scale, absent=lambda b, L: np.zeros(L, bool)):
        O, bound = np.zeros(Q.shape), np.zeros(Q.shape)
        for b in range(self.B):
            L, rows_ = int(self.past[b] + self.new[b]), slice(self.start[b], self.start[b + 1])
            if L == 0 or self.new[b] == 0:
                continue
            (k, sk), (v, sv) = (self.numbers.values(b, w, L) for w in (0, 1))
            sees = sees_of(b, L) & ~absent(b, L)
            for h in range(Q.shape[1]):
                O[rows_, h], bound[rows_, h] = ou.attention(Q[rows_, h], k[:, h // G], v[:, h // G], sk[:, h // G], sv[:, h // G],
                                                            sees, scale)
        return O, bound

    def causal(self, b, L):
        return np.arange(L) <= self.past[b] + np.arange(self.new[b])[:, None]

    def trees(self):
        words = np.zeros(self.T, np.uint64)
        for b in range(self.B):
            for i in range(self.new[b]):
                w = np.uint64(1) << np.uint64(i)
                if i > 0:
                    w |= words[self.start[b] + max(0, i - 1 - int(self.g.integers(0, 6)))]
                words[self.start[b] + i] = w
        return words

    def by_mask(self, words):
        def sees(b, L):
            new = np.arange(L) - self.past[b]
            w = words[self.start[b]: self.start[b + 1], None]
            return (new < 0) | ((w >> np.clip(new, 0, 63).astype(np.uint64)) & np.uint64(1)).astype(bool)
        return sees

    def queries(self, Hq, factor=1.0):
        return (factor * self.g.standard_normal((self.T, Hq, self.D))).astype(np.float16)

    def run(self, Q, mask, scale, workspace=8 << 20, max_rows=None, max_keys=None, table=None, O=None):
        import torch
        import paper_2511_22316_amd as sq
        O = torch.full(Q.shape, 3.0, dtype=torch.float16, device="cuda") if O is None else O
        ws = torch.full((workspace,), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
        sq.sq_tree_attention(dev(Q), self.dstart, self.dcached, None if mask is None else dev(mask.view(np.int64)),
                             self.dtable if table is None else dev(table), self.page, self.cache, self.Hk, scale, O, ws,
                             max_rows=int(self.new.max()) if max_rows is None else max_rows, max_keys=max_keys)
        torch.cuda.synchronize()
        return host(O)


@pytest.mark.parametrize("Hk,D,page", [(1, 64, 16), (3, 64, 64), (2, 128, 16), (8, 128, 64), (5, 128, 1024), (2, 256, 32), (1, 256, 16)])
def test_cache_append_and_read(Hk, D, page):
    import torch
    import paper_2511_22316_amd as sq
    print(f"case cache {Hk} {D} {page}", flush=True)
    s = Setting(D + page, [5, 0, 33, 1], [1, 3, 40, 0], Hk, D, page)
    total = s.past + s.new
    start = np.concatenate([[0], np.cumsum(total)]).astype(np.int32)
    T, W = int(start[-1]), Hk * D
    buf = torch.full((T + 2, 2 * W + 16), 3.0, dtype=torch.float16, device="cuda")
    k, v = buf[:, :W].unflatten(1, (Hk, D)), buf[:, W + 8: 2 * W + 8].unflatten(1, (Hk, D))
    sq.sq_cache_read(s.cache, dev(start), dev(np.zeros(4, np.int32)), s.dtable, page, k, v)
    got = host(buf)
    assert (got[T:] == 3.0).all() and (got[:, W: W + 8] == 3.0).all() and (got[:, 2 * W + 8:] == 3.0).all()
    for b in range(4):
        for which, at in ((0, 0), (1, W + 8)):
            want = s.numbers.values(b, which, int(total[b]))[0].astype(np.float16).reshape(total[b], W)
            assert np.array_equal(got[start[b]: start[b + 1], at: at + W], want), (b, which)
    # slots that no row went to, pages that no sequence has, and what is behind the steps keep their bytes
    raw = host(s.cache)
    untouched = np.setdiff1d(np.arange(raw.shape[0]), [s.table[b, i] for b in range(4) for i in range(-(-int(total[b]) // page))])
    assert (raw[untouched] == 0xFF).all()
    assert (raw[:, Hk * page * (D + 4):] == 0xFF).all()
    last = raw[s.table[0, 5 // page]]                       # sequence 0 holds 6 rows
    free = last[: Hk * page * D].reshape(Hk, 2, page * D // 2)[:, 0].reshape(Hk, page, D // 2)[:, 6:]
    assert (free == 0xFF).all()


def test_cache_rows_that_have_no_place():
    import torch
    import paper_2511_22316_amd as sq
    print("case cache without places", flush=True)
    Hk, D, page = 2, 64, 16
    size = sq.sq_cache_page_bytes(Hk, D, page)
    cache = torch.full((4, size), 0x77, dtype=torch.uint8, device="cuda")
    # sequence 0: its second page is -1, sequence 1: a page beyond the buffer, sequence 2: runs out of pages, 3: cached < 0
    table = np.array([[0, -1], [1, 4], [2, 3], [3, 2]], np.int32)
    cached, start = np.array([14, 15, 30, -1], np.int32), np.array([1, 5, 8, 12, 14], np.int32)
    x = rows(rng(11), 16, Hk * D).reshape(16, Hk, D)
    sq.sq_cache_append(dev(x), dev(x), dev(start), dev(cached), dev(table), page, cache)
    k, v = (torch.full((16, Hk, D), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    sq.sq_cache_read(cache, dev(start), dev(cached), dev(table), page, k, v)
    codes, steps = ou.quantize(x)
    want = np.full((16, Hk, D), 3.0, np.float16)
    for t in (1, 2, 5, 8, 9):                               # rows with a page and a slot; 0 and 14.. belong to no sequence
        want[t] = (codes[t] * steps[t].astype(np.float64)[:, None]).astype(np.float16)
    assert np.array_equal(host(k), want) and np.array_equal(host(v), want)
    raw = host(cache)
    assert (raw[3, : Hk * page * D].reshape(Hk, 2, -1)[:, 0].reshape(Hk, page, D // 2)[:, :14] == 0x77).all()


CASES = [  # past, new, Hq, Hk, D, page, tree
    ([0], [1], 1, 1, 64, 16, False), ([1], [1], 4, 1, 128, 16, False), ([700], [1], 8, 2, 128, 64, False),
    ([15, 16, 17, 0, 300], [1, 1, 1, 1, 1], 10, 2, 128, 16, False), ([63, 64, 31], [1, 0, 1], 16, 1, 64, 32, False),
    ([129, 5], [1, 1], 5, 5, 256, 32, False), ([40, 0, 90], [7, 7, 3], 4, 2, 64, 16, False), ([100, 3], [20, 33], 8, 8, 128, 64, False),
    ([0, 50], [130, 70], 6, 3, 128, 16, False), ([10], [300], 4, 2, 64, 128, False), ([5, 200], [17, 64], 8, 2, 128, 32, True),
    ([0, 33, 511], [64, 1, 40], 4, 1, 128, 16, True), ([90], [61], 16, 2, 256, 64, True), ([1, 2, 3], [2, 3, 4], 3, 3, 64, 16, True),
    ([2000], [5], 32, 4, 128, 64, True), ([1100, 30], [9, 2], 40, 8, 128, 128, True)]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("workspace", [0, 8 << 20])
def test_attention(case, workspace):
    past, new, Hq, Hk, D, page, tree = CASES[case]
    print(f"case attention {CASES[case]} {workspace}", flush=True)
    s = Setting(100 + case, past, new, Hk, D, page, scale_v=[1.0, 2.0 ** -12, 8.0][case % 3])
    Q, scale = s.queries(Hq, 2.0), D ** -0.5
    words = s.trees() if tree else None
    want, bound = s.expect(Q, Hq // Hk, s.by_mask(words) if tree else s.causal, scale)
    ou.held(s.run(Q, words, scale, workspace), want, bound, str(CASES[case]))


def test_attention_masks_that_leave_rows_empty():
    print("case attention empty rows", flush=True)
    for D in (64, 128, 256):
        s = Setting(200 + D, [0, 70, 0], [40, 9, 1], 2, D, 16)
        words = s.trees()
        words[::3] = 0                                      # in sequences without a past: rows that see nothing
        words[7] = np.uint64(1) << np.uint64(63)            # a bit that no new row has
        words[41] = np.uint64(0xFFFFFFFFFFFFFFFF)
        Q = s.queries(4, 3.0)
        sees = s.by_mask(words)
        want, bound = s.expect(Q, 2, sees, 0.125)
        for workspace in (0, 8 << 20):
            got = s.run(Q, words, 0.125, workspace)
            ou.held(got, want, bound, "empty rows")
            assert (got[0] == 0).all() and (got[7] == 0).all()


def test_attention_scores_far_apart():
    """One key that takes all the weight, scores in the hundreds, values of very different size."""
    print("case attention peaks", flush=True)
    for factor in (30.0, 300.0):
        s = Setting(int(factor), [600, 90], [3, 3], 2, 128, 32)
        Q = s.queries(8, factor)
        want, bound = s.expect(Q, 4, s.causal, 0.3)
        ou.held(s.run(Q, None, 0.3), want, bound, f"{factor}")
    s = Setting(77, [600], [1], 1, 128, 32)
    Q = np.zeros((1, 4, 128), np.float16)                   # all scores equal
    want, bound = s.expect(Q, 4, s.causal, 0.3)
    ou.held(s.run(Q, None, 0.3), want, bound, "equal scores")
    Q = (s.queries(4) * np.float16(2.0 ** -14)).astype(np.float16)      # queries below the normal range of fp16
    want, bound = s.expect(Q, 4, s.causal, 1000.0)
    ou.held(s.run(Q, None, 1000.0), want, bound, "tiny queries")


def test_attention_largest_scores():
    """Scores of millions: one key takes it all, nothing overflows; beyond what fp32 tells apart the result is still finite."""
    print("case attention largest scores", flush=True)
    s = Setting(78, [500, 40], [2, 1], 2, 64, 16)
    Q = (s.queries(4) * np.float16(3000)).astype(np.float16)
    got = s.run(Q, None, 5.0)
    assert np.isfinite(got.astype(np.float64)).all()
    for b in range(2):
        k = s.numbers.values(b, 0, int(s.past[b] + s.new[b]))[0]
        v, sv = s.numbers.values(b, 1, int(s.past[b] + s.new[b]))
        for t in range(s.start[b], s.start[b + 1]):
            L = int(s.past[b] + t - s.start[b] + 1)
            for h in range(4):
                order = np.argsort(k[:L, h // 2] @ Q[t, h].astype(np.float64))
                top2 = (k[order[-2:], h // 2] @ Q[t, h].astype(np.float64)) * 5.0
                if top2[1] - top2[0] > 64:                  # the rest is below 2^-90
                    # the weight and the result are rounded to fp16 (half a step each, the second one of the first's
                    # result); the eights come off sums of 16 steps a term, as in operators_util.attention
                    x = v[order[-1], h // 2]
                    bound = (2 * ou.HALF + ou.HALF ** 2 + 8 * ou.EPS32) * np.abs(x) + 40 * ou.EPS32 * 16 * sv[order[-1], h // 2] + ou.TINY
                    ou.held(got[t, h], x, bound, f"{b} {t} {h}")
    Q[:] = 60000.0
    assert np.isfinite(s.run(Q, None, 1e6).astype(np.float64)).all()


def test_attention_pages_that_do_not_exist():
    print("case attention bad pages", flush=True)
    s = Setting(300, [100, 40], [2, 2], 2, 128, 16)
    Q = s.queries(4)
    table = s.table.copy()
    table[0, 2], table[0, 4], table[1, :] = -1, 1 << 30, s.cache.shape[0]
    absent = lambda b, L: np.ones(L, bool) if b == 1 else np.isin(np.arange(L) // 16, (2, 4))    # noqa: E731
    want, bound = s.expect(Q, 2, s.causal, 0.1, absent)
    got = s.run(Q, None, 0.1, table=table)
    ou.held(got, want, bound, "bad pages")
    assert (got[2:] == 0).all()
    # a table too short for the sequences: what it holds
    short = np.ascontiguousarray(s.table[:, :2])
    want, bound = s.expect(Q, 2, s.causal, 0.1, lambda b, L: np.arange(L) >= 32)
    ou.held(s.run(Q, None, 0.1, table=short), want, bound, "short table")


def test_attention_leaves_other_rows_alone_and_takes_strides():
    import torch
    import paper_2511_22316_amd as sq
    print("case attention strides", flush=True)
    s = Setting(400, [30, 20, 10], [3, 2, 4], 2, 64, 16)
    Q = s.queries(6)
    want, bound = s.expect(Q, 3, s.causal, 0.2)
    T, W = s.T, 6 * 64
    buf = torch.full((T + 5, 2 * W + 24), float("nan"), dtype=torch.float16, device="cuda")
    q, o = buf[:, 8: 8 + W].unflatten(1, (6, 64)), buf[:, W + 16: 2 * W + 16].unflatten(1, (6, 64))
    q[:T] = dev(Q)
    buf[:, W + 16:] = 3.0
    start = s.start + 0
    # rows behind the last sequence, rows from max_rows on
    sq.sq_tree_attention(q, dev(start), s.dcached, None, s.dtable, 16, s.cache, 2, 0.2, o, None, max_rows=3)
    torch.cuda.synchronize()
    got = host(buf)[:, W + 16:]
    assert (got[T:] == 3.0).all() and (got[:, W:] == 3.0).all()
    o_ = got[:T, :W].reshape(T, 6, 64)
    assert (o_[8] == 3.0).all()                             # the fourth row of the last sequence
    ou.held(o_[:8], want[:8], bound[:8], "strides")


def test_attention_does_not_depend_on_the_split():
    """max_keys and the workspace say how the work is split, not what comes out."""
    print("case attention splits", flush=True)
    s = Setting(500, [1500, 12, 700], [1, 1, 1], 2, 128, 64)
    Q = s.queries(8)
    want, bound = s.expect(Q, 4, s.causal, 0.1)
    for workspace, max_keys in ((0, None), (16, None), (1 << 14, None), (1 << 16, 64), (8 << 20, 1), (8 << 20, 2 ** 31 - 1), (8 << 20, 0)):
        ou.held(s.run(Q, None, 0.1, workspace, max_keys=max_keys), want, bound, f"{workspace} {max_keys}")


def test_attention_cache_beyond_32_bits():
    import torch
    print("case attention long cache", flush=True)
    more = (5 << 30) // (8 * 64 * 132)                      # 5 GiB of pages in front
    s = Setting(600, [200, 90], [1, 1], 8, 128, 64, pages_more=more)
    assert s.cache.numel() > 1 << 32
    Q = s.queries(16)
    want, bound = s.expect(Q, 2, s.causal, 0.1)
    ou.held(s.run(Q, None, 0.1), want, bound, "long cache")
    del s
    torch.cuda.empty_cache()


def test_decode_step_of_all_operators_captured():
    """Projection, rotary positions, rows into the cache, attention, projection: as a program runs a step, eagerly and as a
    captured graph replayed with other inputs, positions and lengths; another stream."""
    import torch
    import paper_2511_22316_amd as sq
    print("case decode step", flush=True)
    g = rng(12)
    Hq, Hk, D, page, Kin, B, group = 8, 2, 128, 16, 512, 3, 64
    W = (Hq + 2 * Hk) * D
    wq, wo = (g.standard_normal((n, k)).astype(np.float16) * np.float16(0.05) for n, k in ((W, Kin), (Kin, Hq * D)))
    codes = [ou.quantize(w.reshape(w.shape[0], -1, group)) for w in (wq, wo)]
    Qw, sw = [], []
    for w in (wq, wo):
        q = torch.empty(w.shape[0], w.shape[1] // 2, dtype=torch.uint8, device="cuda")
        st = torch.empty(w.shape[0], w.shape[1] // group, dtype=torch.float16, device="cuda")
        sq.sq_quantize_grouped(dev(w), group, q, st)
        Qw.append(q)
        sw.append(st)
    turns_h = sq.sq_rotary_table(D)
    turns = turns_h.cuda()
    table = dev(g.permutation(12).reshape(3, 4).astype(np.int32))
    cache = torch.zeros(12, sq.sq_cache_page_bytes(Hk, D, page), dtype=torch.uint8, device="cuda")
    start = dev(np.arange(B + 1, dtype=np.int32))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    x = torch.zeros(B, Kin, dtype=torch.float16, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    qkv, o, y = (torch.zeros(B, n, dtype=torch.float16, device="cuda") for n in (W, Hq * D, Kin))

    def step(stream=None):
        sq.sq_w4a16_gemm_grouped(x, Qw[0], sw[0], qkv, stream=stream)
        heads = qkv.unflatten(1, (Hq + 2 * Hk, D))
        qk = heads[:, : Hq + Hk]
        sq.sq_rotary_fp16(qk, pos, turns, True, qk, stream=stream)
        sq.sq_cache_append(heads[:, Hq: Hq + Hk], heads[:, Hq + Hk:], start, pos, table, page, cache, stream=stream)
        sq.sq_tree_attention(heads[:, :Hq], start, pos, None, table, page, cache, Hk, D ** -0.5, o.view(B, Hq, D), ws, max_rows=1,
                             max_keys=64, stream=stream)
        sq.sq_w4a16_gemm_grouped(o, Qw[1], sw[1], y, stream=stream)

    # the steps in 64 bits, every rounding to fp16 taken where the library has one
    f = ou.frequencies(D)
    inputs = (g.standard_normal((24, B, Kin))).astype(np.float16)
    seen = [[[], []] for _ in range(B)]
    side = torch.cuda.Stream()
    graph = None
    for i in range(24):
        lengths = np.full(B, i, np.int32)
        x.copy_(dev(inputs[i]))
        pos.copy_(dev(lengths))
        torch.cuda.synchronize()
        if i < 4:
            step()
        elif i < 8:
            side.wait_stream(torch.cuda.current_stream())
            step(side)
        elif graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        got_qkv, got_o, got_y = host(qkv), host(o), host(y)
        p, bound = ou.product(inputs[i], codes[0][0].reshape(W, Kin), codes[0][1], group)
        raw = p.astype(np.float16).reshape(B, -1, D)
        # rotated heads: from the unrotated projection, whose last rounding may differ by a step
        r, rb = ou.rotary(raw[:, : Hq + Hk], lengths, f, True)
        b3 = bound.reshape(B, -1, D)
        i_ = np.arange(D // 2)
        spread = np.zeros_like(rb)
        spread[..., i_] = spread[..., i_ + D // 2] = 2 * (b3[:, : Hq + Hk, : D // 2] + b3[:, : Hq + Hk, D // 2:])
        ou.held(got_qkv.reshape(B, -1, D)[:, : Hq + Hk], r, rb + spread, f"step {i}: rotary")
        heads = got_qkv.reshape(B, -1, D)
        for b in range(B):
            for which, at in ((0, Hq), (1, Hq + Hk)):
                c, s = ou.quantize(heads[b, at: at + Hk])
                seen[b][which].append((c * s.astype(np.float64)[:, None], s.astype(np.float64)))
            k, v = (np.stack([e[0] for e in seen[b][w]]) for w in (0, 1))
            sk, sv = (np.stack([e[1] for e in seen[b][w]]) for w in (0, 1))
            for h in range(Hq):
                hk = h // (Hq // Hk)
                want, ob = ou.attention(heads[b, h][None], k[:, hk], v[:, hk], sk[:, hk], sv[:, hk], np.ones((1, len(k)), bool), D ** -0.5)
                ou.held(got_o.reshape(B, Hq, D)[b, h][None], want, ob, f"step {i}: attention")
        want, yb = ou.product(got_o, codes[1][0].reshape(Kin, Hq * D), codes[1][1], group)
        ou.held(got_y, want, yb, f"step {i}: output")


MANY_KEYS = 2 ** 31 - 1                                     # as a hint: the work is shared out as for long sequences, 32 rows at a time


@pytest.mark.parametrize("case", [n for n, c in enumerate(CASES) if max(c[1]) * (c[2] // c[3]) > 16])
def test_attention_of_many_rows(case):
    past, new, Hq, Hk, D, page, tree = CASES[case]
    print(f"case attention many rows {CASES[case]}", flush=True)
    s = Setting(700 + case, past, new, Hk, D, page, scale_v=[1.0, 2.0 ** -12, 8.0][case % 3])
    Q, scale = s.queries(Hq, 2.0), D ** -0.5
    words = s.trees() if tree else None
    want, bound = s.expect(Q, Hq // Hk, s.by_mask(words) if tree else s.causal, scale)
    for workspace in (0, 8 << 20):
        ou.held(s.run(Q, words, scale, workspace, max_keys=MANY_KEYS), want, bound, f"{CASES[case]} {workspace}")


def test_attention_of_many_rows_empty_ones_bad_pages_and_peaks():
    print("case attention many rows, masks and pages", flush=True)
    for D, page in ((64, 16), (128, 32)):
        s = Setting(800 + D, [0, 170, 0], [40, 19, 1], 2, D, page)
        words = s.trees()
        words[::3] = 0
        words[7] = np.uint64(1) << np.uint64(63)
        words[41] = np.uint64(0xFFFFFFFFFFFFFFFF)
        Q = s.queries(8, 3.0)
        want, bound = s.expect(Q, 4, s.by_mask(words), 0.125)
        got = s.run(Q, words, 0.125, max_keys=MANY_KEYS)
        ou.held(got, want, bound, "empty rows")
        assert (got[0] == 0).all() and (got[7] == 0).all()
        table = s.table.copy()
        table[1, 2], table[1, 4], table[0, :] = -1, 1 << 30, s.cache.shape[0]
        absent = lambda b, L: np.ones(L, bool) if b == 0 else np.isin(np.arange(L) // page, (2, 4)) & (b == 1)    # noqa: E731
        want, bound = s.expect(Q, 4, s.by_mask(words), 0.125, absent)
        got = s.run(Q, words, 0.125, max_keys=MANY_KEYS, table=table)
        ou.held(got, want, bound, "bad pages")
        assert (got[:40] == 0).all()
        for factor in (30.0, 300.0):                        # one key with all the weight; the offset moves on the way
            Q = s.queries(8, factor)
            want, bound = s.expect(Q, 4, s.causal, 0.3)
            ou.held(s.run(Q, None, 0.3, max_keys=MANY_KEYS), want, bound, f"{factor}")


@pytest.mark.parametrize("B", [64, 65])
def test_attention_of_many_rows_in_many_sequences(B):
    """Sequences of equal and of different lengths, some without a row."""
    print(f"case attention many rows {B} sequences", flush=True)
    g = rng(12, B)
    past, new = g.integers(0, 60, B), g.integers(0, 12, B)
    past[10:20], new[10:20] = 33, 9
    s = Setting(900 + B, list(past), list(new), 1, 64, 16)
    Q = s.queries(4)
    want, bound = s.expect(Q, 4, s.causal, 0.2)
    ou.held(s.run(Q, None, 0.2, max_rows=12, max_keys=MANY_KEYS), want, bound, str(B))


@pytest.mark.parametrize("B", [63, 65, 4097, 5000])
def test_cache_of_many_sequences(B):
    import torch
    import paper_2511_22316_amd as sq
    print(f"case cache {B} sequences", flush=True)
    g, Hk, D, page = rng(13, B), 1, 64, 16
    cached, new = g.integers(0, 15, B).astype(np.int32), g.integers(0, 3, B)
    new[B // 3: B // 2] = 0                                 # a run of sequences that share their row_start
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(start[-1])
    table = g.permutation(B).reshape(B, 1).astype(np.int32)
    x = rows(g, T, 2 * Hk * D).reshape(T, 2, Hk, D)
    cache = torch.zeros(B, sq.sq_cache_page_bytes(Hk, D, page), dtype=torch.uint8, device="cuda")
    args = dev(start), dev(cached), dev(table), page
    d = dev(x)
    sq.sq_cache_append(d[:, 0], d[:, 1], *args, cache)
    k, v = (torch.full((T, Hk, D), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    sq.sq_cache_read(cache, *args, k, v)
    codes, steps = ou.quantize(x)
    want = (codes * steps.astype(np.float64)[..., None]).astype(np.float16).reshape(x.shape)
    place = np.repeat(cached, new) + np.arange(T) - np.repeat(start[:-1], new)
    want[place >= page] = 3.0                               # rows beyond a sequence's page
    assert np.array_equal(host(k), want[:, 0]) and np.array_equal(host(v), want[:, 1])


@pytest.mark.parametrize("T,K,N,group", [(1, 256, 4200, 128), (16, 448, 8190, 64), (9, 192, 5000, 32), (20, 256, 4200, 32), (32, 320, 8300, 64),
                                         (17, 256, 11000, 128), (32, 192, 9000, 32), (29, 512, 16384, 256), (20, 256, 16500, 128),
                                         (32, 64, 17000, 32), (40, 256, 33000, 64), (1000, 256, 2500, 32), (300, 128, 9000, 128)])
def test_product_of_many_channels(T, K, N, group):
    """More channels, where the choice of a kernel goes by them."""
    print(f"case product {T} {K} {N} {group}", flush=True)
    g = rng(14, T, K, N, group)
    X, (codes, steps) = rows(g, T, K), weights(g, N, K, group)
    want, bound = ou.product(X, codes, steps, group, T > 32)
    ou.held(run_product(X, codes, steps, 8, 3), want, bound, f"{T} {K} {N} {group}")


def test_a_table_left_on_the_host_is_refused():
    import torch
    import paper_2511_22316_amd as sq
    x = torch.zeros(2, 3, 64, dtype=torch.float16, device="cuda")
    positions = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="device"):
        sq.sq_rotary_fp16(x, positions, sq.sq_rotary_table(32), True, x)
    sq.sq_rotary_fp16(x, positions, sq.sq_rotary_table(32).cuda(), True, x)
    with pytest.raises(ValueError, match="device"):
        sq.sq_quantize_grouped(x[0], 32, torch.zeros(3, 32, dtype=torch.uint8), torch.zeros(3, 2, dtype=torch.float16))
    torch.cuda.synchronize()


def test_product_keeps_an_infinity_where_it_is():
    """A token with an infinity: infinite (or NaN where a code is 0) in its own row, and nothing of it in the others; rows in LDS with
    a K that is no whole number of rounds among them."""
    print("case product infinity", flush=True)
    for T, K, N, group in ((5, 4736, 7200, 128), (5, 4736, 7200, 32), (3, 320, 40, 64), (40, 384, 300, 32)):
        g = rng(15, T, K, N, group)
        X, (codes, steps) = rows(g, T, K), weights(g, N, K, group)
        codes[:, K - 1] = 2 * (codes[:, K - 1] >= 0) - 1    # the place of the infinity: never 0
        want, bound = ou.product(X, codes, steps, group, T > 32)
        X[1, K - 1] = np.inf
        got = run_product(X, codes, steps)
        assert (got[1].astype(np.float64) == np.inf * codes[:, K - 1]).all(), (T, K, N, group)
        others = np.arange(T) != 1
        ou.held(got[others], want[others], bound[others], "others")


def test_attention_rows_that_do_not_see_an_infinity():
    """Keys and values that are not finite, in rows that a mask hides."""
    import paper_2511_22316_amd as sq
    print("case attention hidden infinity", flush=True)
    for D in (64, 128, 256):
        s = Setting(1000 + D, [40, 0], [20, 9], 2, D, 16)
        Q = s.queries(8)
        words = s.trees()
        bad = np.uint64(1) << np.uint64(3)                  # new row 3 of both sequences
        seeing = (words & bad) != 0
        assert seeing.any() and not seeing.all()
        kv = np.full((2, 2, D), np.inf, np.float16)
        kv[:, :, 1::2] = np.nan
        slots = dev(np.array([0, 1, 2], np.int32)), dev((s.past + 3).astype(np.int32)), s.dtable
        sq.sq_cache_append(dev(kv), dev(kv), *slots, 16, s.cache)
        want, bound = s.expect(Q, 4, s.by_mask(words & ~bad), 0.2)
        for max_keys in (None, MANY_KEYS):
            got = s.run(Q, words, 0.2, max_keys=max_keys)
            ou.held(got[~seeing], want[~seeing], bound[~seeing], f"hidden {D}")


def test_attention_scores_of_one_sign_far_from_zero():
    """A score near -10^27 or +10^27 with no other beside it: the value, not zeros."""
    print("case attention scores far below zero", flush=True)
    for sign in (-1, 1):
        one = Setting(80, [0], [1], 1, 64, 16)
        key, value = one.numbers.values(0, 0, 1)[0][0, 0], one.numbers.values(0, 1, 1)[0][0, 0]
        Q = np.broadcast_to((sign * np.sign(key) * 60000).astype(np.float16), (1, 2, 64))
        got = one.run(np.ascontiguousarray(Q), None, 9e19)
        # the weight and the result are rounded to fp16; the eights come off sums of 16 steps
        step = np.abs(value).max() / 7
        bound = (2 * ou.HALF + ou.HALF ** 2 + 8 * ou.EPS32) * np.abs(value) + 40 * ou.EPS32 * 16 * step + ou.TINY
        ou.held(got[0], np.broadcast_to(value, (2, 64)), np.broadcast_to(bound, (2, 64)), f"{sign}")


def test_attention_of_a_sequence_with_a_negative_length():
    print("case attention negative length", flush=True)
    s = Setting(81, [20, 30], [2, 3], 2, 64, 16)
    Q = s.queries(4)
    want, bound = s.expect(Q, 2, s.causal, 0.2)
    s.dcached = dev(np.array([20, -1], np.int32))
    got = s.run(Q, None, 0.2)
    ou.held(got[:2], want[:2], bound[:2], "the other sequence")
    assert (got[2:] == 0).all()


def test_cache_keeps_infinities_as_large_numbers():
    import torch
    import paper_2511_22316_amd as sq
    print("case cache infinity", flush=True)
    x = np.ones((3, 2, 128), np.float16)
    x[0, 0, 5], x[1, 1, 7], x[2, 0, 9] = np.inf, -np.inf, np.nan
    cache = torch.zeros(1, sq.sq_cache_page_bytes(2, 128, 16), dtype=torch.uint8, device="cuda")
    args = dev(np.array([0, 3], np.int32)), dev(np.zeros(1, np.int32)), dev(np.zeros((1, 1), np.int32)), 16
    sq.sq_cache_append(dev(x), dev(x), *args, cache)
    k, v = (torch.empty(3, 2, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    sq.sq_cache_read(cache, *args, k, v)
    k, v = host(k), host(v)
    assert np.array_equal(k[0, 0], np.where(np.arange(128) == 5, np.inf, 0.0)) and np.array_equal(v[0, 0], k[0, 0])
    assert np.array_equal(k[1, 1], np.where(np.arange(128) == 7, -np.inf, 0.0)) and np.array_equal(v[1, 1], k[1, 1])
    other = np.arange(128) != 9
    assert (k[2, 0][other] == 0).all() and (k[0, 1] == k[2, 1]).all() and abs(float(k[0, 1, 0]) - 1) < 0.01
    steps = host(cache).view(np.float16)[0, (2 * 16 * 128) // 2: (2 * 16 * 132) // 2]
    assert np.isfinite(steps).all()


@pytest.mark.parametrize("T,K,N,group", [(32, 2048, 4200, 32), (17, 2304, 4100, 256), (25, 2176, 8300, 64), (31, 2048, 9000, 128), (24, 1024, 17000, 128),
                                         (32, 1152, 16500, 32), (16, 5120, 16400, 64), (13, 6528, 8200, 128), (16, 5120, 9000, 32),
                                         (12, 8192, 4300, 32), (16, 5376, 7000, 256)])
def test_product_in_parts(T, K, N, group):
    """Token rows that pass through LDS in parts."""
    print(f"case product in parts {T} {K} {N} {group}", flush=True)
    g = rng(16, T, K, N, group)
    X, (codes, steps) = rows(g, T, K), weights(g, N, K, group)
    codes[:, K - 1] = 2 * (codes[:, K - 1] >= 0) - 1
    want, bound = ou.product(X, codes, steps, group)
    ou.held(run_product(X, codes, steps, 8, 3), want, bound, f"{T} {K} {N} {group}")
    X[T - 1, K - 1] = np.inf                                # stays in its row, also where the last part is not full
    got = run_product(X, codes, steps)
    assert (got[T - 1].astype(np.float64) == np.inf * codes[:, K - 1]).all()
    ou.held(got[: T - 1], want[: T - 1], bound[: T - 1], "others")


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(40, 5, 80, 40), (33, 6, 96, 24), (5, 3, 20, 8), (9, 2, 36, 12), (3, 2, 10, 4), (1000, 9, 80, 20), (6, 3, 44, 40)])
def test_rotary_narrow_units(T, H, D, rot, half):
    """Widths that go in units of 2, 4 or 8 pairs, and the same rows at places that allow fewer: the same bits."""
    import torch
    import paper_2511_22316_amd as sq
    print(f"case rotary units {T} {H} {D} {rot} {half}", flush=True)
    g = rng(17, T, H, D, rot)
    X = rows(g, T, H * D).reshape(T, H, D)
    pos = g.integers(0, 2 ** 20, T).astype(np.int32)
    turns = sq.sq_rotary_table(rot).cuda()
    want, bound = ou.rotary(X, pos, ou.frequencies(rot), half, 1.0)
    got = None
    for at, row in ((0, 0), (4, 4), (2, 6), (1, 3)):        # halves in front of the rows and behind each
        buf = torch.full((at + T * (H * D + row) + 8,), 3.0, dtype=torch.float16, device="cuda")
        out = buf.clone()
        view = lambda b: b[at: at + T * (H * D + row)].view(T, H * D + row)[:, : H * D].unflatten(1, (H, D))     # noqa: E731
        view(buf)[:] = dev(X)
        sq.sq_rotary_fp16(view(buf), dev(pos), turns, half, view(out))
        sq.sq_rotary_fp16(view(buf), dev(pos), turns, half, view(buf))
        assert torch.equal(out, buf)                        # in place and beside, and nothing around them
        y = host(view(out).contiguous())
        if got is None:
            ou.held(y, want, bound, "units")
            got = y
        assert np.array_equal(y, got)
        view(out)[:] = 3.0
        assert (out == 3.0).all()


@pytest.mark.parametrize("T,K,N,group", [(33, 256, 1000, 64), (64, 384, 1500, 128), (100, 320, 2000, 64), (200, 256, 2040, 32), (2000, 128, 200, 128),
                                         (64, 320, 16384, 32), (65, 320, 16384, 32), (500, 192, 5000, 64), (700, 256, 6000, 32)])
def test_product_between_few_and_many(T, K, N, group):
    print(f"case product {T} {K} {N} {group}", flush=True)
    g = rng(18, T, K, N, group)
    X, (codes, steps) = rows(g, T, K), weights(g, N, K, group)
    want, bound = ou.product(X, codes, steps, group, True)
    ou.held(run_product(X, codes, steps, 8, 3), want, bound, f"{T} {K} {N} {group}")


@pytest.mark.parametrize("Hq,Hk,D,page,new,tree", [(8, 2, 64, 16, [1, 1, 1, 1], False), (4, 4, 128, 64, [1, 0, 1, 1], False), (6, 2, 256, 32, [1, 1, 1, 1], False),
                                                   (8, 1, 128, 16, [9, 3, 1, 17], True), (5, 1, 64, 128, [2, 7, 4, 1], False)])
def test_attention_of_split_sequences(Hq, Hk, D, page, new, tree):
    print(f"case attention split {Hq} {Hk} {D} {page} {new} {tree}", flush=True)
    s = Setting(1100 + D + page, [2500, 900, 0, 3000], new, Hk, D, page)
    Q, scale = s.queries(Hq, 2.0), D ** -0.5
    words = s.trees() if tree else None
    want, bound = s.expect(Q, Hq // Hk, s.by_mask(words) if tree else s.causal, scale)
    for max_keys in (None, 3000, 8000):
        ou.held(s.run(Q, words, scale, max_keys=max_keys), want, bound, f"{max_keys}")


def test_calls_without_work():
    import torch
    import paper_2511_22316_amd as sq
    print("case empty calls", flush=True)
    h = lambda *n: torch.full(n, 3.0, dtype=torch.float16, device="cuda")       # noqa: E731
    u = lambda *n: torch.zeros(n, dtype=torch.uint8, device="cuda")             # noqa: E731
    i = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")             # noqa: E731
    turns = sq.sq_rotary_table(32).cuda()
    sq.sq_quantize_grouped(h(0, 64), 32, u(0, 32), h(0, 2))
    sq.sq_w4a16_gemm_grouped(h(0, 64), u(5, 32), h(5, 2), h(0, 5))
    sq.sq_w4a16_gemm_grouped(h(3, 64), u(0, 32), h(0, 2), h(3, 0))
    sq.sq_rotary_fp16(h(0, 3, 64), i(0), turns, True, h(0, 3, 64))
    sq.sq_rotary_fp16(h(2, 0, 64), i(2), turns, True, h(2, 0, 64))
    size = sq.sq_cache_page_bytes(2, 64, 16)
    for B, T, per, pages in ((0, 0, 0, 0), (0, 0, 2, 3), (2, 0, 1, 3), (2, 4, 0, 3), (2, 4, 2, 0)):
        start = dev(np.array([0, 1, T][: B] + [T], np.int32)) if B else i(1)
        table, cache, k, v, o = torch.full((B, per), -1, dtype=torch.int32, device="cuda"), u(pages, size), h(T, 2, 64), h(T, 2, 64), h(T, 4, 64)
        sq.sq_cache_append(k, v, start, i(B), table, 16, cache)
        sq.sq_cache_read(cache, start, i(B), table, 16, k, v)
        sq.sq_tree_attention(h(T, 4, 64), start, i(B), None, table, 16, cache, 2, 0.1, o, max_rows=4)
        torch.cuda.synchronize()
        assert (k == 3).all() and (v == 3).all() and not cache.any()
        assert (o == 0).all()                               # rows of a sequence without keys


def test_cache_read_into_parts_of_rows_and_shared_pages():
    """Two sequences with the same first pages, read and attended to; K and V are written into wider rows."""
    import torch
    import paper_2511_22316_amd as sq
    print("case shared pages", flush=True)
    s = Setting(1200, [64, 64], [1, 1], 2, 128, 32)
    s.table[1, :2] = s.table[0, :2]                         # the pages of the 64 old rows
    table = dev(s.table)
    s.numbers.rows[1][0][:64] = s.numbers.rows[0][0][:64]
    s.numbers.rows[1][1][:64] = s.numbers.rows[0][1][:64]
    Q = s.queries(8)
    want, bound = s.expect(Q, 4, s.causal, 0.1)
    ou.held(s.run(Q, None, 0.1, table=s.table), want, bound, "shared")
    buf = torch.full((2, 2 * 256 + 16), 3.0, dtype=torch.float16, device="cuda")
    k, v = buf[:, :256].unflatten(1, (2, 128)), buf[:, 264: 264 + 256].unflatten(1, (2, 128))
    sq.sq_cache_read(s.cache, s.dstart, s.dcached, table, 32, k, v)
    for b in range(2):
        assert np.array_equal(host(k)[b], s.numbers.values(b, 0, 65)[0][64].astype(np.float16))
        assert np.array_equal(host(v)[b], s.numbers.values(b, 1, 65)[0][64].astype(np.float16))
    assert (buf[:, 256: 264] == 3).all() and (buf[:, 520:] == 3).all()


def test_two_streams_at_once():
    """The same calls on two streams, each with a cache and a workspace of its own, against one after the other."""
    import torch
    import paper_2511_22316_amd as sq
    print("case two streams", flush=True)
    g = rng(21)
    B, Hq, Hk, D, page, K = 4, 8, 2, 128, 64, 512
    W = (Hq + 2 * Hk) * D
    codes, steps = weights(g, W, K, 128)
    Qw, sw, turns = dev(ou.pack(codes)), dev(steps), sq.sq_rotary_table(D).cuda()
    start, table = dev(np.arange(B + 1, dtype=np.int32)), dev(np.arange(B * 20, dtype=np.int32).reshape(B, 20))
    cached = dev(np.array([1000, 1100, 1200, 900], np.int32))
    filled = torch.randint(0, 256, (B * 20, sq.sq_cache_page_bytes(Hk, D, page)), dtype=torch.uint8, device="cuda")
    filled.view(torch.float16)[:, Hk * page * D // 2:] = 0.05
    X = [dev(rows(g, B, K)) for _ in range(2)]

    def step(n, stream):
        cache, qkv = filled.clone(), torch.empty(B, W, dtype=torch.float16, device="cuda")
        O, ws = torch.empty(B, Hq, D, dtype=torch.float16, device="cuda"), torch.empty(4 << 20, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        def go():
            for _ in range(20):
                sq.sq_w4a16_gemm_grouped(X[n], Qw, sw, qkv, stream=stream)
                heads = qkv.unflatten(1, (Hq + 2 * Hk, D))
                qk = heads[:, : Hq + Hk]
                sq.sq_rotary_fp16(qk, cached, turns, True, qk, stream=stream)
                sq.sq_cache_append(qk[:, Hq:], heads[:, Hq + Hk:], start, cached, table, page, cache, stream=stream)
                sq.sq_tree_attention(qk[:, :Hq], start, cached, None, table, page, cache, Hk, D ** -0.5, O, ws, stream=stream)
        return go, (cache, qkv, O)

    alone = []
    for n in range(2):
        go, out = step(n, None)
        go()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in out])
    both = [step(n, torch.cuda.Stream()) for n in range(2)]
    for go, _ in both:
        go()
    torch.cuda.synchronize()
    for (_, out), want in zip(both, alone):
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert not torch.equal(alone[0][2], alone[1][2])


def test_rotary_lengths_of_one_with_any_stride():
    import torch
    import paper_2511_22316_amd as sq
    g = rng(22)
    turns, pos = sq.sq_rotary_table(32).cuda(), dev(np.arange(7, dtype=np.int32))
    x = dev(rows(g, 7, 5 * 64).reshape(7, 5, 64))
    want = torch.empty_like(x)
    sq.sq_rotary_fp16(x, pos, turns, True, want)
    y = torch.empty(1, 5, 64, dtype=torch.float16, device="cuda")
    sq.sq_rotary_fp16(x[3:4].as_strided((1, 5, 64), (0, 64, 1), 3 * 320), pos[3:4].contiguous(), turns, True, y)
    assert torch.equal(y, want[3:4])
    y = torch.empty(7, 1, 64, dtype=torch.float16, device="cuda")
    sq.sq_rotary_fp16(x.as_strided((7, 1, 64), (320, 1, 1), 2 * 64), pos, turns, True, y)
    assert torch.equal(y, want[:, 2:3])
    # rows whose last head ends where the next begins, and heads that overlap
    gap = torch.zeros(7 * 5 * 72, dtype=torch.float16, device="cuda")
    tight = gap.as_strided((7, 5, 64), (4 * 72 + 64, 72, 1))
    tight.copy_(x)
    out = torch.empty_like(want)
    sq.sq_rotary_fp16(tight, pos, turns, True, out)
    assert torch.equal(out, want)
    with pytest.raises((ValueError, sq.SQError)):
        sq.sq_rotary_fp16(x[:, :1].expand(7, 5, 64), pos, turns, True, want)

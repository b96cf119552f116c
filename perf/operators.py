"""The measured cases of the operators around the quantized layers: products with weight codes that have a step per
group, rotary positions, the paged 4-bit cache and the attention that reads it.

A case is one pass, named by ``path``:

  quantize   fp16 rows to 4-bit codes with a step per group (offline, for weights)
  product    fp16 rows times weight codes with a step per group
  rotary     rotary positions on the query and key heads of a projection's output
  cache      new rows of K and V into the pages of the cache, and the same rows read back
  attention  drafted tokens (or one token a sequence) over the cache

``own`` chooses between the library's calls and their plain form in elementary torch operations.  The plain form reads and
writes the same buffers; the layout of a page is in ``_write_pages`` and ``_read_pages``.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # weights of a down projection, offline
        {"name": "weights_down_proj", "path": "quantize", "T": 4096, "K": 11008, "group": 128},
        # a few hundred rows in the smallest groups
        {"name": "rows_small_groups", "path": "quantize", "T": 333, "K": 5120, "group": 32},
        # one token through an attention projection: the smallest product of a decode step
        {"name": "one_token_product", "path": "product", "T": 1, "K": 4096, "N": 4096, "group": 128},
        # decoding a small batch through an up projection: one pass over the weights
        {"name": "batch_product", "path": "product", "T": 8, "K": 8192, "N": 28672, "group": 64},
        # a short prompt of odd length through the same weights
        {"name": "prompt_product", "path": "product", "T": 333, "K": 5120, "N": 13824, "group": 32},
        # one new token far into a long text, interleaved pairs
        {"name": "rotary_one_token", "path": "rotary", "T": 1, "Hq": 32, "Hk": 8, "D": 128, "rot": 128, "half": False,
         "scaling": "parts", "far": 1000000},
        # a prompt, halves, the first half of each head only
        {"name": "rotary_prompt", "path": "rotary", "T": 8192, "Hq": 32, "Hk": 8, "D": 128, "rot": 64, "half": True,
         "scaling": "none", "far": 8192},
        # one decode step of a batch: one row a sequence
        {"name": "cache_step", "path": "cache", "B": 32, "rows": 1, "Hk": 8, "D": 128, "page": 64, "keys": 2048},
        # prompts of odd lengths
        {"name": "cache_prompts", "path": "cache", "B": 5, "rows": 1999, "Hk": 8, "D": 128, "page": 16, "keys": 2048},
        # one sequence, one token, a long cache: the latency of a single stream
        {"name": "attention_one_token", "path": "attention", "B": 1, "rows": 1, "tree": False, "Hq": 32, "Hk": 8, "D": 128,
         "page": 64, "keys": 16384},
        # a batch of sequences of different lengths, one token each
        {"name": "attention_batch", "path": "attention", "B": 48, "rows": 1, "tree": False, "Hq": 32, "Hk": 8, "D": 128,
         "page": 64, "keys": 8192},
        # trees of drafted tokens to be verified at once
        {"name": "attention_trees", "path": "attention", "B": 16, "rows": 61, "tree": True, "Hq": 32, "Hk": 8, "D": 128,
         "page": 32, "keys": 4096},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    path = rng.choice(["quantize", "product", "product", "product", "rotary", "cache", "attention", "attention", "attention"])
    group = rng.choice([32, 64, 128, 256])
    if path == "quantize":
        K = group * _log_int(rng, 1, 14336 // group)
        return {"path": path, "T": _log_int(rng, 1, min(16384, 45000000 // K)), "K": K, "group": group}
    if path == "product":
        unit = max(64, group)
        K = unit * _log_int(rng, max(1, 256 // unit), 14336 // unit)
        N = _log_int(rng, 100, min(28672, 200000000 // K))
        T = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 512)])
        T = max(1, min(T, 20000000000 // (K * N)))
        return {"path": path, "T": T, "K": K, "N": N, "group": group}
    D = rng.choice([64, 128, 128, 256])
    Hk = rng.choice([1, 2, 4, 8, 5, 16])
    Hq = Hk * rng.choice([1, 2, 4, 5, 8])
    if path == "rotary":
        D = rng.choice([D, 80, 96])
        return {"path": path, "T": _log_int(rng, 1, max(2, 41943040 // ((Hq + Hk) * D))), "Hq": Hq, "Hk": Hk, "D": D,
                "rot": rng.choice([D, D // 2, D // 4]), "half": rng.random() < 0.5,
                "scaling": rng.choice(["none", "linear", "base", "parts"]), "far": _log_int(rng, 16, 1000000)}
    page = rng.choice([16, 32, 64, 128])
    if path == "cache":
        B = _log_int(rng, 1, 64)
        rows = _log_int(rng, 1, max(2, min(4096, 10000000 // (B * Hk * D))))
        return {"path": path, "B": B, "rows": rows, "Hk": Hk, "D": D, "page": page, "keys": rows + _log_int(rng, 1, 4096)}
    tree = rng.random() < 0.5
    rows = rng.randint(2, 64) if tree else rng.choice([1, 1, _log_int(rng, 2, 300)])
    B = _log_int(rng, 1, 64)
    most = min(48 * 8192 * 8 * 128 // (B * Hk * D), 16 * 61 * 4096 * 32 * 128 // (B * rows * Hq * D))
    return {"path": path, "B": B, "rows": rows, "tree": tree, "Hq": Hq, "Hk": Hk, "D": D, "page": page,
            "keys": _log_int(rng, rows, max(rows + 1, min(32768, most)))}


# ---- inputs ---------------------------------------------------------------------------------------


def _rows(rows, width, gen):
    """fp16 activations: a Gaussian body, a few channels of massive outliers, some moderate ones."""
    x = torch.randn(rows, width, device="cuda", generator=gen)
    hit = torch.rand(rows, width, device="cuda", generator=gen) < 0.005
    x = torch.where(hit, 20.0 * x, x)
    x[:, torch.randperm(width, device="cuda", generator=gen)[:2]] *= 30.0
    return x.half()


def _steps_and_codes(x):
    """Step and codes over the last dimension: step = fp16(max / 7) (1 where that is 0), code = floor(x / step + 1/2)."""
    x = x.float()
    seven = torch.full((), 7.0, device=x.device)         # a tensor: torch multiplies by the reciprocal of a number
    step = (x.abs().amax(-1) / seven).half()
    step = torch.where(step == 0, torch.ones_like(step), step)
    codes = torch.floor(x / step.float()[..., None] + 0.5).clamp_(-8.0, 7.0)
    return step, codes


def _pack(codes):
    """Whole numbers in 0 .. 15 -> bytes, the even channel in the low nibble."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).to(torch.uint8)


def _signed(Q):
    """Bytes of two's-complement nibbles -> int8 codes."""
    shift = torch.tensor([4, 0], dtype=torch.int8, device=Q.device)
    return ((Q.view(torch.int8)[..., None] << shift) >> 4).reshape(*Q.shape[:-1], 2 * Q.shape[-1])


def _page_bytes(Hk, D, page):
    return (Hk * page * (D + 4) + 255) // 256 * 256


def _pieces(pages, Hk, D, page):
    """Views into pages uint8 [..., page_bytes]: K codes [..., Hk, page, D/2], V codes [..., Hk, page/16, 4, 16, 4, D/32]
    (slot 16 b + 4 q + r, channels o D/16 .. of it at [b, q, o, r]), steps fp16 [..., 2, Hk, page] of K and V."""
    lead = pages.shape[:-1]
    codes = pages[..., : Hk * page * D].unflatten(-1, (Hk, 2, page * D // 2))
    steps = pages[..., Hk * page * D: Hk * page * (D + 4)].view(torch.float16).reshape(*lead, 2, Hk, page)
    return (codes[..., 0, :].unflatten(-1, (page, D // 2)), codes[..., 1, :].unflatten(-1, (page // 16, 4, 16, 4, D // 32)), steps)


def _v_rows(v, page, D):
    """The V codes of _pieces as rows [..., Hk, page, D/2]."""
    n = v.dim()
    return v.permute(*range(n - 4), n - 4, n - 2, n - 3, n - 1).reshape(*v.shape[:-5], page, D // 2)


def _new_pages(count, Hk, D, page, gen):
    """Pages full of quantized rows: keys with a few strong channels, values without.  [count, page_bytes]"""
    out = torch.zeros(count, _page_bytes(Hk, D, page), dtype=torch.uint8, device="cuda")
    strong = torch.where(torch.rand(Hk, 1, D, device="cuda", generator=gen) < 0.05, 3.0, 1.0)
    part = max(1, (1 << 26) // (Hk * page * D))
    for a in range(0, count, part):
        n = min(part, count - a)
        rows = torch.randn(2, n, Hk, page, D, device="cuda", generator=gen)
        rows[0] *= strong
        step, codes = _steps_and_codes(rows.half())
        bytes_ = _pack(codes.to(torch.int32) + 8)
        out[a:a + n, : Hk * page * D] = torch.stack((
            bytes_[0].reshape(n, Hk, -1),
            bytes_[1].reshape(n, Hk, page // 16, 4, 4, 16, D // 32).permute(0, 1, 2, 3, 5, 4, 6).reshape(n, Hk, -1)), 2).reshape(n, -1)
        out[a:a + n, Hk * page * D: Hk * page * (D + 4)] = step.transpose(0, 1).contiguous().reshape(n, -1).view(torch.uint8)
    return out


def _frequencies(rot, scaling):
    """Radians per position of the rot / 2 pairs; `parts`: slow pairs interpolated, fast ones kept, a ramp between them."""
    base, factor, trained, low, high = 10000.0, 8.0, 8192.0, 1.0, 32.0
    if scaling == "base":
        base *= factor ** (rot / (rot - 2))
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        keep = np.clip((trained * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
    return f


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    path = c["path"]
    if path == "quantize":
        c["X"] = (0.02 * torch.randn(c["T"], c["K"], device="cuda", generator=gen)).half()
        c["Q"] = torch.empty(c["T"], c["K"] // 2, dtype=torch.uint8, device="cuda")
        c["steps"] = torch.empty(c["T"], c["K"] // c["group"], dtype=torch.float16, device="cuda")
        return c
    if path == "product":
        T, K, N, g = c["T"], c["K"], c["N"], c["group"]
        c["X"] = _rows(T, K, gen)
        c["Qw"] = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda")
        c["sw"] = torch.empty(N, K // g, dtype=torch.float16, device="cuda")
        for a in range(0, N, 4096):
            w = (0.02 * torch.randn(min(4096, N - a), K // g, g, device="cuda", generator=gen)).half()
            c["sw"][a:a + 4096], codes = _steps_and_codes(w)
            c["Qw"][a:a + 4096] = _pack((codes.to(torch.int32) & 15).flatten(1))
        c["Y"] = torch.empty(T, N, dtype=torch.float16, device="cuda")
        return c
    if path == "rotary":
        T, H, D, rot = c["T"], c["Hq"] + c["Hk"], c["D"], c["rot"]
        # the query and key heads of a row that holds the value heads too
        c["X"] = _rows(T, (H + c["Hk"]) * D, gen)[:, : H * D].unflatten(1, (H, D))
        first = torch.randint(0, max(1, c["far"] - T), (1,), device="cuda", generator=gen)
        c["positions"] = (first + torch.arange(T, device="cuda")).int()
        f = _frequencies(rot, c["scaling"])
        c["f"] = torch.from_numpy(f).cuda()
        turns = [int(round(float(v) / (2 * math.pi) * 2.0 ** 64)) for v in f]
        c["turns"] = torch.from_numpy(np.array(turns, dtype=np.uint64).view(np.int64)).cuda()
        c["magnitude"] = 0.1 * math.log(8.0) + 1.0 if c["scaling"] == "parts" else 1.0
        c["Y"] = torch.empty(T, H, D, dtype=torch.float16, device="cuda")
        return c
    B, Hk, D, page, keys, rows = (c[k] for k in ("B", "Hk", "D", "page", "keys", "rows"))
    # lengths of the sequences from all of `keys` down to a half, rows likewise, in the order of the seed
    spread = lambda most: (most - torch.arange(B, device="cuda") * (most // 2) // max(1, B - 1))[   # noqa: E731
        torch.randperm(B, device="cuda", generator=gen)].int()
    total, n = spread(keys), spread(rows)
    total = torch.maximum(total, n)
    c["cached"] = total - n
    c["row_start"] = torch.cat((torch.zeros(1, dtype=torch.int32, device="cuda"), n.cumsum(0).int()))
    T = int(c["row_start"][-1])
    per = (keys + page - 1) // page
    count = B * per + 3
    c["table"] = torch.randperm(count, device="cuda", generator=gen)[: B * per].view(B, per).int()
    c["cache"] = _new_pages(count, Hk, D, page, gen)
    if path == "cache":
        kv = _rows(T, 2 * Hk * D, gen)
        c["K"], c["V"] = kv[:, : Hk * D].unflatten(1, (Hk, D)), kv[:, Hk * D:].unflatten(1, (Hk, D))
        c["Kr"], c["Vr"] = (torch.empty(T, Hk, D, dtype=torch.float16, device="cuda") for _ in range(2))
        return c
    c["Q"] = (2.0 * torch.randn(T, c["Hq"], D, device="cuda", generator=gen)).half()
    c["O"] = torch.empty(T, c["Hq"], D, dtype=torch.float16, device="cuda")
    c["scale"] = D ** -0.5
    c["mask"] = None
    if c["tree"]:
        # every drafted token's parent is one of the eight before it; a row sees its ancestors and itself
        i = torch.arange(rows, device="cuda")
        parent = (i - 1 - torch.randint(0, 8, (B, rows), device="cuda", generator=gen)).clamp_(min=0)
        sees = torch.eye(rows, dtype=torch.bool, device="cuda").repeat(B, 1, 1)
        for k in range(1, rows):
            sees[:, k] |= sees[torch.arange(B, device="cuda"), parent[:, k]]
        words = (sees.long() << i).sum(-1)
        local = torch.arange(T, device="cuda") - c["row_start"][:-1].long().repeat_interleave(n.long())
        c["mask"] = words[torch.arange(B, device="cuda").repeat_interleave(n.long()), local]
    c["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")       # one for all layers of a program
    return c


# ---- plain form -----------------------------------------------------------------------------------


def _row_places(c):
    """Sequence and place in it of every new row."""
    start, T = c["row_start"].long(), c["K"].shape[0]
    row = torch.arange(T, device="cuda")
    b = torch.searchsorted(start, row, right=True) - 1
    return b, c["cached"].long()[b] + row - start[b]


def _write_pages(c):
    b, at = _row_places(c)
    Hk, D, page = c["Hk"], c["D"], c["page"]
    where, slot = c["table"][b, at // page].long(), at % page
    k, v, steps = _pieces(c["cache"], Hk, D, page)
    for which, x in ((0, c["K"]), (1, c["V"])):
        step, codes = _steps_and_codes(x)
        bytes_ = _pack(codes.to(torch.int32) + 8)
        steps[where, which, :, slot] = step
        if which == 0:
            k[where, :, slot] = bytes_
        else:
            v[where, :, slot // 16, slot % 16 // 4, :, slot % 4] = bytes_.unflatten(-1, (16, D // 32))


def _values(bytes_, step):
    """Bytes of nibbles holding code + 8, steps -> fp32 values."""
    u = torch.stack((bytes_ & 15, bytes_ >> 4), -1).flatten(-2)
    return (u.float() - 8.0) * step.float()[..., None]


def _read_rows(c):
    b, at = _row_places(c)
    Hk, D, page = c["Hk"], c["D"], c["page"]
    where, slot = c["table"][b, at // page].long(), at % page
    k, v, steps = _pieces(c["cache"], Hk, D, page)
    vb = v[where, :, slot // 16, slot % 16 // 4, :, slot % 4].flatten(-2)
    return {"K": _values(k[where, :, slot], steps[where, 0, :, slot]).half(), "V": _values(vb, steps[where, 1, :, slot]).half()}


def _sequences(c):
    """K and V of all sequences, padded: fp32 [B, Hk, L, D] each."""
    B, Hk, D, page = c["B"], c["Hk"], c["D"], c["page"]
    k, v, steps = _pieces(c["cache"][c["table"].long()], Hk, D, page)      # [B, pages, ...]
    join = lambda x: x.transpose(1, 2).flatten(2, 3)                       # noqa: E731
    return (join(_values(k, steps[:, :, 0])), join(_values(_v_rows(v, page, D), steps[:, :, 1])))


def _visible(c, T, L):
    """bool [T, L]: which cached rows every query row sees."""
    start, cached = c["row_start"].long(), c["cached"].long()
    row = torch.arange(T, device="cuda")
    b = torch.searchsorted(start, row, right=True) - 1
    key = torch.arange(L, device="cuda")
    new = key - cached[b][:, None]                                         # which drafted row a key is
    if c["mask"] is None:
        return b, new <= (row - start[b])[:, None]
    n = (start[1:] - start[:-1])[b]
    bit = (c["mask"][:, None] >> new.clamp(0, 63)) & 1
    return b, (new < 0) | ((bit == 1) & (new < n[:, None]))


def _attention(c):
    Q, B, Hq, Hk, D, rows = c["Q"], c["B"], c["Hq"], c["Hk"], c["D"], c["rows"]
    T, G = Q.shape[0], c["Hq"] // c["Hk"]
    K, V = _sequences(c)
    L = K.shape[2]
    b, sees = _visible(c, T, L)
    local = torch.arange(T, device="cuda") - c["row_start"].long()[b]
    # rows padded to [B, Hk, rows * G]
    q = torch.zeros(B, rows, Hq, D, device="cuda")
    q[b, local] = Q.float() * c["scale"]
    q = q.view(B, rows, Hk, G, D).transpose(1, 2).reshape(B, Hk, rows * G, D)
    mask = torch.zeros(B, rows, L, dtype=torch.bool, device="cuda")
    mask[b, local] = sees
    s = torch.matmul(q, K.transpose(2, 3).contiguous()).view(B, Hk, rows, G, L)
    s = s.masked_fill_(~mask[:, None, :, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp_(min=-1e30))
    p = p / p.sum(-1, keepdim=True).clamp_(min=1e-30)
    o = torch.matmul(p.view(B, Hk, rows * G, L), V)
    o = o.view(B, Hk, rows, G, D).transpose(1, 2).reshape(B, rows, Hq, D)
    return o[b, local].half()


def _rotary(c):
    x, D, rot, m = c["X"], c["D"], c["rot"], c["magnitude"]
    angle = c["positions"].double()[:, None] * c["f"]                      # far positions need 64 bits
    cos, sin = (torch.cos(angle) * m).float()[:, None], (torch.sin(angle) * m).float()[:, None]
    v = x[..., :rot].float()
    if c["half"]:
        a, b = v[..., : rot // 2], v[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = v[..., 0::2], v[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned.half(), x[..., rot:]), -1)


def run(c):
    if own:
        return _run_own(c)
    path = c["path"]
    if path == "quantize":
        step, codes = _steps_and_codes(c["X"].unflatten(1, (-1, c["group"])))
        return {"codes": codes.flatten(1).to(torch.int8), "steps": step}
    if path == "product":
        w = _signed(c["Qw"]).unflatten(1, (-1, c["group"])).float() * c["sw"].float()[..., None]
        return {"Y": torch.matmul(c["X"].float(), w.flatten(1).t()).half()}
    if path == "rotary":
        return {"Y": _rotary(c)}
    if path == "cache":
        _write_pages(c)
        return _read_rows(c)
    return {"O": _attention(c)}


def _run_own(c):
    import paper_2511_22316_amd as sq
    path = c["path"]
    if path == "quantize":
        sq.sq_quantize_grouped(c["X"], c["group"], c["Q"], c["steps"])
        return {"codes": _signed(c["Q"]), "steps": c["steps"]}
    if path == "product":
        sq.sq_w4a16_gemm_grouped(c["X"], c["Qw"], c["sw"], c["Y"])
        return {"Y": c["Y"]}
    if path == "rotary":
        sq.sq_rotary_fp16(c["X"], c["positions"], c["turns"], c["half"], c["Y"], magnitude=c["magnitude"])
        return {"Y": c["Y"]}
    if path == "cache":
        sq.sq_cache_append(c["K"], c["V"], c["row_start"], c["cached"], c["table"], c["page"], c["cache"])
        sq.sq_cache_read(c["cache"], c["row_start"], c["cached"], c["table"], c["page"], c["Kr"], c["Vr"])
        return {"K": c["Kr"], "V": c["Vr"]}
    sq.sq_tree_attention(c["Q"], c["row_start"], c["cached"], c["mask"], c["table"], c["page"], c["cache"], c["Hk"], c["scale"],
                         c["O"], c["workspace"], max_rows=c["rows"], max_keys=c["keys"])
    return {"O": c["O"]}


# ---- 64 bits --------------------------------------------------------------------------------------


def _codes_at(cache, where, what, Hk, D, page):
    """fp64 values [rows, Hk, D] of K (what = 0) or V (1) at `where` = (page number, slot) of every row, byte by byte."""
    number, slot = where
    flat = cache.reshape(-1)
    base = number * cache.shape[1]
    h, d = torch.arange(Hk, device="cuda")[None, :, None], torch.arange(D, device="cuda")[None, None, :]
    at = base[:, None, None] + h * (page * D)
    s = slot[:, None, None]
    if what == 0:
        at = at + s * (D // 2) + d // 2
    else:
        width = D // 16                                   # channels of a unit
        at = at + page * D // 2 + (s // 16) * (8 * D) + (((s % 16) // 4 * 16 + d // width) * 4 + s % 4) * (width // 2) + d % width // 2
    code = ((flat[at].long() >> (4 * (d % 2))) & 15) - 8
    place = (base + Hk * page * D)[:, None] + 2 * ((what * Hk + h[:, :, 0]) * page + slot[:, None])
    step = flat.view(torch.float16)[place // 2].double()
    return code.double() * step[..., None]


def exact(case, seed):
    c = prepare(case, seed)
    path = c["path"]
    if path == "quantize":
        top = c["X"].double().unflatten(1, (-1, c["group"])).abs().amax(-1)
        return {"codes": None, "steps": torch.where(top == 0, torch.full_like(top, 7.0), top) / 7}
    if path == "product":
        T, K, N, g = c["T"], c["K"], c["N"], c["group"]
        y = torch.zeros(T, N, dtype=torch.float64, device="cuda")
        for a in range(0, N, 2048):
            Q = c["Qw"][a:a + 2048]
            w = torch.empty(Q.shape[0], K, dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = ((Q.long() & 15) ^ 8) - 8, ((Q.long() >> 4) ^ 8) - 8
            w *= c["sw"][a:a + 2048].double().repeat_interleave(g, 1)
            y[:, a:a + 2048] = c["X"].double() @ w.T
        return {"Y": y}
    if path == "rotary":
        y = c["X"].double().clone()
        rot, m = c["rot"], c["magnitude"]
        f = torch.from_numpy(_frequencies(rot, c["scaling"])).cuda()
        for i in range(rot // 2):
            p, q = (i, i + rot // 2) if c["half"] else (2 * i, 2 * i + 1)
            t = c["positions"].double()[:, None] * f[i]
            a, b = c["X"][..., p].double(), c["X"][..., q].double()
            y[..., p], y[..., q] = m * (a * t.cos() - b * t.sin()), m * (a * t.sin() + b * t.cos())
        return {"Y": y}
    B, Hk, D, page = c["B"], c["Hk"], c["D"], c["page"]
    start, cached = c["row_start"].tolist(), c["cached"].tolist()
    if path == "cache":
        return {"K": _quantized(c["K"]), "V": _quantized(c["V"])}
    T, Hq = c["Q"].shape[0], c["Hq"]
    o = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, past = start[b + 1] - start[b], cached[b]
        key = torch.arange(past + n, device="cuda")
        where = (c["table"][b].long()[key // page], key % page)
        k, v = (_codes_at(c["cache"], where, what, Hk, D, page) for what in (0, 1))
        row = torch.arange(n, device="cuda")[:, None]
        sees = key <= past + row
        if c["mask"] is not None:
            words = c["mask"][start[b]: start[b + 1]]
            sees = (key < past) | ((words[:, None] & (1 << (key - past).clamp(min=0, max=63))) != 0)
        for h in range(Hq):
            g = h // (Hq // Hk)
            s = (c["Q"][start[b]: start[b + 1], h].double() @ k[:, g].T) * c["scale"]
            s[~sees] = -math.inf
            o[start[b]: start[b + 1], h] = torch.softmax(s, -1) @ v[:, g]
    return {"O": o}


def _quantized(x):
    """Rows behind the quantizer, in 64 bits: the step is the fp16 number the cache holds."""
    step = (x.double().abs().amax(-1, keepdim=True) / 7).half().double()
    step[step == 0] = 1.0
    return (x.double() / step + 0.5).floor().clamp(-8, 7) * step


def work(case):
    path = case["path"]
    if path in ("quantize", "product"):
        T, K, g = case["T"], case["K"], case["group"]
        if path == "quantize":
            return {"bytes": 2.5 * T * K + 2 * T * K / g, "flops": 4 * T * K}
        N = case["N"]
        return {"bytes": 0.5 * N * K + 2 * N * K / g + 2 * T * (K + N), "flops": 2 * T * K * N}
    if path == "rotary":
        values = case["T"] * (case["Hq"] + case["Hk"]) * case["D"]
        return {"bytes": 4 * values + 4 * case["T"], "flops": 3 * values}
    B, Hk, D, keys, rows = (case[k] for k in ("B", "Hk", "D", "keys", "rows"))
    T, cached = rows * (1 + 0.75 * (B - 1)), keys * (1 + 0.75 * (B - 1))
    if path == "cache":                                    # 16-bit rows in, records out; records in, 16-bit rows out
        return {"bytes": 2 * (2 * T * Hk * 2 * D + 2 * T * Hk * (D / 2 + 2)), "flops": 8 * T * Hk * D}
    return {"bytes": cached * Hk * (D + 4) + 4 * T * case["Hq"] * D, "flops": 4 * rows * cached * case["Hq"] * D}

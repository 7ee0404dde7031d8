"""The operators of a step that checks drafted tokens, as a serving program calls them, and their plain forms in torch.

Behind a prompt each sequence holds `start` cached positions. A draft adds up to some dozens of tokens in the form of a tree:
row i of a sequence follows another row of it, or the last cached token. One step of the full model checks them all.

  gemv    projections of few rows with 4-bit weights: weight = (code - zero) * scale, codes 0 .. 15, one scale (and one zero;
          8 without) for each `group` consecutive inputs of an output row. fp32 stored or added, or the gated form in
          bf16: silu(gate) * up with the weight rows in blocks of 128 gate rows and the 128 matching up rows
  append  rows of a QKV projection to the bf16 paged cache: per-head RMSNorm of q and k (if the model has it), rotation by
          the position start + depth of the row in its tree, entries at start + row
  attend  each row over the cached positions and its ancestors (the drafted slots whose bits its mask has), with a window of
          positions if the layer has one
  keep    the accepted path: entries of its slots move to start, start + 1, ..., in all layers

4-bit weights lie as the kernels read them: tiles of 16 rows and 128 inputs, codes uint8 [rows / 16][inputs / 128][16][64].
The 64 bytes of a row are 16 words of 8 codes, word 4 t + j for inputs 32 j + 8 t .. + 7; nibble p of a word is the code of its
input 2 p, or 2 (p - 4) + 1 from p = 4 on. Scales bf16 and zeros uint8 [rows / 16][inputs / 128][16][128 / group], row r of a
tile at 2 (r % 8) + r / 8.

`own` false: elementary torch operations in fp32, for whole batches; `own` true: the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
WORKSPACE_BYTES = 64 << 20      # covers every attention call (POP_TREE_WORKSPACE_BYTES of the library)


# ------------------------------------------------------------------------------------------------ cases
def _gemv(name, rows, n, k, group, mode, zeros=False):
    return {"name": name, "op": "gemv", "rows": rows, "n": n, "k": k, "group": group, "mode": mode, "zeros": zeros}


def _append(name, batch, rows, start, n_q, n_kv, hd, page, ragged=False, x="fp32", norm=False):
    return {"name": name, "op": "append", "batch": batch, "rows": rows, "start": start, "n_q": n_q, "n_kv": n_kv, "hd": hd,
            "page": page, "ragged": ragged, "x": x, "norm": norm}


def _attend_case(name, batch, rows, start, n_q, n_kv, hd, page, window=0, ragged=False, tree=True):
    return {"name": name, "op": "attend", "batch": batch, "rows": rows, "start": start, "n_q": n_q, "n_kv": n_kv, "hd": hd,
            "page": page, "window": window, "ragged": ragged, "tree": tree}


def _keep(name, batch, rows, start, layers, n_kv, hd, page, ragged=False):
    return {"name": name, "op": "keep", "batch": batch, "rows": rows, "start": start, "layers": layers, "n_kv": n_kv,
            "hd": hd, "page": page, "ragged": ragged}


def listed():
    return [
        # the QKV projection of the small model (configuration c1) for one token: the smallest call, where latency counts
        _gemv("gemv 1 x 256 -> 512", 1, 512, 256, 32, "store"),
        # one token through the gate and up projections of configuration c2
        _gemv("gemv 1 x 4096 -> 28672 gated", 1, 28672, 4096, 128, "gated"),
        # a short draft through the down projection, added to the residual stream
        _gemv("gemv 12 x 14336 -> 4096 add", 12, 4096, 14336, 64, "add", zeros=True),
        # the drafts of a few sequences together through a QKV projection
        _gemv("gemv 64 x 4096 -> 6144", 64, 6144, 4096, 128, "store"),
        # eight drafted tokens of one sequence behind configuration c2's prompt
        _append("append 1 x 8", 1, 8, 8192, 32, 8, 128, 128),
        # trees of a serving batch, heads normalised (configuration c3), projections in bf16
        _append("append 48 x up to 33, norm", 48, 33, 6000, 32, 8, 128, 64, ragged=True, x="bf16", norm=True),
        # the small model, a chain of five
        _attend_case("attend 1 x 5 of 300", 1, 5, 300, 4, 2, 64, 16, tree=False),
        # a wide tree behind configuration c2's prompt
        _attend_case("attend 1 x 64 of 8192", 1, 64, 8192, 32, 8, 128, 128),
        # a serving batch with unequal contexts and trees
        _attend_case("attend 24 x 27 of up to 12001", 24, 27, 12001, 32, 8, 128, 64, ragged=True),
        # a local layer of configuration c4: head size 256, 1024 positions in the window
        _attend_case("attend 16 x 12 window 1024", 16, 12, 9000, 16, 8, 256, 128, window=1024, ragged=True),
        # the accepted path of one sequence, all layers of configuration c2
        _keep("keep 1 x 5, 32 layers", 1, 8, 1000, 32, 8, 128, 128),
        # of a serving batch
        _keep("keep 48 x up to 33, 32 layers", 48, 33, 150, 32, 8, 128, 64, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gemv", "gemv", "gemv", "append", "attend", "attend", "keep"])
    if op == "gemv":
        mode = rng.choice(["store", "store", "add", "gated"])
        rows = rng.choice([1, 1, 2, _log(rng, 1, 64)])
        k = 8 * _log(rng, 8, 2000)
        n = _log(rng, 16, max(32, min(30000, 100000000 // k)))
        if mode == "gated":
            n = 256 * max(1, n // 256)
        c = _gemv("", rows, n, k, rng.choice([32, 64, 128]), mode, zeros=rng.random() < 0.5)
        del c["name"]
        return c
    hd = rng.choice([64, 128, 128, 256])
    n_kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128, 256])
    ragged = rng.random() < 0.6
    if op == "append":
        batch = _log(rng, 1, 64)
        rows = _log(rng, 1, max(2, min(128, 1500 // batch)))
        c = _append("", batch, rows, _log(rng, 1, 9000) if rng.random() < 0.9 else 0, n_kv * group, n_kv, hd, page, ragged,
                    rng.choice(["fp32", "bf16"]), rng.random() < 0.5)
    elif op == "attend":
        batch, rows = _log(rng, 1, 48), _log(rng, 1, 64)
        start = _log(rng, 1, max(2, min(30000, int(24 * 12001 * 4096 / (batch * n_kv * hd * 4)),
                                        int(24 * 12001 * 32 * 32 / (batch * rows * n_kv * group)))))
        c = _attend_case("", batch, rows, start, n_kv * group, n_kv, hd, page, rng.choice([0, 0, 0, _log(rng, 1, 2000)]),
                         ragged, rng.random() < 0.8)
    else:
        batch, rows, layers = _log(rng, 1, 32), _log(rng, 2, 48), rng.randint(1, 32)
        c = _keep("", batch, rows, _log(rng, 1, max(2, min(600, 200000000 // (batch * layers * n_kv * hd)))), layers, n_kv,
                  hd, page, ragged)
    del c["name"]
    return c


def _spread(n, lo, hi, by):
    """n lengths over lo .. hi, the first hi, the second lo."""
    return [hi if i == 0 else lo if i == 1 else lo + int((hi - lo) * ((i * by) % 1.0)) for i in range(n)]


def _lengths(c):
    """(drafted rows, positions in front of them) of each sequence."""
    if not c["ragged"]:
        return [c["rows"]] * c["batch"], [c["start"]] * c["batch"]
    return _spread(c["batch"], 1, c["rows"], 0.7548776662), _spread(c["batch"], c["start"] // 16, c["start"], 0.6180339887)


def _kept_of(c):
    """Accepted rows of each sequence: every third of the drafted ones, at least one."""
    rows, _ = _lengths(c)
    return [1 + (2 * r) // 3 if r < 9 else 2 + r // 3 for r in rows]


def work(c):
    if c["op"] == "gemv":
        n, k, r = c["n"], c["k"], c["rows"]
        out = {"store": 4, "add": 8, "gated": 1}[c["mode"]]
        scales = n * -(-k // c["group"]) * (3 if c["zeros"] else 2)
        return {"bytes": n * k / 2 + scales + r * k * 2 + r * n * out, "flops": 2.0 * r * n * k}
    rows, starts = _lengths(c)
    kv, hd = c["n_kv"], c["hd"]
    if c["op"] == "append":
        return {"bytes": sum(rows) * hd * ((c["n_q"] + 2 * kv) * (4 if c["x"] == "fp32" else 2) + (c["n_q"] + 2 * kv) * 2),
                "flops": 0}
    if c["op"] == "keep":
        return {"bytes": sum(_kept_of(c)) * c["layers"] * kv * hd * 8.0, "flops": 0}
    read = pairs = 0.0
    for r, n in zip(rows, starts):
        seen = min(n, c["window"] or n)
        read += seen + r
        pairs += r * (seen + min(r, 6))
    return {"bytes": read * kv * hd * 4.0 + sum(rows) * c["n_q"] * hd * 4.0, "flops": 4.0 * hd * c["n_q"] * pairs}


# ------------------------------------------------------------------------------------------------ plain forms
def _weights(s):
    """fp32 weights [n, k] of the 4-bit tiles."""
    codes = s["codes"]
    nt, kt = codes.shape[:2]
    word = codes.view(torch.int32).view(nt, kt, 16, 4, 4)                               # [.., row, t, j]
    at = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], dtype=torch.int32, device=codes.device)
    c = (word[..., None] >> at) & 15                                                   # [.., row, t, j, input of the word]
    c = c.permute(0, 2, 1, 4, 3, 5).reshape(nt * 16, kt * 128)[:s["n"], :s["k"]]
    per_group = lambda v: (v.view(nt, kt, 8, 2, -1).permute(0, 3, 2, 1, 4).reshape(nt * 16, -1)[:s["n"]]  # noqa: E731
                           .repeat_interleave(s["group"], 1)[:, :s["k"]])
    zero = 8 if s["zeros"] is None else per_group(s["zeros"]).int()
    return (c - zero).float() * per_group(s["scales"]).float()


def _plain_gemv(s):
    y = s["x"].float() @ _weights(s).t()
    if s["mode"] == "store":
        return [y]
    if s["mode"] == "add":
        s["out"] += y
        return [s["out"]]
    y = y.view(y.shape[0], -1, 2, 128)
    gate, up = y[:, :, 0], y[:, :, 1]
    return [(gate / (1 + torch.exp(-gate)) * up).reshape(y.shape[0], -1).to(torch.bfloat16)]


def _turned(x, gain, cos, sin, eps):
    """RMSNorm per head (if gain) and rotation of x [rows, heads, hd]; cos, sin [rows, hd / 2]."""
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gain
    a, b = x.chunk(2, -1)
    cos, sin = cos[:, None, :], sin[:, None, :]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _row_of(s, rows):
    """(sequence, row in it) of each packed row."""
    cu = s["cu"].long()
    r = torch.arange(rows, device=cu.device)
    b = torch.searchsorted(cu, r, right=True) - 1
    return b, r - cu[b]


def _plain_append(s):
    n_q, n_kv, hd, page = s["n_q"], s["n_kv"], s["hd"], s["page"]
    x = s["x"].float().view(s["x"].shape[0], -1, hd)
    b, i = _row_of(s, x.shape[0])
    cs = s["rope"][s["start"].long()[b] + s["depth"].long()]
    q = _turned(x[:, :n_q], s["q_gain"], cs[..., 0], cs[..., 1], s["eps"])
    k = _turned(x[:, n_q:n_q + n_kv], s["k_gain"], cs[..., 0], cs[..., 1], s["eps"])
    at = s["start"].long()[b] + i
    where = s["table"].long()[b, at // page], at % page
    s["k"].index_put_(where, k.to(torch.bfloat16))
    s["v"].index_put_(where, x[:, n_q + n_kv:].to(torch.bfloat16))
    return [q.to(torch.bfloat16).view(q.shape[0], -1), s["k"], s["v"]]


def _plain_attend(s):
    n_q, n_kv, hd, page = s["n_q"], s["n_kv"], s["hd"], s["page"]
    b, i = _row_of(s, s["q"].shape[0])
    start, rows = s["start"].long(), s["max_rows"]
    key = torch.arange(s["max_len"], device=DEV)
    slot = key[None] - start[:, None]                                                   # [B, n] drafted slot of a position
    mine = s["cu"].long()[1:] - s["cu"].long()[:-1]
    live = slot < mine[:, None]
    bit = slot.clamp(0, rows - 1)
    depth = torch.zeros(start.numel(), rows, dtype=torch.long, device=DEV)
    bits = torch.zeros(start.numel(), rows, -(-rows // 32), dtype=torch.long, device=DEV)
    depth[b, i] = s["depth"].long() if s["depth"] is not None else i
    if s["mask"] is not None:
        bits[b, i] = s["mask"].long()
        drafted = (bits.gather(2, (bit // 32)[:, None, :].expand(-1, rows, -1)) >> (bit % 32)[:, None, :]) & 1 == 1
    else:
        drafted = bit[:, None, :] <= torch.arange(rows, device=DEV)[None, :, None]
    at = torch.where(slot >= 0, start[:, None] + depth.gather(1, bit), key[None])       # position of a cache entry
    seen = torch.where(slot[:, None, :] < 0, True, drafted) & live[:, None, :]
    if s["window"]:
        seen &= at[:, None, :] > (start[:, None] + depth)[..., None] - s["window"]
    pages, off = s["table"].long()[:, key // page], (key % page)[None].expand(start.numel(), -1)
    k, v = s["k"][pages, off].float(), s["v"][pages, off].float()                       # [B, n, kv, hd]
    v = torch.where(live[..., None, None], v, torch.zeros((), device=DEV))
    q = torch.zeros(start.numel(), rows, n_q, hd, device=DEV)
    q[b, i] = s["q"].float().view(-1, n_q, hd) / math.sqrt(hd)
    q = q.view(-1, rows, n_kv, n_q // n_kv, hd).permute(0, 2, 1, 3, 4).reshape(start.numel(), n_kv, -1, hd)
    w = (q @ k.permute(0, 2, 3, 1)).view(start.numel(), n_kv, rows, n_q // n_kv, -1)
    w.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    w -= w.amax(-1, keepdim=True).clamp_min(torch.finfo(w.dtype).min)
    w.exp_()
    total = w.sum(-1, keepdim=True).clamp_min(1e-30)
    o = (w.view(start.numel(), n_kv, -1, w.shape[-1]) @ v.permute(0, 2, 1, 3)).view(start.numel(), n_kv, rows, -1, hd) / total
    o = o.permute(0, 2, 1, 3, 4).reshape(start.numel(), rows, n_q * hd)
    return [o[b, i].to(torch.bfloat16)]


def _plain_keep(s):
    page, start = s["page"], s["start"].long()
    b, i = torch.nonzero(torch.arange(s["kept"].shape[1], device=DEV)[None] < s["n_kept"][:, None], as_tuple=True)
    src, dst = start[b] + s["kept"].long()[b, i], start[b] + i
    t = s["table"].long()
    for pool in (s["k"], s["v"]):
        pool[:, t[b, dst // page], dst % page] = pool[:, t[b, src // page], src % page]
    return [s["k"], s["v"]]


# ------------------------------------------------------------------------------------------------ inputs
def _tables(g, batch, pages_each, spare=3):
    n = batch * pages_each + spare
    return torch.randperm(n, generator=g, device=DEV)[:batch * pages_each].view(batch, pages_each).int(), n


def _trees(c, rows, seed, tree):
    """(depth [rows], mask [rows, words] or None) of the packed rows: each row follows one of the rows in front of it, half
    of the time a recent one, or the last cached token."""
    if not tree:
        return torch.cat([torch.arange(r) for r in rows]).int(), None
    g = torch.Generator().manual_seed(seed)
    most, batch = max(rows), len(rows)
    words = -(-most // 32)
    depth = torch.zeros(batch, most, dtype=torch.long)
    sees = torch.zeros(batch, most, words * 32, dtype=torch.bool)
    every = torch.arange(batch)
    for i in range(most):
        far = (torch.rand(batch, generator=g) * (i + 1)).long() - 1
        near = i - 1 - (torch.rand(batch, generator=g) * min(i + 1, 3)).long()
        parent = torch.where(torch.rand(batch, generator=g) < 0.5, far, near).clamp(-1, i - 1)
        has = parent >= 0
        p = parent.clamp_min(0)
        depth[:, i] = torch.where(has, depth[every, p] + 1, 0)
        sees[:, i] = sees[every, p] & has[:, None]
        sees[:, i, i] = True
    bits = (sees.view(batch, most, words, 32).long() << torch.arange(32)).sum(-1)
    bits = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).int()
    live = torch.arange(most)[None] < torch.tensor(rows)[:, None]
    return depth[live].int(), bits[live]


def _rope_rows(n, hd, theta=1e6):
    a = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * theta ** (
        -torch.arange(0, hd, 2, device=DEV, dtype=torch.float64) / hd)
    return torch.stack([a.cos(), a.sin()], -1).float()


def _prepare_gemv(c, g):
    n, k, rows, group = c["n"], c["k"], c["rows"], c["group"]
    nt, kt, shape = -(-n // 16), -(-k // 128), (-(-n // 16), -(-k // 128), 16, 128 // group)
    s = {"op": "gemv", "mode": c["mode"], "n": n, "k": k, "group": group}
    s["codes"] = torch.randint(0, 256, (nt, kt, 16, 64), generator=g, device=DEV, dtype=torch.uint8)
    # weights of a size of 1 / sqrt(k) with unequal groups
    s["scales"] = ((0.5 + torch.rand(shape, generator=g, device=DEV)) * 0.25 / math.sqrt(k)).to(torch.bfloat16)
    s["zeros"] = torch.randint(5, 12, shape, generator=g, device=DEV, dtype=torch.uint8) if c["zeros"] else None
    s["x"] = torch.randn(rows, k, generator=g, device=DEV).to(torch.bfloat16)
    if c["mode"] == "gated":
        s["out"] = torch.empty(rows, n // 2, dtype=torch.bfloat16, device=DEV)
    else:
        s["out"] = torch.randn(rows, n, generator=g, device=DEV)
    return s


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if c["op"] == "gemv":
        return _prepare_gemv(c, g)
    rows, starts = _lengths(c)
    n_kv, hd, page, batch, total = c["n_kv"], c["hd"], c["page"], c["batch"], sum(rows)
    top = max(r + n for r, n in zip(rows, starts))
    as_int = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = {"op": c["op"], "n_kv": n_kv, "hd": hd, "page": page, "batch": batch, "max_rows": max(rows), "max_len": top,
         "max_start": max(starts), "start": as_int(starts), "cu": as_int([sum(rows[:i]) for i in range(batch + 1)])}
    s["table"], pages = _tables(g, batch, -(-top // page))
    if c["op"] == "keep":
        shape = (c["layers"], pages, page, n_kv, hd)
        s["k"], s["v"] = (torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        n_kept = [min(m, r) for m, r in zip(_kept_of(c), rows)]
        order = torch.rand(batch, max(rows), generator=g, device=DEV)
        order = torch.where(torch.arange(max(rows), device=DEV)[None] < as_int(rows)[:, None], order, 2.0)
        chosen = order.argsort(1).argsort(1) < as_int(n_kept)[:, None]                  # a path's slots, in rising order
        slots = torch.where(chosen, torch.arange(max(rows), device=DEV)[None], 1 << 20).sort(1).values[:, :max(n_kept)]
        s["kept"], s["n_kept"] = slots.int().contiguous(), as_int(n_kept)
        return s
    s["n_q"] = c["n_q"]
    shape = (pages, page, n_kv, hd)
    s["k"] = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    s["v"] = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    tree = c.get("tree", True)
    depth, mask = _trees(c, rows, seed, tree)
    s["depth"], s["mask"] = depth.to(DEV), None if mask is None else mask.to(DEV).contiguous()
    if c["op"] == "append":
        x = torch.randn(total, (c["n_q"] + 2 * n_kv) * hd, generator=g, device=DEV) * 1.3
        s["x"] = x if c["x"] == "fp32" else x.to(torch.bfloat16)
        s["eps"] = 1e-6
        s["q_gain"], s["k_gain"] = ((0.5 + torch.rand(hd, generator=g, device=DEV)) if c["norm"] else None for _ in range(2))
        s["rope"] = _rope_rows(top, hd)
        s["q_out"] = torch.empty(total, c["n_q"] * hd, dtype=torch.bfloat16, device=DEV)
    else:
        s["window"] = c["window"]
        if not tree:
            s["depth"] = None
        s["q"] = (torch.randn(total, c["n_q"] * hd, generator=g, device=DEV) * 1.5).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["workspace"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _own(s):
    from paper_2602_03295_b200 import lib
    L, op = lib(), s["op"]
    if op == "gemv":
        L.gemv_w4(s["x"], s["codes"], s["scales"], s["zeros"], s["out"], s["n"], s["group"],
                  mode={"store": 0, "add": 2, "gated": 3}[s["mode"]])
        return [s["out"]]
    if op == "append":
        L.rope_cache_tree(s["x"], s["q_out"], s["k"], s["v"], s["table"], s["rope"], s["n_q"], s["n_kv"], s["hd"],
                          s["max_rows"], start=s["start"], cu_rows=s["cu"], depth=s["depth"], q_gain=s["q_gain"],
                          k_gain=s["k_gain"], eps=s["eps"])
        return [s["q_out"], s["k"], s["v"]]
    if op == "attend":
        L.tree_attention(s["q"], s["k"], s["v"], s["table"], s["out"], s["n_q"], s["n_kv"], s["hd"], s["max_rows"],
                         s["max_start"], start=s["start"], cu_rows=s["cu"], mask=s["mask"], depth=s["depth"],
                         window=s["window"], workspace=s["workspace"])
        return [s["out"]]
    L.cache_keep(s["k"], s["v"], s["table"], s["kept"], start=s["start"], n_kept=s["n_kept"])
    return [s["k"], s["v"]]


def run(s):
    if own:
        return _own(s)
    return {"gemv": _plain_gemv, "append": _plain_append, "attend": _plain_attend, "keep": _plain_keep}[s["op"]](s)


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_gemv(s):
    """By the definition of the layout: the code of row r and input i, read nibble by nibble."""
    n, k, group = s["n"], s["k"], s["group"]
    i = torch.arange(k, device=DEV)
    e = i % 8
    nibble = torch.where(e % 2 == 0, e // 2, e // 2 + 4)
    word = 4 * ((i % 32) // 8) + (i % 128) // 32
    byte, high = 4 * word + nibble // 2, nibble % 2
    y = torch.empty(s["x"].shape[0], n, dtype=torch.float64, device=DEV)
    x = s["x"].double()
    for r0 in range(0, n, 4096):
        r = torch.arange(r0, min(n, r0 + 4096), device=DEV)[:, None]
        b = s["codes"][r // 16, (i // 128)[None], r % 16, byte[None]].long()
        code = torch.where(high[None] == 1, b // 16, b % 16).double()
        where = r // 16, (i // 128)[None], r % 8 * 2 + r % 16 // 8, (i % 128 // group)[None]
        scale = s["scales"][where].double()
        zero = 8.0 if s["zeros"] is None else s["zeros"][where].double()
        y[:, r0:r0 + r.shape[0]] = x @ ((code - zero) * scale).t()
    if s["mode"] == "add":
        return [s["out"].double() + y]
    if s["mode"] == "store":
        return [y]
    at = torch.arange(n // 2, device=DEV)
    gate, up = y[:, at // 128 * 256 + at % 128], y[:, at // 128 * 256 + 128 + at % 128]
    return [gate * torch.sigmoid(gate) * up]


def _exact_append(s):
    n_q, n_kv, hd, page = s["n_q"], s["n_kv"], s["hd"], s["page"]
    k_pool, v_pool, qs = s["k"].double(), s["v"].double(), []
    cu, start = s["cu"].tolist(), s["start"].tolist()
    for b in range(s["batch"]):
        lo, hi = cu[b], cu[b + 1]
        x = s["x"][lo:hi].double().view(hi - lo, -1, hd)
        z = torch.view_as_complex(s["rope"][start[b] + s["depth"][lo:hi].long()].double().contiguous())[:, None]
        turned = []
        for part, gain in ((x[:, :n_q], s["q_gain"]), (x[:, n_q:n_q + n_kv], s["k_gain"])):
            if gain is not None:
                part = part / torch.sqrt(part.pow(2).mean(-1, keepdim=True) + s["eps"]) * gain.double()
            w = torch.complex(part[..., :hd // 2].contiguous(), part[..., hd // 2:].contiguous()) * z
            turned.append(torch.cat([w.real, w.imag], -1))
        qs.append(turned[0].reshape(hi - lo, -1))
        pos = start[b] + torch.arange(hi - lo, device=DEV)
        pg = s["table"][b].long()[pos // page]
        k_pool[pg, pos % page], v_pool[pg, pos % page] = turned[1], x[:, n_q + n_kv:]
    return [torch.cat(qs), k_pool, v_pool]


def _exact_attend(s):
    hd, n_q, n_kv, page = s["hd"], s["n_q"], s["n_kv"], s["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    cu, starts = s["cu"].tolist(), s["start"].tolist()
    for b in range(s["batch"]):
        lo, r, n = cu[b], cu[b + 1] - cu[b], starts[b]
        pos = torch.arange(n + r, device=DEV)
        pg, slot = s["table"][b].long()[pos // page], pos % page
        row = torch.arange(r, device=DEV)
        depth = row if s["depth"] is None else s["depth"][lo:lo + r].long()
        if s["mask"] is None:
            tree = row[None, :] <= row[:, None]
        else:
            tree = (s["mask"][lo:lo + r].long()[:, row // 32] & (1 << (row % 32))[None]) != 0
        seen = torch.cat([torch.ones(r, n, dtype=torch.bool, device=DEV), tree], 1)
        if s["window"]:
            at = torch.cat([torch.arange(n, device=DEV), n + depth])
            seen &= (n + depth)[:, None] - at[None, :] < s["window"]
        for h in range(n_q):
            kv = h // (n_q // n_kv)
            w = s["q"][lo:lo + r, h * hd:(h + 1) * hd].double() @ s["k"][pg, slot, kv].double().t() / math.sqrt(hd)
            p = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
            out[lo:lo + r, h * hd:(h + 1) * hd] = torch.nan_to_num(p) @ s["v"][pg, slot, kv].double()
    return [out]


def _exact_keep(s):
    page, res = s["page"], []
    start, n_kept, kept, table = s["start"].tolist(), s["n_kept"].tolist(), s["kept"].tolist(), s["table"].tolist()
    for pool in (s["k"], s["v"]):
        new = pool.clone()
        for b in range(s["batch"]):
            for i in range(n_kept[b]):
                src, dst = start[b] + kept[b][i], start[b] + i
                new[:, table[b][dst // page], dst % page] = pool[:, table[b][src // page], src % page]
        res.append(new.double())
    return res


def exact(c, seed):
    s = prepare(c, seed)
    return {"gemv": _exact_gemv, "append": _exact_append, "attend": _exact_attend, "keep": _exact_keep}[c["op"]](s)

"""The operators of a step that checks drafted tokens on the GPU against plain 64-bit arithmetic (tests/tree_ref.py): products
with 4-bit weights, append of a tree's rows, their attention, keeping of the accepted path, and all of them together."""
import math

import pytest
import torch

from tests import tree_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def L():
    import paper_2602_03295_b200 as pk
    return pk.lib()


@pytest.fixture(autouse=True)
def _clean_status(request):
    yield
    if "L" in request.fixturenames:
        assert request.getfixturevalue("L").dll.pop_k_status(None) == 0


def gen(seed):
    return torch.Generator().manual_seed(seed)


def within(got, want, bound, what=""):
    got = got.detach().cpu().double()
    off = (got - want).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off - bound).max())} beyond the bound, {float(off.max())} off"


# ---------------------------------------------------------------------------------------------- 4-bit weights
def weights(n, k, group, zeros, g, whole=False):
    """(codes, scales, zeros) as plain tensors; whole: scales that are powers of two."""
    groups = -(-k // group)
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    if whole:
        scales = torch.exp2(torch.randint(-3, 4, (n, groups), generator=g).double()).to(torch.bfloat16)
    else:
        scales = (torch.rand(n, groups, generator=g) + 0.1).to(torch.bfloat16) * torch.randint(0, 2, (n, groups), generator=g).mul(2).sub(1)
    return codes, scales, torch.randint(0, 16, (n, groups), generator=g, dtype=torch.uint8) if zeros else None


def laid_out(L, codes, scales, zeros, group, poison=True):
    """The tiles on the GPU; what lies behind the last row and input is garbage, NaN scales among it."""
    from paper_2602_03295_b200 import pack_w4
    c, s, z = pack_w4(codes, scales, zeros, group)
    if poison:
        n, k = codes.shape
        nt, kt = c.shape[:2]
        ones = torch.ones(n, -(-k // group))
        live = pack_w4(torch.full((n, k), 15, dtype=torch.uint8), ones, None, group)
        c = torch.where(live[0] == 0, torch.full_like(c, 0x5a), c)
        s = torch.where(live[1] == 0, torch.full_like(s, math.nan), s)
        if z is not None:
            z = torch.where(live[1] == 0, torch.full_like(z, 255), z)
    return c.cuda(), s.cuda(), None if z is None else z.cuda()


GEMV = [  # B, N, K, group, zeros
    (1, 1, 8, 32, False), (1, 16, 128, 128, True), (1, 17, 136, 64, True), (2, 512, 256, 32, False), (3, 100, 1000, 128, True),
    (8, 33, 384, 64, False), (9, 48, 2056, 32, True), (16, 700, 512, 128, False), (17, 64, 264, 64, True), (33, 80, 1288, 128, True),
    (64, 272, 768, 32, True), (65, 16, 40, 64, False), (130, 31, 128, 128, False), (1, 4096, 4096, 128, False),
    (5, 4096, 14336, 64, True), (24, 6000, 4096, 128, False), (1, 40, 40000, 128, True), (1, 9000, 96, 32, True),
    (2, 2400, 8192, 64, True), (300, 144, 640, 128, True),
    # long and wide ones of more rows than a warp-level product takes, and their ends
    (9, 4000, 14336, 128, True), (12, 16, 40000, 32, True), (48, 20000, 520, 64, False), (20, 129, 8, 32, True), (32, 256, 264, 32, False),
    (16, 1000, 4096, 32, True), (64, 128, 2176, 128, False),
    # large enough for the products on TMEM accumulators: each of their widths, groups and zeros, with ends inside tiles and steps
    (9, 2051, 4104, 32, True), (10, 2051, 4104, 32, False), (16, 1030, 8200, 64, False), (15, 1030, 8200, 64, True), (13, 4111, 2056, 128, True),
    (16, 4111, 2056, 128, False), (17, 1400, 4008, 32, True), (32, 2070, 2040, 32, False), (32, 2070, 2040, 64, True), (26, 4200, 1032, 64, False),
    (25, 4200, 1032, 128, True), (31, 1100, 4104, 128, False), (33, 1700, 2000, 32, True), (130, 1000, 1032, 32, False), (64, 520, 4104, 64, True),
    (50, 1030, 2600, 64, False), (65, 260, 8072, 128, True), (64, 2111, 1000, 128, False),
]


@pytest.mark.parametrize("B,N,K,group,zeros", GEMV)
def test_gemv_w4(L, B, N, K, group, zeros):
    g = gen(B * 1000 + N + K)
    plain = weights(N, K, group, zeros, g)
    tiles = laid_out(L, *plain, group)
    x = torch.randn(B, K + 24, generator=g).to(torch.bfloat16)[:, :K]
    want, bound = ref.gemv(x, ref.w4_values(*plain, group), group)
    wide = torch.full((B, K + 24), math.nan, dtype=torch.bfloat16, device=DEV)          # NaN behind the row's inputs
    wide[:, :K] = x.cuda()
    out = torch.full((B + 2, N + 5), 7.0, device=DEV)
    L.gemv_w4(wide[:, :K], *tiles, out[1:B + 1, :N], N, group)
    within(out[1:B + 1, :N], want, bound)
    assert (out[0] == 7).all() and (out[B + 1] == 7).all() and (out[:, N:] == 7).all()
    again = torch.empty(B, N, device=DEV)
    L.gemv_w4(wide[:, :K], *tiles, again, N, group)
    assert torch.equal(again, out[1:B + 1, :N])
    base = torch.randn(B, N, generator=g)
    acc = base.cuda()
    L.gemv_w4(wide[:, :K], *tiles, acc, N, group, mode=2)
    within(acc, base.double() + want, bound + ref.FP32 * (base.double().abs() + want.abs() + bound))


@pytest.mark.parametrize("B,N,K,group,zeros", [(1, 40, 264, 32, True), (7, 90, 512, 64, True), (12, 64, 2048, 128, True),
                                               (40, 300, 640, 32, False), (1, 3000, 1024, 128, False),
                                               (12, 8200, 1032, 128, True), (40, 6600, 512, 32, False), (20, 6600, 1000, 64, True)])
def test_gemv_w4_is_exact_where_fp32_is(L, B, N, K, group, zeros):
    """Whole inputs up to 8 and scales that are powers of two: every partial sum is a multiple of 1/8 below 2^21."""
    g = gen(N + K)
    plain = weights(N, K, group, zeros, g, whole=True)
    x = torch.randint(-8, 9, (B, K), generator=g).to(torch.bfloat16)
    w = ref.w4_values(*plain, group)
    assert float((x.double().abs() @ w.abs().t()).max()) < 2 ** 21
    out = torch.empty(B, N, device=DEV)
    L.gemv_w4(x.cuda(), *laid_out(L, *plain, group), out, N, group)
    assert torch.equal(out.cpu().double(), x.double() @ w.t())


@pytest.mark.parametrize("B,F,K,group,zeros,act,n_valid", [
    (1, 128, 64, 32, True, 0, 128), (1, 688, 256, 64, False, 0, 688), (6, 256, 1032, 128, True, 1, 200), (13, 384, 512, 32, False, 1, 384),
    (40, 512, 768, 128, True, 0, 500), (1, 14336, 4096, 128, False, 0, 14336), (70, 128, 136, 64, True, 0, 127),
    (9, 896, 4096, 32, True, 0, 890), (17, 20000, 256, 128, False, 1, 20000), (64, 300, 1000, 64, False, 0, 300),
    (12, 2000, 2056, 64, True, 0, 1990), (40, 900, 1640, 128, False, 0, 897), (64, 1000, 1032, 32, True, 1, 1000)])
def test_gemv_w4_gated(L, B, F, K, group, zeros, act, n_valid):
    N = -(-F // 128) * 256
    g = gen(F + K + B)
    codes, scales, z = weights(N, K, group, zeros, g)
    scales = scales * (4 / math.sqrt(K * 30))
    x = torch.randn(B, K, generator=g).to(torch.bfloat16)
    y, e = ref.gemv(x, ref.w4_values(codes, scales, z, group), group)
    want, bound = ref.gated(y, e, act)
    out = torch.full((B, N // 2 + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    L.gemv_w4(x.cuda(), *laid_out(L, codes, scales, z, group), out, N, group, mode=3, act=act, n_valid=n_valid)
    within(out[:, :n_valid], want[:, :n_valid], bound[:, :n_valid])
    assert (out[:, n_valid:] == 7).all()


@pytest.mark.parametrize("B", [1, 2, 5, 8, 9, 16, 30, 64])
def test_gemv_w4_of_all_magnitudes(L, B):
    """Rows from 2^-90 to 2^90, inputs within a chunk up to 2^20 apart. Those below 2^-27 of a chunk's largest are off by 2^-36 of it."""
    g = gen(B)
    N, K, group = 100 if B in (1, 2, 5, 8, 16) else 7300, 1152, 64
    plain = weights(N, K, group, True, g)
    x = torch.randn(B, K, generator=g) * torch.exp2(torch.randint(-20, 1, (B, K), generator=g).float())
    x = (x * torch.exp2(torch.linspace(-90, 90, B)[:, None].round())).to(torch.bfloat16)
    want = x.double() @ ref.w4_values(*plain, group).t()
    # the sums of code x and zero x are rounded apart: magnitudes of 15 + 15 steps for each weight
    steps = plain[1].double().abs().repeat_interleave(group, 1)[:, :K] * 30
    out = torch.empty(B, N, device=DEV)
    L.gemv_w4(x.cuda(), *laid_out(L, *plain, group), out, N, group)
    within(out, want, ref.gemv(x, steps, group)[1])


def test_gemv_w4_of_more_than_2_to_the_32_weights(L):
    g = gen(1)
    N, K, last = (1 << 19) + 40, 8448, 200
    gd = torch.Generator(device=DEV).manual_seed(1)
    nt, kt = -(-N // 16), K // 128
    codes = torch.randint(0, 256, (nt, kt, 16, 64), generator=gd, device=DEV, dtype=torch.uint8)
    scales = (torch.rand(nt, kt, 16, 1, generator=gd, device=DEV) * 0.02 + 0.01).to(torch.bfloat16)
    assert codes.numel() > 1 << 31
    from paper_2602_03295_b200 import unpack_w4
    tail = -(-last // 16)
    w = unpack_w4(codes[-tail:].contiguous(), scales[-tail:].contiguous(), None, N - (nt - tail) * 16, K).double().cpu()
    for B in (1, 12):
        x = torch.randn(B, K, generator=g).to(torch.bfloat16)
        out = torch.empty(B, N, device=DEV)
        L.gemv_w4(x.cuda(), codes, scales, None, out, N, 128)
        want, bound = ref.gemv(x, w, 128)
        within(out[:, -w.shape[0]:], want, bound)


def test_gemv_w4_workspaces_of_two_streams(L):
    """Calls on two streams at once, each with a workspace of its own, and with those that the binding takes."""
    g = gen(6)
    plain = weights(4200, 2048, 128, False, g)
    tiles = laid_out(L, *plain, 128)
    xs = [torch.randn(24, 2048, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
    want = [torch.empty(24, 4200, device=DEV) for _ in range(2)]
    for x, o in zip(xs, want):
        L.gemv_w4(x, *tiles, o, 4200, 128)
    torch.cuda.synchronize()
    need = L.dll.pop_k_gemv_w4_workspace_bytes(24, 4200, 2048, 128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for given in (True, False):
        got = [torch.zeros(24, 4200, device=DEV) for _ in range(2)]
        ws = [torch.full((need,), 255, dtype=torch.uint8, device=DEV) if given else None for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for x, o, w, st in zip(xs, got, ws, streams):
                L.gemv_w4(x, *tiles, o, 4200, 128, workspace=w, stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gemv_w4_captured(L):
    """Calls with and without a launch that converts, captured together and replayed on another stream."""
    g = gen(16)
    sizes = [(20, 6000, 1032), (64, 2111, 1000), (12, 300, 512), (8, 500, 2048), (3, 200, 256)]
    made = []
    for B, N, K in sizes:
        made.append((torch.randn(B, K, generator=g).to(torch.bfloat16).cuda(), laid_out(L, *weights(N, K, 64, True, g), 64), N,
                     torch.empty(B, N, device=DEV), torch.empty(B, N, device=DEV)))
    for x, tiles, N, a, _ in made:
        L.gemv_w4(x, *tiles, a, N, 64)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        for x, tiles, N, _, b in made:
            L.gemv_w4(x, *tiles, b, N, 64)
    with torch.cuda.stream(s):
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for _, _, _, a, b in made)


def test_gemv_w4_rows_do_not_meet(L):
    """NaN and infinities of one activation row make that row NaN and reach no other."""
    g = gen(5)
    for B, N in ((4, 96), (12, 96), (40, 96), (12, 17000), (40, 7000)):
        plain = weights(N, 512, 64, True, g)
        x = torch.randn(B, 512, generator=g).to(torch.bfloat16)
        x[1, 3], x[2, 100], x[3] = math.nan, math.inf, 0
        out = torch.empty(B, N, device=DEV)
        L.gemv_w4(x.cuda(), *laid_out(L, *plain, 64), out, N, 64)
        w = ref.w4_values(*plain, 64)
        want, bound = ref.gemv(x.nan_to_num(0, 0, 0), w, 64)
        keep = [b for b in range(B) if b not in (1, 2)]
        within(out[keep], want[keep], bound[keep])
        assert out[1].isnan().all() and out[2].isnan().all() and (out[3] == 0).all()


def test_quantize_w4(L):
    """The loaders' rounding: codes nearest to the weight in the group's scale, scales as stated, read back by the kernel."""
    from paper_2602_03295_b200 import quantize_w4, unpack_w4
    g = gen(3)
    w = (torch.randn(70, 300, generator=g) * 0.02).to(torch.bfloat16)
    w[3, :128] = 0
    for group in (32, 64, 128):
        for sym in (True, False):
            tiles = [t if t is None else t.cuda() for t in quantize_w4(w, group, sym)]
            back = unpack_w4(*tiles, 70, 300)
            eye = torch.eye(300, dtype=torch.bfloat16)
            eye = torch.nn.functional.pad(eye, (0, 4))
            out = torch.empty(300, 70, device=DEV)
            L.gemv_w4(eye.cuda()[:, :304], *tiles, out, 70, group)                       # K = 304: four inputs of zero
            assert torch.equal(out.t(), back)
            grp = torch.nn.functional.pad(w.float(), (0, -300 % group)).view(70, -1, group)
            step = grp.abs().amax(-1) / 7 if sym else (grp.amax(-1).clamp_min(0) - grp.amin(-1).clamp_max(0)) / 15
            # half a step, a bf16 rounding of the scale times 15 steps, and a zero that is rounded to a whole code
            most = step.repeat_interleave(group, 1)[:, :300] * (1.01 if not sym else 0.54)
            assert bool(((back.cpu() - w.float()).abs() <= most + 1e-9).all())


# ---------------------------------------------------------------------------------------------- cache and drafts
def pools(seed, batch, length, n_kv, hd, page, layers=None, spare=2):
    g = gen(seed)
    each = max(1, -(-length // page))
    pages = batch * each + spare
    shape = (pages, page, n_kv, hd) if layers is None else (layers, pages, page, n_kv, hd)
    k, v = (torch.randn(shape, generator=g).to(torch.bfloat16) for _ in range(2))
    return k, v, torch.randperm(pages, generator=g)[:batch * each].view(batch, each).int()


def places(table, b, pos, page):
    return table[b].long()[pos // page], pos % page


def prefix(rows):
    return torch.tensor([0] + list(torch.tensor(rows).cumsum(0)), dtype=torch.int32)


def rope_rows(n, hd):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
    return torch.stack([a.cos(), a.sin()], -1).float()


APPEND = [  # rows, starts, n_q, n_kv, hd, page, bf16, norm, tree
    ([1], [0], 1, 1, 64, 16, False, False, True), ([5], [300], 4, 2, 64, 16, False, True, False),
    ([8], [1000], 32, 8, 128, 128, False, False, True), ([3, 0, 33, 1], [17, 5, 0, 126], 6, 3, 128, 32, True, True, True),
    ([12, 40], [63, 500], 8, 8, 256, 64, True, False, True), ([7] * 9, list(range(0, 90, 10)), 5, 1, 64, 256, False, True, True),
    ([130], [64], 2, 2, 256, 128, False, True, True), ([4, 2], [9, 10], 0, 2, 128, 16, False, True, True),
    # so many that a group of lanes has four heads of a row, of one kind or of several
    ([33] * 44 + [0, 20], list(range(46)), 7, 3, 128, 64, True, True, True), ([40] * 60, [5] * 60, 10, 3, 64, 32, False, False, False),
    ([20] * 50, list(range(50)), 6, 2, 256, 16, False, True, True), ([25] * 100, [1] * 100, 0, 4, 128, 64, True, True, False)]


@pytest.mark.parametrize("rows,starts,n_q,n_kv,hd,page,bf16,norm,tree", APPEND)
def test_append_of_a_tree(L, rows, starts, n_q, n_kv, hd, page, bf16, norm, tree):
    g = gen(len(rows) * 100 + hd + sum(rows))
    top = max(r + s for r, s in zip(rows, starts))
    k, v, table = pools(hd, len(rows), top, n_kv, hd, page)
    total, width = sum(rows), (n_q + 2 * n_kv) * hd
    x = torch.randn(total, width + 8, generator=g)
    x = (x.to(torch.bfloat16) if bf16 else x)
    depth = torch.cat([ref.sees(ref.random_tree(r, g))[1] for r in rows if r]) if tree else None
    gains = [0.5 + torch.rand(hd, generator=g) if norm else None for _ in range(2)]
    rope = rope_rows(top, hd)
    cu = prefix(rows)
    kd, vd = k.cuda(), v.cuda()
    q_out = torch.full((total, n_q * hd + 4), 7.0, dtype=torch.bfloat16, device=DEV) if n_q else None
    L.rope_cache_tree(x.cuda()[:, :width], None if not n_q else q_out[:, :n_q * hd], kd, vd, table.cuda(), rope.cuda(), n_q, n_kv,
                      hd, max(rows), start=torch.tensor(starts, dtype=torch.int32, device=DEV), cu_rows=cu.cuda(),
                      depth=None if depth is None else depth.cuda(), q_gain=None if not norm else gains[0].cuda(),
                      k_gain=None if not norm else gains[1].cuda(), eps=1e-6)
    touched = torch.zeros(k.shape[:2], dtype=torch.bool)
    for b, (r, s) in enumerate(zip(rows, starts)):
        if r == 0:
            continue
        xb = x[cu[b]:cu[b + 1], :width].double().view(r, -1, hd)
        d = depth[cu[b]:cu[b + 1]].long() if tree else torch.arange(r)
        at = places(table, b, s + torch.arange(r), page)
        touched[at] = True
        want, e = ref.turned(xb[:, n_q:n_q + n_kv], rope[s + d], gains[1], 1e-6)
        within(kd.cpu()[at], want, e + ref.BF16 * (want.abs() + e))
        assert torch.equal(vd.cpu()[at], xb[:, n_q + n_kv:].to(torch.bfloat16))
        if n_q:
            want, e = ref.turned(xb[:, :n_q], rope[s + d], gains[0], 1e-6)
            within(q_out[cu[b]:cu[b + 1], :n_q * hd].view(r, n_q, hd), want, e + ref.BF16 * (want.abs() + e))
    if n_q:
        assert (q_out[:, n_q * hd:] == 7).all()
    assert torch.equal(kd.cpu()[~touched], k[~touched]) and torch.equal(vd.cpu()[~touched], v[~touched])


def test_append_with_gains_anywhere(L):
    g = gen(8)
    n_q, n_kv, hd = 6, 2, 128
    rope, table = rope_rows(64, hd).cuda(), torch.arange(4, dtype=torch.int32, device=DEV)[None]
    for rows in (3, 50):
        x, outs = torch.randn(rows, (n_q + 2 * n_kv) * hd, generator=g).cuda(), []
        gain = 0.5 + torch.rand(hd, generator=g)
        for shift in (0, 1, 2, 3):
            at = torch.zeros(hd + 4, device=DEV)
            at[shift:shift + hd] = gain.cuda()
            k, v = (torch.zeros(4, 16, n_kv, hd, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            q = torch.empty(rows, n_q * hd, dtype=torch.bfloat16, device=DEV)
            L.rope_cache_tree(x, q, k, v, table, rope, n_q, n_kv, hd, rows, pos0=2, q_gain=at[shift:shift + hd], k_gain=at[shift:shift + hd], eps=1e-5)
            outs.append((q, k, v))
        assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(o, outs[0]))


def test_pools_beyond_32_bits(L):
    """Append, attention and keeping in pages whose bytes and entries lie beyond 2^32 give what they give in the first pages."""
    n_q, n_kv, hd, page, n, start = 16, 8, 128, 128, 12, 250
    g = gen(21)
    pages = (1 << 32) // (page * n_kv * hd) + 8                     # entries, not only bytes
    big = [torch.empty(1, pages, page, n_kv, hd, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    small = [torch.zeros(1, 8, page, n_kv, hd, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    low = torch.tensor([[2, 0, 5]], dtype=torch.int32, device=DEV)
    high = torch.tensor([[pages - 1, pages - 4, pages - 7]], dtype=torch.int32, device=DEV)
    for i in range(2):
        small[i][0, low[0].long()] = torch.randn(3, page, n_kv, hd, generator=g).to(torch.bfloat16).cuda()
        for a, b in zip(high[0].tolist(), low[0].tolist()):
            big[i][0, a] = small[i][0, b]
    x, rope = torch.randn(n, (n_q + 2 * n_kv) * hd, generator=g).cuda(), rope_rows(400, hd).cuda()
    res = []
    for (k, v), table in ((small, low), (big, high)):
        q, out = (torch.empty(n, n_q * hd, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        L.rope_cache_tree(x, q, k[0], v[0], table, rope, n_q, n_kv, hd, n, pos0=start)
        L.tree_attention(q, k[0], v[0], table, out, n_q, n_kv, hd, n, start)
        L.cache_keep(k, v, table, torch.tensor([[1, 3, 4, 10]], dtype=torch.int32, device=DEV), pos0=start)
        res.append([q, out] + [p[0, t] for p in (k, v) for t in table[0].tolist()])
    assert all(torch.equal(a, b) for a, b in zip(*res))


ATTEND = [  # rows, starts, n_q, n_kv, hd, page, window, kind
    ([1], [0], 1, 1, 64, 16, 0, "tree"), ([1], [63], 4, 2, 64, 16, 0, "tree"), ([5], [300], 4, 2, 64, 16, 0, "chain"),
    ([16], [2000], 32, 8, 128, 128, 0, "tree"), ([64], [1500], 32, 8, 128, 64, 0, "tree"),
    ([3, 0, 33, 1, 17], [17, 5, 0, 126, 700], 6, 3, 128, 32, 0, "tree"), ([12, 30], [63, 500], 8, 8, 256, 64, 0, "tree"),
    ([7] * 9, list(range(0, 900, 100)), 5, 1, 64, 256, 0, "tree"), ([130], [64], 8, 2, 128, 128, 0, "tree"),
    ([200, 3], [100, 2000], 8, 4, 64, 16, 0, "bits"), ([40], [3000], 16, 8, 256, 128, 1024, "tree"),
    ([33, 20], [500, 90], 8, 2, 128, 16, 100, "tree"), ([70], [40], 4, 4, 64, 32, 5, "chain"), ([64], [10], 8, 1, 128, 64, 3, "tree"),
    ([9, 8, 40], [5, 0, 200], 7, 1, 128, 128, 0, "bits"), ([2, 2], [64, 128], 128, 1, 64, 64, 0, "tree"),
    ([1] * 70, [(37 * i) % 400 for i in range(70)], 8, 8, 128, 16, 0, "tree"), ([6], [20000], 8, 2, 64, 256, 0, "tree"),
    ([6, 1], [9000, 12], 3, 1, 256, 128, 0, "bits"), ([30, 31], [1100, 0], 24, 1, 128, 128, 0, "tree"),
    ([4] * 40, [0] * 40, 2, 1, 64, 16, 0, "chain"), ([300], [0], 4, 4, 128, 128, 0, "chain"), ([500], [70], 2, 1, 256, 16, 64, "chain"),
    # short ones, an item to a CTA
    ([3, 0, 33, 1, 17], [17, 5, 0, 126, 100], 6, 3, 128, 32, 0, "tree"), ([20, 3], [150, 40], 8, 2, 256, 64, 30, "tree"),
    ([130, 3], [50, 10], 8, 4, 64, 16, 0, "bits"), ([2] * 60, [(7 * i) % 180 for i in range(60)], 4, 2, 128, 64, 0, "tree"),
    ([60, 70], [120, 100], 16, 1, 64, 128, 0, "tree")]


def drafts(rows, kind, g):
    """(seen by rows of each sequence, depth, packed mask or None)."""
    words = max(1, -(-max(rows) // 32))
    m, d, bits = [], [], []
    for r in rows:
        if kind == "chain":
            seen, depth = torch.ones(r, r).tril().bool(), torch.arange(r, dtype=torch.int32)
        else:
            seen, depth = ref.sees(ref.random_tree(r, g))
            if kind == "bits":                                      # any bits; a row may see later slots, or none at all
                seen = torch.rand(r, r, generator=g) < 0.4
                seen[r // 2] = False
        junk = torch.rand(r, words * 32, generator=g) < 0.5         # bits behind the sequence's rows
        junk[:, :r] = seen
        m.append(seen)
        d.append(depth)
        bits.append(ref.pack_bits(junk, words))
    return m, torch.cat(d), None if kind == "chain" else torch.cat(bits)


def attend_all(rows, starts, n_q, n_kv, hd, page, window, q, k, v, table, seen, depth):
    """(out, bound) [rows, n_q hd] in fp64."""
    cu = prefix(rows).tolist()
    out, bound = (torch.zeros(sum(rows), n_q * hd, dtype=torch.float64) for _ in range(2))
    for b, (r, s) in enumerate(zip(rows, starts)):
        if r == 0:
            continue
        pg, slot = places(table, b, torch.arange(s + r), page)
        d = depth[cu[b]:cu[b + 1]].long()
        m = torch.cat([torch.ones(r, s, dtype=torch.bool), seen[b]], 1)
        if window:
            m &= (s + d)[:, None] - torch.cat([torch.arange(s), s + d])[None] < window
        for h in range(n_q):
            kb, vb = k[pg, slot, h * n_kv // n_q], v[pg, slot, h * n_kv // n_q]
            live = m.any(0)                                         # nobody sees the others: they may be anything
            o, e = ref.attend(q[cu[b]:cu[b + 1], h * hd:(h + 1) * hd], kb[live], vb[live], m[:, live])
            out[cu[b]:cu[b + 1], h * hd:(h + 1) * hd], bound[cu[b]:cu[b + 1], h * hd:(h + 1) * hd] = o, e
    return out, bound


def poison(k, v, table, rows, starts, page, window):
    """NaN wherever no row may look: behind the drafts, in unused pages, in front of every window."""
    live = torch.zeros(k.shape[:2], dtype=torch.bool)
    for b, (r, s) in enumerate(zip(rows, starts)):
        if r:
            live[places(table, b, torch.arange(max(0, s - window + 1) if window else 0, s + r), page)] = True
    k[~live] = math.nan
    v[~live] = math.nan


def run_attend(L, rows, starts, n_q, n_kv, hd, page, window, kind, seed, q_scale=1.5, **more):
    g = gen(seed)
    top = max(r + s for r, s in zip(rows, starts))
    k, v, table = pools(seed, len(rows), top, n_kv, hd, page)
    poison(k, v, table, rows, starts, page, window)
    seen, depth, mask = drafts(rows, kind, g)
    total = sum(rows)
    q = (torch.randn(total, n_q * hd, generator=g) * q_scale).to(torch.bfloat16)
    want, bound = attend_all(rows, starts, n_q, n_kv, hd, page, window, q, k, v, table, seen, depth)
    if window:                                                      # pages in front of every window: any entry
        for b, s in enumerate(starts):
            table[b, :max(0, s - window + 1) // 64 * 64 // page] = 1 << 20
    qd = torch.full((total, n_q * hd + 8), math.nan, dtype=torch.bfloat16, device=DEV)
    qd[:, :n_q * hd] = q.cuda()
    out = torch.full((total + 2, n_q * hd + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    args = dict(start=torch.tensor(starts, dtype=torch.int32, device=DEV), cu_rows=prefix(rows).cuda(),
                mask=None if mask is None else mask.cuda(), depth=None if kind == "chain" else depth.cuda(), window=window)
    args.update(more)
    call = lambda o: L.tree_attention(qd[:, :n_q * hd], k.cuda(), v.cuda(), table.cuda(), o, n_q, n_kv, hd, max(rows), max(starts),  # noqa: E731
                                      **args)
    call(out[1:total + 1, :n_q * hd])
    within(out[1:total + 1, :n_q * hd], want, bound)
    assert (out[0] == 7).all() and (out[total + 1] == 7).all() and (out[:, n_q * hd:] == 7).all()
    again = torch.empty(total, n_q * hd, dtype=torch.bfloat16, device=DEV)
    call(again)
    assert torch.equal(again, out[1:total + 1, :n_q * hd])


@pytest.mark.parametrize("rows,starts,n_q,n_kv,hd,page,window,kind", ATTEND)
def test_tree_attention(L, rows, starts, n_q, n_kv, hd, page, window, kind):
    run_attend(L, rows, starts, n_q, n_kv, hd, page, window, kind, seed=sum(rows) + hd)


def test_tree_attention_of_large_and_tiny_queries(L):
    for scale in (60.0, 1e-3, 0.0):
        run_attend(L, [20, 3], [700, 150], 8, 2, 128, 64, 0, "tree", seed=9, q_scale=scale)


def test_rows_that_see_nothing_are_zeros(L):
    rows, n_q, hd = [6, 40], 4, 128
    k, v, table = pools(3, 2, 64, 2, hd, 16)
    q = torch.randn(46, n_q * hd).to(torch.bfloat16).cuda()
    mask = torch.zeros(46, 2, dtype=torch.int32)
    mask[3, 0] = 1                                                  # row 3 sees slot 0 alone: its output is that value
    out = torch.full_like(q, 7.0)
    L.tree_attention(q, k.cuda(), v.cuda(), table.cuda(), out, n_q, 2, hd, 40, 0, cu_rows=prefix(rows).cuda(), mask=mask.cuda())
    want = torch.zeros(46, n_q, hd, dtype=torch.bfloat16)
    want[3] = v[places(table, 0, torch.tensor(0), 16)].repeat_interleave(2, 0)
    assert torch.equal(out.cpu().view(46, n_q, hd), want)


def test_nan_and_infinite_queries_stay_in_their_rows(L):
    rows, starts, n_q, hd = [9], [5000], 4, 128
    g = gen(8)
    k, v, table = pools(8, 1, 5009, 2, hd, 128)
    seen, depth, mask = drafts(rows, "tree", g)
    q = torch.randn(9, n_q * hd, generator=g).to(torch.bfloat16)
    want, bound = attend_all(rows, starts, n_q, 2, hd, 128, 0, q, k, v, table, seen, depth)
    q[2, 5], q[4, hd + 7] = math.nan, math.inf
    out = torch.empty(9, n_q * hd, dtype=torch.bfloat16, device=DEV)
    L.tree_attention(q.cuda(), k.cuda(), v.cuda(), table.cuda(), out, n_q, 2, hd, 9, 5000, mask=mask.cuda())
    hit = torch.zeros(9, n_q, dtype=torch.bool)
    hit[2, 0] = hit[4, 1] = True
    o = out.cpu().view(9, n_q, hd)
    assert o[hit].isnan().all()
    within(o[~hit], want.view(9, n_q, hd)[~hit], bound.view(9, n_q, hd)[~hit])


def test_bad_lengths_and_pages_touch_their_own_sequence(L):
    from paper_2602_03295_b200 import POP_E_INVALID
    n_q, n_kv, hd, page, rows, starts = 4, 2, 64, 16, [4, 4, 4, 4, 4], [30, 200, 40, 20, 33]
    k, v, table = pools(1, 5, 80, n_kv, hd, page)
    g = gen(1)
    seen, depth, mask = drafts(rows, "tree", g)
    q = torch.randn(20, n_q * hd, generator=g).to(torch.bfloat16)
    good = [0, 3]
    want, bound = attend_all([4] * 5, [30, 33, 40, 20, 33], n_q, n_kv, hd, page, 0, q, k, v, table, seen, depth)
    bad = table.clone()
    bad[2, 1] = 1 << 24                                             # a page outside the pool
    bad[4, 0] = -3
    start = torch.tensor(starts, dtype=torch.int32)                 # 200: beyond max_start
    out = torch.full((20, n_q * hd), 7.0, dtype=torch.bfloat16, device=DEV)
    L.tree_attention(q.cuda(), k.cuda(), v.cuda(), bad.cuda(), out, n_q, n_kv, hd, 4, 60, start=start.cuda(), mask=mask.cuda())
    assert L.dll.pop_k_status(None) == POP_E_INVALID
    for b in good:
        within(out[4 * b:4 * b + 4], want[4 * b:4 * b + 4], bound[4 * b:4 * b + 4])
    assert (out[4:8] == 7).all()
    # prefix sums that leave the rows, and more rows than stated
    cu = torch.tensor([0, 4, 10, 12, 16, 40], dtype=torch.int32)
    out.fill_(7.0)
    L.tree_attention(q.cuda(), k.cuda(), v.cuda(), table.cuda(), out, n_q, n_kv, hd, 4, 60, start=torch.tensor([30, 33, 40, 20, 33],
                     dtype=torch.int32).cuda(), cu_rows=cu.cuda(), mask=mask.cuda())
    assert L.dll.pop_k_status(None) == POP_E_INVALID
    within(out[:4], want[:4], bound[:4])
    within(out[12:16], want[12:16], bound[12:16])
    assert (out[4:10] == 7).all() and (out[16:] == 7).all()
    # the append: the same checks
    x = torch.randn(20, (n_q + 2 * n_kv) * hd, generator=g).cuda()
    rope = rope_rows(100, hd).cuda()
    kd, vd, qo = k.cuda(), v.cuda(), torch.full((20, n_q * hd), 7.0, dtype=torch.bfloat16, device=DEV)
    L.rope_cache_tree(x, qo, kd, vd, bad.cuda(), rope, n_q, n_kv, hd, 4, start=torch.tensor([30, -1, 14, 20, 99], dtype=torch.int32).cuda(),
                      depth=depth.cuda())
    assert L.dll.pop_k_status(None) == POP_E_INVALID
    assert (qo[4:8] == 7).all() and (qo[:4] != 7).any() and (qo[12:16] != 7).any()
    page0 = places(table, 0, torch.arange(30, 34), page)
    assert torch.equal(vd.cpu()[page0], x[:4, (n_q + n_kv) * hd:].cpu().view(4, n_kv, hd).to(torch.bfloat16))


# ---------------------------------------------------------------------------------------------- the accepted path
@pytest.mark.parametrize("layers,n_kv,hd,page,starts,kept", [
    (1, 1, 64, 16, [0], [[0]]), (2, 2, 64, 16, [13], [[0, 2, 3, 9]]), (3, 8, 128, 32, [100, 31, 64], [[1, 2, 3], [], [0, 1, 2]]),
    (2, 3, 256, 128, [126, 5], [[2, 5, 6, 7, 11, 12, 13, 14, 20, 29, 30], [4]]), (1, 1, 64, 16, [7], [list(range(1, 200, 2))]),
    (2, 8, 256, 64, [60], [list(range(3, 90))])])
def test_keeping_a_path(L, layers, n_kv, hd, page, starts, kept):
    top = max(s + (max(x) if x else 0) for s, x in zip(starts, kept)) + 1
    k, v, table = pools(7, len(starts), top, n_kv, hd, page, layers=layers)
    most = max(len(x) for x in kept)
    lists = torch.tensor([x + [-5] * (most + 1 - len(x)) for x in kept], dtype=torch.int32)[:, :most]    # row stride most + 1
    kd, vd = k.cuda(), v.cuda()
    L.cache_keep(kd, vd, table.cuda(), lists.cuda(), start=torch.tensor(starts, dtype=torch.int32).cuda(),
                 n_kept=torch.tensor([len(x) for x in kept], dtype=torch.int32).cuda())
    for pool, got in ((k, kd), (v, vd)):
        want = pool.clone()
        for b, (s, x) in enumerate(zip(starts, kept)):
            src, dst = places(table, b, s + torch.tensor(x).long(), page), places(table, b, s + torch.arange(len(x)), page)
            want[:, dst[0], dst[1]] = pool[:, src[0], src[1]]
        assert torch.equal(got.cpu(), want)


def test_bad_paths_leave_their_sequence_alone(L):
    from paper_2602_03295_b200 import POP_E_INVALID
    k, v, table = pools(7, 5, 60, 2, 64, 16, layers=2)
    table[3, 2] = 1 << 20
    lists = torch.tensor([[1, 3, 4], [1, 1, 4], [-1, 2, 3], [1, 3, 4], [1, 2, 900]], dtype=torch.int32)
    start = torch.tensor([20, 20, 20, 30, 20], dtype=torch.int32)
    kd, vd = k.cuda(), v.cuda()
    L.cache_keep(kd, vd, table.cuda(), lists.cuda(), start=start.cuda())
    assert L.dll.pop_k_status(None) == POP_E_INVALID
    want = k.clone()
    src, dst = places(table, 0, 20 + torch.tensor([1, 3, 4]), 16), places(table, 0, 20 + torch.arange(3), 16)
    want[:, dst[0], dst[1]] = k[:, src[0], src[1]]
    assert torch.equal(kd.cpu(), want)


# ---------------------------------------------------------------------------------------------- streams, graphs, together
def test_captured_and_on_another_stream(L):
    """All four captured into a graph and replayed on a stream of its own give the bits of eager calls."""
    n_q, n_kv, hd, page, rows, starts = 8, 2, 128, 64, [9, 4], [600, 75]
    g = gen(2)
    k, v, table = pools(2, 2, 700, n_kv, hd, page)
    seen, depth, mask = drafts(rows, "tree", g)
    d = lambda t: t.cuda()  # noqa: E731
    N, K = (n_q + 2 * n_kv) * hd, 512
    tiles = laid_out(L, *weights(N, K, 64, True, g), 64)
    x, rope, tab, cu, st = d(torch.randn(13, K, generator=g).to(torch.bfloat16)), d(rope_rows(700, hd)), d(table), d(prefix(rows)), \
        torch.tensor(starts, dtype=torch.int32, device=DEV)
    m, dp, kept = d(mask), d(depth), torch.tensor([[0, 3, 8], [1, 2, 3]], dtype=torch.int32, device=DEV)

    def step(kd, vd, qkv, q, out, ws, stream=None):
        L.gemv_w4(x, *tiles, qkv, N, 64, stream=stream)
        L.rope_cache_tree(qkv, q, kd, vd, tab, rope, n_q, n_kv, hd, 9, start=st, cu_rows=cu, depth=dp, stream=stream)
        L.tree_attention(q, kd, vd, tab, out, n_q, n_kv, hd, 9, 600, start=st, cu_rows=cu, mask=m, workspace=ws, stream=stream)
        L.cache_keep(kd[None], vd[None], tab, kept, start=st, stream=stream)

    def buffers():
        from paper_2602_03295_b200.binding import POP_TREE_WORKSPACE_BYTES
        return [d(k), d(v), torch.empty(13, N, device=DEV), torch.empty(13, n_q * hd, dtype=torch.bfloat16, device=DEV),
                torch.empty(13, n_q * hd, dtype=torch.bfloat16, device=DEV), torch.empty(POP_TREE_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)]

    eager, captured, side = buffers(), buffers(), buffers()
    step(*eager)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        step(*captured)
    for t, src in zip(captured[:2], (k, v)):
        t.copy_(src)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph.replay()
    s2 = torch.cuda.Stream()
    step(*side, stream=s2)
    torch.cuda.synchronize()
    for a, b, c in zip(eager[:5], captured[:5], side[:5]):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_calls_argument_by_argument(L):
    """The four entry points called directly give the bits of the binding, which hands them packed words."""
    n_q, n_kv, hd, page, rows, start, K = 4, 2, 64, 32, 6, 100, 256
    g = gen(31)
    N = (n_q + 2 * n_kv) * hd
    tiles = laid_out(L, *weights(N, K, 32, True, g), 32)
    k, v, table = pools(31, 1, start + rows, n_kv, hd, page, layers=1)
    x, rope, tab, gain = torch.randn(rows, K, generator=g).to(torch.bfloat16).cuda(), rope_rows(200, hd).cuda(), table.cuda(), torch.rand(hd, generator=g).cuda()
    kept = torch.tensor([[1, 2, 5]], dtype=torch.int32, device=DEV)
    res = []
    for direct in (False, True):
        kd, vd = k.cuda(), v.cuda()
        qkv, q, out = torch.empty(rows, N, device=DEV), *(torch.empty(rows, n_q * hd, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ws = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
        if direct:
            s, p = torch.cuda.current_stream().cuda_stream, lambda t: t.data_ptr()  # noqa: E731
            pages = (kd.shape[1], tab.shape[1])
            assert L.dll.pop_k_gemv_w4(p(x), K, p(tiles[0]), p(tiles[1]), p(tiles[2]), 32, p(ws), ws.numel(), p(qkv), N, rows, N, K, 0, 0, N, s) == 0
            assert L.dll.pop_k_rope_cache_tree(p(qkv), 0, N, rows, None, rows, None, start, None, 1, p(q), n_q * hd, p(kd), p(vd), p(tab), page,
                                               *pages, p(gain), p(gain), 1e-3, p(rope), 200, n_q, n_kv, hd, s) == 0
            assert L.dll.pop_k_tree_attention(p(q), n_q * hd, rows, None, rows, None, start, None, 0, None, p(kd), p(vd), p(tab), page, *pages,
                                              p(ws), ws.numel(), p(out), n_q * hd, 1, n_q, n_kv, hd, 0, s) == 0
            assert L.dll.pop_k_cache_keep(p(kd), p(vd), kd.stride(0), 1, p(tab), page, *pages, p(kept), 3, None, 3, None, start, 1, n_kv, hd, s) == 0
        else:
            L.gemv_w4(x, *tiles, qkv, N, 32)
            L.rope_cache_tree(qkv, q, kd[0], vd[0], tab, rope, n_q, n_kv, hd, rows, pos0=start, q_gain=gain, k_gain=gain, eps=1e-3)
            L.tree_attention(q, kd[0], vd[0], tab, out, n_q, n_kv, hd, rows, start)
            L.cache_keep(kd, vd, tab, kept, pos0=start)
        res.append((qkv, q, out, kd, vd))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_a_checked_path_is_what_decoding_gives(L):
    """A tree is projected, appended and attended at once; its accepted path is kept. The same tokens decoded one by one with
    the calls that the library has had (projection by the bf16 GEMV over the same weights, append of one row, single-query
    attention) leave the same cache and outputs."""
    from paper_2602_03295_b200 import tree_mask, unpack_w4, quantize_w4
    n_q, n_kv, hd, page, start, dim = 8, 2, 128, 64, 333, 384
    g = gen(11)
    k, v, table = pools(11, 1, 400, n_kv, hd, page)
    parents = [-1, 0, 0, 1, 2, 2, 4, 6, 3]
    path = [0, 2, 4, 6, 7]
    mask, depth = tree_mask(parents)
    N = (n_q + 2 * n_kv) * hd
    tiles = [t if t is None else t.cuda() for t in quantize_w4(torch.randn(N, dim, generator=g) * 0.05, 64, False)]
    w = unpack_w4(*tiles, N, dim)
    x = torch.randn(9, dim, generator=g).to(torch.bfloat16).cuda()
    rope = rope_rows(400, hd).cuda()
    tab = table.cuda()
    kd, vd = k.cuda(), v.cuda()
    qkv, q, out = torch.empty(9, N, device=DEV), torch.empty(9, n_q * hd, dtype=torch.bfloat16, device=DEV), \
        torch.empty(9, n_q * hd, dtype=torch.bfloat16, device=DEV)
    L.gemv_w4(x, *tiles, qkv, N, 64)
    L.rope_cache_tree(qkv, q, kd, vd, tab, rope, n_q, n_kv, hd, 9, pos0=start, depth=depth.cuda())
    L.tree_attention(q, kd, vd, tab, out, n_q, n_kv, hd, 9, start, mask=mask.cuda(), depth=depth.cuda())
    L.cache_keep(kd[None], vd[None], tab, torch.tensor([path], dtype=torch.int32, device=DEV), pos0=start)
    ke, ve = k.cuda(), v.cuda()
    for i, r in enumerate(path):
        row = x[r:r + 1].float() @ w.t()
        q1, o1 = torch.empty(1, n_q * hd, dtype=torch.bfloat16, device=DEV), torch.empty(1, n_q * hd, dtype=torch.bfloat16, device=DEV)
        L.rope_cache(row, q1, ke[None], ve[None], 0, tab, page, None, None, rope, n_q, n_kv, hd, 1, 1, start + i, 0.0)
        L.decode_attention(q1, ke, ve, tab, o1, n_q, n_kv, hd, start + i + 1, page)
        # the projections differ by fp32 sums, so bf16 entries by a step; the outputs by bf16 weights and steps of q, k, v
        assert torch.allclose(out[r].float(), o1[0].float(), rtol=4 * ref.BF16, atol=4 * ref.BF16 * float(o1.float().abs().max()))
    n = start + len(path)
    at = places(table, 0, torch.arange(n), page)
    for a, b in ((kd, ke), (vd, ve)):
        assert torch.equal(a.cpu()[at][:start], b.cpu()[at][:start])
        assert torch.allclose(a.cpu()[at].float(), b.cpu()[at].float(), rtol=2 * ref.BF16, atol=1e-5)

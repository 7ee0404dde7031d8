"""The operators of a step that checks drafted tokens at the ends of what their header allows."""
import pytest
import torch

from tests import test_gpu_tree as base
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


def int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------------------------- windows
FREED = [  # rows, starts, n_q, n_kv, hd, page, window: cut into stretches, and short ones that go whole to a CTA
    ([20, 3, 9], [500, 90, 210], 8, 2, 128, 16, 100), ([20, 3, 9], [500, 90, 210], 4, 2, 64, 32, 100),
    ([9, 5], [3000, 777], 4, 2, 256, 16, 300), ([40], [700], 8, 8, 128, 32, 1), ([33, 20], [1000, 460], 4, 1, 128, 128, 200),
    ([12, 5], [150, 99], 8, 2, 128, 16, 30), ([6], [120], 4, 2, 256, 32, 40), ([70], [100], 4, 4, 64, 16, 5)]


@pytest.mark.parametrize("entry", [-1, 1 << 20])
@pytest.mark.parametrize("rows,starts,n_q,n_kv,hd,page,window", FREED)
def test_entries_of_pages_in_front_of_every_window(L, rows, starts, n_q, n_kv, hd, page, window, entry):
    """Whole pages in front of start - window + 1 may have been given back: any entry, with no effect and no complaint. The
    first page that a row sees is still looked at."""
    from paper_2602_03295_b200 import POP_E_INVALID
    g = base.gen(sum(rows) + page)
    k, v, table = base.pools(page, len(rows), max(r + s for r, s in zip(rows, starts)), n_kv, hd, page)
    base.poison(k, v, table, rows, starts, page, window)
    _, depth, mask = base.drafts(rows, "tree", g)
    q = torch.randn(sum(rows), n_q * hd, generator=g).to(torch.bfloat16).cuda()
    kd, vd = k.cuda(), v.cuda()

    def call(entries):
        out = torch.full_like(q, 7.0)
        L.tree_attention(q, kd, vd, entries.cuda(), out, n_q, n_kv, hd, max(rows), max(starts), start=int32(starts),
                         cu_rows=base.prefix(rows).cuda(), mask=mask.cuda(), depth=depth.cuda(), window=window)
        return out

    want, freed = call(table), table.clone()
    assert L.dll.pop_k_status(None) == 0
    for b, s in enumerate(starts):
        freed[b, :max(0, s - window + 1) // page] = entry
    assert not torch.equal(freed, table)
    got = call(freed)
    assert L.dll.pop_k_status(None) == 0
    assert torch.equal(got, want)
    freed[0, max(0, starts[0] - window + 1) // page] = entry
    call(freed)
    assert L.dll.pop_k_status(None) == POP_E_INVALID


@pytest.mark.parametrize("rows,starts,hd,window", [
    ([300, 7], [1000, 64], 128, 0x7ffffff0), ([130, 9], [20, 500], 64, 0x7ffffff0), ([40], [3000], 256, 0x7ffffff0),
    ([300, 7], [1000, 64], 128, 1300), ([70, 60], [100, 90], 128, 0x7fffffe0), ([200], [500], 64, 1 << 30)])
def test_windows_that_hide_nothing(L, rows, starts, hd, window):
    """A window that reaches beyond every position is no window, up to the largest that is taken."""
    n_q, n_kv, page = 4, 2, 64
    g = base.gen(hd + sum(rows))
    k, v, table = (t.cuda() for t in base.pools(hd, len(rows), max(r + s for r, s in zip(rows, starts)), n_kv, hd, page))
    _, depth, mask = base.drafts(rows, "tree", g)
    q = torch.randn(sum(rows), n_q * hd, generator=g).to(torch.bfloat16).cuda()
    outs = []
    for w in (0, window):
        outs.append(torch.empty_like(q))
        L.tree_attention(q, k, v, table, outs[-1], n_q, n_kv, hd, max(rows), max(starts), start=int32(starts),
                         cu_rows=base.prefix(rows).cuda(), mask=mask.cuda(), depth=depth.cuda(), window=w)
    assert torch.equal(*outs)


# ---------------------------------------------------------------------------------------------- 4-bit weights
PLACES = [(1, 512, 512), (2, 256, 256), (8, 2048, 2048), (9, 4096, 2048), (30, 4096, 1024), (64, 4096, 512)]


@pytest.mark.parametrize("B,N,K", PLACES)
def test_gemv_w4_small_inputs_beside_a_large_one(L, B, N, K):
    """Every chunk of 128 inputs has a largest of 1; each row of weights takes one input alone, with code 15 and zero 0. Inputs
    down to 2^-28 are exact there, smaller ones off by at most 2^-36 times the code (and one rounding of fp32)."""
    g = base.gen(B)
    x = (1 + torch.randint(0, 128, (B, K), generator=g) / 128) * torch.exp2(-torch.randint(20, 40, (B, K), generator=g).float())
    x *= torch.randint(0, 2, (B, K), generator=g) * 2 - 1
    x[:, ::128] = 1
    x = x.to(torch.bfloat16)
    at = torch.arange(N) % K
    codes = torch.zeros(N, K, dtype=torch.uint8)
    codes[torch.arange(N), at] = 15
    tiles = base.laid_out(L, codes, torch.ones(N, K // 128, dtype=torch.bfloat16), torch.zeros(N, K // 128, dtype=torch.uint8), 128)
    out = torch.empty(B, N, device=DEV)
    L.gemv_w4(x.cuda(), *tiles, out, N, 128)
    want = 15 * x.double()[:, at]
    exact = want.abs() >= 15 * 2.0 ** -28
    assert bool(exact.any()) and bool((~exact).any())
    assert torch.equal(out.cpu().double()[exact], want[exact])
    base.within(out, want, 15 * 2.0 ** -36 + ref.FP32 * want.abs())


@pytest.mark.parametrize("B,N,K", [(1, 100, 512), (2, 40, 136), (7, 600, 1536), (12, 64, 256), (9, 4200, 2056), (24, 4200, 1032), (50, 2100, 1032)])
@pytest.mark.parametrize("zeros", [False, True])
def test_gemv_w4_whose_sums_of_inputs_leave_fp32(L, B, N, K, zeros):
    """Inputs near the largest bf16, all of one sign: their sums are beyond fp32, the products are not."""
    g = base.gen(B + K)
    codes, _, z = base.weights(N, K, 64, zeros, g)
    scales = torch.full((N, -(-K // 64)), 2.0 ** -30, dtype=torch.bfloat16)
    x = ((1 + torch.rand(B, K, generator=g)) * 2.0 ** 126).to(torch.bfloat16)
    assert float(x.double()[:, :64].sum(1).min()) > 2.0 ** 128
    out = torch.empty(B, N, device=DEV)
    L.gemv_w4(x.cuda(), *base.laid_out(L, codes, scales, z, 64), out, N, 64)
    want = x.double() @ ref.w4_values(codes, scales, z, 64).t()
    # the sums of code x and zero x are rounded apart: magnitudes of 15 + 15 steps for each weight
    base.within(out, want, ref.gemv(x, torch.full((N, K), 30 * 2.0 ** -30, dtype=torch.float64), 64)[1])


def test_packed_weights_are_there(L):
    """The products read weights ahead of the stream's order: tiles made on the GPU are complete when their maker returns."""
    from paper_2602_03295_b200 import pack_w4, quantize_w4
    w = torch.randn(8192, 4096, device=DEV)
    codes, scales = torch.zeros(8192, 4096, dtype=torch.uint8, device=DEV), torch.ones(8192, 32, device=DEV)
    zeros = torch.zeros(8192, 32, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for make in (lambda: pack_w4(codes, scales), lambda: pack_w4(codes, scales, zeros), lambda: quantize_w4(w), lambda: quantize_w4(w, symmetric=False)):
        for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
            with torch.cuda.stream(stream):
                make()
                made = stream.query()
            torch.cuda.synchronize()
            assert made


# ---------------------------------------------------------------------------------------------- the accepted path
def test_lists_of_paths_with_a_row_stride(L):
    """Lists that are columns of a wider tensor; what lies behind a sequence's list is not looked at."""
    starts, kept = [100, 31, 64, 7], [[1, 2, 5], [], [0, 1, 7], [4, 6]]
    k, v, table = base.pools(7, 4, 120, 2, 64, 16, layers=2)
    wide = torch.full((4, 9), -5, dtype=torch.int32)
    for b, x in enumerate(kept):
        wide[b, :len(x)] = torch.tensor(x, dtype=torch.int32)
    lists = wide.cuda()[:, :3]
    assert lists.stride() == (9, 1)
    kd, vd = k.cuda(), v.cuda()
    L.cache_keep(kd, vd, table.cuda(), lists, start=int32(starts), n_kept=int32([len(x) for x in kept]))
    for pool, got in ((k, kd), (v, vd)):
        want = pool.clone()
        for b, (s, x) in enumerate(zip(starts, kept)):
            src, dst = base.places(table, b, s + torch.tensor(x).long(), 16), base.places(table, b, s + torch.arange(len(x)), 16)
            want[:, dst[0], dst[1]] = pool[:, src[0], src[1]]
        assert torch.equal(got.cpu(), want)


# ---------------------------------------------------------------------------------------------- calls at once
def test_calls_of_three_streams_at_once(L):
    """Attention of two head sizes and products on tensor memory, each on a stream of its own with a workspace of its own, give the
    bits that they give one after the other."""
    g = base.gen(41)
    tiles = base.laid_out(L, *base.weights(4200, 2048, 64, True, g), 64)
    x = torch.randn(40, 2048, generator=g).to(torch.bfloat16).cuda()
    calls = [lambda o, w, s: L.gemv_w4(x, *tiles, o, 4200, 64, workspace=w, stream=s)]
    outs = [torch.zeros(40, 4200, device=DEV)]
    for hd, rows, starts in ((128, [12, 30, 5], [3000, 70, 900]), (256, [9, 20], [2500, 400])):
        k, v, table = (t.cuda() for t in base.pools(hd, len(rows), max(r + s for r, s in zip(rows, starts)), 2, hd, 64))
        _, depth, mask = base.drafts(rows, "tree", g)
        q = torch.randn(sum(rows), 8 * hd, generator=g).to(torch.bfloat16).cuda()
        calls.append(lambda o, w, s, q=q, k=k, v=v, t=table, hd=hd, rows=rows, more=dict(
            start=int32(starts), cu_rows=base.prefix(rows).cuda(), mask=mask.cuda(), depth=depth.cuda(), window=2000), top=max(starts):
            L.tree_attention(q, k, v, t, o, 8, 2, hd, max(rows), top, workspace=w, stream=s, **more))
        outs.append(torch.zeros_like(q))
    spaces = [torch.empty(64 << 20, dtype=torch.uint8, device=DEV) for _ in calls]
    for call, o, w in zip(calls, outs, spaces):
        call(o, w, None)
    torch.cuda.synchronize()
    want, streams = [o.clone() for o in outs], [torch.cuda.Stream() for _ in calls]
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    for _ in range(100):
        for call, o, w, s in zip(calls, outs, spaces, streams):
            call(o, w, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))

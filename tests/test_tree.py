"""The operators of a step that checks drafted tokens without a GPU: layout of 4-bit weights, masks of trees, and every refusal
of the C calls and of their binding (decided on the host before any device work)."""
import pytest
import torch

from tests import tree_ref as ref


@pytest.fixture(scope="module")
def library():
    from paper_2602_03295_b200 import _build, binding
    _build.build()
    return binding.PopLibrary()


# ---------------------------------------------------------------------------------------- layout, masks
@pytest.mark.parametrize("n,k,group,zeros", [(1, 8, 32, False), (16, 128, 128, True), (37, 200, 32, True), (100, 1000, 64, False),
                                             (48, 392, 128, True)])
def test_tiles_hold_the_weights(n, k, group, zeros):
    from paper_2602_03295_b200 import pack_w4, unpack_w4
    g = torch.Generator().manual_seed(n + k)
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    scales = torch.rand(n, -(-k // group), generator=g).to(torch.bfloat16)
    z = torch.randint(0, 16, scales.shape, generator=g, dtype=torch.uint8) if zeros else None
    tiles = pack_w4(codes, scales, z, group)
    assert tiles[0].shape == (-(-n // 16), -(-k // 128), 16, 64) and tiles[1].shape == tiles[0].shape[:3] + (128 // group,)
    want = ref.w4_values(codes, scales, z, group)
    assert torch.equal(unpack_w4(*tiles, n, k).double(), want)
    for _ in range(40):                                             # the layout as the header states it
        r, i = int(torch.randint(n, (1,), generator=g)), int(torch.randint(k, (1,), generator=g))
        e, word = i % 8, 4 * (i % 32 // 8) + i % 128 // 32
        nibble = e // 2 + (4 if e % 2 else 0)
        byte = int(tiles[0][r // 16, i // 128, r % 16, 4 * word + nibble // 2])
        assert (byte >> (4 * (nibble % 2))) & 15 == int(codes[r, i])
        assert tiles[1][r // 16, i // 128, 2 * (r % 8) + r % 16 // 8, i % 128 // group] == scales[r, i // group]


def test_rounding_of_weights():
    from paper_2602_03295_b200 import quantize_w4, unpack_w4
    w = torch.randn(20, 96, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16)
    w[1] = 0
    for group in (32, 64, 128):
        back = unpack_w4(*quantize_w4(w, group), 20, 96)
        assert (back[1] == 0).all()
        blocks = torch.nn.functional.pad(w.float(), (0, -96 % group)).view(20, -1, group)
        scale = torch.where(blocks.abs().amax(-1) > 0, blocks.abs().amax(-1) / 7, 1.0).to(torch.bfloat16).float()
        code = torch.nn.functional.pad(back, (0, -96 % group)).view(20, -1, group) / scale[..., None]
        assert torch.equal(code.round(), code) and code.abs().max() <= 8
        assert ((code - blocks / scale[..., None]).abs() <= 0.5 + 7 * ref.BF16).all()


def test_masks_of_trees():
    from paper_2602_03295_b200 import PopError, tree_mask
    g = torch.Generator().manual_seed(4)
    rows = [70, 0, 1, 33]
    parents = [ref.random_tree(r, g) for r in rows]
    cu = [0, 70, 70, 71, 104]
    mask, depth = tree_mask(sum(parents, []), cu)
    assert mask.shape == (104, 3)
    for b, p in enumerate(parents):
        seen, d = ref.sees(p)
        if p:
            assert torch.equal(mask[cu[b]:cu[b + 1]], ref.pack_bits(seen, 3)) and torch.equal(depth[cu[b]:cu[b + 1]], d)
    for bad in ([0], [-1, 1], [-2], [-1, 0, 3]):
        with pytest.raises(PopError):
            tree_mask(bad)


# ---------------------------------------------------------------------------------------- the C calls' refusals
A = 1 << 20          # an aligned address that nothing dereferences
CALLS = {
    "pop_k_gemv_w4": dict(x=A, ldx=128, codes=A, scales=A, zeros=None, group=128, workspace=None, workspace_bytes=0, out=A, ldo=16,
                          B=2, N=16, K=128, mode=0, act=0, n_valid=0, stream=None),
    "pop_k_rope_cache_tree": dict(x=A, in_bf16=0, ld_in=192, rows=2, cu_rows=None, max_rows=2, start=None, pos0=0, depth=None,
                                  batch=1, q_out=A, ldq=64, k_pool=A, v_pool=A, block_table=A, page_size=16, num_pages=4,
                                  max_pages=4, q_gain=None, k_gain=None, eps=0.0, rope_table=A, table_rows=64, n_q=1, n_kv=1,
                                  head_dim=64, stream=None),
    "pop_k_tree_attention": dict(q=A, ldq=64, rows=2, cu_rows=None, max_rows=2, start=None, max_start=9, mask=None, mask_words=0,
                                 depth=None, k_pool=A, v_pool=A, block_table=A, page_size=16, num_pages=4, max_pages=4,
                                 workspace=A, workspace_bytes=64 << 20, out=A, ldo=64, batch=1, n_q=1, n_kv=1, head_dim=64,
                                 window=0, stream=None),
    "pop_k_cache_keep": dict(k_pool=A, v_pool=A, layer_stride=1024, layers=2, block_table=A, page_size=16, num_pages=4,
                             max_pages=4, kept=A, ld_kept=4, n_kept=None, max_kept=4, start=None, pos0=0, batch=2, n_kv=1,
                             head_dim=64, stream=None),
}
CACHE = [dict(k_pool=None), dict(v_pool=None), dict(block_table=None), dict(page_size=48), dict(page_size=0), dict(num_pages=0),
         dict(max_pages=0), dict(k_pool=A + 8), dict(v_pool=A + 4), dict(head_dim=80), dict(head_dim=0), dict(batch=0), dict(n_kv=0)]
REFUSED = {
    "pop_k_gemv_w4": [dict(x=None), dict(codes=None), dict(scales=None), dict(out=None), dict(B=0), dict(N=0), dict(K=0), dict(K=12),
                      dict(mode=1), dict(mode=4), dict(group=16), dict(group=96), dict(group=0), dict(x=A + 8), dict(ldx=132),
                      dict(ldx=120), dict(B=65536), dict(workspace=A + 8), dict(codes=A + 8), dict(scales=A + 4), dict(zeros=A + 4), dict(out=A + 2), dict(ldo=8),
                      dict(mode=3), dict(mode=3, N=256, ldo=128, n_valid=129), dict(mode=3, N=256, ldo=128, n_valid=-1),
                      dict(mode=3, N=256, ldo=128, n_valid=128, act=2)],
    "pop_k_rope_cache_tree": CACHE + [dict(x=None), dict(q_out=None), dict(rope_table=None), dict(x=A + 4), dict(ld_in=193),
                                      dict(q_out=A + 2), dict(ldq=66), dict(ldq=60), dict(table_rows=0), dict(pos0=-1),
                                      dict(max_rows=-1), dict(rows=-1), dict(rows=1), dict(batch=70000), dict(n_q=-1),
                                      dict(rope_table=A + 8), dict(max_rows=70000, rows=70000)],
    "pop_k_tree_attention": CACHE + [dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 2), dict(ldq=68), dict(ldo=60),
                                     dict(ldq=56), dict(ldo=56), dict(n_q=3, n_kv=2), dict(n_q=0), dict(n_q=129, ldq=9000, ldo=9000),
                                     dict(max_start=-1), dict(window=-1), dict(max_rows=-1), dict(rows=-1), dict(rows=1),
                                     dict(batch=4097, rows=1 << 20), dict(workspace=A + 4), dict(mask=A, mask_words=0),
                                     dict(batch=4096, rows=1 << 18, max_rows=64, n_q=512, n_kv=512, ldq=1 << 15, ldo=1 << 15,
                                          max_pages=1 << 20, max_start=1 << 23)],
    "pop_k_cache_keep": CACHE + [dict(kept=None), dict(layers=0), dict(layers=40000), dict(batch=70000), dict(max_kept=-1),
                                 dict(max_kept=1025, ld_kept=1025), dict(ld_kept=3), dict(pos0=-1), dict(layer_stride=1028),
                                 dict(num_pages=1 << 30)],
}
NOSPACE = [("pop_k_rope_cache_tree", dict(pos0=63)), ("pop_k_tree_attention", dict(max_start=63)),
           ("pop_k_tree_attention", dict(max_start=65, start=A)), ("pop_k_tree_attention", dict(workspace_bytes=1 << 20)),
           ("pop_k_tree_attention", dict(workspace=None)), ("pop_k_gemv_w4", dict(B=9, N=1 << 16, ldo=1 << 16, K=1024, ldx=1024)),
           ("pop_k_gemv_w4", dict(B=9, N=1 << 16, ldo=1 << 16, K=1024, ldx=1024, workspace=A, workspace_bytes=9000)),
           ("pop_k_gemv_w4", dict(B=8, K=4096, ldx=4096)), ("pop_k_cache_keep", dict(pos0=61))]
NOTHING = [("pop_k_rope_cache_tree", dict(max_rows=0)), ("pop_k_rope_cache_tree", dict(rows=0, cu_rows=A)),
           ("pop_k_tree_attention", dict(max_rows=0)), ("pop_k_tree_attention", dict(rows=0, cu_rows=A)),
           ("pop_k_cache_keep", dict(max_kept=0))]


@pytest.mark.parametrize("call,change", [(c, ch) for c in REFUSED for ch in REFUSED[c]])
def test_refused(library, call, change):
    from paper_2602_03295_b200 import POP_E_INVALID
    assert set(change) <= set(CALLS[call])
    assert getattr(library.dll, call)(*{**CALLS[call], **change}.values()) == POP_E_INVALID


@pytest.mark.parametrize("call,change", NOSPACE)
def test_no_space(library, call, change):
    from paper_2602_03295_b200 import POP_E_NOSPACE
    assert getattr(library.dll, call)(*{**CALLS[call], **change}.values()) == POP_E_NOSPACE


@pytest.mark.parametrize("call,change", NOTHING)
def test_nothing_to_do(library, call, change):
    assert getattr(library.dll, call)(*{**CALLS[call], **change}.values()) == 0


PACKED = ("pop_k_gemv_w4", "pop_k_rope_cache_tree", "pop_k_tree_attention", "pop_k_cache_keep")


@pytest.mark.parametrize("call,change", [(c, ch) for c in REFUSED for ch in REFUSED[c]] + NOSPACE + NOTHING)
def test_packed_words_are_the_same_call(library, call, change):
    import struct
    args = {**CALLS[call], **change}
    words = struct.pack("=" + "".join("d" if n == "eps" else "q" for n in args), *[0 if v is None else v for v in args.values()])
    assert library.dll.pop_k_packed(PACKED.index(call), words) == getattr(library.dll, call)(*args.values())


def test_packed_words_outside_their_type(library):
    import struct
    from paper_2602_03295_b200 import POP_E_INVALID
    for n, call in enumerate(PACKED):
        args = CALLS[call]
        for name in ("rows", "batch", "n_q", "n_kv", "head_dim", "B", "N", "K", "group", "mode", "max_rows", "page_size"):
            if name in args:
                big = {**args, name: args[name] + (1 << 32)}            # the right value in its low half
                words = struct.pack("=" + "".join("d" if k == "eps" else "q" for k in big), *[0 if v is None else v for v in big.values()])
                assert library.dll.pop_k_packed(n, words) == POP_E_INVALID, (call, name)
    assert library.dll.pop_k_packed(4, words) == POP_E_INVALID and library.dll.pop_k_packed(0, None) == POP_E_INVALID


def test_binding_wants_the_current_device(library):
    from paper_2602_03295_b200 import PopError
    x = torch.zeros(2, 128, dtype=torch.bfloat16)
    k = torch.zeros(4, 16, 1, 64, dtype=torch.bfloat16)
    t = torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(PopError):
        library.gemv_w4(x, torch.zeros(1, 1, 16, 64, dtype=torch.uint8), torch.zeros(1, 1, 16, 1, dtype=torch.bfloat16), None,
                        torch.zeros(2, 16), 16, 128)
    with pytest.raises(PopError):
        library.rope_cache_tree(torch.zeros(2, 192), x[:, :64], k, k, t, torch.zeros(64, 32, 2), 1, 1, 64, 2)
    with pytest.raises(PopError):
        library.tree_attention(x[:, :64], k, k, t, x[:, :64], 1, 1, 64, 2, 9)
    with pytest.raises(PopError):
        library.cache_keep(k[None], k[None], t, t)


def test_pack_refuses_what_does_not_belong_together():
    from paper_2602_03295_b200 import PopError, pack_w4
    codes, scales = torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 2)
    pack_w4(codes, scales, None, 32)
    for bad in ((codes, scales, None, 64), (codes, scales, None, 16), (codes, scales, torch.zeros(8, 1), 32), (codes, scales[:7], None, 32)):
        with pytest.raises(PopError):
            pack_w4(*bad)

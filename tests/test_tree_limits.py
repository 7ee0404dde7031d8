"""Refusals of the calls that check drafted tokens which need no GPU, beside those of tests/test_tree.py."""
import pytest
import torch


@pytest.fixture(scope="module")
def library():
    from paper_2602_03295_b200 import _build, binding
    _build.build()
    return binding.PopLibrary()


class Recorder:
    """Stands for the library: takes every call, and does nothing."""

    def __init__(self):
        self.calls = 0

    def pop_k_gemv_w4_workspace_bytes(self, *args):
        return 1 << 16

    def pop_k_packed(self, *args):
        self.calls += 1
        return 0


@pytest.fixture
def recorded(monkeypatch):
    """A binding on tensors of the CPU whose calls reach a recorder instead of the library."""
    from paper_2602_03295_b200 import binding
    monkeypatch.setattr(binding.PopLibrary, "_here", staticmethod(lambda t, others, what: 0))
    lib = object.__new__(binding.PopLibrary)
    lib.dll = Recorder()
    return lib


def test_workspaces_with_gaps_are_refused(recorded):
    """The products write their workspace as one piece: views with gaps, and one element expanded, are none."""
    from paper_2602_03295_b200 import PopError
    x, out = torch.zeros(9, 256, dtype=torch.bfloat16), torch.zeros(9, 16)
    tiles = torch.zeros(1, 2, 16, 64, dtype=torch.uint8), torch.zeros(1, 2, 16, 1, dtype=torch.bfloat16), None
    recorded.gemv_w4(x, *tiles, out, 16, 128, workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    recorded.gemv_w4(x, *tiles, out, 16, 128, workspace=torch.zeros(1 << 8, 1 << 6))
    assert recorded.dll.calls == 2
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(1 << 16), torch.zeros(1 << 17, dtype=torch.uint8)[::2],
                torch.zeros(1 << 8, 1 << 9, dtype=torch.uint8)[:, :1 << 8]):
        with pytest.raises(PopError):
            recorded.gemv_w4(x, *tiles, out, 16, 128, workspace=bad)
    assert recorded.dll.calls == 2


def test_layers_that_lie_over_each_other_are_refused(library):
    """Layers are moved at the same time: with less than a page between two of them a page would be moved twice. A page apart is
    enough, as in pools that interleave the pages of the layers."""
    from paper_2602_03295_b200 import POP_E_INVALID
    from tests.test_tree import CALLS
    name = "pop_k_cache_keep"
    page = CALLS[name]["page_size"] * CALLS[name]["n_kv"] * CALLS[name]["head_dim"]
    keep = lambda **change: getattr(library.dll, name)(*{**CALLS[name], **change}.values())  # noqa: E731
    for stride in (0, 8, page - 8, -8, 8 - page):
        assert keep(layer_stride=stride) == POP_E_INVALID
        assert keep(layer_stride=stride, layers=1, max_kept=0) == 0
    for stride in (page, -page, 1 << 40, -(1 << 63)):
        assert keep(layer_stride=stride, max_kept=0) == 0


def test_masks_and_vectors_off_their_words_are_refused(library):
    """Arrays of 32-bit words are read as such: an address between two of them is no address of one."""
    from paper_2602_03295_b200 import POP_E_INVALID
    from tests.test_tree import A, CALLS
    arrays = {"pop_k_rope_cache_tree": ("cu_rows", "start", "depth", "block_table", "q_gain", "k_gain"),
              "pop_k_tree_attention": ("cu_rows", "start", "depth", "block_table", "mask"),
              "pop_k_cache_keep": ("kept", "n_kept", "start", "block_table")}
    for call, names in arrays.items():
        for name in names:
            for off in (1, 2, 3):
                args = {**CALLS[call], name: A + off}
                if name == "mask":
                    args["mask_words"] = 1
                assert getattr(library.dll, call)(*args.values()) == POP_E_INVALID, (call, name, off)


def test_prefix_sums_of_trees_that_leave_the_rows_are_refused():
    """Sequences lie one behind the other within the rows; rows of no sequence see nothing."""
    from paper_2602_03295_b200 import PopError, tree_mask
    mask, depth = tree_mask([-1, -1, 0, -1], [1, 1, 3])
    assert mask.tolist() == [[0], [1], [3], [0]] and depth.tolist() == [0, 0, 1, 0]
    for cu in ([0, 5], [-1, 3], [0, 3, 2], [2, 0], [0, 2, 9]):
        with pytest.raises(PopError):
            tree_mask([-1, -1, 0, -1], cu)

"""The 8-bit paged cache without a GPU: the scale's bit arithmetic, and every refusal of the C calls and of their binding
(decided on the host before any device work)."""
import math

import pytest
import torch

from tests import cache8_ref as ref


@pytest.fixture(scope="module")
def library():
    from paper_2602_03295_b200 import _build, binding
    _build.build()
    return binding.PopLibrary()


def _bits_rule(amax):
    """csrc/cache8.cuh: c8_scale_exp on the fp32 bits."""
    b = int(torch.tensor(amax, dtype=torch.float32).view(torch.int32))
    e = ((b + 0x1fffff) >> 23) - 8
    return e if 63 < e < 247 else 63 if e <= 63 else 247


def test_scale_rule_is_the_smallest_power_of_two():
    g = torch.Generator().manual_seed(1)
    values = [0.0, 1e-38, 448.0, 448.0 * 2 ** -64, 3.3e38, math.inf, 1e-45]
    for k in range(-60, 100, 7):
        edge = torch.tensor(448.0 * 2.0 ** k, dtype=torch.float32)
        values += [float(edge), float(torch.nextafter(edge, torch.tensor(0.0))), float(torch.nextafter(edge, torch.tensor(math.inf)))]
    values += (torch.randn(200, generator=g).abs() * 10 ** (torch.rand(200, generator=g) * 20 - 10)).tolist()
    for v in values:
        v = float(torch.tensor(v, dtype=torch.float32))
        assert _bits_rule(v) == ref.scale_exp(v), v


def test_reference_rounding_is_torchs_cast():
    x = torch.randn(20000, generator=torch.Generator().manual_seed(2)) * 60
    x = torch.cat([x, x * 1e-3, torch.tensor([0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -11])]).clamp(-448, 448)
    assert torch.equal(ref.round_e4m3(x.double()), x.to(torch.float8_e4m3fn).double())
    every = torch.arange(256, dtype=torch.uint8)
    assert torch.equal(ref.code_values(every).nan_to_num(7e9), every.view(torch.float8_e4m3fn).double().nan_to_num(7e9))


# ---------------------------------------------------------------------------------------- the C calls' refusals
A = 1 << 20          # an aligned address that nothing dereferences

QUANT = dict(k_pool=A, v_pool=A, src_layer_stride=8, src_table=A, src_page_size=16, src_num_pages=4, src_max_pages=4,
             k_codes=A, v_codes=A, k_scales=A, v_scales=A, code_layer_stride=16, scale_layer_stride=1, block_table=A,
             page_size=16, num_pages=4, max_pages=4, seq_lens=None, max_len=64, layers=1, batch=1, n_kv=1, head_dim=64,
             stream=None)
APPEND = dict(x=A, in_bf16=0, ld_in=192, cu_rows=None, max_rows=1, start=None, pos0=0, batch=1, q_out=A, ldq=64, k_codes=A,
              v_codes=A, k_scales=A, v_scales=A, block_table=A, page_size=16, num_pages=4, max_pages=4, q_gain=None,
              k_gain=None, eps=0.0, rope_table=A, table_rows=64, positions=None, ld_pos=0, pair_axis=None, n_axes=0, n_q=1,
              n_kv=1, head_dim=64, stream=None)
DECODE = dict(q=A, ldq=64, k_codes=A, v_codes=A, k_scales=A, v_scales=A, block_table=A, page_size=16, num_pages=4,
              max_pages=400, seq_lens=None, kv_len=64, workspace=A, workspace_bytes=64 << 20, out=A, ldo=64, batch=1, n_q=1,
              n_kv=1, head_dim=64, window=0, stream=None)
PROMPT = dict(q=A, ldq=64, cu_rows=None, max_rows=1, k_codes=A, v_codes=A, k_scales=A, v_scales=A, block_table=A,
              page_size=16, num_pages=4, max_pages=400, seq_lens=None, kv_len=64, workspace=A, workspace_bytes=64 << 20,
              out=A, ldo=64, batch=1, n_q=1, n_kv=1, head_dim=64, window=0, stream=None)
CACHE = [dict(k_codes=None), dict(v_codes=None), dict(k_scales=None), dict(v_scales=None), dict(block_table=None),
         dict(page_size=48), dict(page_size=8), dict(page_size=0), dict(num_pages=0), dict(max_pages=0),
         dict(k_codes=A + 8), dict(v_codes=A + 4), dict(head_dim=80), dict(head_dim=0), dict(batch=0), dict(n_kv=0)]
REFUSED = {
    "quant": CACHE + [dict(k_pool=None), dict(v_pool=None), dict(src_table=None), dict(src_page_size=24),
                      dict(src_num_pages=0), dict(max_len=-1), dict(layers=0), dict(batch=70000), dict(k_pool=A + 2),
                      dict(src_layer_stride=4), dict(code_layer_stride=8)],
    "append": CACHE + [dict(x=None), dict(q_out=None), dict(rope_table=None), dict(x=A + 4), dict(ld_in=193),
                       dict(q_out=A + 2), dict(ldq=66), dict(table_rows=0), dict(pos0=-1), dict(max_rows=-1),
                       dict(positions=A), dict(pair_axis=A), dict(positions=A, pair_axis=A, n_axes=300), dict(positions=A, pair_axis=A + 2, n_axes=3), dict(n_q=-1),
                       dict(batch=70000), dict(batch=60000, max_rows=60000)],
    "decode": CACHE + [dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 2), dict(ldq=65), dict(ldo=68),
                       dict(n_q=3, n_kv=2), dict(n_q=0), dict(kv_len=-1), dict(window=-1), dict(batch=4097),
                       dict(workspace=A + 4)],
    "prompt": CACHE + [dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 2), dict(ldq=65), dict(ldo=68),
                       dict(n_q=3, n_kv=2), dict(n_q=0), dict(kv_len=-1), dict(window=-1), dict(max_rows=-1),
                       dict(max_rows=65), dict(batch=70000), dict(workspace=A + 4)],
}
NOSPACE = {
    "quant": [dict(max_len=65), dict(max_len=65, max_pages=5)],
    "append": [dict(pos0=64), dict(pos0=60, max_rows=5)],
    "decode": [dict(kv_len=6401), dict(kv_len=64000, max_pages=4000, workspace_bytes=1000),
               dict(kv_len=64000, max_pages=4000, workspace=None)],
    "prompt": [dict(kv_len=6401), dict(kv_len=64000, max_pages=4000, workspace_bytes=1000),
               dict(kv_len=64000, max_pages=4000, workspace=None), dict(kv_len=6400, max_rows=64, workspace_bytes=1000),
               dict(kv_len=6400, max_rows=64, workspace=None)],
}
CALLS = {"quant": ("pop_k_quant_cache_e4m3", QUANT), "append": ("pop_k_rope_cache_e4m3", APPEND),
         "decode": ("pop_k_decode_attention_e4m3", DECODE), "prompt": ("pop_k_attention_e4m3", PROMPT)}


@pytest.mark.parametrize("op,change", [(op, c) for op in CALLS for c in REFUSED[op]], ids=lambda v: str(v))
def test_c_call_refuses(library, op, change):
    from paper_2602_03295_b200 import POP_E_INVALID
    name, args = CALLS[op]
    assert set(change) <= set(args)
    assert getattr(library.dll, name)(*{**args, **change}.values()) == POP_E_INVALID


@pytest.mark.parametrize("op,change", [(op, c) for op in CALLS for c in NOSPACE[op]], ids=lambda v: str(v))
def test_c_call_says_that_space_is_short(library, op, change):
    from paper_2602_03295_b200 import POP_E_NOSPACE
    name, args = CALLS[op]
    assert getattr(library.dll, name)(*{**args, **change}.values()) == POP_E_NOSPACE


def test_workspace_constant_is_the_headers():
    import os
    import re
    from paper_2602_03295_b200 import binding
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pop_kernels.h")).read()
    m = re.search(r"POP_E4M3_WORKSPACE_BYTES \((\d+) \* (\d+) \* (\d+)\)", text)
    assert binding.POP_E4M3_WORKSPACE_BYTES == int(m[1]) * int(m[2]) * int(m[3])


def test_binding_refuses_tensors_that_are_not_on_the_device(library):
    from paper_2602_03295_b200 import POP_E_INVALID, PopError
    c = torch.zeros(2, 1, 16, 64, dtype=torch.uint8)
    s = torch.zeros(2, 1, 1, dtype=torch.uint8)
    bt = torch.zeros(1, 2, dtype=torch.int32)
    q = torch.zeros(1, 64, dtype=torch.bfloat16)
    with pytest.raises(PopError) as e:
        library.decode_attention_e4m3(q, c, c, s, s, bt, q.clone(), 1, 1, 64, 16)
    assert e.value.code == POP_E_INVALID


@pytest.mark.parametrize("op", ["decode", "prompt"])
def test_lengths_and_windows_behind_the_largest_are_refused(library, op):
    from paper_2602_03295_b200 import POP_E_INVALID
    name, args = CALLS[op]
    for change in (dict(kv_len=0x7fff0001), dict(window=0x7ffffff1)):
        assert getattr(library.dll, name)(*{**args, "max_pages": 1 << 28, **change}.values()) == POP_E_INVALID


def test_output_rows_over_each_other_are_refused(library):
    from paper_2602_03295_b200 import POP_E_INVALID
    dll = library.dll
    assert dll.pop_k_decode_attention_e4m3(*{**DECODE, "batch": 2, "ldo": 56}.values()) == POP_E_INVALID
    assert dll.pop_k_attention_e4m3(*{**PROMPT, "max_rows": 2, "ldo": 0}.values()) == POP_E_INVALID
    assert dll.pop_k_rope_cache_e4m3(*{**APPEND, "max_rows": 2, "ldq": 60}.values()) == POP_E_INVALID


def test_fill_from_takes_a_length_of_zero_for_what_it_is():
    from types import SimpleNamespace
    from paper_2602_03295_b200.binding import KVCache, KVCacheE4M3
    cfg = SimpleNamespace(n_layers=1, n_kv_heads=1, head_dim=64)
    a, c, asked = KVCache(cfg, 1, 40, 16, device="cpu"), KVCacheE4M3(cfg, 1, 32, 16, device="cpu"), []
    fake = SimpleNamespace(quant_cache_e4m3=lambda *args, **kw: asked.append(args[8]))
    for n in (0, 7, None):
        c.fill_from(a, n, library=fake)
    assert asked == [0, 7, 32]
    assert [t.shape[1] for t in c.gather(0, 0)] == [0, 0] and [t.shape[1] for t in c.gather(0)] == [32, 32]


def test_conversion_of_lengths_behind_the_largest_is_refused(library):
    """As those of the attention calls: a block number times 16 has to stay a 32-bit position in every thread of the grid."""
    from paper_2602_03295_b200 import POP_E_INVALID
    big = {**QUANT, "max_pages": 1 << 28, "src_max_pages": 1 << 28}
    for n in (0x7fff0001, 0x7fffff81, 0x7fffffff):
        assert library.dll.pop_k_quant_cache_e4m3(*{**big, "max_len": n}.values()) == POP_E_INVALID


def test_the_count_of_sms_is_asked_for_once_by_all_threads(tmp_path):
    """The host code under ThreadSanitizer: two threads whose first calls come at the same time."""
    import os
    import subprocess
    from paper_2602_03295_b200 import _build
    (tmp_path / "main.cu").write_text("""
#include <thread>
namespace pop { int device_sms(); }
int main() {
  int a = 0, b = 0;
  std::thread x([&] { a = pop::device_sms(); }), y([&] { b = pop::device_sms(); });
  x.join();
  y.join();
  return a == b && a > 0 ? 0 : 1;
}
""")
    flags = [os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17",
             "-Xcompiler", "-fsanitize=thread"]
    files = [tmp_path / "main.cu"] + [_build.CSRC + "/" + n for n in ("cache8.cu", "runtime.cu")]
    subprocess.run(flags + ["-o", str(tmp_path / "race")] + [str(f) for f in files], check=True, capture_output=True, text=True)
    got = subprocess.run([str(tmp_path / "race")], capture_output=True, text=True, timeout=120)
    if "unexpected memory mapping" in got.stderr:
        pytest.skip("ThreadSanitizer cannot place its memory under this kernel's address randomisation")
    assert got.returncode == 0, got.stderr[-3000:]


def test_limits_that_the_header_states(library):
    """Refused one behind the limit; at the limit the call is taken, as far as a machine without a GPU takes it."""
    from paper_2602_03295_b200 import POP_E_INVALID
    call = lambda op, **change: getattr(library.dll, CALLS[op][0])(*{**CALLS[op][1], "max_pages": 1 << 20, **change}.values())  # noqa: E731
    for hd, n_q, most in ((64, 128, 131070), (128, 200, 131070), (256, 128, 65535), (64, 60, 262140), (256, 1, 8388480)):
        for n in (most, most + 1):
            got = call("prompt", head_dim=hd, n_q=n_q, ldq=n_q * hd, ldo=n_q * hd, max_rows=n, kv_len=n)
            assert (got == POP_E_INVALID) == (n > most), (hd, n_q, n, got)
    for op in ("decode", "prompt"):
        for batch, refused in ((15, False), (16, True), (17, True)):          # times 2^27 blocks
            got = call(op, batch=batch, kv_len=0x7fff0000, max_pages=1 << 28)
            assert (got == POP_E_INVALID) == refused, (op, batch, got)
    for pages in ((1 << 27) - 1, 1 << 27):                                    # of 16 positions
        assert (call("prompt", num_pages=pages, max_rows=40) == POP_E_INVALID) == (pages >= 1 << 27)

"""Pins of the reference definitions in oracle/generation.py by small hand-worked cases and invariants, and the argument checks
of the calls they define (no GPU)."""
import ctypes
import math
import os

import pytest
import torch

from oracle import generation as G
from test_library_host import _header_struct_fields


@pytest.fixture(scope="module")
def binding():
    from paper_2603_06588_amd import binding as b, build
    if build.lib_is_stale():
        build.build_lib()
    return b


# ---- rotary positions ---------------------------------------------------------------------------------------

def test_axes_of_pairs():
    assert G.rope_axes([2, 1, 1], cyclic=False) == [0, 0, 1, 2]
    assert G.rope_axes([4, 2, 2], cyclic=True) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert G.rope_axes([3], cyclic=True) == [0, 0, 0]


def test_quarter_turns():
    # pair 0 by a quarter turn, pair 1 by half of one
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    f = torch.tensor([math.pi / 2, math.pi], dtype=torch.float64)
    y = G.rope(x, torch.tensor([1]), f)
    assert torch.allclose(y, torch.tensor([[[-3.0, -2.0, 1.0, -4.0, 9.0]]]).double(), atol=1e-12)
    y = G.rope(x, torch.tensor([1]), f, neighbours=True)
    assert torch.allclose(y, torch.tensor([[[-2.0, 1.0, -3.0, -4.0, 9.0]]]).double(), atol=1e-12)


@pytest.mark.parametrize("neighbours", [False, True])
def test_scores_depend_on_distance_alone_and_inverse_undoes(neighbours):
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn((1, 1, 16), generator=g).double(), torch.randn((1, 1, 16), generator=g).double()
    f = 100.0 ** (-torch.arange(8, dtype=torch.float64) / 8)
    score = lambda a, b: float((G.rope(q, torch.tensor([a]), f, neighbours=neighbours) * G.rope(k, torch.tensor([b]), f, neighbours=neighbours)).sum())  # noqa: E731
    assert abs(score(7, 3) - score(1007, 1003)) < 1e-9
    pos = torch.tensor([[5], [9]])
    y = G.rope(q, pos, f, [5, 3], neighbours, True)
    assert torch.allclose(G.rope(y, pos, f, [5, 3], neighbours, True, inverse=True), q, atol=1e-12)


def test_inverse_is_the_gradient_against_differences():
    # d/dx <w, rope(x)> = rope_inverse(w)
    g = torch.Generator().manual_seed(4)
    x, w = torch.randn((2, 1, 6), generator=g).double(), torch.randn((2, 1, 6), generator=g).double()
    f, pos = torch.tensor([1.0, 0.3], dtype=torch.float64), torch.tensor([3, -4])
    want = G.rope(w, pos, f, inverse=True)
    for i in range(x.numel()):
        h = torch.zeros_like(x)
        h.view(-1)[i] = 1e-5
        slope = ((G.rope(x + h, pos, f) - G.rope(x - h, pos, f)) * w).sum() / 2e-5
        assert abs(float(slope) - float(want.reshape(-1)[i])) < 1e-9


# ---- pages --------------------------------------------------------------------------------------------------

def test_fork_shares_cuts_and_frees():
    table = [[3, 1, 0], [2, 5, 0]]
    rows, lens, refs, status = G.fork([0, 0, -1, 0], table, [20, 32], [0, 1, 1, 1, 0, 1], src_lens=[99, 16, 5, 0])
    assert rows == [[3, 1], [3], [], []] and lens == [20, 16, 0, 0] and status == 0
    assert refs == [0, 1, 0, 2, 0, 0]       # row 1's pages 2 and 5 are free, page 3 has two holders


def test_append_copies_until_one_holder_is_left():
    # three rows share page 4 (8 tokens); a fourth holder keeps it in the second case
    table = [[4, 9, 9]] * 3
    rows, lens, refs, copies, status = G.append([0, 1, 2, 3], table, [8, 8, 8], [0, 0, 1, 0, 3])
    assert copies == [(4, 0, 8), (4, 1, 8)] and rows == [[0], [1], [4]] and lens == [9, 9, 9] and refs == [1, 1, 1, 0, 1] and status == 0
    rows, lens, refs, copies, status = G.append([0, 1, 2, 3], table, [8, 8, 8], [0, 0, 1, 0, 4])
    assert rows == [[0], [1], [3]] and refs == [1, 1, 1, 1, 1] and len(copies) == 3
    # no room for the third copy: nothing happens
    rows, lens, refs, copies, status = G.append([0, 1, 2, 3], table, [8, 8, 8], [0, 0, 1, 1, 4])
    assert rows == [[4]] * 3 and lens == [8, 8, 8] and refs == [0, 0, 1, 1, 4] and copies == [] and status == G.FULL
    # a full last page is not copied; new pages follow in order
    rows, lens, refs, copies, status = G.append([0, 17, 17], [[2, 0, 0], [2, 0, 0]], [16, 16], [0, 0, 2, 0])
    assert rows == [[2, 0, 1], [2]] and lens == [33, 16] and copies == [] and refs == [1, 1, 2, 0]
    # a row longer than the table
    assert G.append([0, 17], [[2, 0]], [16], [0, 0, 2, 0])[4] == G.FULL


def test_compact_moves_the_lowest_to_the_lowest():
    rows, refs, page_map, live, moves, status = G.compact([[5, 2], [7, 9]], [32, 10], [0, 0, 1, 0, 0, 2, 0, 1])
    assert live == 3 and moves == [(5, 0), (7, 1)] and page_map == [-1, -1, 2, -1, -1, 0, -1, 1]
    assert rows == [[0, 2], [1]] and refs == [2, 1, 1, 0, 0, 0, 0, 0] and status == 0


# ---- logits -------------------------------------------------------------------------------------------------

def test_logits_by_hand():
    x = torch.tensor([[2.0, -2.0, 1.0, 0.5]])
    y = G.steer_logits(x, [[0, 1, 1, 7, -1]], [1], [2.0], [0.25], [0.5], [[(2, 1.0), (2, 3.0), (9, 1.0)]], torch.tensor([[0b0111]], dtype=torch.int32))
    # 0 is in the prompt alone; 1 was generated twice; of 2's two entries the last counts; 3 is barred
    assert y.tolist() == [[1.0, -4.0 - 0.5 - 0.5, 4.0, -math.inf]]
    assert G.steer_logits(x, mask=torch.zeros((1, 1), dtype=torch.int32)).tolist() == [[-math.inf] * 4]
    assert torch.equal(G.steer_logits(x, mask=torch.zeros((1, 1), dtype=torch.int32), mask_rows=[-1]), x.double())


# ---- argument checks of the library (nothing is launched) ---------------------------------------------------

P = 4096      # a pointer that is never followed


def _rope(binding, **kw):
    a = binding.HookRopeArgs()
    base = dict(num_tokens=4, num_q_heads=8, num_kv_heads=2, head_dim=128, rotary_dim=128, num_axes=1, positions=P, inv_freq=P, q=P, k=P)
    pairs = kw.pop("axis_pairs", (64,))
    for i, n in enumerate(pairs):
        a.axis_pairs[i] = n
    for key, v in {**base, **kw}.items():
        setattr(a, key, v)
    return binding.load_library().hook_rope(ctypes.byref(a))


def test_structs_match_the_header(binding):
    for struct, cls in (("hook_rope_args", binding.HookRopeArgs), ("hook_pages_args", binding.HookPagesArgs),
                        ("hook_steer_logits_args", binding.HookSteerLogitsArgs)):
        names = [n.split("[")[0].replace("const*", "").strip(" *") for n in _header_struct_fields(struct)]
        assert names == [f[0] for f in cls._fields_]


def test_struct_layouts_match_the_header(binding, tmp_path):
    """Sizes and offsets as a C compiler sees them."""
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pairs = [("hook_rope_args", binding.HookRopeArgs), ("hook_pages_args", binding.HookPagesArgs), ("hook_steer_logits_args", binding.HookSteerLogitsArgs)]
    lines, want = [], []
    for name, cls in pairs:
        for f in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f[0]}));')
            want.append(getattr(cls, f[0]).offset)
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
    src = tmp_path / "layout.c"
    src.write_text('#include "hook_api.h"\n#include <stdio.h>\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", exe], check=True)
    assert [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()] == want


def test_rope_refusals(binding):
    lib = binding.load_library()
    assert lib.hook_rope(None) == 1
    assert _rope(binding) == 1                                                     # no outputs
    assert _rope(binding, q_out=P) == 1                                            # none for k
    assert _rope(binding, q_out=P, k_out=P, positions=0) == 1
    assert _rope(binding, q_out=P, k_out=P, inv_freq=0) == 1
    assert _rope(binding, num_tokens=-1) == 2
    assert _rope(binding, rotary_dim=130) == 2
    assert _rope(binding, rotary_dim=127) == 3
    assert _rope(binding, head_dim=514) == 3
    assert _rope(binding, dtype=2) == 3
    assert _rope(binding, layout=2) == 2 and _rope(binding, axis_order=-1) == 2
    assert _rope(binding, num_axes=0) == 2 and _rope(binding, num_axes=5) == 2
    assert _rope(binding, axis_pairs=(63,)) == 2                                   # the pairs do not add up
    assert _rope(binding, num_axes=2, axis_pairs=(65, -1)) == 2
    assert _rope(binding, num_axes=2, axis_pairs=(31, 33), axis_order=1) == 2      # the second axis runs out of pairs
    assert _rope(binding, q_out=P, k_out=P, q_stride=100) == 2                     # rows on top of each other
    assert _rope(binding, q_out=P, k_out=2 * P, q_stride=1024, q_out_stride=2048) == 2      # its own input at another stride
    assert _rope(binding, q_out=2 * P, k_out=P, q_stride=1 << 41) == 3
    assert _rope(binding, q=P + 1, q_out=P, k_out=P) == 3                          # not aligned to an element
    cache = dict(q_out=P, k_cache=P, v_cache=P, v=P, num_seqs=1, block_size=16, max_blocks_per_seq=4, num_blocks=4, block_table=P, seq_lens=P,
                 cu_q_lens=P)
    for missing in ("v", "k", "k_cache", "v_cache", "block_table", "seq_lens", "cu_q_lens"):
        assert _rope(binding, **{**cache, missing: 0}) == 1, missing
    assert _rope(binding, **{**cache, "block_size": 32}) == 3
    assert _rope(binding, **{**cache, "num_blocks": 0}) == 2
    assert _rope(binding, **{**cache, "num_seqs": 0}) == 2
    assert _rope(binding, **{**cache, "kv_dtype": 2}) == 2
    assert _rope(binding, **{**cache, "kv_dtype": 1}) == 1                         # no scales
    assert _rope(binding, **{**cache, "kv_dtype": 1, "dtype": 1}) == 3
    assert _rope(binding, num_tokens=0) == 0                                       # nothing to do
    assert _rope(binding, q=0, k=0) == 0


def _pages(binding, **kw):
    a = binding.HookPagesArgs()
    base = dict(num_seqs=2, max_blocks_per_seq=4, num_blocks=8, block_size=16, block_table=P, seq_lens=2 * P, ref_counts=3 * P, block_table_out=4 * P,
                seq_lens_out=5 * P, ref_counts_out=3 * P, status=6 * P, num_rows=2, src_rows=7 * P, cu_q_lens=8 * P, page_map=9 * P,
                num_live=10 * P, workspace=16 * P, workspace_bytes=1 << 20)
    caches = kw.pop("cache_list", None)
    for key, v in {**base, **kw}.items():
        setattr(a, key, v)
    if caches is not None:
        a.num_caches, a.caches = len(caches), (ctypes.c_void_p * len(caches))(*caches)
    return a


def test_pages_refusals(binding):
    lib = binding.load_library()
    calls = (lib.hook_pages_fork, lib.hook_pages_append, lib.hook_pages_compact)
    for call in calls:
        assert call(None) == 1
        assert call(_pages(binding, num_seqs=-1)) == 2
        assert call(_pages(binding, num_blocks=0)) == 2
        assert call(_pages(binding, max_blocks_per_seq=0)) == 2
        assert call(_pages(binding, block_size=32)) == 3
        assert call(_pages(binding, max_blocks_per_seq=(1 << 26) + 1)) == 3
        for missing in ("block_table", "seq_lens", "ref_counts", "block_table_out", "ref_counts_out", "status"):
            assert call(_pages(binding, **{missing: 0})) == 1, missing
        assert call(_pages(binding, ref_counts_out=3 * P + 4)) == 2               # partly the input
    fork, append, compact = calls
    assert fork(_pages(binding, num_rows=-1)) == 2
    assert fork(_pages(binding, src_rows=0)) == 1 and fork(_pages(binding, seq_lens_out=0)) == 1
    assert fork(_pages(binding, block_table_out=P)) == 2 and fork(_pages(binding, seq_lens_out=2 * P + 4)) == 2      # in place
    assert fork(_pages(binding, num_seqs=0, num_rows=0)) == 0                     # nothing to do
    assert append(_pages(binding, cu_q_lens=0)) == 1
    assert append(_pages(binding, block_table_out=P + 16)) == 2
    assert compact(_pages(binding, page_map=0)) == 1 and compact(_pages(binding, num_live=0)) == 1
    need = lib.hook_pages_workspace_bytes(_pages(binding))
    assert need > 0 and need % 16 == 0 and lib.hook_pages_workspace_bytes(None) == 0
    for call in (append, compact):
        assert call(_pages(binding, workspace=0)) == 4
        assert call(_pages(binding, workspace=16 * P + 8)) == 4
        assert call(_pages(binding, workspace_bytes=need - 1)) == 4
        geometry = dict(num_kv_heads=2, row_bytes=256)
        assert call(_pages(binding, num_caches=-1)) == 2
        assert call(_pages(binding, cache_list=[P], num_kv_heads=0, row_bytes=256)) == 2
        assert call(_pages(binding, cache_list=[P], num_kv_heads=2, row_bytes=72)) == 3
        assert call(_pages(binding, cache_list=[0], **geometry)) == 1
        assert call(_pages(binding, cache_list=[P + 8], **geometry)) == 3
        assert call(_pages(binding, cache_list=[P] * 257, **geometry)) == 3
        assert call(_pages(binding, num_caches=1, **geometry)) == 1               # no list


def _logits(binding, **kw):
    a = binding.HookSteerLogitsArgs()
    for key, v in {**dict(num_rows=2, vocab=100, logits=P, out=P), **kw}.items():
        setattr(a, key, v)
    return binding.load_library().hook_steer_logits(ctypes.byref(a))


def test_logits_refusals(binding):
    assert binding.load_library().hook_steer_logits(None) == 1
    assert _logits(binding, num_rows=-1) == 2 and _logits(binding, vocab=-1) == 2 and _logits(binding, history_len=-1) == 2
    assert _logits(binding, dtype=3) == 3
    assert _logits(binding, vocab=1 << 29, num_rows=1 << 20) == 3
    assert _logits(binding, logits_stride=99) == 2 and _logits(binding, out_stride=99) == 2
    assert _logits(binding, logits_stride=104) == 2                               # its own input at another stride
    assert _logits(binding, logits_stride=1 << 41, out=2 * P) == 3
    assert _logits(binding, history_len=(1 << 30) + 1, history=P, cu_history=P) == 3
    assert _logits(binding, bias_len=(1 << 30) + 1, cu_bias=P, bias_ids=P, bias_values=P) == 3
    assert _logits(binding, logits=0) == 1 and _logits(binding, out=0) == 1
    assert _logits(binding, history_len=5, history=P) == 1 and _logits(binding, history_len=5, cu_history=P) == 1
    assert _logits(binding, bias_len=5, cu_bias=P, bias_ids=P) == 1
    assert _logits(binding, logits=P + 1, out=2 * P) == 3                         # not aligned to an element
    assert _logits(binding, num_rows=0) == 0 and _logits(binding, vocab=0, logits=0) == 0


def test_binding_refuses_what_it_can_see(binding):
    """Tensors in host memory, before anything else happens to them."""
    x, i = torch.zeros((2, 1, 4)), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(binding.HookError):
        binding.hook_rope(x, None, i, torch.ones(2))
    with pytest.raises(binding.HookError):
        binding.hook_rope(None, None, i, torch.ones(2))
    with pytest.raises(binding.HookError):
        binding.hook_pages_fork(i, i.view(1, 2), i[:1], i, i.view(2, 1), i, i[:1])
    with pytest.raises(binding.HookError):
        binding.hook_steer_logits(torch.zeros((2, 8)))


def test_fork_of_no_rows_still_needs_both_counts(binding):
    fork = binding.load_library().hook_pages_fork
    none = dict(num_seqs=0, num_rows=0)
    assert fork(_pages(binding, **none, ref_counts_out=0)) == 1 and fork(_pages(binding, **none, ref_counts=0)) == 1
    assert fork(_pages(binding, **none, ref_counts=0, ref_counts_out=0)) == 0     # no counts that could change


def test_sizes_beyond_a_launch_are_refused(binding):
    """2^32 threads or more, in workgroups of 256 (rotation, append, compact, capture), 512 and 1024 (logits) and 1024 (fork); nothing is launched."""
    lib = binding.load_library()
    assert _rope(binding, num_tokens=1 << 24, q_out=2 * P, k_out=2 * P) == 3
    assert _rope(binding, num_tokens=599, num_q_heads=65536, num_kv_heads=65536, head_dim=512, rotary_dim=0, axis_pairs=(0,), dtype=1, q_out=2 * P,
                 k_out=2 * P) == 3                                                # 32768 workgroups to a token
    assert lib.hook_pages_fork(_pages(binding, num_rows=1 << 22)) == 3
    assert lib.hook_pages_fork(_pages(binding, num_rows=1 << 19, max_blocks_per_seq=8192)) == 3
    in_place = dict(num_seqs=1 << 24, block_table_out=P, seq_lens_out=2 * P, workspace_bytes=1 << 40)
    for call in (lib.hook_pages_append, lib.hook_pages_compact):
        assert call(_pages(binding, **in_place)) == 3
    assert _logits(binding, num_rows=1 << 22, vocab=8) == 3
    assert _logits(binding, num_rows=1 << 23, vocab=8, out=P + 2) == 3            # rows off the borders: single elements
    assert _logits(binding, num_rows=1 << 20, vocab=32769, dtype=1, out=P + 4) == 3
    a = binding.HookCaptureQkArgs()
    for key, v in dict(num_seqs=1 << 20, total_q=1 << 20, num_q_heads=64, num_kv_heads=8, head_dim=128, block_size=16, max_blocks_per_seq=4, num_blocks=4,
                       num_probe_heads=64, max_sel_q=64, q=P, cu_q_lens=P, probe_heads=P, query_sel=P, q_out=P).items():
        setattr(a, key, v)
    assert lib.hook_capture_qk(a) == 3
    a.max_sel_q, a.num_capture_kv_heads, a.total_k = 1, 1, (1 << 28) + 16
    a.k_cache = a.block_table = a.seq_lens = a.capture_kv_heads = a.cu_k_lens = a.k_out = P
    assert lib.hook_capture_qk(a) == 3                                            # (2^30 threads for the queries: those alone would run)
    # an attention call of one kind is not held to the threads of the other (no workspace: nothing is launched)
    attn = binding.HookAttnProbeArgs()
    for key, v in dict(num_seqs=300000, total_q=300000, num_q_heads=256, num_kv_heads=32, head_dim=64, block_size=16, max_blocks_per_seq=4, num_blocks=4,
                       batch_kind=binding.BATCH_DECODE_ONLY, q=P, k_cache=P, v_cache=P, block_table=P, seq_lens=P, cu_q_lens=P, out=P).items():
        setattr(attn, key, v)
    assert lib.hook_attn_probe(attn) == 4


@pytest.mark.parametrize("m", [1.0, 1.25])
def test_inverse_with_a_magnitude(m):
    """By the same magnitude the gradient, by one over it the way back."""
    g = torch.Generator().manual_seed(5)
    x, w = torch.randn((2, 1, 6), generator=g).double(), torch.randn((2, 1, 6), generator=g).double()
    f, pos = torch.tensor([1.0, 0.3], dtype=torch.float64), torch.tensor([3, -4])
    assert torch.allclose(G.rope(G.rope(x, pos, f, magnitude=m), pos, f, inverse=True, magnitude=1 / m), x, atol=1e-12)
    want = G.rope(w, pos, f, inverse=True, magnitude=m)
    for i in range(x.numel()):
        h = torch.zeros_like(x)
        h.view(-1)[i] = 1e-5
        slope = ((G.rope(x + h, pos, f, magnitude=m) - G.rope(x - h, pos, f, magnitude=m)) * w).sum() / 2e-5
        assert abs(float(slope) - float(want.reshape(-1)[i])) < 1e-9


def test_append_looks_at_the_last_page_alone():
    # page 99 lies outside: full in row 0, the last one of rows that take nothing and that begin a new page, and one that takes a token
    rows, lens, refs, copies, status = G.append([0, 1, 1, 2], [[99, 0, 7], [99, 7, 7], [99, 7, 7]], [20, 9, 16], [1, 0, 0])
    assert rows == [[99, 0], [99], [99, 1]] and lens == [21, 9, 17] and refs == [1, 1, 0] and status == 0 and copies == []
    assert G.append([0, 1], [[99, 7]], [9], [1, 0, 0])[4] == G.BAD_PAGE

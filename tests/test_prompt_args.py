"""Refusals of prompt attention, shared prefixes and positions of several axes (CPU: nothing is launched)."""
import ctypes as C

import pytest
import torch

import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return spx.load_library()


def _attn(**over):
    a = binding.AttnArgs()
    a.batch, a.total_q, a.max_q_len = 4, 900, 0
    a.num_q_heads, a.num_kv_heads, a.head_dim, a.page_size = 8, 2, 64, 16
    a.num_pages, a.max_pages_per_req, a.kv_dtype = 400, 80, binding.BF16
    a.kv_stride_page, a.kv_stride_head, a.kv_stride_token = 2 * 16 * 64, 16 * 64, 64
    a.q = a.k_cache = a.v_cache = a.block_table = a.seq_lens = a.q_indptr = a.out = 4096
    for k, v in over.items():
        setattr(a, k, v)
    return a


INVALID, UNSUPPORTED = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED


@pytest.mark.parametrize("over,code", [
    (dict(batch=-1), INVALID), (dict(total_q=-1), INVALID), (dict(num_kv_heads=0), INVALID), (dict(page_size=0), INVALID), (dict(sm_scale=-1.0), INVALID),
    (dict(sm_scale=float("nan")), INVALID), (dict(kv_dtype=7), INVALID), (dict(kv_stride_token=32), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(seq_lens=None), INVALID), (dict(q=4104), INVALID), (dict(out=4100), INVALID), (dict(kv_stride_head=1028), INVALID), (dict(cache_format=3), INVALID),
    (dict(cache_format=binding.CACHE_E4M3, scale_block=16), INVALID), (dict(num_groups=-1), INVALID),
    (dict(head_dim=96, kv_stride_token=96), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED), (dict(num_q_heads=7), UNSUPPORTED),
    (dict(num_q_heads=258), UNSUPPORTED), (dict(num_groups=1, group_indptr=4096, prefix_lens=4096), UNSUPPORTED)])
def test_prompt_refusals(lib, over, code):
    status = C.c_int32(0)
    assert lib.spx_prompt_attention(C.byref(_attn(**over)), None, 0, C.byref(status), None) == code
    if code == UNSUPPORTED:
        assert lib.spx_prompt_workspace_size(C.byref(_attn(**over))) == 0


def test_prompt_sizes(lib):
    """Rows far beyond the verify step's limit, fewer rows than requests, none at all; too small a workspace is refused."""
    status = C.c_int32(0)
    sizes = [lib.spx_prompt_workspace_size(C.byref(_attn(total_q=n))) for n in (0, 1, 900, 1 << 20)]
    assert all(s > 0 for s in sizes) and sizes == sorted(sizes)
    for a in (_attn(), _attn(max_q_len=1000), _attn(total_q=2), _attn(num_q_heads=256)):
        need = lib.spx_prompt_workspace_size(C.byref(a))
        assert need > 0
        assert lib.spx_prompt_attention(C.byref(a), None, 0, C.byref(status), None) == binding.ERR_WORKSPACE
        assert lib.spx_prompt_attention(C.byref(a), C.c_void_p(1 << 20), need - 1, C.byref(status), None) == binding.ERR_WORKSPACE
        assert lib.spx_prompt_attention(C.byref(a), C.c_void_p((1 << 20) + 8), need, C.byref(status), None) == binding.ERR_WORKSPACE
    assert lib.spx_prompt_attention(C.byref(_attn(total_q=900)), C.c_void_p(1 << 20), 1 << 40, None, None) == INVALID
    assert lib.spx_prompt_attention(None, None, 0, C.byref(status), None) == INVALID


@pytest.mark.parametrize("over,code", [(dict(num_groups=-2), INVALID), (dict(num_groups=2), INVALID), (dict(num_groups=2, group_indptr=4096), INVALID),
                                       (dict(num_groups=2, prefix_lens=4096), INVALID)])
def test_prefix_refusals(lib, over, code):
    status = C.c_int32(0)
    assert lib.spx_verify_attention(C.byref(_attn(total_q=20, max_q_len=5, **over)), None, 0, C.byref(status), None) == code


def test_prefix_workspace_is_larger_and_zero_groups_change_nothing(lib):
    plain = lib.spx_workspace_size(C.byref(_attn(total_q=20, max_q_len=5)), None)
    assert lib.spx_workspace_size(C.byref(_attn(total_q=20, max_q_len=5, num_groups=0, group_indptr=4096, prefix_lens=4096)), None) == plain
    assert lib.spx_workspace_size(C.byref(_attn(total_q=20, max_q_len=5, num_groups=3, group_indptr=4096, prefix_lens=4096)), None) > plain


def test_binding_checks_groups():
    q = torch.zeros(6, 8, 64)
    pool = torch.zeros(4, 2, 16, 64)
    ints = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    args = (q, pool, pool, pool.stride()[:3], ints([[0], [1]]), ints([3, 3]), ints([0, 3, 6]), 2, 16, 4, q)
    binding.make_attn_args(*args, group_indptr=ints([0, 2]), prefix_lens=ints([0]))
    for kw in (dict(group_indptr=ints([0, 2])), dict(prefix_lens=ints([1])), dict(group_indptr=ints([0, 2]), prefix_lens=ints([1, 2])),
               dict(group_indptr=torch.tensor([0, 2]), prefix_lens=ints([1])), dict(group_indptr=ints([0, 9, 2])[::2], prefix_lens=ints([1]))):
        with pytest.raises(spx.SpxError):
            binding.make_attn_args(*args, **kw)


def _append(sections=(16, 24, 24), **over):
    a = binding.KvAppendArgs()
    a.batch, a.total_q, a.num_kv_heads, a.head_dim, a.page_size, a.num_pages = 2, 40, 2, 128, 16, 40
    a.max_pages_per_req, a.kv_dtype = 8, binding.BF16
    a.kv_stride_page, a.kv_stride_head, a.kv_stride_token = 2 * 16 * 128, 16 * 128, 128
    a.new_k = a.new_v = a.k_cache = a.v_cache = a.block_table = a.seq_lens = a.q_indptr = a.positions = 4096
    a.rope_base, a.rope_axes, a.position_stride = 10000.0, len(sections), 40
    for i, n in enumerate(sections[:4]):
        a.rope_sections[i] = n
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("sections,over,code", [
    ((16, 24, 23), {}, INVALID), ((16, 24, 25), {}, INVALID), ((-1, 40, 25), {}, INVALID), ((16, 24, 24), dict(positions=None), INVALID),
    ((16, 24, 24), dict(positions=4098), INVALID), ((16, 24, 24), dict(position_stride=39), INVALID), ((16, 24, 24), dict(rope_base=0.0), INVALID),
    ((16, 24, 24), dict(rope_axes=-1), INVALID), ((16, 24, 24), dict(rope_interleaved=2), INVALID), ((10, 40, 14), dict(rope_interleaved=1), INVALID),
    ((16, 16, 16, 16), dict(rope_axes=5), UNSUPPORTED)])
@pytest.mark.parametrize("kind", ["rows", "e4m3"])
def test_axes_refusals(lib, sections, over, code, kind):
    more = dict(cache_format=binding.CACHE_E4M3, scale_block=16, k_scales=4096, v_scales=4096) if kind == "e4m3" else {}
    status = C.c_int32(0)
    assert lib.spx_kv_append(C.byref(_append(sections, **more, **over)), C.byref(status), None) == code


def test_binding_checks_positions():
    rows, pool = torch.zeros(4, 2, 64), torch.zeros(4, 2, 16, 64)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for kw in (dict(positions=ints(3, 4)), dict(rope_sections=[8, 12, 12]), dict(positions=ints(2, 4), rope_sections=[8, 12, 12])):
        with pytest.raises((spx.SpxError, TypeError)):
            spx.kv_append(rows, rows, pool, pool, pool.stride()[:3], ints(1, 1), ints(1), ints(2), 16, 4, rope_base=1e4, **kw)

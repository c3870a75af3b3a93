"""Query rows of the append whose two tensors overlap (CPU: refused before anything is launched)."""
import ctypes as C

import pytest

import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build

ROW = 4 * 64 * 2   # bytes of a position's query rows
AT = 1 << 20


@pytest.fixture(scope="module")
def lib():
    build.build()
    return spx.load_library()


@pytest.mark.parametrize("fmt", [binding.CACHE_KV_DTYPE, binding.CACHE_E4M3])
@pytest.mark.parametrize("shift", [16, ROW, 5 * ROW, 6 * ROW - 16, -16, -ROW, -(6 * ROW - 16)])
def test_an_output_that_overlaps_the_rows_in_part_is_refused(lib, fmt, shift):
    """A row would be rotated into a place from which another is still to be read."""
    a = binding.KvAppendArgs()
    a.batch, a.total_q, a.num_kv_heads, a.head_dim, a.page_size, a.num_pages, a.max_pages_per_req = 2, 6, 2, 64, 16, 40, 17
    a.kv_dtype = binding.BF16
    a.kv_stride_page, a.kv_stride_head, a.kv_stride_token = 2 * 16 * 64, 16 * 64, 64
    a.new_k = a.new_v = a.k_cache = a.v_cache = a.block_table = a.seq_lens = a.q_indptr = 4096
    if fmt == binding.CACHE_E4M3:
        a.cache_format, a.scale_block, a.k_scales, a.v_scales = fmt, 16, 4096, 4096
    a.rope_base, a.num_q_heads, a.q_rows, a.q_out = 10000.0, 4, AT, AT + shift
    status = C.c_int32(0)
    assert lib.spx_kv_append(C.byref(a), C.byref(status), None) == binding.ERR_INVALID_ARG

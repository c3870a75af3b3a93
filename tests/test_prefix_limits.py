"""Groups past what a plan can hold are refused by every call before anything is queued (CPU: nothing is launched)."""
import ctypes as C

import pytest

import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build

TOO_MANY = (1 << 22) + 1           # a row block for each group at least, and 2^22 row blocks a plan


@pytest.fixture(scope="module")
def lib():
    build.build()
    return spx.load_library()


def _attn(groups):
    a = binding.AttnArgs()
    a.batch, a.total_q, a.max_q_len = 4, 20, 5
    a.num_q_heads, a.num_kv_heads, a.head_dim, a.page_size = 8, 2, 64, 16
    a.num_pages, a.max_pages_per_req, a.kv_dtype = 400, 80, binding.BF16
    a.kv_stride_page, a.kv_stride_head, a.kv_stride_token = 2 * 16 * 64, 16 * 64, 64
    a.q = a.k_cache = a.v_cache = a.block_table = a.seq_lens = a.q_indptr = a.out = 4096
    a.num_groups, a.group_indptr, a.prefix_lens = groups, 4096, 4096
    return a


def _sample():
    s = binding.SampleArgs()
    s.batch, s.total_q, s.vocab, s.logits_dtype = 4, 20, 512, binding.BF16
    s.logits_row_stride = 512
    for f in ("target_logits", "draft_logits", "draft_token_ids", "q_indptr", "u_accept", "u_sample", "accepted_len", "out_tokens"):
        setattr(s, f, 4096)
    return s


def test_too_many_groups(lib):
    a, s, status = _attn(TOO_MANY), _sample(), C.c_int32(0)
    fits = lib.spx_workspace_size(C.byref(_attn(3)), C.byref(s))
    assert fits > 0
    assert lib.spx_workspace_size(C.byref(a), None) == 0 and lib.spx_workspace_size(C.byref(a), C.byref(s)) == 0
    assert lib.spx_host_step_arena_size(C.byref(a), C.byref(s), 1 << 20) == 0
    assert lib.spx_host_step_arena_size(C.byref(_attn(3)), C.byref(s), 1 << 20) > 0
    ws, room = C.c_void_p(1 << 20), 1 << 40
    assert lib.spx_verify_attention(C.byref(a), ws, room, C.byref(status), None) == binding.ERR_UNSUPPORTED
    assert lib.spx_verify_step(C.byref(a), C.byref(s), ws, room, C.byref(status), None) == binding.ERR_UNSUPPORTED
    assert lib.spx_verify_step_host(C.byref(a), C.byref(s), 1 << 20, ws, room, C.byref(status), None) == binding.ERR_INVALID_ARG

"""Refusals of the 8-bit cache and of the log-probability call (CPU: nothing is launched), and the references' own checks."""
import ctypes as C

import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return spx.load_library()


def _attn(**over):
    a = binding.AttnArgs()
    a.batch, a.total_q, a.max_q_len = 4, 20, 5
    a.num_q_heads, a.num_kv_heads, a.head_dim, a.page_size = 8, 2, 64, 16
    a.num_pages, a.max_pages_per_req, a.kv_dtype = 40, 17, binding.BF16
    a.kv_stride_page, a.kv_stride_head, a.kv_stride_token = 2 * 16 * 64, 16 * 64, 64
    a.q = a.k_cache = a.v_cache = a.block_table = a.seq_lens = a.q_indptr = a.out = 4096
    a.cache_format, a.scale_block, a.k_scales, a.v_scales = binding.CACHE_E4M3, 16, 4096, 4096
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code", [
    (dict(cache_format=2), binding.ERR_INVALID_ARG), (dict(cache_format=-1), binding.ERR_INVALID_ARG),
    (dict(scale_block=0), binding.ERR_INVALID_ARG), (dict(scale_block=-4), binding.ERR_INVALID_ARG),
    (dict(scale_block=3), binding.ERR_UNSUPPORTED), (dict(scale_block=32), binding.ERR_UNSUPPORTED),
    (dict(k_scales=None), binding.ERR_INVALID_ARG), (dict(v_scales=None), binding.ERR_INVALID_ARG), (dict(v_scales=4098), binding.ERR_INVALID_ARG),
    (dict(kv_stride_token=72), binding.ERR_INVALID_ARG), (dict(k_cache=4104), binding.ERR_INVALID_ARG)])
def test_attention_refusals(lib, over, code):
    a = _attn(**over)
    status = C.c_int32(0)
    assert lib.spx_verify_attention(C.byref(a), None, 0, C.byref(status), None) == code


def test_attention_fields_are_ignored_for_pools_of_the_kv_dtype(lib):
    a = _attn(cache_format=0, scale_block=-7, k_scales=None)
    status = C.c_int32(0)
    assert lib.spx_verify_attention(C.byref(a), None, 0, C.byref(status), None) == binding.ERR_WORKSPACE
    assert lib.spx_workspace_size(C.byref(a), None) == lib.spx_workspace_size(C.byref(_attn()), None) > 0


def test_arena_counts_bytes_and_scales(lib):
    s = binding.SampleArgs()
    s.batch, s.total_q, s.vocab, s.logits_row_stride, s.logits_dtype = 4, 20, 1024, 1024, binding.BF16
    wide = lib.spx_host_step_arena_size(C.byref(_attn(cache_format=0)), C.byref(s), 1 << 20)
    narrow = lib.spx_host_step_arena_size(C.byref(_attn()), C.byref(s), 1 << 20)
    assert wide - narrow == 2 * (1 << 20) - 2 * 512     # 40 * 2 * 1 floats a pool, in 256-byte steps


def _append(**over):
    a = binding.KvAppendArgs()
    a.batch, a.total_q, a.num_kv_heads, a.head_dim, a.page_size, a.num_pages, a.max_pages_per_req = 2, 500, 2, 64, 16, 40, 17
    a.kv_dtype = binding.BF16
    a.kv_stride_page, a.kv_stride_head, a.kv_stride_token = 2 * 16 * 64, 16 * 64, 64
    a.new_k = a.new_v = a.k_cache = a.v_cache = a.block_table = a.seq_lens = a.q_indptr = 4096
    a.cache_format, a.scale_block, a.k_scales, a.v_scales = binding.CACHE_E4M3, 16, 4096, 4096
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code", [
    (dict(cache_format=9), binding.ERR_INVALID_ARG), (dict(scale_block=0), binding.ERR_INVALID_ARG), (dict(scale_block=6), binding.ERR_UNSUPPORTED),
    (dict(scale_block=32), binding.ERR_UNSUPPORTED), (dict(k_scales=None), binding.ERR_INVALID_ARG), (dict(head_dim=96, kv_stride_token=96), binding.ERR_UNSUPPORTED),
    (dict(head_dim=256, kv_stride_token=256), binding.ERR_UNSUPPORTED), (dict(page_size=256), binding.ERR_UNSUPPORTED),
    (dict(kv_stride_token=72), binding.ERR_INVALID_ARG), (dict(new_k=None), binding.ERR_INVALID_ARG), (dict(rope_base=-1.0), binding.ERR_INVALID_ARG),
    (dict(rope_base=1e4, q_rows=4096, num_q_heads=0), binding.ERR_INVALID_ARG),
    (dict(rope_base=1e4, q_rows=4096, num_q_heads=4, q_out=4100), binding.ERR_INVALID_ARG),
    (dict(q_rows=4096, num_q_heads=4, q_out=4096), binding.ERR_INVALID_ARG), (dict(rope_base=1e4, q_out=4096), binding.ERR_INVALID_ARG)])
def test_append_refusals(lib, over, code):
    a = _append(**over)
    status = C.c_int32(0)
    assert lib.spx_kv_append(C.byref(a), C.byref(status), None) == code


def test_empty_append_is_fine(lib):
    a = _append(batch=0, total_q=0)
    status = C.c_int32(0)
    assert lib.spx_kv_append(C.byref(a), C.byref(status), None) == binding.OK


def _logprob(**over):
    a = binding.LogprobArgs()
    a.rows, a.vocab, a.logits_row_stride, a.logits_dtype, a.top_n = 4, 1000, 1000, binding.BF16, 3
    a.logits = a.token_ids = a.logprobs = a.entropy = a.top_ids = a.top_logprobs = 4096
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), binding.ERR_INVALID_ARG), (dict(vocab=0), binding.ERR_INVALID_ARG), (dict(logits_row_stride=999), binding.ERR_INVALID_ARG),
    (dict(logits_row_stride=1001), binding.ERR_INVALID_ARG), (dict(logits_dtype=3), binding.ERR_INVALID_ARG), (dict(top_n=-1), binding.ERR_INVALID_ARG),
    (dict(top_n=33), binding.ERR_UNSUPPORTED), (dict(vocab=1 << 25, logits_row_stride=1 << 25), binding.ERR_UNSUPPORTED),
    (dict(logits=None), binding.ERR_INVALID_ARG), (dict(logits=4104), binding.ERR_INVALID_ARG), (dict(token_ids=None), binding.ERR_INVALID_ARG),
    (dict(top_n=0), binding.ERR_INVALID_ARG)])
def test_logprob_refusals(lib, over, code):
    a = _logprob(**over)
    status = C.c_int32(0)
    assert lib.spx_token_logprobs(C.byref(a), None, 0, C.byref(status), None) == code


def test_logprob_workspace(lib):
    status = C.c_int32(0)
    a = _logprob()
    need = lib.spx_token_logprobs_workspace(C.byref(a))
    assert need > 0 and need % 256 == 0
    assert lib.spx_token_logprobs_workspace(C.byref(_logprob(top_n=40))) == 0
    assert lib.spx_token_logprobs(C.byref(a), None, 0, C.byref(status), None) == binding.ERR_WORKSPACE
    assert lib.spx_token_logprobs(C.byref(a), 4096, need - 1, C.byref(status), None) == binding.ERR_WORKSPACE
    assert lib.spx_token_logprobs(C.byref(a), 4096, need, None, None) == binding.ERR_INVALID_ARG
    assert lib.spx_token_logprobs(C.byref(_logprob(rows=0)), None, 0, C.byref(status), None) == binding.OK


def test_binding_refuses_host_tensors_and_bad_scales():
    pool = torch.zeros(4, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    ints = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(spx.SpxError):
        spx.token_logprobs(torch.zeros(2, 8, dtype=torch.bfloat16))
    q = torch.zeros(1, 8, 64, dtype=torch.bfloat16)
    make = lambda k, v, ks, vs: binding.make_attn_args(q, k, v, (2048, 1024, 64), torch.zeros(1, 1, dtype=torch.int32), ints[:1], ints, 2, 16, 4, q, k_scales=ks, v_scales=vs)  # noqa: E731
    good = torch.ones(4, 2, 4)
    assert make(pool, pool, good, good).scale_block == 4
    for ks, vs in ((good, None), (None, None), (good.half(), good), (good[:, :1], good), (good.transpose(0, 1), good), (torch.ones(4, 2, 3), torch.ones(4, 2, 3)), (good, good[:3])):
        with pytest.raises((spx.SpxError, TypeError)):
            make(pool, pool, ks, vs)
    with pytest.raises(TypeError):
        make(pool.view(torch.uint8).to(torch.bfloat16), pool, good, good)


def test_the_references_rounding_is_the_formats():
    """Every code decodes and encodes to itself; ties go to the even pattern; torch's conversion agrees."""
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    v = R.decode(codes)
    fine = ~np.isnan(v)
    assert fine.sum() == 254 and v[0x7E] == 448 and v[1] == 2.0 ** -9
    assert (R.encode(v[fine]) == codes.numpy()[fine]).all()
    x = np.concatenate((np.random.RandomState(0).uniform(-448, 448, 20000), np.random.RandomState(1).normal(0, 0.02, 20000), (R.VALUES[1:] + R.VALUES[:-1]) / 2))
    assert (torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy() == R.encode(x.astype(np.float32).astype(np.float64))).all()
    assert R.scale_of(448.0) == 1.0 and R.scale_of(448.0001) == 2.0 and R.scale_of(0.0) == 1.0 and R.scale_of(1e-40) == 2.0 ** -126

"""The warp-wide bounded wait of the attention over 8-bit pools, where its limit runs out: in a wait-test build of the library
(limit 100k cycles) two warps wait for a signal that never comes.  Nothing faults, the kernel returns by itself."""
import ctypes as C
import time

import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_the_wait_runs_out_and_the_context_stays_usable():
    lib = C.CDLL(build.build_wait_test())
    lib.spx_debug_warp_wait_expiry.restype = C.c_int
    lib.spx_debug_warp_wait_expiry.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    report = torch.full((6,), -1, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    assert lib.spx_debug_warp_wait_expiry(report.data_ptr(), status.data_ptr(), None) == binding.OK
    torch.cuda.synchronize()
    elapsed = time.perf_counter() - t0
    rep = report.cpu().tolist()
    assert elapsed < 0.5, elapsed
    assert int(status.item()) == spx.DEV_TIMEOUT
    assert rep[4] != 0 and rep[5] == 0, rep                        # the flag is up, no wait was satisfied
    # 64 sleeps of some 20 us between two looks at the limit: 1.3 ms, 2.6 million cycles, and as much again at most
    assert max(rep[0:2]) >= 100000 and max(rep[0:4]) < 6000000, rep
    # the regular library refuses the call, and a call afterwards is right
    assert spx.load_library().spx_debug_warp_wait_expiry(report.data_ptr(), status.data_ptr(), None) == binding.ERR_UNSUPPORTED
    c = R.Cache([200, 30], 2, 64, 16, 16, seed=1)
    q = torch.randn(4, 8, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    k, v, strides, table, ks, vs = c.on(DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, ints([200, 30]), ints([0, 2, 4]), 2, 16, c.num_pages, k_scales=ks, v_scales=vs)
    assert int(ws.status.item()) == 0
    ref, _, spread, reach = R.attention(c, q, [200, 30], [2, 2])
    tol, _ = R.attention_bounds(ref, spread, reach, 200, 64, q.dtype)
    assert (abs(out.cpu().double().numpy() - ref) <= tol).all()


def test_the_regular_build_refuses():
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert spx.load_library().spx_debug_warp_wait_expiry(None, status.data_ptr(), None) == binding.ERR_UNSUPPORTED

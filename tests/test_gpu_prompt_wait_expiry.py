"""The bounded wait of the attention of prompts and shared prefixes, where its limit runs out: in a wait-test build of the library
(limit 100k cycles) two warps wait for a signal that never comes.  Nothing faults, the kernel returns by itself."""
import ctypes as C
import time

import pytest
import torch

import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build
from prompt_util import DEV, Batch, prompt

pytestmark = pytest.mark.gpu


def test_the_wait_runs_out_and_the_context_stays_usable():
    lib = C.CDLL(build.build_wait_test())
    lib.spx_debug_prompt_wait_expiry.restype = C.c_int
    lib.spx_debug_prompt_wait_expiry.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    report = torch.full((6,), -1, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    assert lib.spx_debug_prompt_wait_expiry(report.data_ptr(), status.data_ptr(), None) == binding.OK
    torch.cuda.synchronize()
    elapsed = time.perf_counter() - t0
    rep = report.cpu().tolist()
    assert elapsed < 0.5, elapsed
    assert int(status.item()) == spx.DEV_TIMEOUT
    assert rep[4] != 0 and rep[5] == 0, rep                        # the flag is up, no wait was satisfied
    # the limit and some sleeps in the barrier, of some 20 us (40,000 cycles) each and no more than a hundred of them
    assert max(rep[0:2]) >= 100000 and max(rep[0:4]) < 6000000, rep
    # the regular library refuses the call, and a call afterwards is right
    assert spx.load_library().spx_debug_prompt_wait_expiry(report.data_ptr(), status.data_ptr(), None) == binding.ERR_UNSUPPORTED
    b = Batch([200, 300], [200, 7], 8, 2, 64, 16, seed=1)
    out, lse, bits = prompt(b)
    assert bits == 0
    b.check(out, lse)


def test_the_regular_build_refuses():
    assert spx.load_library().spx_debug_prompt_wait_expiry(None, None, None) == binding.ERR_UNSUPPORTED

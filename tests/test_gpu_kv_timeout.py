"""The bounded waits of the prompt attention, made to run out on purpose.

Every mbarrier wait of the kernel gives up after about one second of clock cycles
and records LOGQ_ERR_TIMEOUT in the caller's workspace; the warp leaves its role,
the others' waits run out in turn, the kernel waits for the multiply-adds it
issued, frees its tensor memory and returns.  That path never runs in a correct
launch, so this test builds the library once more with the test-only hook
(-DLOGQ_TEST_WAIT_HOOK; the shipped library has no such code): when the workspace
holds the trigger word, an MMA warp first waits on a barrier that nothing
completes.  No fault, trap or unbounded wait is involved.
"""
import ctypes

import pytest
import torch

from gpu_common import lib
from kv_common import attention_ref, check_attention

pytestmark = pytest.mark.gpu

STALL_WORD = 0x57A11
ROLE_WAITS = (0x100, 0x101, 0x102, 0x104)        # MMA, softmax, decode, planner


def test_wait_bound_reports_timeout_and_recovers(tmp_path):
    from paper_2607_01127_gb300 import build
    logq = lib()
    out_path = str(tmp_path / "liblogq_hook.so")
    build.build_library(extra=("-DLOGQ_TEST_WAIT_HOOK",), out=out_path)
    L = ctypes.CDLL(out_path)
    L.logq_kv_attention.argtypes = logq.lib.logq_kv_attention.argtypes
    L.logq_workspace_status.argtypes = logq.lib.logq_workspace_status.argtypes
    gen = torch.Generator(device="cuda").manual_seed(0)
    n, hq, heads, d, page = 200, 8, 2, 64, 32
    cache = logq.new_kv_cache(8, page, heads, d, torch.bfloat16, 1.5, 1.6)
    kv = torch.randn(2, n, heads, d, generator=gen, device="cuda").to(torch.bfloat16)
    logq.logq_kv_append(cache, kv[0], kv[1], torch.arange(n, device="cuda"))
    q = torch.randn(n, hq, d, generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    q_start, kv_len = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [n]))
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    ws = logq.new_kv_workspace(hq, heads, d)
    stream = torch.cuda.current_stream().cuda_stream

    def call():
        st = L.logq_kv_attention(cache._ref, q.data_ptr(), hq * d, hq, n, q_start.data_ptr(), kv_len.data_ptr(), 1,
                                 table.data_ptr(), 8, d ** -0.5, 0, n, out.data_ptr(), ws.data_ptr(), ws.numel(), stream)
        assert st == logq.LOGQ_OK                         # the launch itself succeeds
        detail = ctypes.c_uint32(0)
        return L.logq_workspace_status(ws.data_ptr(), stream, ctypes.byref(detail)), detail.value

    ws.view(torch.int32)[4] = STALL_WORD                  # reserved[0]
    st, detail = call()
    assert st == logq.LOGQ_ERR_TIMEOUT and detail in ROLE_WAITS, (st, detail)
    torch.cuda.synchronize()                              # the context is still usable
    ws.zero_()
    out.fill_(float("nan"))
    assert call() == (logq.LOGQ_OK, 0)
    check_attention(out, *attention_ref(cache, q, [0, n], [n], table, d ** -0.5, 0, 1.5, 1.6))

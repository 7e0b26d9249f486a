"""The calls around the linears give Python's lock back while they enqueue: a full queue of one thread stops no other."""
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["swiglu", "layernorm", "gemv", "ckpt8"])
def test_other_threads_run_while_the_queue_is_full(which):
    from paper_2510_27527_b200 import binding as b

    x, out = torch.randn(2, 64, device="cuda").bfloat16(), torch.empty(2, 64, device="cuda").bfloat16()
    W, gamma, ck = b.nvfp4_quantize(torch.randn(64, 64, device="cuda").bfloat16()), torch.ones(64, device="cuda"), b.alloc_ckpt8(2, 64)
    call = {"swiglu": lambda: b.nvfp4_swiglu_fwd(x, x, 0, out), "layernorm": lambda: b.nvfp4_layernorm_fwd(x, gamma, None, 1e-5, 0, out),
            "gemv": lambda: b.nvfp4_gemv(x, W, out=out), "ckpt8": lambda: b.nvfp4_ckpt8_pack(x, ck)}[which]
    call()
    torch.cuda.synchronize()
    stream, spent = torch.cuda.Stream(), []

    def work():
        with torch.cuda.stream(stream):
            torch.cuda._sleep(3_000_000_000)  # (a kernel of one to two seconds)
            t0 = time.perf_counter()
            for _ in range(6000):  # more than a queue holds
                call()
            spent.append(time.perf_counter() - t0)

    worker = threading.Thread(target=work)
    worker.start()
    longest, last = 0.0, time.perf_counter()
    while worker.is_alive():
        time.sleep(0.002)
        now = time.perf_counter()
        longest, last = max(longest, now - last), now
    worker.join()
    torch.cuda.synchronize()
    assert spent[0] > 0.6, "the queue was never full"
    assert longest < 0.5 * spent[0], (longest, spent[0])

"""The compiled marshalling of the row operators as a part of a Python process."""
import ctypes as C
import subprocess
import threading
import time

import pytest
import torch

from paper_2406_00023_b200 import etr

pytestmark = pytest.mark.gpu

SLOW = """
#include <time.h>
int slow(const void* cfg, void* X, void* w, void* N, void* rstd, void* stream) {
  struct timespec t = {0, 500000000};
  nanosleep(&t, 0);
  return 0;
}
"""


def test_other_threads_run_during_a_call(tmp_path):
    """A function of half a second in the place of etr_prenorm: a thread that wakes every 5 ms goes on meanwhile."""
    src, so = tmp_path / "slow.c", tmp_path / "slow.so"
    src.write_text(SLOW)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)])
    slow = C.cast(C.CDLL(str(so)).slow, C.c_void_p).value
    cfg = etr.make_norm_config(T=4, d=64, dtype=etr.BF16)
    X, N = (torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    etr.prenorm(cfg, X, None, N)                           # binds the library's functions
    from paper_2406_00023_b200 import _args
    extra = ("etr_sort_n_rows", "etr_norm_workspace_bytes", "etr_validate")
    real = [C.cast(getattr(etr.lib(), n), C.c_void_p).value for n in _args.names + extra]
    woken, stop = [], threading.Event()

    def tick():
        while not stop.is_set():
            woken.append(time.monotonic())
            time.sleep(0.005)

    thread = threading.Thread(target=tick)
    thread.start()
    try:
        _args.bind(*[slow if n == "etr_prenorm" else a for n, a in zip(_args.names + extra, real)])
        beg = time.monotonic()
        etr.prenorm(cfg, X, None, N)
        end = time.monotonic()
    finally:
        _args.bind(*real)
        stop.set()
        thread.join()
    assert end - beg >= 0.5
    # a hundred times if nothing else runs; the thread that holds the lock lets it wake twice at most, before and after
    assert sum(beg + 0.05 < t < end - 0.05 for t in woken) >= 10
    etr.prenorm(cfg, X, None, N)
    torch.cuda.synchronize()

"""The compiled marshalling of the row operators as a part of a Python process."""
import ctypes as C
import subprocess
import threading
import time

import pytest
import torch

from paper_2406_00023_b200 import etr

pytestmark = pytest.mark.gpu

FAKES = """
#include <time.h>
#include <stdexcept>
extern "C" int slow(const void* cfg, void* X, void* w, void* N, void* rstd, void* stream) {
  struct timespec t = {0, 500000000};
  nanosleep(&t, 0);
  return 0;
}
extern "C" int throws(const void* cfg, void* X, void* w, void* N, void* rstd, void* stream) { throw std::runtime_error("no memory for a record"); }
"""
EXTRA = ("etr_sort_n_rows", "etr_norm_workspace_bytes", "etr_validate")


@pytest.fixture
def prenorm_by(tmp_path):
    """Binds a function of FAKES in the place of etr_prenorm, which is put back afterwards."""
    src, so = tmp_path / "fakes.cpp", tmp_path / "fakes.so"
    src.write_text(FAKES)
    subprocess.check_call(["g++", "-shared", "-fPIC", "-o", str(so), str(src)])
    fakes = C.CDLL(str(so))
    X, N = (torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cfg = etr.make_norm_config(T=4, d=64, dtype=etr.BF16)
    etr.prenorm(cfg, X, None, N)                           # binds the library's functions
    from paper_2406_00023_b200 import _args
    real = {n: C.cast(getattr(etr.lib(), n), C.c_void_p).value for n in _args.names + EXTRA}

    def bind(name):
        _args.bind(*dict(real, etr_prenorm=C.cast(getattr(fakes, name), C.c_void_p).value).values())
        return lambda: etr.prenorm(cfg, X, None, N)

    yield bind
    _args.bind(*real.values())
    etr.prenorm(cfg, X, None, N)
    torch.cuda.synchronize()


def test_other_threads_run_during_a_call(prenorm_by):
    """A function of half a second: a thread that wakes every 5 ms goes on meanwhile."""
    woken, stop = [], threading.Event()

    def tick():
        while not stop.is_set():
            woken.append(time.monotonic())
            time.sleep(0.005)

    call, thread = prenorm_by("slow"), threading.Thread(target=tick)
    thread.start()
    try:
        beg = time.monotonic()
        call()
        end = time.monotonic()
    finally:
        stop.set()
        thread.join()
    assert end - beg >= 0.5
    # a hundred times if nothing else runs; where the call keeps the lock, never
    assert sum(beg + 0.05 < t < end - 0.05 for t in woken) >= 10


def test_an_exception_of_the_library_is_a_python_one(prenorm_by):
    call = prenorm_by("throws")
    for _ in range(2):
        with pytest.raises(RuntimeError, match="no memory for a record"):
            call()

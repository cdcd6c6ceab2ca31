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


def test_two_threads_at_once():
    """Two Python threads, each with its stream and buffers, in the library at the same time: the bits of either alone."""
    T, d, h, E, k = 300, 256, 128, 8, 2
    cfg = etr.make_config(T=T, d=d, D=8, E=E, k=k, h=h, capacity=T, dtype=etr.BF16)
    n = etr.make_norm_config(T=T, d=d, dtype=etr.BF16, post_norm=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).bfloat16()                 # noqa: E731
    W = [rand(E, h, d, scale=d ** -0.5), rand(E, h, d, scale=d ** -0.5), rand(E, d, h, scale=h ** -0.5)]
    sets = [dict(X=rand(T, d), ids=torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32),
                 w=torch.rand(T, k, generator=g, device="cuda")) for _ in range(2)]

    def state():
        f32, rows = (lambda *s: torch.zeros(*s, device="cuda")), (lambda: torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"))
        return dict(buf=etr.LayerBuffers(cfg), plan=etr.SortBuffers(etr.routed_sort_config(cfg)), N=rows(), Y=rows(), Xo=rows(), dX=rows(), dN=rows(),
                    r=f32(T), ry=f32(T), dw=f32(T, k), dgain=f32(d), dW=[torch.zeros_like(t) for t in W],
                    ws=torch.empty(etr.norm_workspace_bytes(n), dtype=torch.uint8, device="cuda"))

    def step(x, s):
        etr.prenorm(n, x["X"], None, s["N"], s["r"])
        etr.routed_forward(cfg, s["N"], x["ids"], x["w"], *W, s["buf"], s["plan"], s["Y"])
        etr.join(n, x["X"], s["Y"], None, None, None, s["Xo"], None, s["ry"])
        etr.routed_backward(cfg, x["w"], *W, s["Xo"], s["buf"], s["plan"], s["dN"], s["dw"], *s["dW"])
        etr.prenorm_bwd(n, s["dN"], x["X"], None, s["r"], None, s["dX"], s["dgain"], s["ws"])

    def outputs(s):
        return [s[name] for name in ("N", "Y", "Xo", "dX", "dN", "dw", "dgain")] + s["dW"]

    alone = []
    for x in sets:
        s = state()
        step(x, s)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in outputs(s)])
    both, failed = [state(), state()], []
    torch.cuda.synchronize()
    start = threading.Barrier(2)

    def work(x, s):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(60)
                for _ in range(100):
                    step(x, s)
                torch.cuda.current_stream().synchronize()
        except Exception as e:                             # noqa: BLE001  handed to the test's own thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(sets, both)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for s, ref in zip(both, alone):
        assert all(torch.equal(a, b) for a, b in zip(outputs(s), ref))

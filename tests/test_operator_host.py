"""The operators' host code without a GPU: what is launched for which call, and who is told of waits that ran out.

Every test runs in a process of its own in which a stand-in for the CUDA runtime (host/fake_operators.c) is preloaded."""
import ctypes as C
import os
import subprocess
import sys
import threading

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
OK, TIMEOUT = 0, -6


@pytest.fixture(scope="session")
def fake_runtime(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("fake") / "libfakeoperators.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-shared", "-fPIC", "-pthread", "-I", "/usr/local/cuda/include", "-o", so,
                    os.path.join(HERE, "host", "fake_operators.c")], check=True)
    return so


# ------------------------------------------------------------------ in the process with the stand-in

def _fake():
    f = C.CDLL(os.environ["LD_PRELOAD"])
    f.fake_launch_name.restype = C.c_char_p
    return f


def _in_a_thread(call):
    result = []
    t = threading.Thread(target=lambda: result.append(call()))
    t.start()
    t.join()
    return result[0]


def every_thread_is_told_of_a_timeout():
    """A wait that ran out on the device is told once to every thread that asks, whoever asked before, and so is the next one."""
    import paper_2108_09413_b200 as isc
    f, lib = _fake(), isc.lib()
    status = lambda: lib.isc_operator_status(None)  # noqa: E731
    go, asked, results = threading.Semaphore(0), threading.Semaphore(0), []

    def other():
        while True:
            go.acquire()
            results.append(status())
            asked.release()
    thread = threading.Thread(target=other, daemon=True)
    thread.start()

    def theirs():
        go.release()
        assert asked.acquire(timeout=60)
        return results[-1]
    files = f.fake_timeouts(0, 0)
    assert files == 3 and (status(), theirs()) == (OK, OK)
    for file in range(files):
        f.fake_timeouts(file, 1 + file)
        assert status() == TIMEOUT, file
        assert status() == OK, file
        assert theirs() == TIMEOUT, file                # not taken away by the first
    assert (status(), theirs()) == (OK, OK)
    f.fake_timeouts(1, 1)
    assert theirs() == TIMEOUT and status() == TIMEOUT and theirs() == OK and status() == OK
    assert _in_a_thread(status) == TIMEOUT              # a thread's first: since the library was loaded


AT = 0x10000                                  # an aligned address nobody owns


def a_sum_s_pitch_counts_only_with_a_sum():
    """Which form of the norm runs does not depend on what a caller who wants no sum passes as its pitch."""
    import paper_2108_09413_b200 as isc
    f = _fake()

    def kernel(total, lds, rows=20000, width=4096):
        f.fake_reset()
        assert isc.lib().isc_rms_norm_quant(AT, width, AT, width, AT, 0, 0, rows, width, 1e-6, total, lds, AT, width, AT, None) == OK
        assert f.fake_launches() == 1
        return next(n for n in ("k_norm_ring", "k_norm_block") if n in f.fake_launch_name(0).decode())
    for lds in (0, 1, 4095, 4097, -1, 2**40 + 1):
        assert kernel(None, lds) == "k_norm_ring", lds
    assert kernel(AT, 4096) == "k_norm_ring" and kernel(AT, 4097) == "k_norm_block"


def nothing_is_launched_for_a_refused_projection():
    """A projection of more tiles than are supported is refused as a whole: the adapters' inner sums are not computed either."""
    import paper_2108_09413_b200 as isc
    from paper_2108_09413_b200.operators import _Adapters
    f, lib = _fake(), isc.lib()
    parts = _Adapters(AT, AT, AT, AT, 0, 4, 16)

    def call(rows, n):
        f.fake_reset()
        size = C.c_int64()
        assert lib.isc_quant_linear_work_space(rows, 16, C.byref(size)) == OK
        return lib.isc_quant_linear(AT, 64, AT, rows, AT, 64, AT, 64, n, None, C.addressof(parts), AT, n, 0, AT, size.value, None), f.fake_launches()
    assert call(2**29, 2**29) == (-3, 0)
    assert call(2**20, 2**30 - 2) == (-3, 0)
    assert call(300, 1000) == (OK, 2) and call(1, 1000) == (OK, 2)


TESTS = [every_thread_is_told_of_a_timeout, a_sum_s_pitch_counts_only_with_a_sum, nothing_is_launched_for_a_refused_projection]


@pytest.mark.parametrize("test", [t.__name__ for t in TESTS])
def test_host(fake_runtime, test):
    run = subprocess.run([sys.executable, os.path.abspath(__file__), test], env=dict(os.environ, LD_PRELOAD=fake_runtime), cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    globals()[sys.argv[1]]()

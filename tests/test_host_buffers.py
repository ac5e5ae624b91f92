"""When a context's buffer counts as cleared: the header's host functions, compiled alone, with a clearing that is told to fail."""
import ctypes
import subprocess

import pytest

from paper_2411_11925_b200 import build


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("hostio")
    src = d / "hostio.cpp"
    src.write_text('#include "hostio.h"\n'
                   'static csd::HostIo b;\n'
                   'static int calls = 0;\n'
                   'extern "C" int ask(int captured, int rc) { return csd::clear_once(b, captured != 0, [&] { ++calls; return rc; }); }\n'
                   'extern "C" int count() { return calls; }\n'
                   'extern "C" int drop() { b.base = &b; b.cap = 5; b.in_graph = true; b.drop(); return b.base == nullptr && b.cap == 0 && !b.in_graph; }\n')
    so = d / "hostio.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{build.CSRC}", str(src), "-o", str(so)], check=True)
    return ctypes.CDLL(str(so))


def test_a_clearing_that_failed_is_done_again(lib):
    assert lib.ask(0, -7) == -7 and lib.count() == 1
    assert lib.ask(0, -7) == -7 and lib.count() == 2     # the buffer has its size by now, but nobody has cleared it
    assert lib.ask(1, 0) == 0 and lib.count() == 3       # in a graph only
    assert lib.ask(0, 0) == 0 and lib.count() == 4
    assert lib.ask(0, 0) == 0 and lib.ask(1, 0) == 0 and lib.count() == 4
    assert lib.drop() == 1                               # another buffer
    assert lib.ask(0, 0) == 0 and lib.count() == 5

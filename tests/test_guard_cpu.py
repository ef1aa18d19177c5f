"""wf_guard.h (compiled for the host): what a C entry leaves behind where its work throws."""
import ctypes
import pathlib
import subprocess

import pytest

SRC = pathlib.Path(__file__).parents[1] / "paper_2609_32869_amd" / "csrc"
CODE = """
#include <new>
#include "%s/wf_guard.h"
struct Handle { std::string err = "an older call's"; };
static Handle held;
static std::string thread;
extern "C" int run(int throws, int with_handle) {
  held.err = thread = "an older call's";
  return wf::guarded(with_handle ? &held : nullptr, thread, -1, [&] {
    if (throws == 1) throw std::bad_alloc();
    if (throws == 2) throw 7;
    return 5;
  });
}
extern "C" const char* message(int of_handle) { return of_handle ? held.err.c_str() : thread.c_str(); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("guard")
    (folder / "guard.cpp").write_text(CODE % SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", folder / "guard.so", folder / "guard.cpp"], check=True)
    lib = ctypes.CDLL(str(folder / "guard.so"))
    lib.message.restype = ctypes.c_char_p
    return lib


@pytest.mark.parametrize("throws", [1, 2])
def test_the_message_is_where_the_caller_looks(lib, throws):
    assert lib.run(throws, 1) == -1
    assert lib.message(1) == lib.message(0) == b"out of host memory"
    assert lib.run(throws, 0) == -1
    assert lib.message(0) == b"out of host memory" and lib.message(1) == b"an older call's"


def test_results_and_messages_of_their_own_stay(lib):
    assert lib.run(0, 1) == lib.run(0, 0) == 5
    assert lib.message(1) == lib.message(0) == b"an older call's"

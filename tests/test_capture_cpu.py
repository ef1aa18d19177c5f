"""wf_capture.h (compiled for the host, over a runtime of counters): a capture ends however its scope is left."""
import ctypes
import pathlib
import subprocess

import pytest

SRC = pathlib.Path(__file__).parents[1] / "paper_2609_32869_amd" / "csrc"
FAKE = """
#include <new>
#include "%s/wf_capture.h"
struct Fake {
  using Error = int;
  using Stream = int*;
  using Graph = int*;
  using Exec = int*;
  static constexpr int ok = 0;
  static inline int fails, open, graphs, execs, g, x;
  static int begin(Stream) { if (fails == 1) return 7; ++open; return 0; }
  static int end(Stream, Graph* to) { --open; if (fails == 2) { *to = nullptr; return 8; } ++graphs; *to = &g; return 0; }
  static int instantiate(Exec* to, Graph) { if (fails == 3) return 9; ++execs; *to = &x; return 0; }
  static void destroy(Graph) { --graphs; }
  static void destroy_exec(Exec) { --execs; }
};
// fails: 0 nothing, 1 .. 3 the runtime's call, 4 the work throws, 5 what follows the instantiation throws, 6 the work is refused
extern "C" int run(int fails, int* left) {
  Fake::fails = fails;
  Fake::open = Fake::graphs = Fake::execs = 0;
  bool on = false, was_on = false;
  int r = 0;
  try {
    wf::Capture<Fake> cap(nullptr, on);
    r = [&] {
      if (int e = cap.begin()) return e;
      was_on = on;
      if (fails == 4) throw std::bad_alloc();
      const int e = cap.end();
      if (fails == 6) return 10;
      if (e) return e;
      if (int e1 = cap.instantiate()) return e1;
      if (fails == 5) throw std::bad_alloc();
      cap.release();
      return 0;
    }();
  } catch (const std::bad_alloc&) { r = -1; }
  left[0] = Fake::open; left[1] = Fake::graphs; left[2] = Fake::execs; left[3] = on; left[4] = was_on;
  return r;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("capture")
    (folder / "capture.cpp").write_text(FAKE % SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", folder / "capture.so", folder / "capture.cpp"], check=True)
    return ctypes.CDLL(str(folder / "capture.so"))


@pytest.mark.parametrize("fails,result", [(0, 0), (1, 7), (2, 8), (3, 9), (4, -1), (5, -1), (6, 10)])
def test_nothing_is_left_open(lib, fails, result):
    left = (ctypes.c_int * 5)()
    assert lib.run(fails, left) == result
    # no stream in capture, no graph, the executable graph where it was handed on, and the flag down again
    assert list(left) == [0, 0, 1 if fails == 0 else 0, 0, 0 if fails == 1 else 1]

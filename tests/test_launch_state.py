"""Launch set-up belongs to a device: no launcher keeps a count of its
multiprocessors, or that a limit was raised there, in a variable of the process,
where a second device would find the first one's, and two threads would race."""
import glob
import os
import re

from tests.conftest import ROOT

KEPT = re.compile(r"^\s+static\s+(?:int|bool|unsigned|size_t|long|float|"
                  r"cuda\w+)\b[^()]*(?:=|;|\{)")


def test_no_launcher_keeps_what_belongs_to_a_device():
    files = glob.glob(os.path.join(ROOT, "paper_2608_15797_gb300", "csrc", "*"))
    assert len(files) > 20
    kept = []
    for path in sorted(files):
        with open(path) as f:
            kept += [f"{os.path.basename(path)}:{n}: {line.strip()}"
                     for n, line in enumerate(f, 1) if KEPT.match(line)]
    assert not kept, kept


def test_what_is_looked_for():
    for line in ("  static int sms = 0;", "  static bool ready = false;",
                 "    static cudaError_t e;", "  static unsigned n{};"):
        assert KEPT.match(line)
    for line in ("  static constexpr int kCols = 8;", "  int sms = 0;",
                 "  static const int order[7][2] = {{4, 2}};",
                 "static __device__ int f(int x);"):
        assert not KEPT.match(line)

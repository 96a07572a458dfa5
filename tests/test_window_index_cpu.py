"""Which of a call's tokens a window cache keeps (csrc/bm_window_dev.h), computed by the device
code's own functions, compiled for the host with signed overflow trapped, against the
definition in numbers of any size (no GPU needed)."""
import itertools
import subprocess

import pytest

from paper_2412_05693_amd.build import CSRC, INCLUDE, hipcc

PROGRAM = r"""
#include <algorithm>
#include <cstdio>

#include "bm_window_dev.h"

int main() {
  int t0, pad, n_tok, window, sinks;
  while (scanf("%d %d %d %d %d", &t0, &pad, &n_tok, &window, &sinks) == 5) {
    const int kept = std::min(n_tok, window), lead = std::min(sinks, n_tok - kept);
    const int r0 = bm::index_of(t0, pad);
    for (int r = 0; r < kept + lead; ++r) {
      const int t = bm::kept_token(r, lead, n_tok, window, sinks, r0);
      if (t >= 0) printf("%d:%d ", t, r0 + t);
    }
    printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("host")
    (d / "kept.hip").write_text(PROGRAM)
    subprocess.run([hipcc(), "--offload-host-only", "-std=c++17", "-O1", "-Xarch_host", "-fsanitize=undefined",
                    "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", CSRC, "-I", INCLUDE, str(d / "kept.hip"),
                    "-o", str(d / "kept")], check=True, capture_output=True, text=True)
    return d / "kept"


def test_kept_tokens(program):
    top = 2 ** 31 - 1
    cases = []
    for t0, pad, n_tok, (window, sinks) in itertools.product(
            (0, 1, 5, 40, 2 ** 30 - 200), (0, 1, 4, 7, 39, 40, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 7, top - 5, top - 1, top),
            (1, 2, 9, 33, 200), ((1, 0), (1, 6), (8, 4), (32, 1), (32, 40), (300, 5))):
        cases.append((t0, pad, n_tok, window, sinks))
    run = subprocess.run([program], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
    lines = run.stdout.splitlines()
    assert len(lines) == len(cases)
    for (t0, pad, n_tok, window, sinks), line in zip(cases, lines):
        want = {t: t0 + t - pad for t in range(n_tok)
                if t0 + t - pad >= 0 and (t0 + t - pad < sinks or t >= n_tok - window)}
        got = [tuple(map(int, x.split(":"))) for x in line.split()]
        assert len(got) == len(want) and dict(got) == want, (t0, pad, n_tok, window, sinks)

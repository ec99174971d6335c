"""The host rules of the serving operators' kernels on the CPU, compiled from
the headers that the kernels are built from."""
import os
import subprocess

import pytest

from paper_2601_18999_amd import build

SERVE = os.path.join(build.HERE, "csrc_serve")


def compiled(tmp_path, text, *flags):
    """Output of a host program that includes the serving operators' headers."""
    src, exe = tmp_path / "rule.cpp", tmp_path / "rule"
    src.write_text(text)
    subprocess.run([build.hipcc(), "-std=c++17", "-O1", *flags, "-I", SERVE, str(src), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_lanes_reach_what_32_bits_address(dim, tmp_path):
    # a load of 64 lanes, 16 bytes each: its rows' offsets from the first one's, in 32 and in 64 bits
    rows = 512 // dim
    last = (2 ** 32 - 2 * dim) // (rows - 1) // 16 * 16  # the last stride, of those on 16 bytes, that 32 bits hold
    strides = [0, 2 * dim, last - 16, last, last + 16, 2 ** 31 - 16]
    out = compiled(tmp_path, """
#include <cstdio>
#include "kvr_serve.h"
int main() {
  const int dim = %d, chunks = dim / 8;
  for (const long long stride : {%s}) {
    bool same = true;
    for (int lane = 0; lane < 64; ++lane) {
      const uint32_t row = lane / chunks, at = lane %% chunks * 16;
      same &= (uint32_t)(row * (uint32_t)stride + at) == (uint64_t)row * (uint64_t)stride + at;
    }
    std::printf("%%d %%d\\n", kvr::lanes_reach(dim, stride), same);
  }
}
""" % (dim, ", ".join(f"{s}ll" for s in strides)))
    got = [(int(a), int(b)) for a, b in zip(out[::2], out[1::2])]
    assert all(reach == same for reach, same in got), got
    fits = [s <= last for s in strides]
    assert [bool(r) for r, _ in got] == fits

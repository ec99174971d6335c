"""The host rules of the serving operators' kernels on the CPU, compiled from
the headers that the kernels are built from."""
import os
import re
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


def test_partial_rows_fit_their_room(tmp_path):
    # the plan's own rules over random requests and groups, those of the largest shared and split units among them
    out = compiled(tmp_path, """
#include <cstdio>
#include <random>
#include <vector>
#include "kvr_plan.h"
using namespace kvr;

struct Request { int rows, own, group; };

// partial rows of a plan, counted unit by unit
static int64_t partial_rows(const std::vector<Request>& reqs, const std::vector<int>& prefix, int slots, int few, int kv) {
  const int groups = (int)prefix.size();
  std::vector<int> apart(groups), rows(groups), shared(groups);
  for (const Request& r : reqs)
    if (groups) apart[r.group] += row_waves(r.rows, few), rows[r.group] += r.rows;
  for (int j = 0; j < groups; ++j)
    shared[j] = worth_sharing(apart[j], row_waves(rows[j], few), steps_of(prefix[j]), kv);
  struct U { int rows, steps, cost; bool partial; };
  std::vector<U> units;
  auto tiles = [&](int n, int steps, bool partial) {
    for (int at = 0; at < n; at += kTileRows) {
      const int r = n - at < kTileRows ? n - at : kTileRows;
      units.push_back({r, steps, steps * row_waves(r, few), partial});
    }
  };
  for (int j = 0; j < groups; ++j)
    if (shared[j]) tiles(rows[j], steps_of(prefix[j]), true);
  for (const Request& r : reqs) {
    const bool s = groups && shared[r.group];
    tiles(r.rows, steps_of(r.own) + (groups && !s ? steps_of(prefix[r.group]) : 0), s);
  }
  int64_t total = 0, sum = 0;
  for (const U& u : units) total += u.cost;
  const int chunk = chunk_of(total, slots, few);
  for (const U& u : units) {
    const Cut c = cut_of(u.steps, u.cost, chunk);
    if (u.partial || c.splits > 1) sum += (int64_t)c.splits * u.rows;
  }
  return sum;
}

int main() {
  std::mt19937 rng(5);
  auto upto = [&](int n) { return (int)(rng() %% (unsigned)n); };
  const int sizes[] = {1, 2, 16, 32, 33, 100, 127, 128, 129, 160, 161, 256, 257, 288, 289, 384, 385};
  int64_t cases = 0, over = 0, shared_near = 0, split_near = 0;
  for (int i = 0; i < 60000; ++i) {
    const int few = upto(2) ? 1 : 4, kv = 1 << upto(11), slots = kAttendSlots / kv > 0 ? kAttendSlots / kv : 1;
    const int n = 1 + upto(upto(2) ? 12 : 200), groups = upto(3) ? 1 + upto(n < 5 ? n : 5) : 0;
    std::vector<int> prefix(groups);
    for (int& p : prefix) p = upto(upto(2) ? 400 : 20000);
    std::vector<Request> reqs(n);
    const int same = upto(2) ? sizes[upto(17)] : 0, lengths = 1 + upto(upto(2) ? 200 : 30000);
    int64_t rows = 0;
    for (int r = 0; r < n; ++r) {
      reqs[r] = {same ? same : upto(600), 1 + upto(lengths), groups ? r * groups / n : 0};
      rows += reqs[r].rows;
    }
    const int64_t most = most_partial_rows(rows, n, groups > 0, slots), have = partial_rows(reqs, prefix, slots, few, kv);
    ++cases;
    over += have > most;
    if (groups) shared_near += have > 2 * 200 * (int64_t)n;
    if (!groups) split_near += 2 * have > most;
  }
  std::printf("%%lld %%lld %%lld %%lld\\n", (long long)cases, (long long)over, (long long)shared_near, (long long)split_near);
}
""".replace("%%", "%"), "-x", "hip", "--offload-arch=gfx950")
    cases, over, shared_near, split_near = map(int, out)
    assert cases == 60000 and over == 0
    assert shared_near > 100 and split_near > 100  # the room is used: more than half of it by many


def test_assembler_names_the_registers_that_it_writes():
    # scalar registers by name: the compiler has to know what it may not keep there
    statements = 0
    for name in sorted(os.listdir(SERVE)):
        text = open(os.path.join(SERVE, name)).read()
        for asm in re.findall(r"\basm\b(?: volatile)?\s*\((.*?)\);", text, re.S):
            code, _, operands = asm.partition('"' + ' ::') if '" ::' in asm else asm.partition('" :')
            for written in re.findall(r"\bs_mov_b(?:32|64) ([a-z_]+[0-9]*),", code):
                statements += 1
                assert f'"{written}"' in operands, (name, asm)
    assert statements == 3

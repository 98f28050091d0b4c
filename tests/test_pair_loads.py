"""What the products of pairs load stays inside their operands, shown on the host by the arithmetic that the kernels use (csrc/tng_pair_loads.hpp).

A matrix of pairs is looked at by tiles of its rows and pieces of its depth, as the products take them: every load of every stage, and those asked for behind
the last one.  A lane reads where its offset is below what its descriptor says there is, and nowhere else.  Every byte that is read has to be one of the tile's
rows, at the load's stage, and together the loads have to read all of those, once; no descriptor may reach beyond the last row's end."""
import shutil
import subprocess

import pytest

from paper_1901_08227_amd import build

PROGRAM = r"""
#include "tng_pair_loads.hpp"
#include <cstdio>
#include <cstdlib>
#include <vector>
using tng::PairRows;

static void check(bool ok, const char* what, uint32_t all, uint32_t tile, uint32_t waves, uint32_t deep, uint32_t first, uint32_t stage, uint32_t stages) {
  if (ok) return;
  printf("%s: %u rows, tiles of %u by %u, depth %u, first row %u, stages %u + %u\n", what, all, tile, waves, deep, first, stage, stages);
  exit(1);
}

int main() {
  const uint32_t kinds[][2] = {{256, 8}, {192, 8}, {128, 8}, {64, 4}, {128, 4}};
  const uint32_t deeps[] = {1, 2, 5};
  const uint64_t p = 1ull << 40;
  for (const auto& kind : kinds)
    for (uint32_t all = 1; all <= 2 * kind[0] + 1; all += all < 70 ? 1 : 13)
      for (uint32_t deep : deeps)
        for (uint32_t pieces = 1; pieces <= (deep == 5 ? 2u : 1u); ++pieces)
          for (uint32_t s = 0; s < pieces; ++s)
            for (uint32_t first = 0; first < all; first += kind[0]) {
              const uint32_t tile = kind[0], waves = kind[1], stage = deep * s / pieces, stages = deep * (s + 1) / pieces - stage;
              const uint64_t ld = deep * 128ull, end = p + all * ld;
              const uint32_t rows = all - first < tile ? all - first : tile;
              PairRows r = PairRows::of(p, ld, all, first, tile, stage, stages);
              auto ok = [&](bool is, const char* what) { check(is, what, all, tile, waves, deep, first, stage, stages); };
              for (uint32_t k = 0; k < stages + 4; ++k, r.next()) {  // (up to four stages are asked for ahead)
                std::vector<char> seen(rows * 128u);
                for (uint32_t j = 0; j * waves * 8 < tile; ++j) {
                  const PairRows::Descriptor d = r.from(j * waves * 8);
                  ok(d.bytes == 0 || (d.base >= p && d.base + d.bytes <= end), "a descriptor reaches beyond the operand");
                  ok(d.bytes < (1u << 31), "a descriptor's bytes");
                  for (uint32_t wave = 0; wave < waves; ++wave)
                    for (uint32_t lane = 0; lane < 64; ++lane) {
                      const uint32_t offset = r.offset(lane, wave);
                      if (offset >= d.bytes) continue;
                      ok(offset + 16 <= d.bytes, "a load that is in bounds only in part");
                      const uint64_t at = d.base + offset - p, row = at / ld, in = at % ld;
                      ok(k < stages, "a stage behind the last one");
                      ok(row >= first && row < first + rows, "another row");
                      ok(in / 128 == stage + k, "another stage");
                      const uint32_t piece = (uint32_t)(row - first) * 128 + in % 128;
                      for (uint32_t b = 0; b < 16; ++b) ok(!seen[piece + b]++, "a byte twice");
                    }
                }
                for (char c : seen) ok(c == (k < stages), "a byte that is not read");
              }
            }
  // the largest: 256 rows of 65536 columns
  const PairRows r = PairRows::of(p, 65536 / 32 * 128, 65536, 65280, 256, 0, 2048);
  if (r.bytes != 256u * 262144u || r.from(248).bytes != 8 * 262144 || r.from(248).base + r.from(248).bytes != p + 65536ull * 262144) return 2;
  return 0;
}
"""


def test_loads_stay_inside_their_operands(tmp_path):
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("no host compiler")
    (tmp_path / "loads.cpp").write_text(PROGRAM)
    program = str(tmp_path / "loads")
    subprocess.run([compiler, "-O2", "-std=c++17", "-Wall", "-Werror", "-D__host__=", "-D__device__=", "-I", build.CSRC, str(tmp_path / "loads.cpp"), "-o", program],
                   check=True)
    ran = subprocess.run([program], capture_output=True, text=True, timeout=100)
    assert ran.returncode == 0, ran.stdout


def test_no_load_has_an_offset_beside_its_descriptor():
    """What the arithmetic above says is all that says where a load goes: loads to LDS have a scalar offset of 0."""
    import os
    import re

    loads = 0
    for name in sorted(os.listdir(build.CSRC)):
        with open(os.path.join(build.CSRC, name)) as f:
            for operand in re.findall(r'"buffer_load_dword\w* %\d, %\d, (\S+) offen lds"', f.read()):
                loads += 1
                assert operand == "0", name
    assert loads >= 2

"""The lists that an attention over a map cuts, against the workspace that its size query reserves.

A piece's sums go to the tile of its workgroup's number and a cut list to the next entry of a table; the kernels clamp
neither, so no list lengths whatever may give more pieces or cut lists than there is room for, and a cut list has to
have two pieces at least (its sums are read from the workspace).  The rules are compiled from the library's header and
applied to random and extreme lengths of every list of a call, as the ordering kernel applies them."""
import shutil
import subprocess

import numpy as np
import pytest

from paper_2609_37001_amd import build

MAIN = r"""
#include <stdio.h>

#include <random>
#include <vector>

#include "psa_pieces.h"

using psa::Cut;
using psa::Pieces;
std::mt19937_64 rng(7);
long cases, cut_cases, most_splits, most_pieces;      // (in thousandths of what fits)

bool order(const std::vector<int32_t>& len, const Pieces& to, int32_t room) {
  unsigned long long work = 0;
  for (int32_t c : len) work += c;
  const int64_t items = len.size();
  const Cut cut(work, (int32_t)items, room, to);
  int64_t splits = 0, pieces = 0;
  for (int32_t c : len)
    if (cut.cuts(c)) {
      const int32_t p = cut.pieces(c);
      if (p < 2 || p > 0xffff || p > c) return false;
      splits++;
      pieces += p;
    }
  cases++;
  cut_cases += splits > 0;
  if (splits) {
    most_splits = std::max<long>(most_splits, 1000 * splits / to.splits);
    most_pieces = std::max<long>(most_pieces, 1000 * pieces / to.pieces);
  }
  return splits <= to.splits && pieces <= to.pieces && pieces + items - splits <= to.grid;
}

// Lists of at most `longest` blocks.
bool lists(int64_t items, int64_t longest, const Pieces& to, int64_t room) {
  if (!to.grid) return true;
  std::vector<int32_t> len(items);
  auto value = [&](int64_t x) { return (int32_t)std::max<int64_t>(0, std::min<int64_t>(longest, x)); };
  auto below = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)n); };
  // some long ones of one length, the others of another: around every count at which cutting starts or ends
  for (int64_t base : {int64_t(0), int64_t(1), below(longest + 1)})
    for (int64_t many : {int64_t(1), int64_t(2), room * 4 / 5 - 1, room * 4 / 5, room * 4 / 5 + 1, room * 2 / 3 - 1, room * 2 / 3, room - 1, room, room + 1,
                         items / 2, items - 1, items, below(items) + 1})
      for (int64_t top : {longest, below(longest) + 1, below(64) + 1, int64_t(13), base + base / 4 + 1}) {
        many = std::max<int64_t>(0, std::min(many, items));
        for (int64_t i = 0; i < items; i++) len[i] = value(i < many ? top : base);
        if (!order(len, to, room)) return false;
      }
  for (int kind = 0; kind < 12; kind++) {
    const double power = 0.5 + kind, keep = 1.0 / (1 + below(40));
    for (int64_t i = 0; i < items; i++) {
      const double u = (rng() >> 11) * 0x1p-53;
      len[i] = value(kind % 3 == 0 ? below(longest + 1) : kind % 3 == 1 ? (int64_t)(longest * pow(u, power)) : (int64_t)(u < keep ? longest : 40 * u));
    }
    if (!order(len, to, room)) return false;
  }
  return true;
}

struct Section { size_t at, bytes; };
bool apart(std::initializer_list<Section> of, size_t total) {
  for (const Section& x : of) {
    if (x.at % 256 || x.at + x.bytes > total) return false;
    for (const Section& y : of)
      if (&x != &y && x.bytes && y.bytes && x.at < y.at + y.bytes && y.at < x.at + x.bytes) return false;
  }
  return true;
}

int main() {
  int n_kv, group, d, nbq, nbk, block;
  while (scanf("%d %d %d %d %d %d", &n_kv, &group, &d, &nbq, &nbk, &block) == 6) {
    const int32_t n_bh = n_kv * group, room = psa::room_of(block);
    const int64_t rows = (int64_t)n_bh * nbq, cols = (int64_t)n_kv * nbk;
    const size_t tile = (size_t)block * d * 4;
    const psa::MapLayout f = psa::map_layout(n_bh, d, nbq, nbk, block);
    const psa::MapBwdLayout b = psa::map_bwd_layout(n_bh, n_kv, d, nbq, nbk, block);
    bool ok = lists(rows, nbk, f.rows, room) && lists(rows, nbk, b.rows, room) && lists(cols, group * nbq, b.cols, room);
    auto order_of = [](size_t at, const Pieces& p) { return Section{at, p.grid * sizeof(int2)}; };
    auto split_of = [](size_t at, const Pieces& p) { return Section{at, p.grid ? (1 + (size_t)p.splits) * sizeof(int4) : 0}; };
    auto counts = [](size_t at, const Pieces& p, size_t n) { return Section{at, p.grid ? 4 * n : 0}; };
    auto tiles = [](const Pieces& p, size_t n, int32_t parts) { return p.grid ? (size_t)p.pieces : parts > 1 ? n * parts : 0; };
    const size_t tf = tiles(f.rows, rows, f.parts), tq = tiles(b.rows, rows, b.parts), tk = tiles(b.cols, cols, b.head_parts * b.list_parts);
    ok = ok && apart({counts(f.row_counts, f.rows, rows), order_of(f.row_order, f.rows), split_of(f.row_split, f.rows),
                      {f.part_o, tf * tile}, {f.part_ml, tf * block * 8}}, f.total);
    const size_t values = (size_t)rows * block * 4;
    ok = ok && apart({{b.neg_lse2, values}, {b.neg_delta, values}, counts(b.row_counts, b.rows, rows), order_of(b.row_order, b.rows),
                      split_of(b.row_split, b.rows), counts(b.col_counts, b.cols, cols), order_of(b.col_order, b.cols),
                      split_of(b.col_split, b.cols), {b.part_q, tq * tile}, {b.part_k, tk * tile}, {b.part_v, tk * tile}}, b.total);
    printf("%d\n", (int)ok);
  }
  fprintf(stderr, "%ld %ld %ld %ld\n", cases, cut_cases, most_splits, most_pieces);
}
"""


def test_no_lists_give_more_pieces_than_the_workspace_holds(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "main.cc", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.run([gxx, "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", build.INCLUDE,
                    "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    rng = np.random.default_rng(5)
    log = lambda hi: int(np.exp(rng.uniform(0, np.log(hi))) + 0.5)
    cases = []
    while len(cases) < 300:
        c = (log(64), log(16), int(rng.choice([64, 128])), log(7936), log(7936), int(rng.choice([64, 128])))
        if c[0] * c[1] * c[3] <= 6000 and c[0] * c[4] <= 6000:
            cases.append(c)
    # a few blocks around the workgroups that share the work, the longest lists, sums past 2^31
    cases += [(n, 1, d, 1, nk, block) for n in (1, 255, 256, 257, 511, 512, 513) for d in (64, 128) for nk in (13, 25)
              for block in (64, 128)]
    cases += [(1, 1, 64, 7936, 7936, 64), (1, 2, 128, 7936, 1, 128), (1, 1, 128, 7936, 600, 128), (1, 400, 128, 40, 40, 128),
              (3, 300, 64, 20, 7936, 64), (1, 512, 128, 1, 7936, 64), (1, 256, 64, 1, 7936, 128)]
    run = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True)
    ok = [int(x) for x in run.stdout.split()]
    assert len(ok) == len(cases) and not [c for c, x in zip(cases, ok) if not x]
    tried, cut, splits, pieces = map(int, run.stderr.split())
    assert tried > 40000 and cut > 10000
    # The lists come near what fits: of more lists than room r shares long, room / r go in floor(2 r + 1) pieces, at most
    # 8 / 3 room (r = 1.5) of 3 room reserved.
    assert splits <= 1000 and 880 <= pieces <= 1000

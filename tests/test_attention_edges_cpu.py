"""CPU tests of the attention calls' edges: the work map over any prefix sums, checked in the code that the kernels
use."""
import os
import subprocess

import pytest

import paper_2506_13771_amd as lb

CSRC = os.path.join(os.path.dirname(lb.LIB_PATH), "csrc")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lb.LIB_PATH):
        from paper_2506_13771_amd import _build
        _build.build()
    return lb.load_library()


MAP = r"""
#include "latent_map.h"
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
using namespace lb;

struct Seq { int64_t q0, nq, items, steps; };

// every slot that the shares of a call are written to: in range, none twice, and an item's as join finds them;
// returns the largest slot and one
static int64_t walk(const std::vector<Seq>& seqs, int step, int64_t slots, bool check) {
  int64_t W = 0, items = 0, most = 0;
  for (auto& s : seqs) W += s.items * s.steps, items += s.items;
  if (W == 0) return 0;
  const int G = groups_of(static_cast<int>(W), step);
  if (G < 1 || G > kG || G > W) { std::printf("G %d of W %lld\n", G, (long long)W); std::exit(1); }
  std::vector<char> used(items + G + 1, 0);
  int64_t x_last = 0;
  for (int g = 0; g < G; ++g) {
    const int64_t x0 = first_step(W, g, G), x1 = first_step(W, g + 1, G);
    if (x0 != x_last || x1 <= x0) { std::printf("share %d\n", g); std::exit(1); }
    x_last = x1;
    for (int64_t x = x0; x < x1;) {
      int64_t sb = 0, ib = 0;
      size_t b = 0;
      while (sb + seqs[b].items * seqs[b].steps <= x) sb += seqs[b].items * seqs[b].steps, ib += seqs[b].items, ++b;
      const int64_t item = (x - sb) / seqs[b].steps, end = sb + (item + 1) * seqs[b].steps, slot = g + ib + item;
      if (slot + 1 > most) most = slot + 1;
      if (check) {
        if (slot >= slots || used[slot]) { std::printf("slot %lld of %lld\n", (long long)slot, (long long)slots); std::exit(1); }
        used[slot] = 1;
        const int g0 = group_of(W, static_cast<int>(end - seqs[b].steps), G), gn = group_of(W, static_cast<int>(end - 1), G);
        if (g < g0 || g > gn) { std::printf("share %d of %d .. %d\n", g, g0, gn); std::exit(1); }
      }
      x = end < x1 ? end : x1;
    }
  }
  if (x_last != W) { std::printf("%lld of %lld steps\n", (long long)x_last, (long long)W); std::exit(1); }
  return most;
}

int main() {
  std::mt19937 rng(7);
  auto below = [&](int n) { return static_cast<int>(rng() % n); };
  int overlapping = 0;
  for (int trial = 0; trial < 600; ++trial) {
    const int T = 1 + below(trial % 3 ? 40 : 3000), H = 1 + below(70), n = 1 + below(trial % 5 ? 9 : 140), kind = trial % 6;
    const int step = 16 << below(4);
    std::vector<int32_t> cu(n + 1), len(n);
    for (int b = 0; b <= n; ++b) {
      switch (kind) {
        case 0: cu[b] = static_cast<int>(static_cast<int64_t>(T) * b / n); break;   // prefix sums
        case 1: cu[b] = b % 2 ? T : 0; break;                                      // rising and falling
        case 2: cu[b] = below(2 * T + 1) - T / 2; break;                            // any
        case 3: cu[b] = b % 2 ? INT32_MAX : INT32_MIN; break;
        case 4: cu[b] = T + 1 + b; break;                                          // all past the end
        default: cu[b] = -1 - b; break;
      }
    }
    for (auto& l : len) l = below(6) ? 1 + below(5000) : 0;
    std::vector<Seq> apart, alone;
    int end = rows_end(0, cu[0], T);
    for (int b = 0; b < n; ++b) {
      const int hi = rows_end(end, cu[b + 1], T);
      if (hi < end || hi > T || end < 0) { std::printf("rows %d .. %d of %d\n", end, hi, T); return 1; }
      const int64_t steps = (len[b] + step - 1) / step;
      apart.push_back({end, hi - end, (static_cast<int64_t>(hi - end) * H + kCols - 1) / kCols, steps});
      end = hi;
      // what sequences would have that are cut to [0, T) each by itself
      const int lo1 = rows_end(0, cu[b], T), hi1 = rows_end(lo1, cu[b + 1], T);
      alone.push_back({lo1, hi1 - lo1, (static_cast<int64_t>(hi1 - lo1) * H + kCols - 1) / kCols, steps});
      if (kind == 0 && (lo1 != apart.back().q0 || hi1 - lo1 != apart.back().nq)) { std::printf("prefix sums\n"); return 1; }
    }
    const int64_t slots = lat_slots(T, n, H);
    walk(apart, step, slots, true);
    if (walk(alone, step, slots, false) > slots) ++overlapping;
  }
  std::printf("%d\n", overlapping);
  return overlapping > 20 ? 0 : 1;  // (the trials reach what the rule is for)
}
"""


def test_work_map_stays_inside_the_workspace(tmp_path):
    src, exe = tmp_path / "map.cpp", str(tmp_path / "map")
    src.write_text(MAP)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(src), "-o", exe],
                   check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr


def test_workspace_holds_every_slot(lib):
    # q' in three terms of two bytes, a factor a row, and a slot's statistics and sums of 32 rows
    for T, n, H, r, dr in ((64, 3, 64, 112, 64), (64, 8, 32, 16, 0), (1, 140, 5, 720, 0), (3000, 1, 7, 33, 16)):
        slots, row, ow = 256 + -(-T * H // 32) + n, lb.lb_latent_row(r, dr), -(-2 * r // 32) * 32
        need = -(-T * H // 32) * 32 * row * 6 + T * H * 4 + slots * 32 * (8 + 4 * ow)
        assert lb.lb_latent_attention_workspace_bytes(T, n, H, r, dr) >= need

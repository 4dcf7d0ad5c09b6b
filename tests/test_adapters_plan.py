"""The rules of the adapters that the host can run: how wavefronts share the slabs of an adapter's rows, and tiles."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_18556_amd", "csrc")


def run(tmp_path, source):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True,
                   capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_every_slab_is_taken_once_and_the_end_stays_the_end(tmp_path):
    """All segments' slabs of 32 rows by 1 to 8 wavefronts, through two places in turn as the sums use them: when a
    wavefront is done, nothing that it asked for is unused."""
    run(tmp_path, r'''
#include <cstdio>
#include <cstdlib>
#include <map>
#include <vector>
#include "gsq_walk.h"
using namespace gsq;
struct Segments {
  const std::vector<int>& rows;
  SlabWalk walk;
  size_t next_segment = 0;
  int64_t before = 0;
  bool next(int64_t& first, int& n, int every) {
    while (!walk.take(32, every, first, n)) {
      if (next_segment == rows.size()) return false;
      before += 1000;                          // segments need not follow one another
      walk.enter(before, before + rows[next_segment]);
      before += rows[next_segment++];
    }
    return true;
  }
};
int main() {
  std::vector<std::vector<int>> cases = {{}, {0}, {0, 0, 0}, {64, 0, 1, 33, 0}, {1, 1, 1, 1, 1, 1, 1, 1, 1}, {31, 32, 33, 0, 640, 1}};
  for (int n = 1; n <= 700; n += n % 32 == 1 || n % 32 == 31 || n % 32 == 0 || n < 70 ? 1 : 5)
    for (const std::vector<int>& more : {std::vector<int>{}, {0, 5}, {256, 0, 0, 100}}) {
      std::vector<int> all{n};
      all.insert(all.end(), more.begin(), more.end());
      cases.push_back(all);
    }
  for (const auto& rows : cases)
    for (int waves = 1; waves <= 8; ++waves) {
      std::map<int64_t, int> want, got;
      int64_t at = 0;
      for (int n : rows) {
        at += 1000;
        for (int k = 0; k < n; k += 32) want[at + k] = n - k < 32 ? n - k : 32;
        at += n;
      }
      for (int w = 0; w < waves; ++w) {
        Segments s{rows, SlabWalk(w)};
        bool waiting[2] = {};
        int64_t first[2];
        int n[2];
        const auto ask = [&](int place) { return waiting[place] = s.next(first[place], n[place], waves); };
        const auto use = [&](int place) {
          if (!waiting[place] || !got.emplace(first[place], n[place]).second) { std::printf("used twice\n"); std::exit(1); }
          return ask(place);
        };
        bool even = ask(0), odd = ask(1);
        while (even) {
          even = use(0);
          if (!odd) break;
          odd = use(1);
        }
        bool bad = waiting[0] || waiting[1];
        int64_t f;
        int r;
        for (int again = 0; again < 20; ++again) bad = bad || s.next(f, r, waves);
        if (bad) { std::printf("asked for and not used: %d rows first, %d waves, wave %d\n", rows[0], waves, w); return 1; }
      }
      if (want != got) { std::printf("not all: %d waves\n", waves); return 1; }
    }
  return 0;
}
''')


def test_chosen_tiles_fit_a_launch(tmp_path):
    """The rule reckons with up to eight wavefronts to a tile; those of 16 x 16 have up to sixteen."""
    run(tmp_path, r'''
#include <cstdio>
#include "gsq_plan.h"
using namespace gsq;
int main() {
  for (int64_t rows = 1; rows <= (int64_t)1 << 29; rows += rows < 64 ? 1 : rows / 19 + 1)
    for (int64_t segments : {1, 2, 3, 16, 100, 1000, 10000, 65535})
      for (int rank : {1, 8, 16, 17, 32, 48, 64, 65, 80, 128, 129, 200, 320, 511, 512})
        for (int slabs : {1, 2, 3, 5, 8, 16, 64, 1000, 32768})
          for (bool tight : {true, false}) {
            const RowsPlan p = plan_adapter(rows, segments, rank, slabs, tight);
            const int waves = std::min(slabs, p.height == 16 && p.width == 16 ? 16 : 8);   // one for each slab at most
            if (p.height && !fits_launch(most_panels(rows, segments, p.height) * tiles_of(rank, p.width), 64 * waves)) {
              std::printf("%lld rows, %lld segments, rank %d\n", (long long)rows, (long long)segments, rank);
              return 1;
            }
          }
  return 0;
}
''')

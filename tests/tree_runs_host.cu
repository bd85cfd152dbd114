// Host code for tests/test_ops_host.py: walks through the runs that the blocks of the tcgen05 kernel of drafted tokens take.
#include <algorithm>
#include <vector>

#include "../paper_2401_06104_b200/csrc/tova_tree_tc.cuh"

namespace {
// A block's run: what the kernel's helper warp finds.
tova::TreeTcRun run_of(const tova::TreeParams& p, int blocks, int block, long long* total_out) {
  const int jobs = p.Hkv * p.row_rounds;
  long long total = 0;
  for (int b = 0; b < p.B; ++b) total += (long long)tova::tree_tc_tiles(p, b) * jobs;
  const long long share = tova::tree_tc_share(total, blocks / p.group, p.least);
  tova::TreeTcRun r{};
  r.at = std::min(total, block / p.group * share);
  r.end = std::min(total, r.at + share);
  r.tiles = tova::tree_tc_tiles(p, 0);
  while (r.at < r.end && r.at >= r.base + (long long)r.tiles * jobs) {
    r.base += (long long)r.tiles * jobs;
    r.tiles = tova::tree_tc_tiles(p, ++r.b);
  }
  r.first = true;
  *total_out = total;
  return r;
}
}  // namespace

// Every tile of every job is in exactly one piece; a job's pieces are the first block's `cut` and what it points at, whether or
// not a wait runs out at some block's piece `fail_at` (-1: none does).  0, or the line where something is wrong.
extern "C" int check_tree_runs(int B, int Hkv, int G, int N, int cap, const int* lens, int n_live, int blocks, int group,
                               int row_rounds, int least, int fail_at) {
  tova::TreeParams p{};
  p.B = B; p.Hkv = Hkv; p.G = G; p.H = Hkv * G; p.N = N; p.M = N * G; p.cap = cap; p.lens = lens; p.n_live = n_live;
  p.group = group; p.row_rounds = row_rounds; p.least = least;
  const int row_blocks = group * row_rounds;
  struct Piece { int block, b, hk, rb, i0, i1, tiles, part; bool last; };
  std::vector<std::vector<Piece>> pieces(blocks);
  std::vector<tova::TreeTcCut> cuts(blocks);
  long long total = 0, seen = 0;
  for (int k = 0; k < blocks; ++k) {
    tova::TreeTcRun r = run_of(p, blocks, k, &total);
    const tova::TreeTcRun start = r;
    while (r.next(p, k)) {
      pieces[k].push_back({k, r.b, r.hk, r.rb, r.i0, r.i1, r.tiles, r.part, r.last});
      seen += r.i1 - r.i0;
    }
    int calls = 0;
    cuts[k] = tova::tree_tc_walk(start, p, k, [&](const tova::TreeTcRun& piece) {
      if (piece.i1 <= piece.n_state) return false;
      return calls++ != fail_at;
    });
    if (fail_at >= 0 && calls > fail_at + 1) return __LINE__;
  }
  if (seen != total * group) return __LINE__;
  std::vector<char> done((size_t)B * Hkv * row_blocks, 0);
  for (int k = 0; k < blocks; ++k) {
    int cut = 0;
    for (const Piece& x : pieces[k]) {
      if (x.rb < 0 || x.rb >= row_blocks || x.hk >= Hkv || x.b >= B) return __LINE__;
      if (x.i0 > 0) continue;                     // found from its job's first piece
      char& d = done[((size_t)x.b * Hkv + x.hk) * row_blocks + x.rb];
      if (d) return __LINE__;
      d = 1;
      if (x.last) {
        if (x.part != -1 || x.i1 != x.tiles) return __LINE__;
        continue;
      }
      if (cut++) return __LINE__;
      const tova::TreeTcCut& c = cuts[k];
      if (c.pieces < 2 || c.b != x.b || c.hk != x.hk || c.rb != x.rb || c.part != x.part) return __LINE__;
      if (x.part != 2 * k && x.part != 2 * k + 1) return __LINE__;
      int at = x.i1;
      for (int i = 1; i < c.pieces; ++i) {
        const int other = k + i * group;
        if (other >= blocks || pieces[other].empty()) return __LINE__;
        const Piece& y = pieces[other][0];
        if (y.b != x.b || y.hk != x.hk || y.rb != x.rb || y.i0 != at || y.part != 2 * other) return __LINE__;
        if (y.last != (i == c.pieces - 1)) return __LINE__;
        at = y.i1;
      }
      if (at != x.tiles) return __LINE__;
    }
    if (!cut && cuts[k].pieces != 0) return __LINE__;
  }
  for (char d : done)
    if (!d) return __LINE__;
  return 0;
}

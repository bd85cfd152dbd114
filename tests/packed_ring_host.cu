// Host code for tests/test_serve_edges_host.py: walks through the places that a block's copies take in the ring of the tcgen05
// kernel of packed prompts.
#include "../paper_2401_06104_b200/csrc/tova_packed_tc.cuh"

// `items` items of copies[i mod n] copies each, beside a count in 64 bits: the slot, its phase and whether it was used before, of
// the first and last 12 copies of every item.  0, or 1 + the item where they differ; *total: the copies passed.
template <int SLOTS>
static long long walk(const int* copies, int n, long long items, long long* total) {
  tova::PackedRing<SLOTS> ring;
  long long at = 0;
  for (long long i = 0; i < items; ++i) {
    const int c = copies[i % n];
    for (int x = 0; x < c; ++x) {
      if (x == 12 && c > 24) x = c - 12;
      const long long pos = at + x;
      if (ring.slot(x) != (int)(pos % SLOTS) || ring.phase(x) != (unsigned)(pos / SLOTS % 2) || ring.again(x) != (pos >= SLOTS)) return i + 1;
    }
    ring.pass(c);
    at += c;
  }
  *total = at;
  return 0;
}

extern "C" long long check_packed_ring(int slots, const int* copies, int n, long long items, long long* total) {
  return slots == tova::PackedTcShape<128>::SLOTS  ? walk<tova::PackedTcShape<128>::SLOTS>(copies, n, items, total)
         : slots == tova::PackedTcShape<64>::SLOTS ? walk<tova::PackedTcShape<64>::SLOTS>(copies, n, items, total)
                                                   : -1;
}

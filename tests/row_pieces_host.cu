// Host program around the reads of rows as 16-byte pieces, for an address sanitizer: every row of 1 to 70 elements of every type,
// at every distance from a 16-byte boundary, its array's last element the row's, and the bytes in front of it forbidden
// as far as they can be (8 at a time). Prints how many pieces were read.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include <sanitizer/asan_interface.h>

#include "mca_rows.cuh"

template <class T>
struct Array {                              // V elements, `off` behind a 16-byte boundary
  char* base;
  T* x;
  int V;
  Array(int V_, int off, int salt) : V(V_) {
    base = static_cast<char*>(std::malloc((size_t)(off + V) * sizeof(T)));
    if (reinterpret_cast<uintptr_t>(base) % 16) std::exit(2);
    x = reinterpret_cast<T*>(base) + off;
    for (int i = 0; i < V; ++i) {
      const unsigned int bits = 0x3c01u + (unsigned int)(i * 7 + salt);
      std::memcpy(x + i, &bits, sizeof(T));
    }
    if (off * sizeof(T) >= 8) ASAN_POISON_MEMORY_REGION(base, 8);
  }
  ~Array() {
    ASAN_UNPOISON_MEMORY_REGION(base, 8);
    std::free(base);
  }
  // Whether q holds the elements from `at` on, -inf outside.
  bool holds(const void* q, int at, int n) const {
    for (int e = 0; e < n; ++e) {
      unsigned int want = sizeof(T) == 4 ? 0xff800000u : none, got = 0;
      if (at + e >= 0 && at + e < V) {
        want = 0;
        std::memcpy(&want, x + at + e, sizeof(T));
      }
      std::memcpy(&got, static_cast<const char*>(q) + e * sizeof(T), sizeof(T));
      if (want != got) return false;
    }
    return true;
  }
  unsigned int none = 0;
};

template <int DT>
long all() {
  using P = mca::Pieces<DT>;
  using T = mca::elem_t<DT>;
  constexpr int N = P::N, es = (int)sizeof(T);
  long n = 0;
  for (int V = 1; V <= 70; ++V)
    for (int off = 0; off < N; ++off) {
      Array<T> a(V, off, 1);
      a.none = DT == MCA_DTYPE_FP16 ? 0xfc00u : 0xff80u;
      const P row(a.x, V);
      if (row.head != off) std::exit(3);
      for (int j = 0; j < row.count; ++j, ++n) {
        const uint4 q = row.bits(j);
        if (!a.holds(&q, row.index(j, 0), N)) std::exit(4);
      }
      // another row of V elements, whose pieces are those of this one
      for (int other = 0; other < N; ++other) {
        Array<T> b(V, other, 2);
        const uintptr_t from = reinterpret_cast<uintptr_t>(b.x - row.head);
        const int by = (int)(from % 16);
        const char* blocks = reinterpret_cast<const char*>(from - by);
        const int lo = mca::first_of_own_blocks(row.head, by, es), hi = mca::end_of_own_blocks(V, row.head, by, es);
        for (int j = 0; j < row.count; ++j) {
          const char* block = blocks + 16 * j;
          const bool own = block >= reinterpret_cast<char*>(b.x) &&
                           block + (by ? 32 : 16) <= reinterpret_cast<char*>(b.x + V);
          if ((j >= lo && j < hi) != own || (own && !row.whole(j))) std::exit(5);
          if (!own) continue;
          uint4 two[2] = {*reinterpret_cast<const uint4*>(block), {}};
          if (by) two[1] = *reinterpret_cast<const uint4*>(block + 16);
          if (!b.holds(reinterpret_cast<const char*>(two) + by, row.index(j, 0), N)) std::exit(6);
          ++n;
        }
      }
    }
  return n;
}

int main() {
  std::printf("%ld\n", all<MCA_DTYPE_FP32>() + all<MCA_DTYPE_FP16>() + all<MCA_DTYPE_BF16>());
  return 0;
}

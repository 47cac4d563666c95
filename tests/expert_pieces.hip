// Addresses that the weight gradient's loaders form, walked on the host: for
// each tile of each expert, each stage and each thread of the kernel's own
// loader, every 16-byte piece has to lie inside the rows that the experts have.
// Prints the first piece that does not and ends with 1.
#include <cstdio>
#include <utility>
#include <vector>

#include "../paper_2609_32398_amd/csrc/expert_gemm.h"

using namespace dol::expert;

namespace {

constexpr uint64_t kBase = 1ull << 44;  // where the operand would lie: no piece is read

// f(0), f(1), .. with constant arguments.
template <int... J, typename F>
void every(std::integer_sequence<int, J...>, F&& f) {
  (f(std::integral_constant<int, J>{}), ...);
}

// One operand, [rows][ld] elements of T, columns in tiles of DIM.
template <typename T, int DIM, int THREADS, bool WIDE>
bool walk(const std::vector<int>& offsets, int ld, const char* what) {
  using Loader = PieceLoader<T, kOuter, DIM, THREADS, WIDE, false>;
  const T* p = reinterpret_cast<const T*>(kBase);
  const uint64_t end = kBase + (uint64_t)offsets.back() * ld * sizeof(T);
  int64_t loaded = 0;
  for (size_t e = 0; e + 1 < offsets.size(); ++e) {
    const int rows = offsets[e + 1] - offsets[e];
    const uint64_t lo = kBase + (uint64_t)offsets[e] * ld * sizeof(T);
    for (int col0 = 0; col0 < ld; col0 += DIM) {
      for (int tid = 0; tid < THREADS; ++tid) {
        const int nk = stages<T>(rows);
        if (nk == 0) continue;  // such a tile is not begun
        Loader l;
        l.start_outer(tid, rows, p + (int64_t)offsets[e] * ld, ld, col0, ld, nullptr, 0, nullptr);
        for (int s = 0; s < nk; ++s) {
          bool ok = true;
          every(std::make_integer_sequence<int, Loader::N>{}, [&](auto j) {
            const uint64_t at = reinterpret_cast<uint64_t>(l.base) +
                                (uint64_t)l.template offset<decltype(j)::value>(tid, 0u, 0u) * (WIDE ? 16 : 1);
            ++loaded;
            if (ok && (at < lo || at + 16 > end)) {
              std::printf("%s: expert %zu of %zu (rows %d to %d), columns from %d, stage %d, thread %d: byte %lld of %lld\n",
                          what, e, offsets.size() - 1, offsets[e], offsets[e + 1], col0, s, tid,
                          (long long)(at - kBase), (long long)(end - kBase));
              ok = false;
            }
          });
          if (!ok) return false;
          l.next(tid);
        }
      }
    }
  }
  std::printf("%s: %zu experts, rows of %d: %lld pieces inside\n", what, offsets.size() - 1, ld, (long long)loaded);
  return true;
}

template <typename T, int DIM, int THREADS>
bool both(const std::vector<int>& offsets, int ld, const char* what) {
  return walk<T, DIM, THREADS, false>(offsets, ld, what) && walk<T, DIM, THREADS, true>(offsets, ld, what);
}

}  // namespace

int main() {
  const std::vector<std::vector<int>> rows = {
      {0, 5, 5},                            // the last expert has none
      {0, 0, 0, 1, 1, 1},                   // only one has, and one row
      {0, 0},                               // nobody has
      {0, 64, 128, 191, 191},               // whole stages, and one row less
      {0, 0, 33, 33, 290, 290, 290},        // none at both ends and in between
      {0, 300, 700},
  };
  bool ok = true;
  for (const auto& o : rows)
    for (int ld : {8, 64, 136, 264}) {
      ok = ok && both<uint16_t, Big::BP, Big::loaders>(o, ld, "bf16, 256 x 256");
      ok = ok && both<uint16_t, Small::BP, Small::loaders>(o, ld, "bf16, 128 x 64, x");
      ok = ok && both<uint16_t, Small::BQ, Small::loaders>(o, ld, "bf16, 128 x 64, dy");
      ok = ok && both<float, Big::BP, Big::loaders>(o, ld, "fp32, 256 x 256");
      ok = ok && both<float, Small::BP, Small::loaders>(o, ld, "fp32, 128 x 64, x");
      ok = ok && both<float, Small::BQ, Small::loaders>(o, ld, "fp32, 128 x 64, dy");
    }
  return ok ? 0 : 1;
}

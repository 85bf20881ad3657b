// Dense softmax attention baseline on the bf16 matrix unit: the shape of a call and its launches.  The kernels are in
// mrt_dense_bf16.hpp.
#include "mrt_dense_bf16.hpp"

#include <algorithm>

namespace mrt {

namespace {

// A call takes as many rounds as its workgroups fill the chip; the shape with the least rounds x cost.
//
// 128 features: a workgroup occupies a compute unit.  A round of 4680 keys costs 61, 79 and 126 us for
// workgroups of 64 (QT = 1, WK = 2), 128 (QT = 2, WK = 2) and 256 (QT = 2) queries (one head of 4680
// tokens 59 | 78 | 122 us, 5 heads 120 | 80 | 123, 12 heads 233 | 159 | 130, 16 heads 294 | 238 | 256).
// Where a mask gives the query tiles different key counts the short ones fill the last round, and the
// largest shape, which reads the keys least often, is taken at 112 (24 heads of 12 one-frame chunks of
// 320 tokens 203 | 173 | 162, 10 heads of 2 chunks of 4680 tokens 575 | 444 | 399, with the tiles head by head, as
// in all figures down to the last paragraph).
//
// 64 features: two workgroups of 64 or 128 queries share a compute unit; a round of up to one per unit
// costs 40 and 57 us, of up to two 54 and 90 (one head of 4680 tokens 38 | 57, 5 heads 53 | 58, 8 heads
// 92 | 87, 16 heads 145 | 134; 40 heads of 1560 tokens 43 | 52).  Workgroups of 256, one per unit, take
// 88 a round: never ahead of 128 by more than 3 %, behind by up to 1.5 x.  Under a mask the workgroups
// count by their share of the longest one's keys (12 heads of 3 chunks of 1040 tokens 50 | 63, 16 heads
// 63 | 64, 32 heads 101 | 98).
//
// Splitting the keys.  Calls of few queries leave most of the chip idle however small their workgroups
// are (one head of 816 queries, 3264 keys: 26 workgroups of 64 queries, 43.6 us), so `parts` workgroups
// share the keys of a query tile and a second launch merges their partial results.  `time` is a model of
// a call fitted to 700 measured shapes of 29 calls (rounds x steps of 64 keys x microseconds a step, the merge
// launch, the partial results' bytes) and, for calls under a mask, to another 1600: there one round lasts as long
// as its longest workgroup, and of several the units that finish early take the next one's workgroups.  A split
// has to promise 6 %: 928 drawn calls that are split so take 0.64 of the unsplit time on average, four of them
// more than that time, up to 1.034.  (Counted as if units could finish early in a single round, 128 features, or as if
// workgroups beyond the last full round cost nothing, 64, calls under a mask took up to 1.43 of the unsplit time.)
// (2 heads of 816 queries of 3264 keys 43.6 -> 19 us, one
// head of 7080 of 21240 244 -> 88, 4 heads of 1989 of 7956 96 -> 49, 6 heads of 7020 of 21060 501 -> 415;
// 64 features: one head of 3240 of 12960 96 -> 30.  No split: 384 keys 10.6 (two parts 12.6), 12 heads of
// 4680 of 4680 132 (155), under a mask 15 heads of 3240 of 6480 172 (201).)
constexpr int kMostParts = 32;
constexpr size_t kMostPartsBytes = (size_t)128 << 20;       // of partial results
constexpr long long kMostSplitRows = 1 << 18;               // 2^18 rows of two parts are more than that

// Under a mask the longest tiles go first, which the figures above do not know: a call then takes as long as its longest
// workgroup, or as all of them on all units and three tenths of the longest (microseconds a step of 64 keys by the number
// of queries; more where all units work at once).  A call that keeps its row statistics goes by that (128 features; us by
// the rule above | by this: 16 heads of 1531 causal tokens sharing 2, batch of 2, 55 | 44, 12 heads of 4096 112 | 83, of 12
// one-frame chunks of 320 102 | 76, 32 heads of 2048 71 | 63, 13 other shapes the same; 64 features would gain 3 % at most);
// dense_attn_fwd keeps its shapes, and with them the last bits of its results.
double masked_time(const KParams& kp, int nbh, int queries, int parts) {
  const double lone = queries == 64 ? 0.71 : queries == 128 ? 1.02 : 1.56, busy = queries == 64 ? 0.85 : queries == 128 ? 1.1 : 1.56;
  const long long first = dense_visible(kp, std::min(queries, kp.Nq) - 1), last = dense_visible(kp, kp.Nq - 1), pairs = (last + 63) / 64;
  const double steps = (double)((pairs + parts - 1) / parts), share = (double)(first + last) / (2 * last);
  const double n = (double)((kp.Nq + queries - 1) / queries) * nbh * parts / compute_units();
  const double joined = parts > 1 ? 5.5 + 1e-6 * 2 * dense_parts_bytes(kp.Nq * nbh, parts, kp.d) / 5.7 : 0.0;
  return 7.5 + steps * (n <= 1 ? lone : std::max(lone, n * share * busy + 0.3 * lone)) + joined;
}

DenseShape dense_shape(const KParams& kp, int nbh, bool may_split, bool save) {
  const long long cus = compute_units(), first = dense_visible(kp, 0), last = dense_visible(kp, kp.Nq - 1);
  auto wgs = [&](int queries) { return (long long)((kp.Nq + queries - 1) / queries) * nbh; };
  DenseShape best;
  if (kp.d == 64) {
    auto cost = [&](int queries, long long one, long long two) {
      const long long n = (wgs(queries) * (first + last) + 2 * last - 1) / (2 * last), rest = n % (2 * cus);
      return n / (2 * cus) * two + (rest > cus ? two : rest > 0 ? one : 0);
    };
    best = {cost(64, 40, 54) < cost(128, 57, 90) ? 64 : 128, 1};
  } else {
    auto cost = [&](int queries, long long unit) { return (wgs(queries) + cus - 1) / cus * unit; };
    const long long c256 = cost(256, first == last ? 126 : 112), c128 = cost(128, 79), c64 = cost(64, 61);
    best = {c64 < c128 && c64 < c256 ? 64 : c128 < c256 ? 128 : 256, 1};
  }
  const bool masked = save && first != last && kp.d == 128;
  if (masked) {
    best.queries = 64;
    for (int queries : {128, 256})
      if (masked_time(kp, nbh, queries, 1) <= masked_time(kp, nbh, best.queries, 1)) best.queries = queries;
  }
  if (!may_split || (long long)kp.Nq * nbh > kMostSplitRows) return best;
  const long long pairs = (last + 63) / 64;
  auto time = [&](int queries, int parts) {
    const double steps = (double)((pairs + parts - 1) / parts), share = (double)(first + last) / (2 * last);
    const long long n = wgs(queries) * parts;
    double us = 0;
    if (kp.d == 64) {
      const double one = queries == 64 ? 0.45 : 0.72, two = queries == 64 ? 0.67 : 1.12;
      const long long rest = n % (2 * cus);
      double full = n / (2 * cus) * two + (rest > cus ? two : rest > 0 ? one : 0);
      if (first != last)
        full = n > 2 * cus ? std::max(two, n * share / (2 * cus) * two + 0.7 * one)
                           : one + (two - one) * std::min(1.0, std::max(0.0, (n - cus) / 64.0));
      us = 6.0 + full * steps;
      if (parts > 1) us += 4.2;
    } else {
      const long long rounds = (n + cus - 1) / cus;
      const double full = first == last ? (double)rounds : std::min((double)rounds, std::max(1.0, n * share / cus + 0.8));
      us = 3.4 + 4.1 * rounds + full * steps * (queries == 64 ? 0.71 : queries == 128 ? 1.02 : 1.56);
      if (parts > 1) us += 5.5;
    }
    const double mb = 1e-6 * 2 * dense_parts_bytes(kp.Nq * nbh, parts, kp.d);      // written, read
    return parts > 1 ? us + mb / (kp.d == 64 ? 3.0 : 5.7) : us;
  };
  const DenseShape one = best;
  // Queries of one run (a workgroup, or its half if it has 256) meet the values of every key that one of
  // them sees, with weights of zero where they don't: an infinite value hidden from some of them shows in
  // them all.  A split takes no run longer than the unsplit call's that a chunk could end inside.
  auto run_ok = [&](int queries) {
    const long long run = std::min(queries, 128);
    return first == last || run <= one.queries || ((long long)kp.cc * kp.hw % run == 0 && (long long)kp.qoff * kp.hw % run == 0);
  };
  double least = (masked ? masked_time(kp, nbh, one.queries, 1) : time(one.queries, 1)) / 1.06;
  for (int queries = 64; queries <= (kp.d == 64 ? 128 : 256); queries *= 2) {
    if (!run_ok(queries)) continue;
    for (int parts = 2; parts <= kMostParts && parts <= pairs; ++parts) {
      if (dense_parts_bytes(kp.Nq * nbh, parts, kp.d) > kMostPartsBytes || wgs(queries) * parts > 6 * cus) break;
      const double us = masked ? masked_time(kp, nbh, queries, parts) : time(queries, parts);
      if (us < least) { least = us; best = {queries, parts}; }
    }
  }
  return best;
}

}  // namespace

DenseShape dense_call_shape(const KParams& kp, int nbh, size_t bytes, bool save) {
  const DenseShape shape = dense_shape(kp, nbh, bytes > 0, save);
  return shape.parts > 1 && bytes < dense_parts_bytes(kp.Nq * nbh, shape.parts, kp.d) ? dense_shape(kp, nbh, false, save) : shape;
}

size_t bf16_dense_workspace_bytes(const KParams& kp, int nbh, bool save) {
  const DenseShape shape = dense_shape(kp, nbh, true, save);
  return shape.parts > 1 ? dense_parts_bytes(kp.Nq * nbh, shape.parts, kp.d) : 0;
}

int bf16_dense_queries(const KParams& kp, int nbh, size_t workspace_bytes, bool save) {
  return dense_call_shape(kp, nbh, workspace_bytes, save).queries;
}

hipError_t launch_bf16_dense(const KParams& kp, int nbh, void* workspace, size_t workspace_bytes, const DenseSave* save, hipStream_t s) {
  const DenseShape shape = dense_call_shape(kp, nbh, workspace ? workspace_bytes : 0, save != nullptr);
  const size_t rows = (size_t)kp.Nq * nbh * shape.parts;
  const bool even = dense_visible(kp, 0) == dense_visible(kp, kp.Nq - 1);
  const DenseParts parts = {(float*)workspace, (float2*)((float*)workspace + rows * kp.d), shape.parts, (unsigned)nbh,
                            even ? 0u : (unsigned)nbh * shape.parts};
  return save ? run_dense_shape(kp, nbh, shape, parts, *save, s) : run_dense_shape(kp, nbh, shape, parts, NoSave{}, s);
}

}  // namespace mrt

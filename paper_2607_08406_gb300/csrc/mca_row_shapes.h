// Which kernel has rows of a size, and how many warps: the rules of the loss against a teacher's list (mca_distill.cu) and of draws
// (mca_draw.cu). Plain C++, so that tests can ask them too.
#pragma once

#include <cstdint>

namespace mca {

constexpr int kSms = 152;
constexpr int kTeamWarps = 8;              // of a CTA that has a row or a part of one
constexpr int kMaxCluster = 8;             // CTAs that have a row

// 16-byte pieces of n elements that a row may have, wherever it starts.
inline int64_t most_pieces(int64_t vocab, int n) { return (vocab + 2 * n - 2) / n; }

// ------------------------------------------------------------------------------------------------
// The loss: a warp with the row in registers, a row in shared memory, CTAs that stay, or a team of warps (or a cluster of
// `split` CTAs) for a row.
// ------------------------------------------------------------------------------------------------
enum class DistillBy { kRegisters, kSharedRow, kStaying, kTeam };

constexpr int kSmallPieces = 256;          // of a row in registers at most: 8 to a lane
constexpr int kRowPieces = 3200;           // of a row in shared memory at most
constexpr int kStreamCtas = 3;             // that stay, per SM
constexpr int64_t kStreamVocab = 1 << 20;  // a thread adds up its terms one after the other: two chains of 2048 then

struct DistillShape {
  DistillBy by;
  int n;                                   // pieces to a lane (kRegisters), or warps
  int split;
};

inline DistillShape distill_shape(int64_t rows, int64_t vocab, int n, bool tail) {
  const int64_t count = most_pieces(vocab, n), bytes = vocab * (16 / n);
  if (count <= 32) return {DistillBy::kRegisters, 1, 1};
  if (count <= 64) return {DistillBy::kRegisters, 2, 1};
  if (count <= 128) return {DistillBy::kRegisters, 4, 1};
  if (count <= kSmallPieces) return {DistillBy::kRegisters, 8, 1};
  if (rows >= 4 * kSms) {
    if (count <= 512) return {DistillBy::kSharedRow, 1, 1};
    if (count <= 1024) return {DistillBy::kSharedRow, 2, 1};
    if (count <= (tail ? kRowPieces : 2048)) return {DistillBy::kSharedRow, 4, 1};
  }
  // CTAs that stay where rows are long enough for one warp to keep up with their lists, and leave few of them without a
  // row at the end (4096 x 128000 179 us -> 162, 2048 x 50001 45 -> 39, 4096 x 32000 fp16 with tail 66 -> 54).
  constexpr int64_t kCtas = kSms * kStreamCtas;
  const int64_t turns = (rows + kCtas - 1) / kCtas;
  if (bytes >= 32768 && vocab <= kStreamVocab && rows >= kCtas * 2 && rows * 100 >= turns * kCtas * 85)
    return {DistillBy::kStaying, kTeamWarps, 1};
  // Else four warps for a row, however many rows there are (4096 x 128000 bf16 329 us with one, 205 with two, 179 with
  // four, 189 with eight; 2048 x 50001 74, 49, 45, 50; 4096 x 32000 fp16 with tail 106, 79, 66, 92; 4000 x 16380 bf16, not
  // long enough for the above, 37 with two, 29 with four), or eight where all rows run at once with these.
  if (rows * kTeamWarps > 32 * kSms) return {DistillBy::kTeam, 4, 1};
  int split = 1;
  while (split < kMaxCluster && rows * split * 2 <= kSms && vocab / (split * 2) >= 2048) split *= 2;
  return {DistillBy::kTeam, kTeamWarps, split};
}

// ------------------------------------------------------------------------------------------------
// Draws. Warps per row: few, so that what a row takes beside its logits is not a warp's all, but as many as run at once (6000
// x 10000 bf16: 147 us with sixteen, 74 with one). A CTA's warps at least where rows are few, or a cluster's CTAs. Rows of a
// round have a kernel of their own, which draws from the steps that it has added up (16384 x 65 bf16 28 us in the others,
// 15 here).
// ------------------------------------------------------------------------------------------------
constexpr int kDrawCtas = 3;               // per SM, of kTeamWarps

struct DrawShape {
  int warps = 1, split = 1;
  bool round;                              // a row has 32 pieces at most, wherever it starts
  DrawShape(int64_t rows, int64_t vocab, int n) : round(most_pieces(vocab, n) <= 32) {
    const int64_t pieces = vocab / n;
    constexpr int64_t kAtOnce = kDrawCtas * kTeamWarps * kSms, kRounds = 8;
    while (warps < kTeamWarps &&
           ((rows * warps < kAtOnce && pieces >= 64 * warps) || pieces >= 32 * 32 * kRounds * warps))
      warps *= 2;
    if (warps == kTeamWarps)
      while (split < kMaxCluster && rows * split * 2 <= kDrawCtas * kSms && pieces / (split * 2) >= 256) split *= 2;
  }
  int64_t grid(int64_t rows) const { return (rows * warps * split + kTeamWarps - 1) / kTeamWarps; }
};

}  // namespace mca

// How the norm's kernels give rows to blocks: rules on sizes alone, for the host.
#pragma once
#include <algorithm>
#include <cstdint>

#include <cuda_runtime.h>

namespace rudra {
namespace {

constexpr uint32_t kPiece = 16;            // values of a row that a thread works on at a time
constexpr uint64_t kMultiprocessors = 148; // of a B200

constexpr uint32_t kMostThreads = 512;
constexpr uint32_t kMostSums = 2 * kMostThreads * kPiece;    // floats of shared memory for the groups' sums
constexpr uint64_t kMostHeld = 2 * kMostThreads * kPiece;    // columns of a row that a block holds in registers: 32 to a thread

// How rows that are held in registers are given to blocks: as many to a block as fill it, and as many blocks as run at once.
// `held`: threads that an SM holds of the kernel.
struct Split {
  uint32_t parts, warps, threads, blocks;
  // most: threads of a block of several rows; held: threads of the kernel that an SM holds; spread: blocks that few rows are given to
  Split(uint64_t rows, uint64_t padded, uint32_t parts_, uint32_t most, uint32_t held, uint64_t spread) : parts(parts_) {
    const uint64_t per_warp = 32 * kPiece * parts;
    warps = (uint32_t)((padded + per_warp - 1) / per_warp);
    // rows that would not fill the SMs otherwise get a block each, or a few to a block
    const uint32_t groups = (uint32_t)std::min<uint64_t>(std::max(1u, most / 32 / warps), (rows + spread - 1) / spread);
    threads = groups * warps * 32;
    blocks = (uint32_t)std::min<uint64_t>((rows + groups - 1) / groups, kMultiprocessors * std::max(1u, held / threads));
  }
  uint32_t length() const { return warps * 32 * kPiece * parts; }     // of a part of the weight's gradient
};

// Blocks of 256 threads, three to an SM, while a row fits one, and more warps where rows lie anyhow and their values are asked for one by
// one (4000 x 4111 bf16 34.6 us with 27 warps to an SM, 44 with 18); 32 values to a thread where a block could not hold a row otherwise.
inline Split forward_split(uint64_t rows, uint64_t padded, bool anyhow) {
  static_assert(kMostHeld <= 1024 * kPiece, "a block holds rows that lie anyhow with 16 values to a thread");
  const uint32_t parts = !anyhow && padded > 768 * kPiece ? 2 : 1;
  return Split(rows, padded, parts, parts == 1 && !anyhow ? padded > 256 * kPiece ? 768 : 256 : 512, parts == 2 ? 512 : anyhow ? 1024 : 768, kMultiprocessors);
}

constexpr uint32_t kMostCluster = 8;      // blocks that add their parts of the weight's gradient themselves
constexpr uint32_t kWideThreads = 640;    // of a block that holds two rows of nine or ten warps
// The gradients of a row in registers: 32 values to a thread where a block could not hold the row otherwise.  Few rows are a
// cluster's.  bf16 rows that lie anyhow (`halves`) are held up by their values one by one: where 16 warps hold one and 20 hold two, 20 are
// faster for all that their threads have fewer registers (4000 x 4111 97 us with 16 and 75 with 20, 3289 x 4999 85 and 69; but 2348 x 7001 69 and 83,
// 4696 x 3501 67 and 79; f32 4000 x 4111 75 and 73, 3651 x 4503 73 and 75).
inline Split backward_split(uint64_t rows, uint64_t cols, bool halves) {
  const uint32_t parts = cols > kMostThreads * kPiece ? 2 : 1;
  const Split few(rows, cols, parts, kMostThreads, kMostThreads, 1);
  if (few.blocks <= kMostCluster) return few;
  const bool wide = halves && parts == 1 && kMostThreads / 32 / few.warps == 1 && kWideThreads / 32 / few.warps == 2;
  const uint32_t most = wide ? kWideThreads : kMostThreads;
  return Split(rows, cols, parts, most, most, kMultiprocessors);
}

constexpr uint32_t kRing = 216 * 1024, kMostSlots = 8;
// Warps that work, and one that copies: forward with 32 values to a thread, backward with 16.
constexpr uint32_t kForwardWarps = 16, kBackwardWarps = 24;

// How rows lie in the ring; host and device.
struct Ring {
  uint32_t matrices, row, pitch, groups, slots;      // bytes of a row, and of its place in a slot
  __host__ __device__ uint32_t slot() const { return groups * matrices * pitch; }
};

// How many rows of bf16 go through rings, if they do: as many groups as leave three slots, and forward 32 values to a thread where
// that still makes twelve warps (backward a thread's sums for the weight take the registers for that).  (f32 rows stay with loads
// by the groups: a warp's 64-byte pieces of shared memory meet in its banks, 8192 x 4096 backward 113 us and 90.)
struct Staged {
  Ring ring = {};
  uint32_t parts = 0, warps = 0, blocks = 0;      // parts 0: not this way
  Staged(uint64_t rows, uint64_t cols, uint32_t element, uint32_t matrices, uint64_t padded, bool backward) {
    if (element != 2 || cols * element % 16) return;
    ring.matrices = matrices;
    ring.row = (uint32_t)(cols * element);
    ring.pitch = (ring.row + 127) / 128 * 128;
    if (ring.pitch * (uint64_t)matrices > kRing / 2) return;
    const uint32_t all = backward ? kBackwardWarps : kForwardWarps, one = (uint32_t)((padded + 511) / 512), two = (uint32_t)((padded + 1023) / 1024);
    const uint32_t most = std::max(1u, kRing / 3 / (ring.pitch * matrices));
    const uint32_t groups1 = one <= all ? std::min(most, all / one) : 0, groups2 = two <= 16 ? std::min(most, 16 / two) : 0;
    const bool wide = !groups1 || (!backward && one != two && groups2 * two >= 12);
    parts = wide ? 2 : 1;
    warps = wide ? two : one;
    const uint32_t groups = std::min(warps > 1 ? 15u : 32u, wide ? groups2 : groups1);      // a barrier each, but for single warps; a lane each
    if (!groups || rows < 3 * kMultiprocessors * groups) parts = 0;       // too few to keep a ring going
    if (!parts) return;
    ring.groups = groups;
    ring.slots = std::min(kMostSlots, kRing / ring.slot());
    blocks = (uint32_t)kMultiprocessors;
  }
  uint32_t threads() const { return ring.groups * warps * 32 + 32; }
  uint32_t length() const { return warps * 32 * kPiece * parts; }
};

}  // namespace
}  // namespace rudra

// Who has been told of the kernels that gave up.  The kernels count them, per device and never back; a stream is told when
// a count is not the one it was last told of, so that no stream's asking takes a report away from another.
#pragma once
#include <array>
#include <cstdint>
#include <map>
#include <mutex>
#include <utility>

namespace rudra {

class Reports {
 public:
  static constexpr int kKernels = 6;   // files that count
  using Counts = std::array<uint32_t, kKernels>;

  // Whether a stream (by its number, which is not given out twice) has not been told of `counts` yet; it now is.
  bool fresh(int device, uint64_t stream, const Counts& counts) {
    std::lock_guard<std::mutex> lock(mutex_);
    const auto at = told_.find({device, stream});
    if (counts == (at == told_.end() ? Counts{} : at->second)) return false;
    told_[{device, stream}] = counts;
    return true;
  }

 private:
  std::mutex mutex_;
  std::map<std::pair<int, uint64_t>, Counts> told_;   // streams without an entry: all zero
};

}  // namespace rudra

// Who has been told of the kernels that gave up.  The kernels count them, per device and never back; a stream is told when
// a count is not the one it was last told of, so that no stream's asking takes a report away from another.
#pragma once
#include <array>
#include <atomic>
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

// Places that calls take while they run, as many as there are.
class Places {
 public:
  static constexpr int kMost = 64;
  // The number of one that is free, now taken; -1: none is.
  int take() {
    uint64_t taken = taken_.load();
    while (~taken) {
      const int i = __builtin_ctzll(~taken);
      if (taken_.compare_exchange_weak(taken, taken | 1ull << i)) return i;
    }
    return -1;
  }
  void give(int i) {
    if (i >= 0) taken_.fetch_and(~(1ull << i));
  }

  // One of them, for as long as it lives.
  struct Place {
    explicit Place(Places& of_) : of(of_), number(of_.take()) {}
    Place(const Place&) = delete;
    ~Place() { of.give(number); }
    Places& of;
    const int number;      // -1: none
  };

 private:
  std::atomic<uint64_t> taken_{0};
};

}  // namespace rudra

// The handles' status words, in plain C++: up to 1024 a device out of one allocation that stays (4 KB), so that making and
// dropping a handle costs no cudaMalloc and cudaFree (13 us instead of 0.8 ms where it is the device's only one).
#pragma once
#include <cstddef>
#include <mutex>

namespace qc {

class StatusWords {
 public:
  static constexpr int kWords = 1024;
  // A word that nobody has, or null where all are taken.  allocate(int** base, bytes) is asked once a device; its error (not 0) is handed back.
  template <typename Allocate>
  auto take(int device, int** word, Allocate&& allocate) -> decltype(allocate(word, size_t())) {
    std::lock_guard<std::mutex> lock(mu_);
    PerDevice& d = per_device_[device & 63];
    *word = nullptr;
    decltype(allocate(word, size_t())) e{};
    if (!d.base) {
      e = allocate(&d.base, kWords * sizeof(int));
      if (e != decltype(e){}) { d.base = nullptr; return e; }
    }
    for (int i = 0; i < kWords && !*word; ++i)
      if (!d.used[i]) { d.used[i] = true; *word = d.base + i; }
    return e;
  }
  // idle: nothing that may write the word is in flight any more.  If that is not known, nobody gets it again: whoever did could be
  // told of another handle's failure.
  void give(int device, int* word, bool idle) {
    if (!idle) return;
    std::lock_guard<std::mutex> lock(mu_);
    PerDevice& d = per_device_[device & 63];
    d.used[word - d.base] = false;
  }

 private:
  struct PerDevice {
    int* base = nullptr;
    bool used[kWords] = {};
  };
  std::mutex mu_;
  PerDevice per_device_[64];
};

}  // namespace qc

// What a kernel needs once on each device before its first launch (no CUDA in here).
#pragma once

#include <atomic>
#include <cstdint>
#include <mutex>
#include <new>

namespace asymspec_impl {

// The kernels prepared so far, as many as there are; looked up without a lock.
class Prepared {
 public:
  // Calls prepare() unless it has returned 0 before for this kernel and device; its result, or 0.
  template <typename F>
  int once(const void* kernel, int device, F prepare) {
    std::atomic<Entry*>& list = lists_[(reinterpret_cast<uintptr_t>(kernel) / 16 + static_cast<unsigned>(device) * 7u) % kLists];
    if (find(list, kernel, device)) return 0;
    std::lock_guard<std::mutex> lock(mutex_);
    if (find(list, kernel, device)) return 0;
    const int status = prepare();
    if (status != 0) return status;
    // (without memory for the entry the next call prepares again)
    Entry* const e = new (std::nothrow) Entry{kernel, device, list.load(std::memory_order_relaxed)};
    if (e) list.store(e, std::memory_order_release);
    return 0;
  }

 private:
  struct Entry {
    const void* kernel;
    int device;
    Entry* next;
  };
  static bool find(const std::atomic<Entry*>& list, const void* kernel, int device) {
    for (const Entry* e = list.load(std::memory_order_acquire); e; e = e->next)
      if (e->kernel == kernel && e->device == device) return true;
    return false;
  }

  static constexpr int kLists = 64;
  std::atomic<Entry*> lists_[kLists] = {};
  std::mutex mutex_;
};

}  // namespace asymspec_impl

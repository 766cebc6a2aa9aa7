// What the library looks up once for each device, for calls from several host threads: the Python calls release the interpreter
// lock, so two threads may make their first call on a device at the same time.  Host code without CUDA headers.
#pragma once
#include <atomic>
#include <mutex>

namespace dq {

constexpr int MAX_DEVICES = 64;

template <typename T>
class PerDevice {
  struct Slot {
    std::atomic<bool> ready{false};
    T value{};
  };
  Slot slots[MAX_DEVICES];
  std::mutex first;

 public:
  // out = device's value, which ask(value) finds out the first time.  ask returns 0, or an error that is returned and not kept.
  // A thread that finds `ready` set sees the whole value: it was set after it (release, acquire).
  template <typename F>
  int get(int device, T& out, F ask) {
    Slot& s = slots[device];
    if (!s.ready.load(std::memory_order_acquire)) {
      std::lock_guard<std::mutex> lock(first);
      if (!s.ready.load(std::memory_order_relaxed)) {
        T value{};
        if (const int error = ask(value)) return error;
        s.value = value;
        s.ready.store(true, std::memory_order_release);
      }
    }
    out = s.value;
    return 0;
  }
};

}  // namespace dq

// A workgroup on the host: one fiber per lane, in one thread.
//
// The lanes of a wave run one after another up to the next point at which they exchange values or meet, and what they
// store until then reaches memory there, after the last of them: loads and stores of one wave keep their program order
// over all of its lanes, as on the device.  Between waves nothing but a barrier orders anything, and that is what is put
// to the test: a wave runs to its next barrier, or to its end, before the wave behind it in `wave_order` starts, so that
// the first of them is as far ahead of the last one as the kernel allows.
#pragma once

#include <setjmp.h>
#include <ucontext.h>

#include <cstdio>
#include <cstdlib>
#include <functional>
#include <memory>
#include <vector>

#include <hip/hip_runtime.h>

dim3 threadIdx, blockIdx, blockDim, gridDim;

namespace fibers {

enum State { kReady, kAtExchange, kAtBarrier, kDone };
struct Store {
  char* p;
  std::vector<char> bytes;
};
struct Lane {
  jmp_buf at;  // where it has stopped (its first entry: a context of its own, whose switch costs a system call)
  ucontext_t context;
  bool entered;
  std::unique_ptr<char[]> stack;
  State state;
  int turn;  // of the exchange buffers
};
constexpr size_t kStack = 64 << 10;

static bool last_wave_first;  // the order of the waves, and of the workgroups
static std::vector<Lane> lanes;
static std::vector<uint32_t> slots[2];
static std::vector<Store> stores;  // of the wave that runs
static jmp_buf scheduler;
static std::function<void()> body;
static long stopped;  // times that a lane has stopped, for the closing line

inline void entry() {
  body();
  lanes[threadIdx.x].state = kDone;
  _longjmp(scheduler, 1);
}
inline void stop(State s) {
  Lane& l = lanes[threadIdx.x];
  ++stopped;
  l.state = s;
  if (_setjmp(l.at) == 0) _longjmp(scheduler, 1);
}
inline void resume(Lane& l) {
  if (_setjmp(scheduler) != 0) return;
  if (l.entered) _longjmp(l.at, 1);
  l.entered = true;
  setcontext(&l.context);
}

// Runs a wave to its next barrier or its end.
inline void run_wave(uint32_t first, uint32_t end) {
  for (;;) {
    for (uint32_t l = first; l < end; ++l)
      if (lanes[l].state == kReady) {
        threadIdx.x = l;
        resume(lanes[l]);
      }
    for (const Store& s : stores) std::memcpy(s.p, s.bytes.data(), s.bytes.size());
    stores.clear();
    bool exchange = false, other = false;
    for (uint32_t l = first; l < end; ++l) (lanes[l].state == kAtExchange ? exchange : other) = true;
    if (!exchange) return;
    if (other) {
      std::printf("lanes of one wave part at an exchange\n");
      std::exit(1);
    }
    for (uint32_t l = first; l < end; ++l) lanes[l].state = kReady;
  }
}

inline void run_workgroup() {
  const uint32_t n = blockDim.x, waves = (n + 63) / 64;
  while (lanes.size() < n) {
    lanes.emplace_back();
    lanes.back().stack.reset(new char[kStack]);
  }
  for (auto& s : slots) s.resize(n);
  for (uint32_t l = 0; l < n; ++l) {
    getcontext(&lanes[l].context);
    lanes[l].context.uc_stack.ss_sp = lanes[l].stack.get();
    lanes[l].context.uc_stack.ss_size = kStack;
    lanes[l].context.uc_link = nullptr;
    makecontext(&lanes[l].context, entry, 0);
    lanes[l].state = kReady;
    lanes[l].turn = 0;
    lanes[l].entered = false;
  }
  for (bool left = true; left;) {
    left = false;
    for (uint32_t i = 0; i < waves; ++i) {
      const uint32_t w = last_wave_first ? waves - 1 - i : i;
      run_wave(w * 64, std::min(n, w * 64 + 64));
    }
    for (uint32_t l = 0; l < n; ++l)  // all that have not ended are at the barrier
      if (lanes[l].state == kAtBarrier) {
        lanes[l].state = kReady;
        left = true;
      }
  }
}

struct Config {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
};
template <typename F>
struct Launch {
  F* f;
  Config c;
  template <typename... A>
  void operator()(A... a) const {
    body = [&] { f(a...); };
    blockDim = c.block;
    gridDim = c.grid;
    for (uint32_t y = 0; y < c.grid.y; ++y)
      for (uint32_t i = 0; i < c.grid.x; ++i) {
        blockIdx = dim3(last_wave_first ? c.grid.x - 1 - i : i, y);
        run_workgroup();
      }
  }
};
template <typename F>
Launch<F> launch(F* f, Config c) {
  return {f, c};
}

}  // namespace fibers

void __syncthreads() { fibers::stop(fibers::kAtBarrier); }
uint32_t lane_read(uint32_t x, uint32_t from) {
  fibers::Lane& l = fibers::lanes[threadIdx.x];
  const uint32_t wave = threadIdx.x / 64 * 64;
  auto& slot = fibers::slots[l.turn];
  l.turn ^= 1;
  slot[threadIdx.x] = x;
  fibers::stop(fibers::kAtExchange);
  return slot[wave + from];
}
void lane_store(void* p, const void* value, size_t n) {
  const char* v = static_cast<const char*>(value);
  fibers::stores.push_back({static_cast<char*>(p), std::vector<char>(v, v + n)});
}

// Runs a grid's work groups one after the other, in any order, and the waves of one in turn for any
// number of steps each: what depends on an order shows by its results.
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <random>
#include <vector>

#include "lanes.hpp"

dim3 blockIdx, threadIdx, gridDim, blockDim;

namespace lanes {

std::mt19937 order;

namespace {

enum State { kReady, kMeeting, kBarrier, kDone };
struct Fiber {
  ucontext_t at;
  std::vector<char> stack;
  State state;
  int site, bytes;
  const void* value;
  Brought got;
};
constexpr int kStack = 1 << 17;
std::vector<Fiber> fibers;
ucontext_t scheduler;
int current, count;
void (*body)(void*);
void* body_args;

void pause() {
  const int me = current;
  swapcontext(&fibers[me].at, &scheduler);
}
void entry() {
  body(body_args);
  fibers[current].state = kDone;
  pause();
}

// Lets every lane of a wave run to its next meeting, barrier or end, and the meeting that comes first
// in the source take place.
bool step(int wave) {
  bool ran = false;
  int site = 0x7fffffff;
  Fiber* const f = &fibers[64 * wave];
  for (int i = 0; i < 64; ++i) {
    if (f[i].state == kReady) {
      current = 64 * wave + i;
      threadIdx = dim3(current);
      swapcontext(&scheduler, &f[i].at);
      ran = true;
    }
    if (f[i].state == kMeeting) site = std::min(site, f[i].site);
  }
  if (site == 0x7fffffff) return ran;
  Brought all;
  all.mask = 0;
  for (int i = 0; i < 64; ++i)
    if (f[i].state == kMeeting && f[i].site == site) {
      memcpy(all.bytes[i], f[i].value, f[i].bytes);
      all.mask |= uint64_t(1) << i;
    }
  for (int i = 0; i < 64; ++i)
    if (all.mask >> i & 1) f[i].got = all, f[i].state = kReady;
  return true;
}

void work_group() {
  for (int i = 0; i < count; ++i) {
    Fiber& f = fibers[i];
    f.stack.resize(kStack);
    getcontext(&f.at);
    f.at.uc_stack.ss_sp = f.stack.data();
    f.at.uc_stack.ss_size = kStack;
    f.at.uc_link = nullptr;
    f.state = kReady;
    makecontext(&f.at, entry, 0);
  }
  std::vector<int> waves;
  for (int w = 0; w < count / 64; ++w) waves.push_back(w);
  for (;;) {
    bool any = false;
    std::shuffle(waves.begin(), waves.end(), order);
    for (int w : waves)
      for (unsigned n = 1 + order() % 40; n > 0; --n) {
        if (!step(w)) break;
        any = true;
      }
    if (any) continue;
    int waiting = 0, done = 0;
    for (int i = 0; i < count; ++i) waiting += fibers[i].state == kBarrier, done += fibers[i].state == kDone;
    if (done == count) return;
    if (done) {
      printf("%d lanes wait at a barrier for %d that have ended\n", waiting, done);
      exit(3);
    }
    for (int i = 0; i < count; ++i) fibers[i].state = kReady;
  }
}

}  // namespace

int lane() { return current & 63; }
const Brought& meet(const void* p, int bytes, int site) {
  Fiber& f = fibers[current];
  f.value = p, f.bytes = bytes, f.site = site, f.state = kMeeting;
  pause();
  return fibers[current].got;
}
void barrier() {
  fibers[current].state = kBarrier;
  pause();
}
void launch(dim3 grid, dim3 block, void (*kernel)(void*), void* args) {
  if (fibers.empty()) fibers.resize(1024);
  gridDim = grid, blockDim = block, count = int(block.x), body = kernel, body_args = args;
  std::vector<dim3> groups;
  for (unsigned y = 0; y < grid.y; ++y)
    for (unsigned x = 0; x < grid.x; ++x) groups.push_back(dim3(x, y));
  std::shuffle(groups.begin(), groups.end(), order);
  for (const dim3& g : groups) {
    blockIdx = g;
    work_group();
  }
}

}  // namespace lanes

// The lanes of hip/hip_runtime.h: fibers on stacks of their own, and buffers between guard pages.
#include <hip/hip_runtime.h>

#include <csetjmp>
#include <map>
#include <string>
#include <sys/mman.h>
#include <ucontext.h>
#include <vector>

namespace {

constexpr size_t kStack = 256 << 10, kPage = 4096, kLdsOfUnit = 160 << 10;

struct Lane {
  void* stack = nullptr;
  jmp_buf at;
  bool started = false, done = false;
};
std::vector<Lane> lanes;
std::vector<Meeting> waves;
int block_arrived, block_turn;
jmp_buf scheduler;
ucontext_t home, fresh;
std::function<void()> kernel_now;
unsigned char* lds_now;
bool from_the_back;
std::string launched;
std::map<unsigned char*, std::pair<unsigned char*, size_t>> mapped;

void pause() {
  const int me = lane_now;
  if (_setjmp(lanes[me].at) == 0) _longjmp(scheduler, 1);
}

void begin() {
  kernel_now();
  lanes[lane_now].done = true;
  _longjmp(scheduler, 1);
}

void resume(int i) {
  lane_now = i;
  if (_setjmp(scheduler) != 0) return;
  if (lanes[i].started) _longjmp(lanes[i].at, 1);
  lanes[i].started = true;
  getcontext(&fresh);
  fresh.uc_stack.ss_sp = lanes[i].stack;
  fresh.uc_stack.ss_size = kStack;
  fresh.uc_link = nullptr;
  makecontext(&fresh, begin, 0);
  setcontext(&fresh);
}

void run_block(int threads) {
  while ((int)lanes.size() < threads) {
    lanes.emplace_back();
    lanes.back().stack = mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
  }
  waves.resize(threads / 64);
  for (Meeting& w : waves) w.arrived = w.turn = 0;
  block_arrived = block_turn = 0;
  for (int i = 0; i < threads; ++i) lanes[i].started = lanes[i].done = false;
  for (bool left = true; left;) {
    left = false;
    for (int k = 0; k < threads; ++k) {
      const int i = from_the_back ? threads - 1 - k : k;
      if (lanes[i].done) continue;
      resume(i);
      left = left || !lanes[i].done;
    }
  }
}

int threads_now;

void meet(int& arrived, int& turn, int count) {
  const int mine = turn;
  if (++arrived == count) arrived = 0, ++turn;
  while (turn == mine) pause();
}

}  // namespace

int lane_now;
dim3 block_now;

hipError_t hipGetLastError() { return hipSuccess; }
Meeting& wave_now() { return waves[lane_now / 64]; }
void wave_meet() {
  Meeting& w = wave_now();
  meet(w.arrived, w.turn, 64);
}
void block_meet() { meet(block_arrived, block_turn, threads_now); }
unsigned char* lanes_lds() { return lds_now; }

// Memory of exactly n bytes (rounded up to what its alignment asks for) that ends, or begins, at a guard page.
extern "C" unsigned char* lanes_alloc(size_t n, size_t alignment, int at_end) {
  const size_t room = (n + kPage - 1) / kPage * kPage + (n == 0 ? kPage : 0);
  unsigned char* base = static_cast<unsigned char*>(
      mmap(nullptr, room + 2 * kPage, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
  mprotect(base, kPage, PROT_NONE);
  mprotect(base + kPage + room, kPage, PROT_NONE);
  memset(base + kPage, 0xff, room);
  unsigned char* p = base + kPage + (at_end ? (room - n) / alignment * alignment : 0);
  mapped[p] = {base, room + 2 * kPage};
  return p;
}
extern "C" void lanes_free(unsigned char* p) {
  munmap(mapped.at(p).first, mapped.at(p).second);
  mapped.erase(p);
}
extern "C" void lanes_order(int back) { from_the_back = back != 0; }
extern "C" const char* lanes_launched() { return launched.c_str(); }  // the launches of the last call of it on, a line each
extern "C" void lanes_forget() { launched.clear(); }

void lanes_launch(const char* what, dim3 grid, dim3 block, size_t lds, hipStream_t, std::function<void()> kernel) {
  if (lds > kLdsOfUnit || block.x % 64 || block.x > 1024 || grid.x == 0 || (uint64_t)grid.x * block.x >= 1ull << 32) abort();
  launched += std::string(what) + " " + std::to_string(grid.x) + " " + std::to_string(block.x) + "\n";
  kernel_now = kernel;
  threads_now = (int)block.x;
  lds_now = lanes_alloc(lds, 16, 1);
  for (unsigned b = 0; b < grid.x; ++b) {
    block_now = dim3(b, 0, 0);
    memset(lds_now, 0xff, lds);  // (what an earlier workgroup left is nobody's business)
    run_block((int)block.x);
  }
  lanes_free(lds_now);
}

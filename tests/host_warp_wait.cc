// warp_wait of csrc/warp_wait.cuh run by 32 threads that stand in for a warp's lanes.  A vote is a barrier of all
// 32: a lane that left on its own would leave the others there.  Prints one line a case: the verdict of every lane
// ('+' or '-'), and which of them gave up ('g', 'L': with its own limit over; '.': not at all).
#include <atomic>
#include <barrier>
#include <cstdio>
#include <functional>
#include <thread>
#include <vector>

#include "warp_wait.cuh"

constexpr int kLanes = 32;

struct Votes {
  std::barrier<> gate{kLanes};
  std::atomic<int> count{0};
  int vote(bool x) {                             // how many lanes say so
    count += x;
    gate.arrive_and_wait();
    const int n = count;
    gate.arrive_and_wait();
    if (x) --count;
    gate.arrive_and_wait();
    return n;
  }
};

struct Lane {
  Votes* votes;
  int lane;
  std::function<bool(int, int)>* ready_at;       // lane, its test's number
  std::function<bool(int)>* sees_flag;
  std::function<uint64_t(int, int)>* clock;      // lane, its reading's number
  char* gave_up;
  int* tests;
  int* reads;
  bool ready() { return (*ready_at)(lane, (*tests)++); }
  bool all(bool x) { return votes->vote(x) == kLanes; }
  bool any(bool x) { return votes->vote(x) > 0; }
  bool gone() { return (*sees_flag)(lane); }
  uint64_t now() { return (*clock)(lane, (*reads)++); }
  void give_up(bool late) { *gave_up = late ? 'L' : 'g'; }
};

void run(const char* name, std::function<bool(int, int)> ready, std::function<bool(int)> flag,
         std::function<uint64_t(int, int)> clock) {
  Votes votes;
  std::vector<char> verdict(kLanes, '?'), gave(kLanes, '.');
  std::vector<std::thread> warp;
  for (int l = 0; l < kLanes; ++l)
    warp.emplace_back([&, l] {
      int tests = 0, reads = 0;
      verdict[l] = lsp::warp_wait(Lane{&votes, l, &ready, &flag, &clock, &gave[l], &tests, &reads}, 100) ? '+' : '-';
    });
  for (auto& t : warp) t.join();
  printf("%s|%.32s|%.32s\n", name, verdict.data(), gave.data());
  fflush(stdout);
}

int main() {
  auto up = [](int) { return true; };
  auto down = [](int) { return false; };
  auto early = [](int, int) { return (uint64_t)7; };
  auto over = [](int, int k) { return (uint64_t)(k ? 1000 : 7); };
  auto at = [](int k) { return [k](int, int n) { return n >= k; }; };
  auto never = [](int, int) { return false; };
  run("complete", at(0), up, over);
  run("complete later", at(20), down, early);
  run("complete after the limit's first look", at(40), down, early);
  run("never", never, down, over);
  run("another role gave up", never, up, early);
  // the limit is over for one lane only, and the others' next test would succeed
  run("one lane late", at(33), down, [](int l, int k) { return (uint64_t)(k && l == 5 ? 1000 : 7); });
  run("one lane sees the flag", at(33), [](int l) { return l == 9; }, early);
  // the last lane to see the barrier complete decides when, also where the others would not see it again
  run("a phase that moves on", [](int l, int n) { return n == (l == 3 ? 12 : l % 5); }, down, early);
  run("all but one lane complete", [](int l, int n) { return l != 31 && n > 2; }, down, over);
}

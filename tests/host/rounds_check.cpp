// Check of the meetings of the warps that fill a ring together
// (csrc/pcs_attend_rounds.h) with a thread per warp: whichever warp's wait runs
// out, and at whichever fill, all of them leave, and none is left waiting at a
// meeting.  Prints "ok" or the first failure.
#include <atomic>
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>
#include <vector>

#include "pcs_attend_rounds.h"

namespace {

constexpr int kWarps = 3;

// Of kWarps threads; a wait for the others has a limit, so that a thread that is
// left alone is found out.
class Meeting {
 public:
  // Whether the others came.
  bool meet() {
    std::unique_lock<std::mutex> l(mu_);
    if (alone_) return false;
    if (++here_ == kWarps) {
      here_ = 0;
      ++round_;
      cv_.notify_all();
      return true;
    }
    const int round = round_;
    if (!cv_.wait_for(l, std::chrono::milliseconds(500), [&] { return round_ != round || alone_; }) || alone_) {
      alone_ = true;
      cv_.notify_all();
      return false;
    }
    return true;
  }

 private:
  std::mutex mu_;
  std::condition_variable cv_;
  int here_ = 0, round_ = 0;
  bool alone_ = false;
};

bool run(int n, int bad_warp, int bad_fill) {
  Meeting meeting;
  std::atomic<bool> left_alone{false};
  bool ok[kWarps] = {};
  int filled[kWarps] = {};
  std::vector<std::thread> warps;
  for (int w = 0; w < kWarps; ++w)
    warps.emplace_back([&, w] {
      ok[w] = pcs::in_rounds(
          n, [&](int i) { return !(w == bad_warp && i == bad_fill); },
          [&] {
            if (!meeting.meet()) left_alone = true;
          },
          [&](int i) { filled[w] += i + 1; });
    });
  for (std::thread& t : warps) t.join();
  const int all = n * (n + 1) / 2;
  bool fine = !left_alone;
  for (int w = 0; w < kWarps; ++w) {
    const bool whole = bad_warp < 0 || bad_fill >= n;
    if (whole) fine = fine && ok[w] && filled[w] == all;
    else fine = fine && ok[w] == (w != bad_warp) && filled[w] == (w == bad_warp ? bad_fill * (bad_fill + 1) / 2 : all);
  }
  if (!fine) std::printf("%d fills, warp %d's wait for fill %d: %s\n", n, bad_warp, bad_fill, left_alone ? "a warp is left waiting" : "wrong fills");
  return fine;
}

}  // namespace

int main() {
  for (int n = 0; n <= 8; n += 2) {
    if (!run(n, -1, 0)) return 1;
    for (int w = 0; w < kWarps; ++w)
      for (int i = 0; i < n; ++i)
        if (!run(n, w, i)) return 1;
  }
  std::puts("ok");
}

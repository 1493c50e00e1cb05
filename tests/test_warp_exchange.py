"""Exchanges between the lanes of a warp, as they stand in the sources, with the lanes as threads of the host."""
from csrc_util import block, run, source

# Lanes as threads; a barrier of the warp is a barrier of theirs, and nothing else orders them.
WARP = """#include <chrono>
#include <condition_variable>
#include <mutex>
#include <thread>
#include <vector>
constexpr int LANES = 32;
struct Barrier {
  std::mutex m;
  std::condition_variable c;
  int waiting = 0, round = 0;
  void wait() {
    std::unique_lock<std::mutex> l(m);
    const int mine = round;
    if (++waiting == LANES) { waiting = 0; ++round; c.notify_all(); }
    else c.wait(l, [&] { return round != mine; });
  }
} barrier;
thread_local int lane = 0;
void __syncwarp() { barrier.wait(); }
template <class F> void warp(F f) {
  std::vector<std::thread> t;
  for (int i = 0; i < LANES; ++i) t.emplace_back([=] { lane = i; f(); });
  for (auto& x : t) x.join();
}
"""


def test_a_slot_cleared_late_does_not_take_the_next_tokens_value():
    """Two tokens in a row whose slots of expert 5 are lane 0's and lane 1's.  Lane 0 comes to its clearing 50 ms after the others."""
    code = block(source("sq_route.cu"), "template <int EPL>\n__device__ __forceinline__ void route_spread(")
    assert code.count("if (put) row[id] = 0.0f;") == 1
    code = code.replace("if (put) row[id] = 0.0f;",
                        "if (put) { if (lane == 0) std::this_thread::sleep_for(std::chrono::milliseconds(50)); row[id] = 0.0f; }")
    rows = run(WARP + code + """
volatile float got[2][32];
float row[32];
int main() {
  warp([] {
    float extra[1];
    route_spread<1>(row, lane == 0, 5, 2.0f, lane, extra);
    got[0][lane] = extra[0];
    route_spread<1>(row, lane == 1, 5, 3.0f, lane, extra);
    got[1][lane] = extra[0];
  });
  for (int t = 0; t < 2; ++t)
    for (int i = 0; i < 32; ++i) printf("%g\\n", got[t][i]);
  for (int i = 0; i < 32; ++i) printf("%g\\n", row[i]);
}""")
    got = [float(r[0]) for r in rows]
    want = [0.0] * 96
    want[5], want[32 + 5] = 2.0, 3.0
    assert got == want


def test_a_warp_of_the_stream_agrees_on_a_landing():
    """One lane runs out of its wait for a landing that the others see: all go on alike (what follows has barriers of the whole warp)."""
    src = source("sq_gemm_gs.cu")
    start = src.index("cp_async_wait<L::DEPTH - 1>();")
    piece = src[start:src.index("__syncwarp();", start)]
    rows = run(WARP + """
struct L { static constexpr int DEPTH = 4; };
enum { GS_FULL = 112 };
template <int N> void cp_async_wait() {}
int votes[LANES];
int __all_sync(unsigned, int v) {
  votes[lane] = v;
  barrier.wait();
  int all = 1;
  for (int i = 0; i < LANES; ++i) all &= votes[i] != 0;
  barrier.wait();
  return all;
}
int late = -1;
bool mbar_wait(uint64_t*, uint32_t, uint32_t, uint32_t) { return lane != late; }
volatile int got[2][32];
int main() {
  for (int t = 0; t < 2; ++t) {
    late = t == 0 ? -1 : 7;
    warp([t] {
      uint64_t full[4] = {};
      int slot = 0;
      uint32_t phase = 0, limit = 100;
      bool ok = true;
      """ + piece + """
      got[t][lane] = ok;
    });
  }
  for (int t = 0; t < 2; ++t)
    for (int i = 0; i < 32; ++i) printf("%d\\n", got[t][i]);
}""")
    assert [int(r[0]) for r in rows] == [1] * 32 + [0] * 32

// Buffers of the scratch pool whose address a captured graph holds, on the fake runtime of fake_cuda/: they must outlive any
// later growth of their lease. Prints the first failed check and exits 1, or "ok".
#include <cuda_runtime.h>

#include "scratch_pool.h"

#define CHECK(x)                                      \
  do {                                                \
    if (!(x)) {                                       \
      std::printf("line %d: %s\n", __LINE__, #x);     \
      return 1;                                       \
    }                                                 \
  } while (0)

namespace {

cudaStream_t stream(int i) { return reinterpret_cast<cudaStream_t>((size_t)i * 16); }

struct Buffers {
  void *ws, *pack;
};
Buffers call(scratch::Pool& pool, cudaStream_t s, size_t ws, size_t pack) {
  scratch::Hold hold(pool, s);
  Buffers b{nullptr, nullptr};
  if (pack) b.pack = hold.pack_buffer(pack);
  if (ws) b.ws = hold.workspace(ws);
  return b;
}
Buffers captured(scratch::Pool& pool, cudaStream_t s, size_t ws, size_t pack) {
  fake::capturing.insert(s);
  const Buffers b = call(pool, s, ws, pack);
  fake::capturing.erase(s);
  return b;
}
bool alive(void* p) { return fake::live.count(p) == 1; }

// `others`: a second stream has been seen before, so that the pool records events.
int run(bool others) {
  fake::live.clear();
  fake::mallocs = fake::frees = fake::syncs = fake::bad = 0;
  scratch::Pool pool;
  if (others) {
    call(pool, stream(7), 10, 10);
    call(pool, stream(8), 10, 10);
  }
  const cudaStream_t s = stream(1);
  // growth without a graph gives the smaller buffer back
  call(pool, s, 1000, 1000);
  call(pool, s, 2000, 2000);
  CHECK(fake::bad == 0);
  const size_t plain = fake::live.size();
  call(pool, s, 3000, 4000);
  CHECK(fake::live.size() == plain);
  // a captured call takes what its lease holds
  const Buffers eager = call(pool, s, 3000, 4000), graph = captured(pool, s, 3000, 4000);
  CHECK(graph.ws == eager.ws && graph.pack == eager.pack);
  // a later, larger call gets another buffer, and the graph's stays
  const Buffers large = call(pool, s, 100000, 100000);
  CHECK(large.ws && large.pack && large.ws != graph.ws && large.pack != graph.pack);
  CHECK(alive(graph.ws) && alive(graph.pack) && alive(large.ws) && alive(large.pack));
  // growth after that is ordinary again
  const Buffers larger = call(pool, s, 200000, 200000);
  CHECK(!alive(large.ws) && !alive(large.pack) && alive(graph.ws) && alive(graph.pack));
  // a second graph on the larger buffers, and one more growth
  const Buffers graph2 = captured(pool, s, 50, 50);
  CHECK(graph2.ws == larger.ws && graph2.pack == larger.pack);
  call(pool, s, 400000, 400000);
  CHECK(alive(graph.ws) && alive(graph.pack) && alive(graph2.ws) && alive(graph2.pack));
  // a captured call that needs more than there is is refused and leaves the capture and the buffers alone
  const int syncs = fake::syncs;
  const Buffers none = captured(pool, s, 900000, 900000);
  CHECK(none.ws == nullptr && none.pack == nullptr && fake::syncs == syncs && fake::bad == 0);
  const Buffers after = call(pool, s, 10, 10);
  CHECK(after.ws && after.pack && alive(after.ws) && alive(after.pack));
  // everything comes back in the end, once
  CHECK(scratch::release_all(pool));
  CHECK(fake::live.empty() && fake::bad == 0 && fake::mallocs == fake::frees);
  CHECK(cudaGetLastError() == cudaSuccess);
  const Buffers fresh = call(pool, s, 100, 100);
  CHECK(alive(fresh.ws) && alive(fresh.pack));
  CHECK(scratch::release_all(pool) && fake::live.empty());
  return 0;
}

}  // namespace

int main() {
  if (run(false) || run(true)) return 1;
  std::printf("ok\n");
  return 0;
}

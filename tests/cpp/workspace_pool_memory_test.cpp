// CPU: the scratch-buffer pool when the host has no memory for its list of buffers.  Nothing is thrown, nothing
// allocated on the device, and the pool works on afterwards.  Prints "ok" or the first failed expectation.
#include <stdio.h>
#include <stdlib.h>

#include <new>

#include "../../paper_2608_10103_b200/csrc/workspace_pool.h"

static bool g_no_memory = false;
void* operator new(size_t n) {
  if (g_no_memory) throw std::bad_alloc();
  if (void* p = malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

static int g_live = 0, g_events = 0;
struct Backend {
  using Stream = int;
  using Event = int;
  int alloc(void** p, size_t bytes, Stream) { return ++g_live, *p = malloc(bytes), 0; }
  int free_after(void* p, Stream) { return --g_live, free(p), 0; }
  int free_now(void* p) { return free_after(p, 0); }
  int event_create(Event* e) { return *e = ++g_events, 0; }
  void event_destroy(Event) {}
  int event_record(Event, Stream) { return 0; }
  bool event_done(Event) { return false; }
  bool capturing(Stream) { return false; }
  int clear(void*, size_t, Stream) { return 0; }
};
using Pool = b200gemm::WorkspacePool<Backend>;

#define EXPECT(x) \
  do { \
    if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } \
  } while (0)

int main() {
  Pool pool;
  Pool::Lease held[64], l;
  int n = 0;
  g_no_memory = true;
  EXPECT(pool.acquire(0, 256, 0, &l) == Pool::kNoHostMemory);
  EXPECT(g_live == 0 && g_events == 0);
  g_no_memory = false;
  for (; n < 40; ++n) {  // whatever room the list has: sooner or later it must grow
    g_no_memory = true;
    const int rc = pool.acquire(n, 256, 0, &held[n]);
    g_no_memory = false;
    EXPECT(rc == 0 || rc == Pool::kNoHostMemory);
    if (rc != 0) {
      EXPECT(g_live == n && pool.buffers() == static_cast<size_t>(n));
      EXPECT(pool.acquire(n, 256, 0, &held[n]) == 0);
    }
    EXPECT(g_live == n + 1);
  }
  while (n--) EXPECT(pool.release(held[n], n) == 0);
  EXPECT(pool.release_all() == 0 && g_live == 0);
  puts("ok");
}

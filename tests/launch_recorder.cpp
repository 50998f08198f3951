// Stands in for the HIP runtime's launch and last-error functions, so that a process without a GPU can see
// which launches a call of the library makes, and what it does where one of them fails. Nothing is executed.
// Loaded into a process of its own before the library (RTLD_GLOBAL).
#include <cstdint>
#include <cstring>

struct Dim3 {
  uint32_t x, y, z;
};
struct Launch {
  Dim3 grid, block;
};

namespace {

constexpr int kMost = 256;
constexpr int kInvalidConfiguration = 9, kOutOfResources = 701;  // hipError_t
Launch g_launch[kMost];
int g_n = 0, g_fail_at = -1, g_last = 0;
struct {
  Dim3 grid, block;
  size_t shared;
  void* stream;
} g_config;

bool too_large(uint32_t n, uint32_t threads) { return (uint64_t)n * threads >= (1ull << 32); }

}  // namespace

extern "C" {

int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t shared, void* stream) {
  g_config = {grid, block, shared, stream};
  return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* shared, void** stream) {
  *grid = g_config.grid;
  *block = g_config.block;
  *shared = g_config.shared;
  *stream = g_config.stream;
  return 0;
}
int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void**, size_t, void*) {
  const int i = g_n++;
  if (i < kMost) g_launch[i] = {grid, block};
  int rc = 0;
  if (i == g_fail_at) rc = kOutOfResources;
  else if (too_large(grid.x, block.x) || too_large(grid.y, block.y) || too_large(grid.z, block.z))
    rc = kInvalidConfiguration;  // as the runtime refuses it
  if (rc) g_last = rc;
  return rc;
}
int hipPeekAtLastError() { return g_last; }
int hipGetLastError() {
  const int rc = g_last;
  g_last = 0;
  return rc;
}

// Forgets the launches so far; the fail_at-th from now on fails (negative: none).
void recorder_reset(int fail_at) {
  g_n = g_last = 0;
  g_fail_at = fail_at;
}
int recorder_launches(Launch* out, int most) {
  memcpy(out, g_launch, sizeof(Launch) * (g_n < most ? g_n : most));
  return g_n;
}

}

// Host code of the update side's operators against a recording stand-in for the HIP runtime: what every launch of a call
// asks for, without a GPU.
#include "embedding.hip"
#include "logprobs.hip"
#include "policy_loss.hip"

namespace {
int g_launches;
uint64_t g_most;  // threads of a dimension of a launch
bool g_bad;       // an empty launch, or one that HIP would refuse
dim3 g_grid, g_block;
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* module;
  return &module;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t*, hipStream_t*) {
  *grid = g_grid;
  *block = g_block;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  const uint64_t x = (uint64_t)grid.x * block.x, y = (uint64_t)grid.y * block.y, z = (uint64_t)grid.z * block.z;
  g_most = std::max(g_most, std::max(x, std::max(y, z)));
  g_bad |= !x || !y || !z || x >> 32 || y >> 16 || z >> 16 || block.x > 1024;
  ++g_launches;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }

int launches() { return g_launches; }
uint64_t most_threads() { return g_most; }

// 0: all launches of the call can be made.  Nothing is dereferenced here.
static int done() { return g_bad; }
static void begin() {
  g_launches = 0;
  g_most = 0;
  g_bad = false;
}
int embedding_backward(int n, int vocab, int dim, int bf16, int accumulate) {
  begin();
  char x[16];
  rollout::launch_embedding_backward(nullptr, bf16, bf16, {x, (int32_t*)x, n, vocab, dim, 1.f, accumulate != 0, x}, x);
  return done();
}
int embedding(int n, int vocab, int dim) {
  begin();
  char x[16];
  rollout::launch_embedding(nullptr, 0, 0, {x, vocab, dim, (int32_t*)x, n, 1.f, x});
  return done();
}
int logprobs(int rows, int vocab, int top, int bf16) {
  begin();
  char x[16];
  float* f = (float*)x;
  rollout::launch_logprobs(nullptr, bf16, {x, vocab, rows, vocab, 1.f, (int32_t*)x, top, f, f, f, (int32_t*)x, f}, x);
  return done();
}
int logprobs_backward(int rows, int vocab, int bf16) {
  begin();
  char x[16];
  float* f = (float*)x;
  rollout::launch_logprobs_backward(nullptr, bf16, {x, vocab, rows, vocab, 1.f, (int32_t*)x, f, f, f, f, x, vocab});
  return done();
}
int policy_loss(int seqs, int max_len, int mean) {
  begin();
  char x[16];
  float* f = (float*)x;
  rollout::launch_policy_loss(nullptr, {f, f, f, f, f, (int32_t*)x, seqs, max_len, 0.2f, 0.2f, 0.f, 0.f, mean, f, f, f, f}, x);
  return done();
}
}

// A recording stand-in for the HIP runtime under the host code of the layers' operators: what every launch of a call asks for,
// without a GPU.  Linked with the operators' own sources.
#include "update.h"

namespace {
int g_launches;
bool g_bad;  // an empty launch, or one that HIP would refuse
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
  g_bad |= !x || !y || !z || x >> 32 || y >> 16 || z >> 16 || block.x > 1024;
  ++g_launches;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }

int launches() { return g_launches; }
static void begin() { g_launches = 0, g_bad = false; }

static rollout::AttentionArgs shape(int heads, int kv, int hd, int seqs, int n_q, int n_k, int causal) {
  rollout::AttentionArgs a = {};
  a.heads = heads, a.kv_heads = kv, a.head_dim = hd, a.n_seqs = seqs, a.n_q = n_q, a.n_k = n_k, a.causal = causal != 0, a.scale = 1.f;
  return a;
}
// 0: all launches of the call can be made.  Nothing is dereferenced here.
int attention(int bf16, int heads, int kv, int hd, int seqs, int n_q, int n_k, int causal) {
  begin();
  char x[16];
  rollout::launch_packed_attention(nullptr, bf16, shape(heads, kv, hd, seqs, n_q, n_k, causal), x);
  return g_bad;
}
int attention_backward(int bf16, int heads, int kv, int hd, int seqs, int n_q, int n_k, int causal) {
  begin();
  char x[16];
  rollout::AttentionGradArgs a = {};
  static_cast<rollout::AttentionArgs&>(a) = shape(heads, kv, hd, seqs, n_q, n_k, causal);
  rollout::launch_packed_attention_backward(nullptr, bf16, a, x);
  return g_bad;
}
int norm(int rows, int dim, int x, int delta, int y) {
  begin();
  char c[16];
  rollout::NormArgs a = {c, delta < 0 ? nullptr : c, nullptr, rows, dim, 1e-6f, c, c, nullptr, nullptr};
  rollout::launch_rms_norm(nullptr, x, delta, y, a);
  return g_bad;
}
int norm_backward(int rows, int dim, int dgain) {
  begin();
  char c[16];
  rollout::NormGradArgs a = {c, c, nullptr, (float*)c, rows, dim, nullptr, c, dgain ? (float*)c : nullptr, 0};
  rollout::launch_rms_norm_backward(nullptr, 0, 0, 0, a, c);
  return g_bad;
}
int adamw(int tensors, int64_t chunks) {
  begin();
  rollout::launch_adamw(nullptr, nullptr, tensors, chunks, {});
  return g_bad;
}
}

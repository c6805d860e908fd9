// Attention of one new token per request over a paged K/V cache.
// (Beyond the paper, whose queries come a chunk at a time.)
#include "pafu_internal.h"

namespace pafu {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float widen(const char* p, int i, bool codes) {
  if (codes) return __builtin_amdgcn_cvt_f32_fp8(reinterpret_cast<const unsigned char*>(p)[i], 0);
  return __uint_as_float((unsigned)reinterpret_cast<const unsigned short*>(p)[i] << 16);
}

// One wave per (request, query head): tokens one after the other, lane l holds D / 64 neighbouring elements of the row.
__global__ __launch_bounds__(64) void paged_attention_kernel(PagedAttention a, PagedPool pool) {
  const int b = blockIdx.x / a.N, h = blockIdx.x % a.N, kvh = h / (a.N / a.N_kv), lane = threadIdx.x;
  const bool codes = a.kv_dtype == PAFU_FP8_E4M3;
  const int per = a.D / 64;
  const long long most = (long long)a.max_pages << pool.page_log2;
  const int len = (int)min((long long)max(a.kv_len[b], 0), most);
  const int lo = a.window > 0 ? max(a.kv_len[b] - a.window, 0) : 0;
  float q[2] = {0.f, 0.f}, o[2] = {0.f, 0.f}, m = -3e38f, l = 0.f;
  const char* qp = static_cast<const char*>(a.Q) + b * a.ld_q + (long long)h * a.D * 2;
  for (int e = 0; e < per; ++e) q[e] = widen(qp, lane * per + e, false);
  for (int j = 0; j < len; ++j) {
    if (j >= a.n_pinned && j < lo) continue;
    const int page = a.table[b * a.ld_table + (j >> pool.page_log2)];
    if (page < 0 || page >= pool.n_pages) continue;
    const long long at = page * pool.ld_page + (j & ((1 << pool.page_log2) - 1)) * pool.ld_token + kvh * pool.ld_head;
    float s = 0.f;
    for (int e = 0; e < per; ++e) s += q[e] * widen(pool.K + at, lane * per + e, codes);
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    s *= a.scale * a.k_scale * kLog2e;
    const float up = fmaxf(m, s), w = __builtin_amdgcn_exp2f(s - up), down = __builtin_amdgcn_exp2f(m - up);
    m = up;
    l = l * down + w;
    for (int e = 0; e < per; ++e) o[e] = o[e] * down + w * widen(pool.V + at, lane * per + e, codes);
  }
  const float inv = l == 0.f ? 0.f : a.v_scale / l;
  char* op = static_cast<char*>(a.O) + b * a.ld_o;
  for (int e = 0; e < per; ++e) {
    const int at = h * a.D + lane * per + e;
    if (a.out_dtype == PAFU_F32) reinterpret_cast<float*>(op)[at] = o[e] * inv;
    else reinterpret_cast<__bf16*>(op)[at] = (__bf16)(o[e] * inv);
  }
}

}  // namespace

size_t paged_attention_workspace_bytes(int B, int N, int N_kv, int D) {
  (void)B; (void)N; (void)N_kv; (void)D;
  return 0;
}

int launch_paged_attention(hipStream_t st, const PagedAttention& a, const PagedPool& pool, void* workspace,
                           size_t workspace_bytes) {
  (void)workspace; (void)workspace_bytes;
  hipLaunchKernelGGL(paged_attention_kernel, dim3((unsigned)(a.B * a.N)), dim3(64), 0, st, a, pool);
  return check_launch();
}

}  // namespace pafu

// Paged K/V cache: block tables and slot maps from request lengths, and rows into the pages.
// (Beyond the paper, whose cache belongs to one video.)
#include "pafu_internal.h"
#include "quant_body.h"

namespace pafu {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

constexpr int kTableThreads = 256, kTableWaves = kTableThreads / 64;

// a + b for non-negative a and b, at most 2^31 - 1
__device__ __forceinline__ int sat_add(int a, int b) {
  const unsigned s = (unsigned)a + (unsigned)b;
  return s > 0x7fffffffu ? 0x7fffffff : (int)s;
}

// Slots (and, with TAKE, pages) for `count` tokens of each request from its token `start` on.
//   rows: exclusive prefix sums of count -> row_start          pages: of want - have, from *free_start on -> first
// Every workgroup forms both sums of all requests by itself (B values from L2; there is no second launch and nothing to
// wait for) and then takes its part of the slots, four neighbouring ones per thread, whose requests it finds by bisection
// in LDS.  A request's first new page is entered by the thread that summed it, further ones by the waves in turn.
template <bool TAKE>
__global__ __launch_bounds__(kTableThreads) void paged_tables_kernel(PagedTables t) {
  extern __shared__ int lds[];
  int* rows = lds;             // [B + 1]
  int* first = lds + t.B + 1;  // [B + 1] (TAKE)
  __shared__ int wave_rows[2][kTableWaves], wave_pages[2][kTableWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int page_mask = (1 << t.page_log2) - 1;
  int row_at = 0, page_at = TAKE && t.free_start ? *t.free_start : 0;
  if (page_at < 0) page_at = 0;
  for (int base = 0, side = 0; base < t.B; base += kTableThreads, side ^= 1) {
    const int b = base + tid;
    int n = 0, have = 0, total = 0, need = 0;
    if (b < t.B) {
      n = max(t.count[b], 0);
      const int s = max(t.start[b], 0);
      total = sat_add(s, n);
      have = (s >> t.page_log2) + ((s & page_mask) != 0);
      need = max((total >> t.page_log2) + ((total & page_mask) != 0) - have, 0);
    }
    int in_rows = n, in_pages = need;  // inclusive sums
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int r = __shfl_up(in_rows, d), p = __shfl_up(in_pages, d);
      if (lane >= d) {
        in_rows = sat_add(in_rows, r);
        in_pages = sat_add(in_pages, p);
      }
    }
    if (lane == 63) {
      wave_rows[side][wave] = in_rows;
      wave_pages[side][wave] = in_pages;
    }
    __syncthreads();
    int before_rows = row_at, before_pages = page_at;
#pragma unroll
    for (int w = 0; w < kTableWaves; ++w) {
      if (w == wave) {
        before_rows = row_at;
        before_pages = page_at;
      }
      row_at = sat_add(row_at, wave_rows[side][w]);
      page_at = sat_add(page_at, wave_pages[side][w]);
    }
    // the exclusive sum is the lower lane's inclusive one
    int ex_rows = __shfl_up(in_rows, 1), ex_pages = __shfl_up(in_pages, 1);
    ex_rows = sat_add(before_rows, lane ? ex_rows : 0);
    ex_pages = sat_add(before_pages, lane ? ex_pages : 0);
    if (b < t.B) {
      rows[b] = ex_rows;
      if (TAKE) first[b] = ex_pages;
      if (blockIdx.x == 0) {
        t.row_start[b] = ex_rows;
        if (TAKE) {
          t.kv_len_out[b] = total;
          if (need > 0 && have < t.max_pages)
            t.table[b * t.ld_table + have] = ex_pages < t.n_free ? t.free_pages[ex_pages] : -1;
        }
      }
    }
  }
  if (tid == 0) {
    rows[t.B] = row_at;
    if (TAKE) first[t.B] = page_at;
    if (blockIdx.x == 0) {
      t.row_start[t.B] = row_at;
      if (TAKE) *t.free_end = page_at;
    }
  }
  __syncthreads();

  if (TAKE) {
    // pages after a request's first new one: request by request, a request's columns over `parts` waves
    const int waves = gridDim.x * kTableWaves, id = blockIdx.x * kTableWaves + wave;
    const int parts = max(waves / t.B, 1);
    for (int job = id; job < t.B * parts; job += waves) {
      const int b = job % t.B, part = job / t.B;
      const int need = first[b + 1] - first[b];
      if (need <= 1 + part * 64) continue;
      const int s = max(t.start[b], 0);
      const int have = (s >> t.page_log2) + ((s & page_mask) != 0);
      const int in_table = min(need, t.max_pages - have);
      for (int i = 1 + part * 64 + lane; i < in_table; i += parts * 64) {
        const int at = sat_add(first[b], i);
        t.table[b * t.ld_table + have + i] = at < t.n_free ? t.free_pages[at] : -1;
      }
    }
  }

  const long long stride = (long long)gridDim.x * kTableThreads * 4;
  for (long long i0 = ((long long)blockIdx.x * kTableThreads + tid) * 4; i0 < t.max_slots; i0 += stride) {
    int b = 0, hi = t.B;  // the last request whose first row is at or before i0
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (rows[mid] <= i0) b = mid;
      else hi = mid;
    }
    int slot[4], page = -1, page_b = -1, s = 0, have = 0;
    unsigned page_col = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = (int)min(i0 + e, (long long)t.max_slots - 1);
      slot[e] = -1;
      if (i >= row_at) continue;
      while (i >= rows[b + 1]) ++b;
      if (b != page_b) {
        s = max(t.start[b], 0);
        have = TAKE ? (s >> t.page_log2) + ((s & page_mask) != 0) : 0x7fffffff;
      }
      const unsigned token = (unsigned)s + (unsigned)(i - rows[b]), col = token >> t.page_log2;
      if (b != page_b || col != page_col) {
        page = -1;
        if (col < (unsigned)t.max_pages) {
          if ((int)col < have) {
            page = t.table[b * t.ld_table + col];
          } else {
            const int nth = (int)col - have, at = sat_add(first[b], nth);
            if (nth < first[b + 1] - first[b] && at < t.n_free) page = t.free_pages[at];
          }
        }
        page_b = b;
        page_col = col;
      }
      if (page >= 0 && page <= (0x7fffffff >> t.page_log2)) slot[e] = (page << t.page_log2) + (int)(token & page_mask);
    }
    if (i0 + 4 <= t.max_slots) {
      *reinterpret_cast<int4*>(t.slots + i0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
      for (int e = 0; i0 + e < t.max_slots; ++e) t.slots[i0 + e] = slot[e];
    }
  }
}

// Rows of K and V to their slots, 8 elements (16 bytes) of each per thread and turn, as bf16 or as E4M3 codes.
struct AppendShape {
  int rows, chunks, head_log2;  // 8-element chunks of a row, log2 of those of a head
  int step_r, step_c;           // the grid's stride in rows and chunks
  long long ld_in;
};
template <bool CODES>
__global__ __launch_bounds__(256) void paged_append_kernel(const char* __restrict__ K, const char* __restrict__ V,
                                                           const int* __restrict__ slots, AppendShape a, PagedPool pool,
                                                           float inv_k, float inv_v) {
  const unsigned i = blockIdx.x * 256u + threadIdx.x;
  int r = i / (unsigned)a.chunks, c = i - (unsigned)r * a.chunks;
  while (r < a.rows) {
    const int slot = slots[r];
    const int page = slot >> pool.page_log2;
    if (slot >= 0 && page < pool.n_pages) {
      const long long src = r * a.ld_in + c * 16ll;
      const long long dst = page * pool.ld_page + (slot & ((1 << pool.page_log2) - 1)) * pool.ld_token +
                            (c >> a.head_log2) * pool.ld_head + (c & ((1 << a.head_log2) - 1)) * (CODES ? 8ll : 16ll);
      const u32x4 in[2] = {*reinterpret_cast<const u32x4*>(K + src), *reinterpret_cast<const u32x4*>(V + src)};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        char* to = const_cast<char*>(x ? pool.V : pool.K) + dst;
        if (CODES) {
          const unsigned words[4] = {in[x][0], in[x][1], in[x][2], in[x][3]};
          unsigned codes[2];
          e4m3_codes8(words, x ? inv_v : inv_k, codes);
          *reinterpret_cast<u32x2*>(to) = u32x2{codes[0], codes[1]};
        } else {
          *reinterpret_cast<u32x4*>(to) = in[x];
        }
      }
    }
    r += a.step_r;
    c += a.step_c;
    if (c >= a.chunks) { c -= a.chunks; ++r; }
  }
}

}  // namespace

int launch_paged_tables(hipStream_t st, const PagedTables& t, bool take_pages) {
  // a workgroup per 1024 slots, at most two per compute unit: each forms the sums of all requests
  long long blocks = ((long long)t.max_slots + kTableThreads * 4 - 1) / (kTableThreads * 4);
  const long long most = 2ll * compute_units();
  blocks = blocks < 1 ? 1 : (blocks > most ? most : blocks);
  const size_t lds = (size_t)(t.B + 1) * 4 * (take_pages ? 2 : 1);
  if (take_pages)
    hipLaunchKernelGGL(paged_tables_kernel<true>, dim3((unsigned)blocks), dim3(kTableThreads), lds, st, t);
  else
    hipLaunchKernelGGL(paged_tables_kernel<false>, dim3((unsigned)blocks), dim3(kTableThreads), lds, st, t);
  return check_launch();
}

int launch_paged_append(hipStream_t st, const void* K, const void* V, long long ld_in_bytes, int rows, const int* slots,
                        int N, int D, const PagedPool& pool, int kv_dtype, int k_scale_log2, int v_scale_log2) {
  AppendShape a;
  a.rows = rows;
  a.chunks = N * D / 8;
  a.head_log2 = D == 128 ? 4 : 3;
  a.ld_in = ld_in_bytes;
  long long blocks = ((long long)rows * a.chunks + 255) / 256;
  const long long most = 16ll * compute_units();
  if (blocks > most) blocks = most;
  a.step_r = (int)(blocks * 256 / a.chunks);
  a.step_c = (int)(blocks * 256 % a.chunks);
  const auto k = static_cast<const char*>(K), v = static_cast<const char*>(V);
  if (kv_dtype == PAFU_FP8_E4M3)
    hipLaunchKernelGGL(paged_append_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, st, k, v, slots, a, pool,
                       ldexpf(1.0f, -k_scale_log2), ldexpf(1.0f, -v_scale_log2));
  else
    hipLaunchKernelGGL(paged_append_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, k, v, slots, a, pool, 1.f, 1.f);
  return check_launch();
}

}  // namespace pafu

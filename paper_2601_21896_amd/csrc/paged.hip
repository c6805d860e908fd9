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

// inclusive saturating sums over the wave's lanes
__device__ __forceinline__ int wave_scan(int x) {
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));  // row_shr:1, 2, 4, 8: within 16 lanes
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // row_bcast:15 into rows 1 and 3
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));  // row_bcast:31 into rows 2 and 3
  return x;
}

__device__ __forceinline__ void load4(const int* p, int at, int n, int (&x)[4]) {  // p 16-byte aligned, at a multiple of 4
  if (at + 4 <= n) {
    const int4 v = *reinterpret_cast<const int4*>(p + at);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = at + e < n ? p[at + e] : 0;
  }
}
__device__ __forceinline__ void store4(int* p, int at, int n, const int (&x)[4]) {
  if (at + 4 <= n) {
    *reinterpret_cast<int4*>(p + at) = make_int4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (at + e < n) p[at + e] = x[e];
  }
}

// Slots (and, with TAKE, pages) for `count` tokens of each request from its token `start` on.
//   rows: exclusive sums of count -> row_start          first: of the pages wanted and not there yet, from *free_start on
// Latency: a list of a few hundred lengths, a table entry and a slot each.  So it is one launch: every workgroup forms both
// sums of all requests by itself, four neighbouring requests per thread (one round for 1024 requests), and keeps them in
// LDS; then it takes its part of the table and of the slots, four neighbouring slots per thread, which finds its request by
// bisection between those of its wave's first and last slot.  A request's first new page (a decode step has no other) is
// entered by the thread that summed it.
template <bool TAKE>
__global__ __launch_bounds__(kTableThreads) void paged_tables_kernel(PagedTables t) {
  extern __shared__ __attribute__((aligned(16))) int lds[];
  const int stride4 = (t.B + 4) / 4 * 4;  // room for B + 1, 16-byte aligned
  int* rows = lds;
  int* begin = lds + stride4;      // each request's start
  int* first = lds + 2 * stride4;  // (TAKE)
  __shared__ int wave_rows[2][kTableWaves], wave_pages[2][kTableWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int page_mask = (1 << t.page_log2) - 1;
  auto pages_of = [&](int tokens) { return (tokens >> t.page_log2) + ((tokens & page_mask) != 0); };
  int row_at = 0, page_at = TAKE && t.free_start ? max(*t.free_start, 0) : 0;
  for (int base = 0, side = 0; base < t.B; base += kTableThreads * 4, side ^= 1) {
    const int b0 = base + tid * 4;
    int n[4], s[4], total[4], need[4], sum_rows = 0, sum_pages = 0;
    load4(t.count, b0, t.B, n);
    load4(t.start, b0, t.B, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      n[e] = max(n[e], 0);
      s[e] = max(s[e], 0);
      if (TAKE) {
        total[e] = sat_add(s[e], n[e]);
        need[e] = pages_of(total[e]) - pages_of(s[e]);
        sum_pages = sat_add(sum_pages, need[e]);
      }
      sum_rows = sat_add(sum_rows, n[e]);
    }
    const int in_rows = wave_scan(sum_rows), in_pages = TAKE ? wave_scan(sum_pages) : 0;
    if (lane == 63) {
      wave_rows[side][wave] = in_rows;
      wave_pages[side][wave] = in_pages;
    }
    __syncthreads();
    int at_row = row_at, at_page = page_at;
#pragma unroll
    for (int w = 0; w < kTableWaves; ++w) {
      if (w == wave) {
        at_row = row_at;
        at_page = page_at;
      }
      row_at = sat_add(row_at, wave_rows[side][w]);
      page_at = sat_add(page_at, wave_pages[side][w]);
    }
    // the sum in front of this thread is the lower lane's inclusive one
    const int lower_rows = __shfl_up(in_rows, 1), lower_pages = __shfl_up(in_pages, 1);
    at_row = sat_add(at_row, lane ? lower_rows : 0);
    at_page = sat_add(at_page, lane ? lower_pages : 0);
    if (b0 < t.B) {
      int r[4], p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        r[e] = at_row;
        at_row = sat_add(at_row, n[e]);
        if (TAKE) {
          p[e] = at_page;
          at_page = sat_add(at_page, need[e]);
        }
      }
      store4(rows, b0, t.B, r);
      store4(begin, b0, t.B, s);
      if (TAKE) store4(first, b0, t.B, p);
    }
  }
  if (tid == 0) {
    rows[t.B] = row_at;
    if (TAKE) first[t.B] = page_at;
  }
  __syncthreads();

  // the last request whose first row is at or before row i, among lo .. hi - 1
  auto request_of = [&](long long i, int lo, int hi) {
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (rows[mid] <= i) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  const long long stride = (long long)gridDim.x * kTableThreads * 4;
  for (long long w0 = ((long long)blockIdx.x * kTableThreads + wave * 64) * 4; w0 < t.max_slots; w0 += stride) {
    // 64 requests at a time: where the wave's rows begin and end
    int lo = 0, hi = t.B;
    for (int range = hi - lo; range > 64; range = hi - lo) {
      const int step = (range + 63) / 64, at = lo + lane * step;
      const unsigned long long below = __ballot(at < hi && rows[min(at, t.B)] <= w0);  // lane 0 always
      lo += (63 - __clzll(below)) * step;
      hi = min(lo + step, hi);
    }
    lo = request_of(w0, lo, hi);
    const long long i0 = w0 + lane * 4;
    hi = lo + 1;  // past the last request that may hold a row of the wave, by steps of 64
    while (hi < t.B) {
      const unsigned long long in = __ballot(hi + lane < t.B && rows[min(hi + lane, t.B)] < w0 + 256);
      hi += __popcll(in);
      if (in != ~0ull) break;
    }
    int b = request_of(i0, lo, hi);
    // four slots at once: the loads of one do not wait for another's
    int of[4], slot[4], page[4];
    const int* from[4];
    unsigned token[4];
    bool found[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      found[e] = i0 + e < row_at;
      if (found[e])
        while (i0 + e >= rows[b + 1]) ++b;
      of[e] = b;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) slot[e] = begin[of[e]];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int s = slot[e];
      token[e] = (unsigned)s + (unsigned)(found[e] ? (int)(i0 + e) - rows[of[e]] : 0);
      const unsigned col = token[e] >> t.page_log2;
      found[e] = found[e] && col < (unsigned)t.max_pages;
      from[e] = t.table + of[e] * t.ld_table + col;
      if (TAKE) {
        const int nth = (int)col - pages_of(s), at = sat_add(first[of[e]], max(nth, 0));
        if (nth >= 0) {
          found[e] = found[e] && nth < first[of[e] + 1] - first[of[e]] && at < t.n_free;
          from[e] = t.free_pages + at;
        }
      }
      if (!found[e]) from[e] = t.start;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) page[e] = *from[e];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      slot[e] = found[e] && page[e] >= 0 && page[e] <= (0x7fffffff >> t.page_log2)
                    ? (page[e] << t.page_log2) + (int)(token[e] & page_mask) : -1;
    if (i0 < t.max_slots) store4(t.slots, (int)i0, t.max_slots, slot);
  }

  // what is told by request, from the launch's last threads: a decode step's slots are the work of its first
  const int threads = gridDim.x * kTableThreads, back = threads - 1 - (int)(blockIdx.x * kTableThreads + tid);
  for (int b0 = back * 4; b0 < t.B; b0 += threads * 4) {
    int r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = rows[min(b0 + e, t.B)];
    store4(t.row_start, b0, t.B, r);
    if (TAKE) {
      int n[4], s[4], total[4], page[4], at[4];
      load4(t.count, b0, t.B, n);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        at[e] = first[min(b0 + e, t.B)];
        page[e] = at[e] < t.n_free && b0 + e < t.B ? t.free_pages[at[e]] : -1;
        s[e] = begin[min(b0 + e, t.B - 1)];
        total[e] = sat_add(s[e], max(n[e], 0));
      }
      store4(t.kv_len_out, b0, t.B, total);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (b0 + e < t.B && pages_of(total[e]) > pages_of(s[e]) && pages_of(s[e]) < t.max_pages)
          t.table[(b0 + e) * t.ld_table + pages_of(s[e])] = page[e];
    }
  }
  if (back == 0) {
    t.row_start[t.B] = row_at;
    if (TAKE) *t.free_end = page_at;
  }

  if (TAKE) {
    // pages after a request's first new one: 64 columns in a row to a wave, every parts-th run of a request's; a wave looks
    // through 64 of its (request, run) pairs at once for those that are not empty
    const int waves = gridDim.x * kTableWaves, id = blockIdx.x * kTableWaves + wave, parts = max(waves / t.B, 1);
    const int jobs = t.B * parts;
    // what a request takes: a difference of the sums, unless they are saturated
    auto pages_taken = [&](int b) {
      const int end = first[b + 1];
      if (end < 0x7fffffff) return end - first[b];
      return pages_of(sat_add(begin[b], max(t.count[b], 0))) - pages_of(begin[b]);
    };
    for (int j0 = id; j0 < jobs; j0 += waves * 64) {
      const int j = j0 + lane * waves, mine = j < jobs ? j % t.B : 0;
      for (unsigned long long todo = __ballot(j < jobs && pages_taken(mine) > 1 + j / t.B * 64); todo;
           todo &= todo - 1) {
        const int job = j0 + (__ffsll(todo) - 1) * waves, b = job % t.B, part = job / t.B, from = first[b];
        const int have = pages_of(begin[b]), in_table = min(pages_taken(b), t.max_pages - have);
        for (int i = 1 + part * 64 + lane; i < in_table; i += parts * 64) {
          const int at = sat_add(from, i);
          t.table[b * t.ld_table + have + i] = at < t.n_free ? t.free_pages[at] : -1;
        }
      }
    }
  }
}

// Rows of K and V to their slots, 8 elements (16 bytes) of each per thread and turn, as bf16 or as E4M3 codes.  Bound by
// HBM.  With STREAM both sides bypass the caches: 65537 rows of 8 x 128 103.7 -> 99.5 us (5.3 TB/s; a large copy 5.2), to
// codes 76 -> 73; but 8000 rows, which the caches hold, 13.2 -> 14.5.
struct AppendShape {
  unsigned rows, chunks, head_log2;  // 8-element chunks of a row, log2 of those of a head
  unsigned step_r, step_c;           // the grid's stride in rows and chunks
  long long ld_in;
};
template <bool STREAM>
__device__ __forceinline__ u32x4 load_row(const char* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return *reinterpret_cast<const u32x4*>(p);
}
template <bool STREAM, typename T>
__device__ __forceinline__ void store_row(char* p, T x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<T*>(p));
  else *reinterpret_cast<T*>(p) = x;
}
template <bool CODES, bool STREAM>
__global__ __launch_bounds__(256) void paged_append_kernel(const char* __restrict__ K, const char* __restrict__ V,
                                                           const int* __restrict__ slots, AppendShape a, PagedPool pool,
                                                           float inv_k, float inv_v) {
  const unsigned i = blockIdx.x * 256u + threadIdx.x;
  unsigned r = i / a.chunks, c = i - r * a.chunks;
  while (r < a.rows) {
    const int slot = slots[r];
    const int page = slot >> pool.page_log2;
    const long long src = r * a.ld_in + c * 16ll;
    u32x4 in[2];
    if constexpr (!STREAM) {  // a small call is a chain of reads: the rows do not wait for their slot
      in[0] = load_row<false>(K + src);
      in[1] = load_row<false>(V + src);
    }
    if (slot >= 0 && page < pool.n_pages) {
      const long long dst = page * pool.ld_page + (slot & ((1 << pool.page_log2) - 1)) * pool.ld_token +
                            (c >> a.head_log2) * pool.ld_head + (c & ((1 << a.head_log2) - 1)) * (CODES ? 8ll : 16ll);
      if constexpr (STREAM) {
        in[0] = load_row<true>(K + src);
        in[1] = load_row<true>(V + src);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        char* to = const_cast<char*>(x ? pool.V : pool.K) + dst;
        if (CODES) {
          const unsigned words[4] = {in[x][0], in[x][1], in[x][2], in[x][3]};
          unsigned codes[2];
          e4m3_codes8(words, x ? inv_v : inv_k, codes);
          store_row<STREAM>(to, u32x2{codes[0], codes[1]});
        } else {
          store_row<STREAM>(to, in[x]);
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
  // a workgroup per 1024 slots, at most four per compute unit
  long long blocks = ((long long)t.max_slots + kTableThreads * 4 - 1) / (kTableThreads * 4);
  const long long most = 4ll * compute_units();
  blocks = blocks < 1 ? 1 : (blocks > most ? most : blocks);
  const size_t lds = (size_t)(t.B + 4) / 4 * 16 * (take_pages ? 3 : 2);
  // (the lists of more than 5000 requests pass 64 KiB)
  static LdsLimit limit[2];
  const int rc = take_pages ? set_lds_limit(limit[1], paged_tables_kernel<true>, 100 << 10)
                            : set_lds_limit(limit[0], paged_tables_kernel<false>, 100 << 10);
  if (rc) return rc;
  if (take_pages)
    hipLaunchKernelGGL(paged_tables_kernel<true>, dim3((unsigned)blocks), dim3(kTableThreads), lds, st, t);
  else
    hipLaunchKernelGGL(paged_tables_kernel<false>, dim3((unsigned)blocks), dim3(kTableThreads), lds, st, t);
  return check_launch();
}

int launch_paged_append(hipStream_t st, const void* K, const void* V, long long ld_in_bytes, int rows, const int* slots,
                        int N, int D, const PagedPool& pool, int kv_dtype, int k_scale_log2, int v_scale_log2) {
  AppendShape a;
  a.rows = (unsigned)rows;
  a.chunks = (unsigned)(N * D / 8);
  a.head_log2 = D == 128 ? 4 : 3;
  a.ld_in = ld_in_bytes;
  long long blocks = ((long long)rows * a.chunks + 255) / 256;
  const long long most = 256ll * compute_units();
  if (blocks > most) blocks = most;
  a.step_r = (unsigned)(blocks * 256 / a.chunks);
  a.step_c = (unsigned)(blocks * 256 % a.chunks);
  const bool codes = kv_dtype == PAFU_FP8_E4M3;
  // Past the caches from 64 MiB of rows on.  Through -> past them, with six sets of rows and pages in turn, which the caches do
  // not hold: 16 MiB 7.8 -> 8.1 us, 32 17.2 -> 14.1, 64 28.8 -> 25.8, 128 53.1 -> 50.4; with two, which they hold in part: 32 14.8
  // -> 15.0, 48 19.1 -> 20.7, 64 25.8 -> 26.5, 80 34.7 -> 32.8, 128 54.2 -> 51.2 (codes and other layouts alike).
  const bool stream = (long long)rows * N * D * 4 >= 64ll << 20;
  const auto kernel = codes ? (stream ? paged_append_kernel<true, true> : paged_append_kernel<true, false>)
                            : (stream ? paged_append_kernel<false, true> : paged_append_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, static_cast<const char*>(K), static_cast<const char*>(V),
                     slots, a, pool, codes ? ldexpf(1.0f, -k_scale_log2) : 1.f, codes ? ldexpf(1.0f, -v_scale_log2) : 1.f);
  return check_launch();
}

}  // namespace pafu

// Attention of one new token per request over a paged K/V cache.
// (Beyond the paper, whose queries come a chunk at a time.)
//
//   O[b,h] = sum_j w_j v[j] / sum_j w_j,   w_j = 2^(s_j - m),   s_j = scale * log2(e) * q[b,h] . k[j]
//
// The tokens of a request are taken in tiles of 32.  A wave works alone: no LDS, no barrier.  For a tile it forms
// S^T = K Q^T (16 query heads of the group as columns), the weights, and O^T += V^T W^T, all on 16x16x32 matrix
// instructions.  The rows of the two S^T blocks of a tile are dealt to tokens so that a lane's eight weights are those
// of eight neighbouring tokens, 8 g .. 8 g + 7 for lane group g, which is the operand layout of the second product: the
// weights never leave their lane.  V is read by rows, a lane its 8 (or 4) neighbouring elements of its group's eight
// tokens, and transposed within the lane by byte permutes; column n of block i is element 8 n + i.  O^T has the queries
// in columns like S^T, so that a raise of the softmax reference is a multiplication in the lane.
//
// Bound by the reads of K and V.  Every product is exact in fp32; a weight goes into the second product as the sum of
// two bf16 numbers (one alone, 2^-9 off, would cost more than the rounding of a bf16 result).
#include "pafu_internal.h"

namespace pafu {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -3.0e38f;   // softmax reference before the first visible token
constexpr float kRaiseAt = 8.f;      // weights up to 2^8: the reference is raised when a score passes it by more
constexpr int kTile = 32;            // tokens
constexpr int kWaves = 4;            // per workgroup; they share nothing but the launch
constexpr int kMinShare = 4;         // tiles that a wave takes at least where requests are cut

// How the work is laid out.  A column is a run of tiles of the requests' concatenated tile lists; every (key head, group of
// query heads) of a column is one wave, and these are neighbours in the launch: they read neighbouring memory.
struct Layout {
  int columns;     // cut: runs of equal length; whole: one per request
  int heads;       // waves per column = N_kv * groups
  int groups;      // of 16 * QT query heads that share a key head
  int cut;
  float* partial;  // [columns][2][N][D]: 0 = the request began in an earlier column, 1 = it goes on in the next one
  float2* stat;    // [columns][2][N]: softmax reference and sum of a partial result
  int2* joins;     // [columns]: request that begins in the column and goes on, number of columns it spans (0: none)
};

// The tiles of a request.  Visible are [0, pin) and [lo, len).
struct Tiles {
  int n, n_pin;  // all, those of [0, pin)
  int pin, lo, len, base;  // base: first token of the first tile of [lo, len)
};
__device__ __forceinline__ int tiles_of(int tokens) { return tokens > 0 ? (tokens - 1) / kTile + 1 : 0; }
__device__ __forceinline__ Tiles request_tiles(const PagedAttention& a, int page_log2, int kv_len) {
  Tiles t;
  const long long most = (long long)a.max_pages << page_log2;
  t.len = kv_len < 0 ? 0 : (kv_len < most ? kv_len : (int)most);
  t.lo = 0;
  t.pin = 0;
  if (a.window > 0 && kv_len > a.window) {
    const int lo = kv_len - a.window, pin = a.n_pinned < t.len ? a.n_pinned : t.len;
    if (lo > pin) {
      t.lo = lo;
      t.pin = pin;
    }
  }
  t.n_pin = tiles_of(t.pin);
  t.base = t.lo & ~(kTile - 1);
  t.n = t.n_pin + (t.lo < t.len ? tiles_of(t.len - t.base) : 0);
  return t;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ int wave_scan(int x, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// A tile's raw rows as one lane holds them.
template <int D, bool KV8>
struct Raw {
  static constexpr int kK = KV8 ? D / 64 : D / 32;        // 16-byte pieces of a K row
  static constexpr int kVWords = KV8 ? D / 64 : D / 32;   // 32-bit words of a V row: D / 16 elements
  u32x4 k[2][kK];
  unsigned v[8][kVWords];
};

template <int WORDS>
__device__ __forceinline__ void load_words(const char* p, unsigned (&w)[WORDS]) {
  if constexpr (WORDS == 4) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  } else if constexpr (WORDS == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    w[0] = x[0];
    w[1] = x[1];
  } else {
    w[0] = *reinterpret_cast<const unsigned*>(p);
  }
}

// two codes of a word -> two bf16 (exact; the tensor's scale is applied elsewhere)
__device__ __forceinline__ unsigned widen2(unsigned w, bool upper) {
  return upper ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))
               : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}

template <int D, bool KV8, int QT, bool OUT_F32>
__global__ __launch_bounds__(64 * kWaves) void paged_attention_kernel(PagedAttention a, PagedPool pool, Layout ly) {
  constexpr int kSteps = D / 32;   // matrix instructions of one S^T block
  constexpr int kBlocks = D / 16;  // blocks of O^T
  using R = Raw<D, KV8>;
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
  const int x = id / ly.heads, head_id = id - x * ly.heads;
  if (x >= ly.columns) return;
  const int kvh = head_id / ly.groups, group = head_id - kvh * ly.groups;
  const int G = a.N / a.N_kv;

  // ---- this column's tiles: request b from its tile `at` on, `left` tiles
  int b = 0, at = 0, left = 0, share = 0, before = 0;  // before: tiles of the requests in front of b
  if (ly.cut) {
    int mine = 0;
    for (int r = lane; r < a.B; r += 64) mine += request_tiles(a, pool.page_log2, a.kv_len[r]).n;
    const int total = wave_sum(mine);
    share = (total + ly.columns - 1) / ly.columns;
    if (share < kMinShare) share = kMinShare;
    const long long first = (long long)x * share;
    if (first < total) {
      left = min(share, total - (int)first);
      for (int r0 = 0; r0 < a.B; r0 += 64) {
        const int r = r0 + lane, t = r < a.B ? request_tiles(a, pool.page_log2, a.kv_len[r]).n : 0;
        const int ends = before + wave_scan(t, lane);
        const unsigned long long beyond = __ballot(ends > (int)first);
        if (beyond) {
          const int l = __ffsll(beyond) - 1;
          b = __builtin_amdgcn_readfirstlane(r0 + l);
          before = __builtin_amdgcn_readfirstlane(__shfl(ends - t, l));
          at = (int)first - before;
          break;
        }
        before = __builtin_amdgcn_readfirstlane(__shfl(ends, 63));
      }
    }
  } else {
    b = x;
    left = 0x7fffffff;
  }
  left = __builtin_amdgcn_readfirstlane(left);

  // ---- requests without tiles
  for (int r = x; r < a.B; r += ly.columns) {
    const int kv_len = __builtin_amdgcn_readfirstlane(a.kv_len[r]);
    if (request_tiles(a, pool.page_log2, kv_len).n > 0) continue;
    const int h0 = kvh * G + group * 16 * QT, rows = min(16 * QT, G - group * 16 * QT);
    char* to = static_cast<char*>(a.O) + r * a.ld_o + (long long)h0 * D * (OUT_F32 ? 4 : 2);
    for (int i = lane; i < rows * D * (OUT_F32 ? 4 : 2) / 16; i += 64) reinterpret_cast<u32x4*>(to)[i] = u32x4{0, 0, 0, 0};
  }

  const float sc = a.scale * a.k_scale * kLog2e;
  int2 join = make_int2(0, 0);
  while (left > 0 && b < a.B) {
    const Tiles t = request_tiles(a, pool.page_log2, __builtin_amdgcn_readfirstlane(a.kv_len[b]));
    const int here = min(t.n - at, left);
    if (here <= 0) {  // no tiles
      if (!ly.cut) break;
      before += t.n;
      ++b;
      at = 0;
      continue;
    }

    // ---- queries: column n of block `qt` is query head h0 + 16 qt + n (the last one again where the group ends)
    bf16x8 q[QT][kSteps];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int hq = min(group * 16 * QT + qt * 16 + n, G - 1);
      const char* qp = static_cast<const char*>(a.Q) + b * a.ld_q + ((long long)kvh * G + hq) * (D * 2);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = KV8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        q[qt][s] = *reinterpret_cast<const bf16x8*>(qp + d * 2);
      }
    }
    f32x4 o[QT][kBlocks];
    float m[QT], l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m[qt] = kNoMax;
      l[qt] = 0.f;
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) o[qt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- addresses: a group of eight tokens lies on one page
    const int* row = a.table + b * a.ld_table;
    const int kgroup = n >> 2;  // the group that this lane's K rows belong to
    const long long head = kvh * pool.ld_head;
    const char* Kl = pool.K + head + (n & 3) * pool.ld_token + g * 16;
    const char* Vl = pool.V + head + n * (D / 16) * (KV8 ? 1 : 2);
    const int mask = (1 << pool.page_log2) - 1;
    auto tile_base = [&](int i) { return i < t.n_pin ? i * kTile : t.base + (i - t.n_pin) * kTile; };
    auto page_at = [&](int token) { return row[min(token >> pool.page_log2, a.max_pages - 1)]; };
    auto offset = [&](int page, int token) {
      page = max(min(page, pool.n_pages - 1), 0);
      return page * pool.ld_page + (token & mask) * pool.ld_token;
    };
    auto load_k = [&](R& raw, int base, int page) {
      const char* p = Kl + offset(page, base + kgroup * 8);
#pragma unroll
      for (int tk = 0; tk < 2; ++tk)
#pragma unroll
        for (int i = 0; i < R::kK; ++i) raw.k[tk][i] = *reinterpret_cast<const u32x4*>(p + tk * 4 * pool.ld_token + i * 64);
    };
    auto load_v = [&](R& raw, int base, int page) {
      const char* p = Vl + offset(page, base + g * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) load_words(p + j * pool.ld_token, raw.v[j]);
    };

    R raw;
    int base = tile_base(at);
    int page_v = page_at(base + g * 8), page_k = page_at(base + kgroup * 8);
    load_k(raw, base, page_k);
    load_v(raw, base, page_v);
    int next_base = here > 1 ? tile_base(at + 1) : base;
    int next_v = page_at(next_base + g * 8), next_k = page_at(next_base + kgroup * 8);

    for (int i = 0; i < here; ++i) {
      // ---- S^T = K Q^T
      f32x4 s[QT][2];
#pragma unroll
      for (int tk = 0; tk < 2; ++tk) {
        bf16x8 k[kSteps];
#pragma unroll
        for (int e = 0; e < kSteps; ++e) {
          if constexpr (KV8) {
            u32x4 w;
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = widen2(raw.k[tk][e >> 1][(e & 1) * 2 + (u >> 1)], u & 1);
            k[e] = __builtin_bit_cast(bf16x8, w);
          } else {
            k[e] = __builtin_bit_cast(bf16x8, raw.k[tk][e]);
          }
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          s[qt][tk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < kSteps; ++e)
            s[qt][tk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[e], q[qt][e], s[qt][tk], 0, 0, 0);
        }
      }
      if (i + 1 < here) load_k(raw, next_base, next_k);

      // ---- what is not visible: s(tk, r) belongs to token base + 8 g + 4 tk + r, V's row j to base + 8 g + j
      const bool pinned = at + i < t.n_pin;
      const int lo = pinned ? 0 : t.lo, hi = pinned ? t.pin : t.len;
      const bool page_ok = page_v >= 0 && page_v < pool.n_pages;
      if (base < lo || hi - base < kTile || __ballot(!page_ok)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int token = base + g * 8 + j;
          const bool seen = page_ok && token >= lo && token < hi;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[qt][j >> 2][j & 3] = seen ? s[qt][j >> 2][j & 3] : -__builtin_inff();
#pragma unroll
          for (int w = 0; w < R::kVWords; ++w) raw.v[j][w] = seen ? raw.v[j][w] : 0u;
        }
      }

      // ---- weights
      bf16x8 hi_w[QT], lo_w[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        float top = s[qt][0][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, s[qt][j >> 2][j & 3]);
        if (__ballot(top * sc > m[qt] + kRaiseAt)) {  // raise the reference: rare after the first tiles
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float up = fmaxf(m[qt], top * sc);
          const float down = __builtin_amdgcn_exp2f(m[qt] - up);
          m[qt] = up;
          l[qt] *= down;
#pragma unroll
          for (int k = 0; k < kBlocks; ++k) o[qt][k] *= down;
        }
        u32x4 upper, lower;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float w0 = __builtin_amdgcn_exp2f(fmaf(s[qt][j >> 2][j & 3], sc, -m[qt]));
          const float w1 = __builtin_amdgcn_exp2f(fmaf(s[qt][j >> 2][(j & 3) + 1], sc, -m[qt]));
          l[qt] += w0 + w1;
          const unsigned u0 = __float_as_uint(w0), u1 = __float_as_uint(w1);
          upper[j >> 1] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);  // the upper halves
          bf16x2 rest;
          rest[0] = (__bf16)(w0 - __uint_as_float(u0 & 0xffff0000u));
          rest[1] = (__bf16)(w1 - __uint_as_float(u1 & 0xffff0000u));
          lower[j >> 1] = __builtin_bit_cast(unsigned, rest);
        }
        hi_w[qt] = __builtin_bit_cast(bf16x8, upper);
        lo_w[qt] = __builtin_bit_cast(bf16x8, lower);
      }

      // ---- O^T += V^T W^T: block k of this lane's elements, rows transposed in the lane
      unsigned v[8][kBlocks / 2];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < kBlocks / 2; ++e) v[j][e] = KV8 ? widen2(raw.v[j][e >> 1], e & 1) : raw.v[j][KV8 ? 0 : e];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = __builtin_amdgcn_perm(v[2 * j + 1][k >> 1], v[2 * j][k >> 1], (k & 1) ? 0x07060302u : 0x05040100u);
        const bf16x8 vt = __builtin_bit_cast(bf16x8, w);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          o[qt][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, hi_w[qt], o[qt][k], 0, 0, 0);
          o[qt][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, lo_w[qt], o[qt][k], 0, 0, 0);
        }
      }
      if (i + 1 < here) {
        load_v(raw, next_base, next_v);
        base = next_base;
        page_v = next_v;
        next_base = tile_base(min(at + i + 2, at + here - 1));
        next_v = page_at(next_base + g * 8);
        next_k = page_at(next_base + kgroup * 8);
      }
    }

    // ---- out: lane (g, n) holds query n's elements (4 g + r) * kBlocks + k
    const bool whole = at == 0 && here == t.n;
    const long long slot = 2ll * x + (at == 0 ? 1 : 0);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      l[qt] += __shfl_xor(l[qt], 16);
      l[qt] += __shfl_xor(l[qt], 32);
      const int hq = group * 16 * QT + qt * 16 + n;
      if (hq >= G) continue;
      const long long h = (long long)kvh * G + hq;
      if (whole) {
        const float inv = l[qt] == 0.f ? 0.f : a.v_scale / l[qt];
        char* to = static_cast<char*>(a.O) + b * a.ld_o + h * D * (OUT_F32 ? 4 : 2);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = (g * 4 + r) * kBlocks;
          if constexpr (OUT_F32) {
#pragma unroll
            for (int k = 0; k < kBlocks; k += 4)
              *reinterpret_cast<f32x4*>(to + (d + k) * 4) =
                  f32x4{o[qt][k][r] * inv, o[qt][k + 1][r] * inv, o[qt][k + 2][r] * inv, o[qt][k + 3][r] * inv};
          } else {
            unsigned w[kBlocks / 2];
#pragma unroll
            for (int k = 0; k < kBlocks; k += 2) {
              bf16x2 y;
              y[0] = (__bf16)(o[qt][k][r] * inv);
              y[1] = (__bf16)(o[qt][k + 1][r] * inv);
              w[k >> 1] = __builtin_bit_cast(unsigned, y);
            }
            if constexpr (kBlocks == 8) *reinterpret_cast<u32x4*>(to + d * 2) = u32x4{w[0], w[1], w[2], w[3]};
            else *reinterpret_cast<u32x2*>(to + d * 2) = u32x2{w[0], w[1]};
          }
        }
      } else {
        float* to = ly.partial + (slot * a.N + h) * D;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int k = 0; k < kBlocks; k += 4)
            *reinterpret_cast<f32x4*>(to + (g * 4 + r) * kBlocks + k) =
                f32x4{o[qt][k][r], o[qt][k + 1][r], o[qt][k + 2][r], o[qt][k + 3][r]};
        if (g == 0) ly.stat[slot * a.N + h] = make_float2(m[qt], l[qt]);
      }
    }
    if (at == 0 && here < t.n) join = make_int2(b, (before + t.n - 1) / share - x + 1);
    if (!ly.cut) break;
    left -= here;
    before += t.n;
    ++b;
    at = 0;
  }
  if (ly.cut && head_id == 0 && lane == 0) ly.joins[x] = join;
}

// Joins the partial results of the request that begins in a column and ends in a later one: one workgroup per (column,
// query head), D / 4 lanes to a partial result, the others take further ones, in a fixed order.
template <int D, bool OUT_F32>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttention a, Layout ly) {
  constexpr int kLanes = D / 4, kSets = 256 / kLanes;
  const int x = blockIdx.x, h = blockIdx.y;
  const int2 join = ly.joins[x];
  if (join.y == 0) return;
  __shared__ float sm[kSets], sl[kSets];
  __shared__ f32x4 so[kSets][kLanes];
  const int set = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  float m = kNoMax, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p = set; p < join.y; p += kSets) {
    const long long at = (2ll * (x + p) + (p == 0 ? 1 : 0)) * a.N + h;
    const float2 st = ly.stat[at];
    const f32x4 part = *reinterpret_cast<const f32x4*>(ly.partial + at * D + lane * 4);
    const float up = fmaxf(m, st.x), keep = __builtin_amdgcn_exp2f(m - up), add = __builtin_amdgcn_exp2f(st.x - up);
    m = up;
    l = l * keep + st.y * add;
    o = o * keep + part * add;
  }
  if (lane == 0) {
    sm[set] = m;
    sl[set] = l;
  }
  so[set][lane] = o;
  __syncthreads();
  if (set > 0) return;
  float up = kNoMax;
#pragma unroll
  for (int i = 0; i < kSets; ++i) up = fmaxf(up, sm[i]);
  l = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kSets; ++i) {
    const float w = __builtin_amdgcn_exp2f(sm[i] - up);
    l += sl[i] * w;
    o += so[i][lane] * w;
  }
  o *= l == 0.f ? 0.f : a.v_scale / l;
  char* to = static_cast<char*>(a.O) + join.x * a.ld_o + ((long long)h * D + lane * 4) * (OUT_F32 ? 4 : 2);
  if constexpr (OUT_F32) {
    *reinterpret_cast<f32x4*>(to) = o;
  } else {
    bf16x2 y0, y1;
    y0[0] = (__bf16)o[0];
    y0[1] = (__bf16)o[1];
    y1[0] = (__bf16)o[2];
    y1[1] = (__bf16)o[3];
    *reinterpret_cast<u32x2*>(to) = u32x2{__builtin_bit_cast(unsigned, y0), __builtin_bit_cast(unsigned, y1)};
  }
}

int query_tiles(int G) { return G <= 16 ? 1 : 2; }
int head_waves(int N, int N_kv) {
  const int G = N / N_kv, rows = 16 * query_tiles(G);
  return N_kv * ((G + rows - 1) / rows);
}
// Columns of a cut launch: 12 waves per compute unit.
int cut_columns(int N, int N_kv) {
  const int columns = 12 * compute_units() / head_waves(N, N_kv);
  return columns < 1 ? 1 : columns;
}
size_t round16(size_t n) { return (n + 15) / 16 * 16; }

template <int D, bool KV8>
int launch(hipStream_t st, const PagedAttention& a, const PagedPool& pool, const Layout& ly) {
  const unsigned blocks = (unsigned)(((long long)ly.columns * ly.heads + kWaves - 1) / kWaves);
  const dim3 threads(64 * kWaves);
  const bool f32 = a.out_dtype == PAFU_F32;
  if (query_tiles(a.N / a.N_kv) == 1) {
    if (f32) hipLaunchKernelGGL((paged_attention_kernel<D, KV8, 1, true>), dim3(blocks), threads, 0, st, a, pool, ly);
    else hipLaunchKernelGGL((paged_attention_kernel<D, KV8, 1, false>), dim3(blocks), threads, 0, st, a, pool, ly);
  } else {
    if (f32) hipLaunchKernelGGL((paged_attention_kernel<D, KV8, 2, true>), dim3(blocks), threads, 0, st, a, pool, ly);
    else hipLaunchKernelGGL((paged_attention_kernel<D, KV8, 2, false>), dim3(blocks), threads, 0, st, a, pool, ly);
  }
  int rc = check_launch();
  if (rc || !ly.cut) return rc;
  const dim3 grid((unsigned)ly.columns, (unsigned)a.N);
  if (f32) hipLaunchKernelGGL((paged_join_kernel<D, true>), grid, dim3(256), 0, st, a, ly);
  else hipLaunchKernelGGL((paged_join_kernel<D, false>), grid, dim3(256), 0, st, a, ly);
  return check_launch();
}

}  // namespace

size_t paged_attention_workspace_bytes(int B, int N, int N_kv, int D) {
  (void)B;
  const size_t columns = (size_t)cut_columns(N, N_kv), rows = columns * 2 * N;
  return rows * D * 4 + round16(rows * 8) + round16(columns * 8);
}

int launch_paged_attention(hipStream_t st, const PagedAttention& a, const PagedPool& pool, void* workspace,
                           size_t workspace_bytes) {
  Layout ly;
  const int G = a.N / a.N_kv;
  ly.heads = head_waves(a.N, a.N_kv);
  ly.groups = ly.heads / a.N_kv;
  (void)G;
  const long long longest = ((((long long)a.max_pages << pool.page_log2) + kTile - 1) / kTile);
  ly.cut = workspace != nullptr && workspace_bytes >= paged_attention_workspace_bytes(a.B, a.N, a.N_kv, a.D) &&
           longest > kMinShare;
  ly.columns = a.B;
  ly.partial = nullptr;
  ly.stat = nullptr;
  ly.joins = nullptr;
  if (ly.cut) {
    const size_t all = (size_t)cut_columns(a.N, a.N_kv);
    const long long useful = (longest * a.B + kMinShare - 1) / kMinShare;
    ly.columns = (int)(useful < (long long)all ? useful : (long long)all);
    char* w = static_cast<char*>(workspace);
    ly.partial = reinterpret_cast<float*>(w);
    w += all * 2 * a.N * a.D * 4;
    ly.stat = reinterpret_cast<float2*>(w);
    w += round16(all * 2 * a.N * 8);
    ly.joins = reinterpret_cast<int2*>(w);
  }
  const bool kv8 = a.kv_dtype == PAFU_FP8_E4M3;
  if (a.D == 128) return kv8 ? launch<128, true>(st, a, pool, ly) : launch<128, false>(st, a, pool, ly);
  return kv8 ? launch<64, true>(st, a, pool, ly) : launch<64, false>(st, a, pool, ly);
}

}  // namespace pafu

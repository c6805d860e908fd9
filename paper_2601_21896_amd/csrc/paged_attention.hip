// Attention of one new token per request over a paged K/V cache.
// (Beyond the paper, whose queries come a chunk at a time.)
//
//   O[b,h] = sum_j w_j v[j] / sum_j w_j,   w_j = 2^(c (s_j - m)),   s_j = q[b,h] . k[j],   c = scale * log2(e)
//
// The tokens of a request are taken in tiles of 32, a wave works on a tile alone.  It forms S^T = K Q^T (16 query heads that
// share a key head as columns), the weights, and O^T += V^T W^T, all on 16x16x32 matrix instructions.  The rows of the two
// S^T blocks of a tile are dealt to tokens so that a lane's eight weights are those of eight neighbouring tokens,
// 8 g .. 8 g + 7 for lane group g, which is the operand layout of the second product: the weights never leave their lane.
// V is read by rows, a lane its 8 (or 4) neighbouring elements of its group's eight tokens, and transposed within the lane
// by byte permutes; column n of block i is element 8 n + i.  O^T has the queries in columns like S^T, so that a raise of
// the softmax reference is a multiplication in the lane.
//
// Bound by the reads of K and V, at up to 6.9 TB/s (a kernel that only reads reaches 7.0; a large copy 5.1).  They bypass the
// caches where one wave alone reads their lines (6.2 TB/s otherwise), except in small calls.  Eight waves per compute unit,
// all of the launch at once, hold enough rows in flight; twelve or sixteen were slower everywhere (more, shorter runs).
// What a call takes beyond the reads: about 5 us until the first rows are there, 7 us for the join and the way to it.
//
// Products of bf16 or widened 8-bit values are exact in fp32.  A weight goes into the second product whole: as the sum of
// three bf16 numbers, which hold eight of its 24 bits each.
#include "pafu_internal.h"

namespace pafu {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -3.4028235e38f;  // softmax reference m before the first visible token
constexpr float kRaiseAt = 8.f;           // weights up to 2^8: the reference is raised when a score passes it by more
constexpr int kTile = 32;            // tokens
constexpr int kWaves = 4;            // per workgroup

// How the work is laid out.  A column is a run of tiles of the requests' concatenated tile lists, or, where nothing is cut, a
// request.  Every (key head, group of query heads) of a column is one wave, neighbouring heads are one workgroup
// ("narrow"), or it is a workgroup, whose waves take the tiles in turn and add up in LDS ("wide").
struct Layout {
  int columns;
  int heads;       // waves or workgroups per column = N_kv * groups
  int groups;      // of 16 * QT query heads that share a key head
  int cut;
  int joined;      // the requests, or, where they are more than the columns, the columns that a request may go on from
  float* partial;  // [columns][2][N][D]: 0 = the request began in an earlier column, 1 = it goes on in the next one
  float2* stat;    // [columns][2][N]: softmax reference and sum of a partial result
  int2* joins;     // [joined]: first column and number of columns of a request that is cut (0 columns: it is not)
};

// The tiles of a request.  Visible are [0, pin) and [lo, len).
struct Tiles {
  int n, n_pin;  // all, those of [0, pin)
  int pin, lo, len, base;  // base: first token of the first tile of [lo, len)
};
__device__ __forceinline__ int tiles_of(int tokens) { return tokens > 0 ? (tokens - 1) / kTile + 1 : 0; }
__device__ __forceinline__ Tiles request_tiles(const PagedAttention& a, int kv_len) {
  Tiles t;
  t.len = min(max(kv_len, 0), a.max_tokens);
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

// c.  Not 0: what is not visible is -infinity times it.
__device__ __forceinline__ float exponent_scale(const PagedAttention& a) {
  return fmaxf(a.scale * a.k_scale * kLog2e, 1.1754944e-38f);
}

// inclusive sums over the wave's lanes
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8: within 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return x;
}

// A tile's rows as one lane reads them.
template <int D, bool KV8>
struct Raw {
  static constexpr int kRow = KV8 ? D : 2 * D;            // bytes
  static constexpr int kK = kRow / 64;                    // 16-byte pieces of a lane's part of a K row
  static constexpr int kVWords = kRow / 64;               // 32-bit words of its part of a V row: D / 16 elements
  // K is read 16 bytes a lane, kLanes lanes to a row (each of the four lane groups kStep rows at once), and turned in LDS, a
  // row 16 bytes longer there to spread the banks.  Read the way the matrix instruction wants it (16 rows and 64 bytes of
  // each at a time) the 8-bit cache of 12 x 128 came at 6.1 TB/s instead of 6.7, the bf16 one of 8 x 128 at 6.80 instead
  // of 6.85; pages of 16 tokens 5 % slower, since K and V no longer share a lane's page.
  static constexpr int kLanes = kRow / 16, kStep = 16 / kLanes, kPitch = kRow + 16;
  // Lane group g's part of a row: 32 neighbouring bytes of every 128 (of a row of 64 bytes 16).
  static constexpr int kPiece = kRow == 64 ? 16 : 32;
  static __device__ constexpr int at(int i) { return (i >> 1) * 128 + (i & 1) * 16; }
  u32x4 k[2 * kK];
  unsigned v[8][kVWords];
};

template <bool ONCE, typename T>
__device__ __forceinline__ T load(const char* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const T*>(p));
  return *reinterpret_cast<const T*>(p);
}
template <bool ONCE, int WORDS>
__device__ __forceinline__ void load_words(const char* p, unsigned (&w)[WORDS]) {
  if constexpr (WORDS == 4) {
    const u32x4 x = load<ONCE, u32x4>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  } else if constexpr (WORDS == 2) {
    const u32x2 x = load<ONCE, u32x2>(p);
    w[0] = x[0];
    w[1] = x[1];
  } else {
    w[0] = load<ONCE, unsigned>(p);
  }
}

// LDS that a wave alone uses: its accesses are carried out in order, so only the compiler has to keep to it.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A float's upper half is a bf16 number, the float with its lower bits cut off; behind: what is cut off (exact).
__device__ __forceinline__ float behind(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ u16x2 upper_halves(float x, float y) {
  return __builtin_bit_cast(u16x2, __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u));
}

// x y; 0 where y is 0, whatever x: a row whose scores are all -infinity is 0 even if 0 times its values gave NaN
__device__ __forceinline__ f32x4 scaled(f32x4 x, float y) {
  const unsigned keep = y == 0.f ? 0u : ~0u;
  return __builtin_bit_cast(f32x4, __builtin_bit_cast(u32x4, x * y) & keep);
}

// two codes of a word -> two bf16 (exact; the tensor's scale is applied elsewhere)
__device__ __forceinline__ unsigned widen2(unsigned w, bool upper) {
  return upper ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))
               : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}

template <int D, bool KV8, int QT, bool WIDE, bool ONCE>  // ONCE: no other wave reads the same lines of K and V
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_kernel(PagedAttention a, PagedPool pool, Layout ly) {
  constexpr int kSteps = D / 32;   // matrix instructions of one S^T block
  constexpr int kBlocks = D / 16;  // blocks of O^T
  using R = Raw<D, KV8>;
  constexpr int kWays = WIDE ? kWaves : 1;
  // K on its way to the matrix instructions, then what the waves of a wide workgroup add up
  constexpr int kStage = kWaves * kTile * R::kPitch, kParts = WIDE ? kWaves * QT * kBlocks * 64 * 16 : 0;
  __shared__ __attribute__((aligned(16))) char lds[kStage > kParts ? kStage : kParts];
  f32x4 (*part)[QT][4][kBlocks / 4][64] = reinterpret_cast<f32x4 (*)[QT][4][kBlocks / 4][64]>(lds);
  __shared__ float2 part_stat[kWays][QT][16];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.N / a.N_kv, out_bytes = a.out_dtype == PAFU_F32 ? 4 : 2;

  // ---- the tiles of all requests, summed over the lanes: a request to each, or, of more than 64, a run of `per`
  int kv = 0, kv0 = 0, mine = 0, ends = 0, total = 0, per = 1;  // kv: length of request kv0 + lane; ends: tiles up to a lane's
  if (ly.cut) {
    if (a.B <= 64) {
      kv = a.kv_len[min(lane, a.B - 1)];
      mine = lane < a.B ? request_tiles(a, kv).n : 0;
    } else {
      per = (a.B + 255) / 256 * 4;
#pragma unroll 4
      for (int i = 0; i < per; i += 4) {
        const int r = lane * per + i;
        if (r + 4 <= a.B) {
          const int4 v = *reinterpret_cast<const int4*>(a.kv_len + r);
          mine += request_tiles(a, v.x).n + request_tiles(a, v.y).n +
                  request_tiles(a, v.z).n + request_tiles(a, v.w).n;
        } else {
          for (int e = r; e < a.B; ++e) mine += request_tiles(a, a.kv_len[e]).n;
        }
      }
    }
    ends = wave_scan(mine);
    total = __builtin_amdgcn_readlane(ends, 63);
  }
  const int columns = ly.columns, sub = WIDE ? wave : 0;
  const int id = WIDE ? blockIdx.x : blockIdx.x * kWaves + wave;
  const int x = id / ly.heads, head_id = id - x * ly.heads;
  if (x >= columns) return;
  const int kvh = head_id / ly.groups, group = head_id - kvh * ly.groups;

  // ---- this column's tiles: request b from its tile `at` on, `left` tiles
  int b = x, at = 0, left = 0x7fffffff, share = 0, before = 0;  // before: tiles of the requests in front of b
  if (ly.cut) {
    share = max(total - 1, 0) / columns + 1;
    if (WIDE && share < kWays) share = kWays;  // a tile for each wave
    left = 0;
    const long long first = (long long)x * share;
    if (first < total) {
      left = min(share, total - (int)first);
      const int l = __ffsll(__ballot(ends > (int)first)) - 1;
      b = l * per;
      before = __builtin_amdgcn_readlane(ends - mine, l);
      while (per > 1) {  // which one of the run
        kv0 = b;
        kv = a.kv_len[min(kv0 + lane, a.B - 1)];
        mine = kv0 + lane < a.B ? request_tiles(a, kv).n : 0;
        ends = before + wave_scan(mine);
        const unsigned long long beyond = __ballot(ends > (int)first);
        if (beyond) {
          b = kv0 + __ffsll(beyond) - 1;
          before = __builtin_amdgcn_readlane(ends - mine, b - kv0);
          break;
        }
        before = __builtin_amdgcn_readlane(ends, 63);
        b += 64;
      }
      at = (int)first - before;
    }
  }

  // joins are told by request, or by column with the request in the first place
  const bool by_request = ly.cut && ly.joined == a.B, tells = ly.cut && head_id == 0 && sub == 0 && lane == 0;
  const float sc = exponent_scale(a);
  int2 join = make_int2(0, 0);  // of the column
  if (!ly.cut) {
    kv0 = b;
    kv = a.kv_len[min(b + lane, a.B - 1)];
  }

  // ---- A wave's tiles in their order.  It goes through them in one pipeline, from a request to the next without a pause: the
  // pages of a tile are asked for two tiles ahead, its rows one.  (One that ran dry at each request's end took 52.5 us instead
  // of 49.8 for 8 requests of 8192 tokens, 8 x 128; rows two tiles ahead gained nothing anywhere.)
  struct Place {  // the i-th of the `here` tiles that the column takes of request b, from its tile `at` on; left: with what follows
    int b, at, here, i, left;
    Tiles t;
  };
  struct Spot {  // first token of a tile, and which are visible
    int base, lo, hi;
  };
  auto settle = [&](Place& p) {  // to request p.b, or the next one that has tiles; here = 0 behind the last
    p.here = 0;
    p.i = sub;
    while (p.left > 0 && p.b < a.B) {
      if (p.b - kv0 >= 64) {
        kv0 = p.b;
        kv = a.kv_len[min(p.b + lane, a.B - 1)];
        asm volatile("" : "+v"(kv));  // waited for here, not on the path without it, where rows are in flight
      }
      p.t = request_tiles(a, __builtin_amdgcn_readlane(kv, p.b - kv0));
      p.here = max(min(p.t.n - p.at, p.left), 0);
      if (p.here > 0 || !ly.cut) return;
      ++p.b;
      p.at = 0;
    }
  };
  auto after = [&](Place p) {
    p.i += kWays;
    if (p.i >= p.here) {
      p.left = ly.cut ? p.left - p.here : 0;
      ++p.b;
      p.at = 0;
      settle(p);
    }
    return p;
  };
  auto spot = [&](const Place& p) {  // (where a wave of a wide workgroup has no tile of a request, nothing is visible)
    if (p.i >= p.here) return Spot{0, 0, 0};
    const int tile = p.at + p.i;
    return tile < p.t.n_pin ? Spot{tile * kTile, 0, p.t.pin} : Spot{p.t.base + (tile - p.t.n_pin) * kTile, p.t.lo, p.t.len};
  };
  // addresses: lane group g reads tokens 8 g .. 8 g + 7 of a tile, which lie on one page
  const long long head = kvh * pool.ld_head;
  const char* Kl = pool.K + head + (n / R::kLanes) * pool.ld_token + (n % R::kLanes) * 16;
  const char* Vl = pool.V + head + n * (R::kRow / 16);
  char* k_in = lds + wave * (kTile * R::kPitch) + (g * 8 + n / R::kLanes) * R::kPitch + (n % R::kLanes) * 16;
  const char* k_out = lds + wave * (kTile * R::kPitch) + ((n >> 2) * 8 + (n & 3)) * R::kPitch + g * R::kPiece;
  const int mask = (1 << pool.page_log2) - 1;
  auto page_of = [&](const Place& p, const Spot& s) {
    return a.table[min(p.b, a.B - 1) * a.ld_table + min((s.base + g * 8) >> pool.page_log2, a.max_pages - 1)];
  };
  auto seen = [&](const Spot& s, int page) {  // is any of this lane's eight tokens visible, on a page of the pool?
    return page >= 0 && page < pool.n_pages && s.base + g * 8 + 7 >= s.lo && s.base + g * 8 < s.hi;
  };
  // Where this lane's rows lie.  Rows that are not seen are the pool's first: one line for all lanes, and loads on every path, in
  // one order (K, page, V), let the compiler wait for just the ones it needs.
  auto offset = [&](const Spot& s, int page) {
    page = max(min(page, pool.n_pages - 1), 0);
    return page * pool.ld_page + ((s.base + g * 8) & mask) * pool.ld_token;
  };
  auto load_k = [&](R& raw, const char* from) {
#pragma unroll
    for (int i = 0; i < 2 * R::kK; ++i) raw.k[i] = load<ONCE, u32x4>(from + i * R::kStep * pool.ld_token);
  };
  auto load_v = [&](R& raw, const char* from) {
#pragma unroll
    for (int j = 0; j < 8; ++j) load_words<ONCE>(from + j * pool.ld_token, raw.v[j]);
  };
  // queries: column n of block `qt` is query head h0 + 16 qt + n (the last one again where the group ends)
  bf16x8 q[QT][kSteps];
  auto load_q = [&](int request) {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int hq = min(group * 16 * QT + qt * 16 + n, G - 1);
      const char* qp = static_cast<const char*>(a.Q) + request * a.ld_q + ((long long)kvh * G + hq) * (D * 2);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = KV8 ? g * (D / 4) + s * 8 : (s >> 1) * 64 + g * 16 + (s & 1) * 8;
        q[qt][s] = *reinterpret_cast<const bf16x8*>(qp + d * 2);
      }
    }
  };
  f32x4 o[QT][kBlocks];
  float m[QT], l[QT];
  auto clear = [&] {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m[qt] = kNoMax;
      l[qt] = 0.f;
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) o[qt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };

  // Where nothing is cut and all tokens are visible, the first pages and the queries do not wait for the length (small calls
  // are chains of reads).
  const bool early = !ly.cut && a.window == 0;
  int page = 0, page1 = 0;
  Place p0{b, at, 0, 0, left, {}};
  if (early) {
    page = page_of(p0, Spot{sub * kTile, 0, 0});
    page1 = page_of(p0, Spot{(sub + kWays) * kTile, 0, 0});
    load_q(b);
  }
  settle(p0);
  if (p0.here > 0) {
    Place p1 = after(p0);
    Spot s0 = spot(p0), s1 = spot(p1);
    R raw;
    if (!early) {
      page = page_of(p0, s0);
      load_q(p0.b);
      page1 = page_of(p1, s1);
    }
    clear();
    bool ok = seen(s0, page);
    const long long from = offset(s0, page);
    page = page1;
    __builtin_amdgcn_sched_barrier(0);
    load_k(raw, ok ? Kl + from : pool.K);
    __builtin_amdgcn_sched_barrier(0);
    load_v(raw, ok ? Vl + from : pool.V);
    __builtin_amdgcn_sched_barrier(0);

    while (true) {
      // ---- S^T = K Q^T
      wave_sync();
#pragma unroll
      for (int j = 0; j < 2 * R::kK; ++j) *reinterpret_cast<u32x4*>(k_in + j * R::kStep * R::kPitch) = raw.k[j];
      wave_sync();
      f32x4 s[QT][2];
#pragma unroll
      for (int tk = 0; tk < 2; ++tk) {
        bf16x8 k[kSteps];
#pragma unroll
        for (int j = 0; j < R::kK; ++j) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(k_out + tk * 4 * R::kPitch + R::at(j));
          if constexpr (KV8) {
            k[2 * j] = __builtin_bit_cast(bf16x8, u32x4{widen2(x[0], false), widen2(x[0], true), widen2(x[1], false), widen2(x[1], true)});
            k[2 * j + 1] = __builtin_bit_cast(bf16x8, u32x4{widen2(x[2], false), widen2(x[2], true), widen2(x[3], false), widen2(x[3], true)});
          } else {
            k[j] = __builtin_bit_cast(bf16x8, x);
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
      const Place p2 = after(p1);
      const Spot s2 = spot(p2);
      const long long next = offset(s1, page);
      const bool next_ok = seen(s1, page);
      load_k(raw, next_ok ? Kl + next : pool.K);
      page = page_of(p2, s2);
      const bool last = p0.i + kWays >= p0.here;  // of this wave's tiles of the request
      if (last) load_q(min(p1.b, a.B - 1));

      // ---- what is not visible: s(tk, r) belongs to token base + 8 g + 4 tk + r, V's row j to base + 8 g + j
      if (s0.base < s0.lo || s0.hi - s0.base < kTile || __ballot(!ok)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int token = s0.base + g * 8 + j;
          const bool visible = ok && token >= s0.lo && token < s0.hi;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[qt][j >> 2][j & 3] = visible ? s[qt][j >> 2][j & 3] : -__builtin_inff();
#pragma unroll
          for (int w = 0; w < R::kVWords; ++w) raw.v[j][w] = visible ? raw.v[j][w] : 0u;
        }
      }

      // ---- weights
      bf16x8 w_parts[QT][3];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        float top = s[qt][0][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, s[qt][j >> 2][j & 3]);
        if (__ballot((top - m[qt]) * sc > kRaiseAt)) {  // raise the reference: rare after the first tiles
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float up = fmaxf(m[qt], top);
          const float down = __builtin_amdgcn_exp2f((m[qt] - up) * sc);
          m[qt] = up;
          l[qt] *= down;
#pragma unroll
          for (int k = 0; k < kBlocks; ++k) o[qt][k] *= down;
        }
        // c s - c m in one operation, unless c m is so large that its rounding shows: from 2^31 on the weights would overflow
        float ref = m[qt] * sc;
        if (__ballot(fabsf(ref) > 64.f)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) s[qt][j >> 2][j & 3] -= m[qt];
          ref = 0.f;
        }
        u32x4 part0, part1, part2;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float w0 = __builtin_amdgcn_exp2f(fmaf(s[qt][j >> 2][j & 3], sc, -ref));
          const float w1 = __builtin_amdgcn_exp2f(fmaf(s[qt][j >> 2][(j & 3) + 1], sc, -ref));
          l[qt] += w0 + w1;
          // A weight's bits eight at a time.  Where none are left, a part of a weight that is not 0 is the least bf16 number: the
          // parts of 0 alone are 0, and 0 times an infinite value is none.
          const float r0 = behind(w0), r1 = behind(w1);
          const u16x2 first = upper_halves(w0, w1), least = __builtin_elementwise_min(first, u16x2{1, 1});
          part0[j >> 1] = __builtin_bit_cast(unsigned, first);
          part1[j >> 1] = __builtin_bit_cast(unsigned, __builtin_elementwise_max(upper_halves(r0, r1), least));
          part2[j >> 1] = __builtin_bit_cast(unsigned, __builtin_elementwise_max(upper_halves(behind(r0), behind(r1)), least));
        }
        w_parts[qt][0] = __builtin_bit_cast(bf16x8, part0);
        w_parts[qt][1] = __builtin_bit_cast(bf16x8, part1);
        w_parts[qt][2] = __builtin_bit_cast(bf16x8, part2);
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
        for (int e = 0; e < 3; ++e)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            o[qt][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w_parts[qt][e], o[qt][k], 0, 0, 0);
      }
      load_v(raw, next_ok ? Vl + next : pool.V);

      if (last) {
        // ---- out: lane (g, n) holds query n's elements (4 g + r) * kBlocks + k.  The waves of a wide workgroup leave what they
        // have in LDS, and wave r adds up the elements of its r.
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          l[qt] += __shfl_xor(l[qt], 16);
          l[qt] += __shfl_xor(l[qt], 32);
        }
        const bool whole = p0.at == 0 && p0.here == p0.t.n;
        const long long slot = 2ll * x + (p0.at == 0 ? 1 : 0);
        if constexpr (WIDE) {
          __syncthreads();  // no wave has K in LDS any more
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int k = 0; k < kBlocks; k += 4)
                part[wave][qt][r][k >> 2][lane] = f32x4{o[qt][k][r], o[qt][k + 1][r], o[qt][k + 2][r], o[qt][k + 3][r]};
            if (g == 0) part_stat[wave][qt][n] = make_float2(m[qt], l[qt]);
          }
          __syncthreads();
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const int hq = group * 16 * QT + qt * 16 + n;
          const long long h = (long long)kvh * G + hq;
          float top = m[qt], sum = l[qt];
          float weight[kWays];
          if constexpr (WIDE) {
            top = kNoMax;
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWays; ++w) top = fmaxf(top, part_stat[w][qt][n].x);
#pragma unroll
            for (int w = 0; w < kWays; ++w) {
              weight[w] = __builtin_amdgcn_exp2f((part_stat[w][qt][n].x - top) * sc);
              sum += part_stat[w][qt][n].y * weight[w];
            }
          }
          if (hq >= G) continue;
          const float inv = !whole ? 1.f : (sum == 0.f ? 0.f : a.v_scale / sum);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            f32x4 y[kBlocks / 4];
            int elements = (g * 4 + r) * kBlocks;
            if constexpr (WIDE) {
              if (r > 0) break;  // (this wave's r is its number)
              elements = (g * 4 + wave) * kBlocks;
#pragma unroll
              for (int k = 0; k < kBlocks / 4; ++k) {
                y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWays; ++w) y[k] += part[w][qt][wave][k][lane] * weight[w];
              }
            } else {
#pragma unroll
              for (int k = 0; k < kBlocks / 4; ++k)
                y[k] = f32x4{o[qt][4 * k][r], o[qt][4 * k + 1][r], o[qt][4 * k + 2][r], o[qt][4 * k + 3][r]};
            }
#pragma unroll
            for (int k = 0; k < kBlocks / 4; ++k) y[k] = scaled(y[k], inv);
            if (!whole || out_bytes == 4) {
              char* to = whole ? static_cast<char*>(a.O) + p0.b * a.ld_o + (h * D + elements) * 4
                               : reinterpret_cast<char*>(ly.partial + (slot * a.N + h) * D + elements);
#pragma unroll
              for (int k = 0; k < kBlocks / 4; ++k) reinterpret_cast<f32x4*>(to)[k] = y[k];
            } else {
              char* to = static_cast<char*>(a.O) + p0.b * a.ld_o + (h * D + elements) * 2;
              unsigned w[kBlocks / 2];
#pragma unroll
              for (int k = 0; k < kBlocks; k += 2) {
                bf16x2 pair;
                pair[0] = (__bf16)y[k >> 2][k & 3];
                pair[1] = (__bf16)y[k >> 2][(k & 3) + 1];
                w[k >> 1] = __builtin_bit_cast(unsigned, pair);
              }
              if constexpr (kBlocks == 8) *reinterpret_cast<u32x4*>(to) = u32x4{w[0], w[1], w[2], w[3]};
              else *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[1]};
            }
          }
          if (!whole && g == 0 && sub == 0) ly.stat[slot * a.N + h] = make_float2(top, sum);
        }
        if (ly.cut && p0.at == 0) {
          const int spans = whole ? 0 : (before + p0.t.n - 1) / share - x + 1;
          if (spans) join = make_int2(p0.b, spans);
          if (by_request && tells) ly.joins[p0.b] = make_int2(x, spans);
        }
        before += p0.t.n;
        if (p1.here == 0) break;
        clear();
        if constexpr (WIDE) __syncthreads();  // the sums are formed: K may come again
      }
      p0 = p1;
      s0 = s1;
      p1 = p2;
      s1 = s2;
      ok = next_ok;
    }
  }
  if (tells && !by_request) ly.joins[x] = join;

  // ---- requests without tiles: every columns-th from x on, looked through 64 at once
  for (int r0 = x; r0 < a.B; r0 += 64 * columns) {
    const long long mine_too = r0 + (long long)lane * columns;
    const bool empty = mine_too < a.B && request_tiles(a, a.kv_len[min(mine_too, a.B - 1ll)]).n == 0;
    for (unsigned long long todo = __ballot(empty); todo; todo &= todo - 1) {
      const int r = r0 + (__ffsll(todo) - 1) * columns;
      const int h0 = kvh * G + group * 16 * QT, bytes = min(16 * QT, G - group * 16 * QT) * D * out_bytes;
      char* to = static_cast<char*>(a.O) + r * a.ld_o + (long long)h0 * D * out_bytes;
      if (sub == 0)
        for (int i = lane * 16; i < bytes; i += 64 * 16) *reinterpret_cast<u32x4*>(to + i) = u32x4{0, 0, 0, 0};
      if (by_request && tells) ly.joins[r] = make_int2(0, 0);
    }
  }
}

// Joins the partial results of a request that is cut: one workgroup per (request, query head), D / 4 lanes to a partial
// result, four of them asked for at once, the others' in a fixed order.
template <int D, bool OUT_F32, int SPLIT>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttention a, Layout ly) {
  constexpr int kLanes = D / 4 / SPLIT, kSets = 256 / kLanes, kAhead = 4;
  const int h = blockIdx.y, first = blockIdx.z * (D / SPLIT);  // first element
  const int2 join = ly.joins[blockIdx.x];
  if (join.y == 0) return;
  const bool by_request = ly.joined == a.B;
  const int x = by_request ? join.x : blockIdx.x, b = by_request ? blockIdx.x : join.x;
  __shared__ float sm[kSets], sl[kSets];
  __shared__ f32x4 so[kSets][kLanes];
  const int set = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const float sc = exponent_scale(a);
  float m = kNoMax, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = set; p0 < join.y; p0 += kSets * kAhead) {
    float2 st[kAhead];
    f32x4 part[kAhead];
    float up = m;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int p = p0 + i * kSets;
      st[i] = make_float2(kNoMax, 0.f);
      part[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (p < join.y) {
        const long long at = (2ll * (x + p) + (p == 0 ? 1 : 0)) * a.N + h;
        st[i] = ly.stat[at];
        part[i] = *reinterpret_cast<const f32x4*>(ly.partial + at * D + first + lane * 4);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) up = fmaxf(up, st[i].x);
    const float keep = __builtin_amdgcn_exp2f((m - up) * sc);
    m = up;
    l *= keep;
    o *= keep;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float w = __builtin_amdgcn_exp2f((st[i].x - up) * sc);
      l += st[i].y * w;
      o += part[i] * w;
    }
  }
  const int sets = min(join.y, kSets);
  if (set < sets) {
    if (lane == 0) {
      sm[set] = m;
      sl[set] = l;
    }
    so[set][lane] = o;
  }
  __syncthreads();
  if (set > 0) return;
  float up = m;
  for (int i = 1; i < sets; ++i) up = fmaxf(up, sm[i]);
  const float keep = __builtin_amdgcn_exp2f((m - up) * sc);
  l *= keep;
  o *= keep;
  for (int i = 1; i < sets; ++i) {
    const float w = __builtin_amdgcn_exp2f((sm[i] - up) * sc);
    l += sl[i] * w;
    o += so[i][lane] * w;
  }
  o = scaled(o, l == 0.f ? 0.f : a.v_scale / l);
  char* to = static_cast<char*>(a.O) + b * a.ld_o + ((long long)h * D + first + lane * 4) * (OUT_F32 ? 4 : 2);
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

// Query heads of a key head: `groups` of up to 16 * qt.
struct Groups {
  int qt, groups;
};
Groups query_groups(int N, int N_kv, int D) {
  const int tiles = (N / N_kv + 15) / 16, most = D == 64 ? 3 : 2, groups = (tiles + most - 1) / most;
  return {(tiles + groups - 1) / groups, groups};
}
// Columns of a cut launch: eight waves per compute unit, which are all there at once.
int cut_columns(int heads, bool wide) {
  const int columns = 8 * compute_units() / (wide ? kWaves : 1) / heads;
  return columns < 1 ? 1 : columns;
}
size_t round16(size_t n) { return (n + 15) / 16 * 16; }

template <int D, int SPLIT>
void launch_join(hipStream_t st, const PagedAttention& a, const Layout& ly) {
  const dim3 grid((unsigned)ly.joined, (unsigned)a.N, SPLIT);
  if (a.out_dtype == PAFU_F32) hipLaunchKernelGGL((paged_join_kernel<D, true, SPLIT>), grid, dim3(256), 0, st, a, ly);
  else hipLaunchKernelGGL((paged_join_kernel<D, false, SPLIT>), grid, dim3(256), 0, st, a, ly);
}
template <int D, bool KV8, int QT, bool ONCE>
int launch(hipStream_t st, const PagedAttention& a, const PagedPool& pool, const Layout& ly, bool wide) {
  const long long jobs = (long long)ly.columns * ly.heads;
  const dim3 threads(64 * kWaves), blocks((unsigned)(wide ? jobs : (jobs + kWaves - 1) / kWaves));
  if (wide) hipLaunchKernelGGL((paged_attention_kernel<D, KV8, QT, true, ONCE>), blocks, threads, 0, st, a, pool, ly);
  else hipLaunchKernelGGL((paged_attention_kernel<D, KV8, QT, false, ONCE>), blocks, threads, 0, st, a, pool, ly);
  int rc = check_launch();
  if (rc || !ly.cut) return rc;
  // few requests in many columns: four workgroups to a row, which ask for four times as many partial results at once
  if (ly.columns >= 128 * ly.joined) launch_join<D, 4>(st, a, ly);
  else launch_join<D, 1>(st, a, ly);
  return check_launch();
}
// Do the rows of neighbouring heads share the 128 bytes of a line?
bool shared_lines(const PagedAttention& a, const PagedPool& pool) {
  return a.D == 64 && a.kv_dtype == PAFU_FP8_E4M3 && a.N_kv > 1 && pool.ld_head < 128;
}
template <int D, bool KV8, int QT>
int launch(hipStream_t st, const PagedAttention& a, const PagedPool& pool, const Layout& ly, bool wide) {
  // Past the caches from 16 MiB of K and V on, which is the most that the table has room for: 16 requests of 1000 tokens in 16
  // places of memory in turn 18.2 -> 16.9 us (in three places, which the caches hold, 15.1 -> 16.4), 32 of 1000 .. 2048
  // 42.5 -> 37.5; below, one of 4096 12.4 -> 12.8.
  const long long seen = a.window > 0 && a.window < a.max_tokens - (long long)a.n_pinned ? (long long)a.window + a.n_pinned : a.max_tokens;
  const bool small = seen * a.B * a.N_kv <= (16ll << 20) / (2 * D * (KV8 ? 1 : 2));
  return ly.groups == 1 && !shared_lines(a, pool) && !small ? launch<D, KV8, QT, true>(st, a, pool, ly, wide)
                                                            : launch<D, KV8, QT, false>(st, a, pool, ly, wide);
}
template <int D, bool KV8>
int launch(hipStream_t st, const PagedAttention& a, const PagedPool& pool, const Layout& ly, bool wide) {
  switch (query_groups(a.N, a.N_kv, D).qt) {
    case 1: return launch<D, KV8, 1>(st, a, pool, ly, wide);
    case 2: return launch<D, KV8, 2>(st, a, pool, ly, wide);
    default: return launch<64, KV8, 3>(st, a, pool, ly, wide);  // (D is 64)
  }
}

}  // namespace

size_t paged_attention_workspace_bytes(int B, int N, int N_kv, int D) {
  (void)B;
  const size_t columns = (size_t)cut_columns(N_kv * query_groups(N, N_kv, D).groups, false), rows = columns * 2 * N;
  return rows * D * 4 + round16(rows * 8) + round16(columns * 8);
}

int launch_paged_attention(hipStream_t st, const PagedAttention& a, const PagedPool& pool, void* workspace,
                           size_t workspace_bytes) {
  Layout ly;
  const Groups split = query_groups(a.N, a.N_kv, a.D);
  ly.groups = split.groups;
  ly.heads = a.N_kv * ly.groups;
  const long long longest = ((long long)a.max_tokens + kTile - 1) / kTile, items = (long long)a.B * ly.heads;
  const int units = compute_units();
  // Short requests are not cut: the join and the way to it (7 us) cost more than an even share is worth.  By the most tiles that
  // a request may have, cut -> whole: 8 tiles, 100 requests of 150 .. 250 tokens, 32 / 8 heads of 128, 26.5 -> 18.9 us; 16
  // tiles, 256 of 300 .. 512 86 -> 73 us, 400 of 100 .. 500 with one key head 27 -> 18; 32 tiles, 4 of 300 .. 1000 11.5 -> 17.4.
  // With more than 512 waves (two workgroups to a unit) and less than 2048 (all that fit) the longest ones decide, and how much
  // longer than the others they are the host does not know.  At 512 to 2048 waves, 9 .. 16 tiles, cut / whole on the average of 25
  // shapes: 1 .. 400 tokens 0.84 (0.66 .. 1.00), 100 .. 512 0.99, 300 .. 512 1.10, 500 .. 512 1.14 (1.00 .. 1.27): cut, for batches
  // are ragged.  Not with more than 16 query heads to a key head, whose partial results are as many: 1.41 (0.92 .. 1.80) of 47.
  const bool one_round = split.groups * split.qt == 1 && ly.heads >= kWaves && items > 2 * units && items < 8 * units;
  ly.cut = workspace != nullptr && workspace_bytes >= paged_attention_workspace_bytes(a.B, a.N, a.N_kv, a.D) &&
           longest > (one_round ? 8 : 16);
  ly.columns = a.B;
  ly.joined = 0;
  ly.partial = nullptr;
  ly.stat = nullptr;
  ly.joins = nullptr;
  // Cut: wide where a workgroup's four heads would not be neighbours in memory; narrow where waves share what they read, so that
  // they do so through one compute unit's cache (48 / 1 heads of 128 202 -> 156 us; 8-bit rows of 64, 8 / 2 heads, 112 -> 72).
  // Whole: wide where the requests may be long, or where the launch has few waves.
  const bool wide = ly.cut ? ly.groups == 1 && ((ly.heads < kWaves && !shared_lines(a, pool)) || pool.ld_head > pool.ld_token)
                           : longest > 16 || items <= 2 * units;
  if (ly.cut) {
    const size_t all = (size_t)cut_columns(ly.heads, false);
    const long long useful = longest * a.B, most = cut_columns(ly.heads, wide);
    ly.columns = (int)(useful < most ? useful : most);
    ly.joined = a.B < ly.columns ? a.B : ly.columns;
    char* w = static_cast<char*>(workspace);
    ly.partial = reinterpret_cast<float*>(w);
    w += all * 2 * a.N * a.D * 4;
    ly.stat = reinterpret_cast<float2*>(w);
    w += round16(all * 2 * a.N * 8);
    ly.joins = reinterpret_cast<int2*>(w);
  }
  const bool kv8 = a.kv_dtype == PAFU_FP8_E4M3;
  if (a.D == 128) return kv8 ? launch<128, true>(st, a, pool, ly, wide) : launch<128, false>(st, a, pool, ly, wide);
  return kv8 ? launch<64, true>(st, a, pool, ly, wide) : launch<64, false>(st, a, pool, ly, wide);
}

}  // namespace pafu

// Attention of many new tokens over the 8-bit cache on the sm_100a tensor cores: prompt chunks, head size 64 or 128.
//
// A CTA takes 256 query rows of a (request, kv head) -- row = new token x query head of the group -- as two tiles of 128, and a chunk
// of the request's keys in steps of 64 (four pages).  Everything the MMAs read is fp16, which holds an e4m3 code exactly: K and V codes
// are converted once per CTA, Q has its rows brought to [2^14, 2^15) by powers of two.  K's page scales multiply the scores.  A V scale is 2^e times a
// mantissa: the mantissa, 1 for the scales that the append writes, goes into the converted values, e into the exponent of the probabilities: P holds
// weights, probability x 2^e x 2^w, with a whole number w for each row that has brought its largest weight so far to at least 2^6 and lets none pass
// 2^15.  (With V relative to the largest scale of the chunk a page of large values took the bits of all others, from rows that did not see it, too.)  The maximum
// is kept as a whole number where its last bit would show beside e: what is added to and taken from an exponent then adds up without a rounding, whatever the
// page.  Roles:
//   warps 0-3, 4-7  softmax of tile 0 and 1, one thread per query row (at first: that row of Q into shared memory).  A row of S is read
//                   from tensor memory once and P written over it in fp16.  The running maximum is raised, and O rescaled, only when
//                   it grows by more than 2^8 or a weight would pass 2^15.  The warps of the two tiles on a scheduler take turns at the exponentials, so that one tile's
//                   scores are read and reduced while the other keeps the special-function unit busy;
//   warps 8, 9      issue S_g = Q_g K^T (M 128, N 64) into one of two buffers per tile, g = 0 and 1;
//   warps 10, 11    issue O_g += P_g V, P as the A operand from tensor memory, V as an MN-major B operand;
//   warps 12-15     request the pages of the next steps, one of each, and write them as the 128-byte-swizzled tiles that the MMAs want, and their scales where the softmax warps read them.  NaN
//                   codes of V are taken out (a zero probability times NaN is NaN) and the first key that has one is kept per dim: a row that
//                   sees it gets its NaN at the end.
// With several chunks of keys partial results go to scratch, as in the kernel for few rows, and are merged by the same kernel.
// Every mbarrier wait is bounded.
//
// Bound by the tensor cores on paper (2 products of rows x keys x hd), in fact by no unit alone.  Four prompt chunks of 509 to 1024 new tokens
// after up to 8192, 32 heads over 8, hd 128: 266 us, 893 TFLOP/s; hd 64: 213.  A step takes 2200 cycles: the tensor cores are at work in 1280
// (an MMA of N 64 takes 3/4 of one of N 128, as all of Q is read for it), the special-function unit in 1024, shared memory, by its bytes, in
// 1500.  Without any exponentials it took 5 % less, without the conversion 4 %, with an eighth of Q K^T 4.5 %.  9 us of a CTA are not its
// loop, and the last round of CTAs leaves 7 % of the SMs idle.  Tried: 16 softmax warps, two threads to a row, 295; 128 keys to a pass of the softmax, 295 (a longer chain from P V to
// the next scores outweighs the fewer hand-overs); without turns 283 (against 271 then).
#include <climits>

#include "../../include/epara.h"
#include "common.cuh"
#include "kernels.h"
#include "kv8.cuh"
#include "tcgen05.cuh"

namespace epara {

namespace {

using namespace tc;

constexpr int KF_STEP = 64, KF_TILE = 128;
constexpr int KF_S_WARP = 8, KF_PV_WARP = 10, KF_CONV_WARP = 12, KF_CONV_WARPS = 4;
constexpr int KF_THREADS = 32 * (KF_CONV_WARP + KF_CONV_WARPS);
constexpr int KF_Q_HALF = KF_TILE * 128, KF_KV_HALF = KF_STEP * 128;          // bytes of 64 columns of a tile
constexpr float KF_RAISE = 8.0f, KF_MOST = 15.0f;    // log2: of a probability, of a weight
constexpr int KF_PAIRS = 64, KF_BINS = 128;
constexpr int KF_INFO = 8;                            // steps whose scales are kept: at most STAGES + 2 are between a converter and the softmax

template <int HD>
struct KfGeo {
  static constexpr int NH = HD / 64;
  static constexpr int Q_BYTES = KF_Q_HALF * NH, KV_BYTES = KF_KV_HALF * NH;   // a tile of Q; a step's K or V
  static constexpr int STAGES = HD == 64 ? 4 : 3;                              // of converted K and V
  static constexpr int RAW = 4, RAW_BYTES = 2 * EPARA_KV_PAGE * HD;            // pages that a converter has requested, K and V of one
  static constexpr int OFF_KV = 2 * Q_BYTES;
  static constexpr int OFF_RAW = OFF_KV + STAGES * 2 * KV_BYTES;
  static constexpr int OFF_NAN = OFF_RAW + KF_CONV_WARPS * RAW * RAW_BYTES;    // first key with a NaN in V, per dim
  static constexpr int OFF_INFO = OFF_NAN + HD * 4;                            // K scales of a step's four pages, exponents of their V scales
  static constexpr int OFF_BAR = OFF_INFO + KF_INFO * 32;
  static constexpr int SMEM = 1024 + OFF_BAR + 512;
  static_assert(STAGES + 2 < KF_INFO, "a step's scales stay until they are read");
  static_assert(SMEM <= 227 * 1024 && 2 * SMEM > 227 * 1024, "one CTA, which takes all of the tensor memory, to an SM");
};
constexpr int KF_S_COL = 0, KF_O_COL = 256;          // TMEM columns: S / P buffers 0, 1 of tile 0, of tile 1; O_0, O_1

enum { KB_Q = 0, KB_S_FULL, KB_P_READY = KB_S_FULL + 4, KB_PV_DONE = KB_P_READY + 4, KB_K_FULL = KB_PV_DONE + 4, KB_K_EMPTY = KB_K_FULL + 6, KB_V_FULL = KB_K_EMPTY + 6,
       KB_V_EMPTY = KB_V_FULL + 6, KB_COUNT = KB_V_EMPTY + 6 };
static_assert(8 * KB_COUNT + 32 <= 512, "barrier area");

__device__ __forceinline__ uint32_t kf_idesc(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }   // fp16 x fp16 -> fp32
__device__ __forceinline__ uint64_t kf_desc_v(uint32_t addr) {
  uint64_t d = make_smem_desc(addr);
  d &= ~((uint64_t)0x3fff << 16);
  return d | (uint64_t)(KF_KV_HALF >> 4) << 16;       // 64-dim halves
}
__device__ __forceinline__ void kf_mma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void kf_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void kf_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t f2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void un_f2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float kf_max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// a (hi + lo), rounded once but for what lo's own product loses
__device__ __forceinline__ uint32_t hscale2(uint32_t a, uint32_t hi, uint32_t lo) {
  uint32_t r;
  asm("{\n\t.reg .b32 t;\n\tmul.rn.f16x2 t, %1, %3;\n\tfma.rn.f16x2 %0, %1, %2, t;\n\t}" : "=r"(r) : "r"(a), "r"(hi), "r"(lo));
  return r;
}

// The turns of the two softmax warps of a scheduler, a barrier each: a warp waits at its own for the other one's arrival.  They have no limit
// of their own: a warp that gives up goes on taking and passing its turns.
__device__ __forceinline__ void turn_wait(int warp) { asm volatile("barrier.cta.sync.aligned %0, 64;" ::"r"(1 + warp) : "memory"); }
__device__ __forceinline__ void turn_pass(int warp) { asm volatile("barrier.cta.arrive.aligned %0, 64;" ::"r"(1 + (warp ^ 4)) : "memory"); }

// The exponents are score x factor - maximum, fused.  Beyond 2^22 a row has score and maximum scaled down to [2^21, 2^22) by a power of two: whole numbers
// that the exponent of a V scale can be added to; the scores' own sums are not as exact as that.  Equal scores have equal weights, others next to none, as
// they should.
__device__ __forceinline__ float scale_down(float m) {
  return fabsf(m) > 4194304.f ? __uint_as_float((275u - (__float_as_uint(fabsf(m)) >> 23)) << 23) : 1.f;
}
// What a row's maximum is kept as: itself, so that the probability of its token is exactly 1, up to 2^10, where the exponent of a V scale adds to it within 2^-15;
// beyond it the next whole number, scaled down, at or above it.
__device__ __forceinline__ float reference(float m) {
  const float d = scale_down(m);
  return fabsf(m) <= 1024.f ? m : ceilf(m * d) / d;
}

template <int HD>
__global__ void __launch_bounds__(KF_THREADS, 1) kv8_flash_kernel(const Kv8Attn a) {
  using Geo = KfGeo<HD>;
  constexpr int ST = Geo::STAGES, NX = HD / 32;       // ... 16-byte pieces of a page tile in a lane
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* const base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  int* const nan_key = reinterpret_cast<int*>(base_ptr + Geo::OFF_NAN);
  const uint32_t bars = base + Geo::OFF_BAR;
  auto bar = [&](int i) { return bars + 8u * i; };
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + Geo::OFF_BAR + 8 * KB_COUNT);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* const any_nan = reinterpret_cast<int*>(tmem_slot + 2);
  float* const info = reinterpret_cast<float*>(base_ptr + Geo::OFF_INFO);              // [KF_INFO][K scales, V exponents][4]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // ---- the work item.  The longest ones start first: requests in order of their lengths, of each one the last rows first.  (In order of
  // the rows alone a long request with few rows came late: 362 us for the four prompt chunks, like this 283.)
  const int kvh = blockIdx.x % a.Hkv, item = blockIdx.x / a.Hkv, chunk = blockIdx.y;
  __shared__ int the_request, the_tile, all_tiles, all_live, warp_tiles[KF_THREADS / 32];
  pdl_wait();
  int b = item / a.tiles, pair = a.tiles - 1 - item % a.tiles;
  if (a.ordered) {
    static_assert(KF_PAIRS * 16 + KF_BINS * 4 + KV8_FLASH_MOST * 4 <= Geo::OFF_RAW, "room for the order");
    int4* const live = reinterpret_cast<int4*>(base_ptr);             // length, request, tiles of those that this launch takes, the first KF_PAIRS
    int* const bins = reinterpret_cast<int*>(live + KF_PAIRS);        // tiles of the requests with lengths like these
    int* const all = bins + KF_BINS;                                  // each request's tiles x KF_BINS + its bin
    const int shift = max(32 - __clz(a.max_len) - 7, 0);
    if (threadIdx.x == 0) { all_tiles = all_live = 0; the_request = -1; }
    if (threadIdx.x < KF_BINS) bins[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.B; i += KF_THREADS) {
      int row0, n;
      new_rows(a.q_rows, i, a.T, row0, n);
      n = min(n, a.max_q);
      all[i] = 0;
      if (n < a.min_n) continue;
      const int tiles = (n * a.G + 2 * KF_TILE - 1) / (2 * KF_TILE), length = min(max(a.kv_lens[i], 0), a.max_len), bin = length >> shift, at = atomicAdd(&all_live, 1);
      if (at < KF_PAIRS) live[at] = make_int4(length, i, tiles, 0);   // (in any order: what follows looks at lengths and requests)
      all[i] = tiles * KF_BINS + bin;
      atomicAdd(&bins[bin], tiles);
      atomicAdd(&all_tiles, tiles);
    }
    __syncthreads();
    if (item >= all_tiles) return;
    if (all_live <= KF_PAIRS) {
      for (int i = threadIdx.x; i < all_live; i += KF_THREADS) {
        const int4 own = live[i];
        int before = 0;
        for (int k = 0; k < all_live; ++k) {
          const int4 other = live[k];
          if (other.x > own.x || (other.x == own.x && other.y < own.y)) before += other.z;
        }
        if (item >= before && item < before + own.z) { the_request = own.y; the_tile = own.z - 1 - (item - before); }
      }
    } else {
      // More requests than that are put in order by the first seven bits of their lengths, the ones that agree in them by their place: the bin that holds
      // this item, from the longest one on, and then the request of the bin.  (All pairs of 1000 requests took 34 us a CTA: with 64 tokens each 3230 us, like
      // this 1450; 500 894 and 695.)
      int own[KF_BINS / 32], sum = 0, upto;
#pragma unroll
      for (int k = 0; k < KF_BINS / 32; ++k) sum += own[k] = bins[KF_BINS - 1 - lane * (KF_BINS / 32) - k];
      auto running = [&](int v) {                     // sum of the lanes up to this one
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) {
          const int other = __shfl_up_sync(0xffffffffu, v, x);
          if (lane >= x) v += other;
        }
        return v;
      };
      upto = running(sum);
      int before = upto - sum, bin = KF_BINS - 1 - lane * (KF_BINS / 32);
      const int from = __ffs(__ballot_sync(0xffffffffu, item >= before && item < upto)) - 1;
#pragma unroll
      for (int k = 0; k < KF_BINS / 32 - 1; ++k)
        if (bin == KF_BINS - 1 - lane * (KF_BINS / 32) - k && item >= before + own[k]) { before += own[k]; --bin; }
      bin = __shfl_sync(0xffffffffu, bin, max(from, 0));
      int rest = item - __shfl_sync(0xffffffffu, before, max(from, 0));
      // each thread some requests in a row
      const int per = (a.B + KF_THREADS - 1) / KF_THREADS, i0 = threadIdx.x * per;
      sum = 0;
      for (int i = i0; i < min(i0 + per, a.B); ++i) if ((all[i] & (KF_BINS - 1)) == bin) sum += all[i] / KF_BINS;
      upto = running(sum);
      if (lane == 31) warp_tiles[warp] = upto;
      __syncthreads();
      for (int w = 0; w < warp; ++w) rest -= warp_tiles[w];
      rest -= upto - sum;
      if (rest >= 0 && rest < sum)
        for (int i = i0; i < min(i0 + per, a.B); ++i) {
          const int tiles = (all[i] & (KF_BINS - 1)) == bin ? all[i] / KF_BINS : 0;
          if (rest >= 0 && rest < tiles) { the_request = i; the_tile = tiles - 1 - rest; }
          rest -= tiles;
        }
    }
    __syncthreads();
    b = the_request;
    pair = the_tile;
    if (b < 0) return;                                // (prefix sums that are none)
  }
  int row0, n;
  new_rows(a.q_rows, b, a.T, row0, n);
  const int G = a.G, len = min(max(a.kv_lens[b], 0), a.max_len);
  const int seen0 = len - n + 1;                      // keys that new token 0 attends to
  if (n > a.max_q) {
    if (threadIdx.x == 0 && pair == 0 && kvh == 0 && chunk == 0) atomicExch(a.status, ERR_ROWS);
    n = a.max_q;
  }
  if (n < a.min_n) return;
  const int r_first = pair * 2 * KF_TILE, rows = min(n * G - r_first, 2 * KF_TILE);
  if (rows <= 0) return;
  const int t_begin = chunk * a.chunk, t_end = min(seen0 + (r_first + rows - 1) / G, t_begin + a.chunk);
  if (t_begin >= t_end) return;
  const int n_mt = rows > KF_TILE ? 2 : 1, steps = (t_end - t_begin + KF_STEP - 1) / KF_STEP;
  const int pg0 = t_begin / EPARA_KV_PAGE, n_pages = (t_end - t_begin + EPARA_KV_PAGE - 1) / EPARA_KV_PAGE;
  const int32_t* const table = a.tables + (size_t)b * a.table_stride + pg0;
  auto page_id = [&](int i) {                         // of the chunk's page i; -1: none, or outside the pool
    int id = i < n_pages ? table[i] : -1;
    return id < a.kv_pages ? id : -1;
  };

  if (threadIdx.x == 0) {
    mbar_init(bar(KB_Q), 8);
    for (int i = 0; i < 4; ++i) { mbar_init(bar(KB_S_FULL + i), 1); mbar_init(bar(KB_P_READY + i), 4); mbar_init(bar(KB_PV_DONE + i), 1); }
    for (int s = 0; s < ST; ++s) {
      mbar_init(bar(KB_K_FULL + s), KF_CONV_WARPS); mbar_init(bar(KB_K_EMPTY + s), n_mt);
      mbar_init(bar(KB_V_FULL + s), KF_CONV_WARPS); mbar_init(bar(KB_V_EMPTY + s), n_mt);
    }
    *abort_flag = 0;
    *any_nan = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = threadIdx.x; i < HD; i += KF_THREADS) nan_key[i] = INT_MAX;
  if (warp == KF_S_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  bool ok = true;
  float m_ref = 0.f, l = 0.f, row_f = 0.f, up_w = 0.f;            // softmax threads: the row's maximum (log2 domain), sum, score factor, w of its weights
  const int g = warp >> 2, row = (warp & 3) * 32 + lane, rr = r_first + g * KF_TILE + row;         // (warps 0 .. 7)
  const bool row_live = warp < 8 && g * KF_TILE + row < rows;
  const int seen = row_live ? seen0 + rr / G : 0;     // keys that the row attends to

  if (warp >= KF_CONV_WARP) {
    // ------------------------------------------------------------------ converters
    const int cw = warp - KF_CONV_WARP;               // this warp's page of a step
    auto look_up = [&](int i) {                       // (each page of the chunk once, by one lane: ids outside the pool are reported here)
      const int id = page_id(i);
      if (id < 0 && i < n_pages) atomicExch(a.status, ERR_PAGE_ATTEND);
      return id;
    };
    int id_cur = look_up(lane * 4 + cw), id_next = look_up((lane + 32) * 4 + cw);      // of 32 steps each
    auto k_scale = [&](int id) { return id >= 0 ? a.scales[(size_t)id * 2 * a.Hkv + kvh] : 0.f; };
    auto v_scale = [&](int id) { return id >= 0 ? a.scales[((size_t)id * 2 + 1) * a.Hkv + kvh] : 0.f; };
    float ks_cur = k_scale(id_cur), ks_next = k_scale(id_next), vs_cur = v_scale(id_cur), vs_next = v_scale(id_next);
    // The pages of the next steps are requested as 16-byte asynchronous copies into a ring of this warp's own: a step is shorter than
    // the way to memory.  (By itself no faster than one step's loads in registers, 359 and 362 us for the four prompt chunks, but these
    // registers are what the conversion needs.)
    const uint32_t raw = base + Geo::OFF_RAW + cw * Geo::RAW * Geo::RAW_BYTES;
    int where[NX], rawat[NX], place[NX];              // of a piece in the page tile, in the ring and in the converted tile (its first half)
#pragma unroll
    for (int x = 0; x < NX; ++x) {
      const int half = HD == 128 ? x & 1 : 0, r = (HD == 128 ? x >> 1 : x) * 8 + (lane >> 2), R = cw * 16 + r;
      where[x] = r * HD + half * 64 + (lane & 3) * 16;
      rawat[x] = HD == 128 ? where[x] ^ ((r & 1) << 6) : where[x];             // (rows in turn in different banks)
      place[x] = half * KF_KV_HALF + R * 128 + ((((lane & 3) * 2) ^ (R & 7)) << 4);
    }
    auto request = [&](int j) {
      if (j < steps) {
        const int id = __shfl_sync(0xffffffffu, (j & 32) == 0 ? id_cur : id_next, j & 31);
        const uint32_t dst = raw + (j % Geo::RAW) * Geo::RAW_BYTES;
        const unsigned char* p = a.codes + ((size_t)max(id, 0) * 2 * a.Hkv + kvh) * EPARA_KV_PAGE * HD;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
          for (int x = 0; x < NX; ++x) cp16_zfill(dst + kv * (EPARA_KV_PAGE * HD) + rawat[x], p + (size_t)kv * a.Hkv * EPARA_KV_PAGE * HD + where[x], id >= 0);
      }
      cp_commit();
    };
    auto fetch = [&](int j, int is_v, uint4* u) {
#pragma unroll
      for (int x = 0; x < NX; ++x) u[x] = lds16(raw + (j % Geo::RAW) * Geo::RAW_BYTES + is_v * (EPARA_KV_PAGE * HD) + rawat[x]);
    };
    auto put = [&](unsigned char* tile, int x, const uint4& u, bool scaled, uint32_t hi2, uint32_t lo2) {
      uint4 lo = make_uint4(to_f16x2(u.x), to_f16x2(u.x >> 16), to_f16x2(u.y), to_f16x2(u.y >> 16));
      uint4 hi = make_uint4(to_f16x2(u.z), to_f16x2(u.z >> 16), to_f16x2(u.w), to_f16x2(u.w >> 16));
      if (scaled) {
        lo.x = hscale2(lo.x, hi2, lo2); lo.y = hscale2(lo.y, hi2, lo2); lo.z = hscale2(lo.z, hi2, lo2); lo.w = hscale2(lo.w, hi2, lo2);
        hi.x = hscale2(hi.x, hi2, lo2); hi.y = hscale2(hi.y, hi2, lo2); hi.z = hscale2(hi.z, hi2, lo2); hi.w = hscale2(hi.w, hi2, lo2);
      }
      *reinterpret_cast<uint4*>(tile + place[x]) = lo;
      *reinterpret_cast<uint4*>(tile + (place[x] ^ 16)) = hi;
    };
#pragma unroll
    for (int j = 0; j < Geo::RAW - 1; ++j) request(j);
    for (int j = 0; j < steps; ++j) {
      const int slot = j % ST;
      const uint32_t parity = ((j / ST) & 1u) ^ 1u;
      if ((j & 31) == 0 && j > 0) {                   // the 32 steps after the next ones
        const int id = look_up((lane + j + 32) * 4 + cw);
        if (j & 32) { id_cur = id; ks_cur = k_scale(id); vs_cur = v_scale(id); } else { id_next = id; ks_next = k_scale(id); vs_next = v_scale(id); }
      }
      unsigned char* const kt = base_ptr + Geo::OFF_KV + slot * 2 * Geo::KV_BYTES;
      request(j + Geo::RAW - 1);                      // into the place that the step before has left
      cp_wait<Geo::RAW - 1>();
      __syncwarp();
      uint4 kx[NX], vx[NX];
      fetch(j, 0, kx);
      fetch(j, 1, vx);
      if (j >= ST && !mbar_wait(bar(KB_K_EMPTY + slot), parity, abort_flag)) { ok = false; if (lane == 0) atomicExch(a.status, 23); break; }
#pragma unroll
      for (int x = 0; x < NX; ++x) put(kt, x, kx[x], false, 0u, 0u);
      const float ks = __shfl_sync(0xffffffffu, (j & 32) == 0 ? ks_cur : ks_next, j & 31), vs = __shfl_sync(0xffffffffu, (j & 32) == 0 ? vs_cur : vs_next, j & 31);
      const uint32_t vb = __float_as_uint(vs);
      const float mant = vb < 0x00800000u ? vs * 8.5070592e37f : __uint_as_float((vb & 0x007fffffu) | 0x3f800000u);        // (x 2^126)
      if (lane == 0) {
        float* const to = info + (j % KF_INFO) * 8 + cw;
        to[0] = ks;
        to[4] = (float)((int)max(vb >> 23, 1u) - 127);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(KB_K_FULL + slot));
      const bool scaled = mant != 1.f;
      const uint32_t mant_hi = pack_f16(mant, mant);
      const float rest = mant - __half2float(__ushort_as_half((unsigned short)mant_hi));
      const uint32_t mant_lo = pack_f16(rest, rest);
      const int t0 = t_begin + j * KF_STEP + cw * 16;
      uint32_t nan = 0;
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        if (t0 + 16 > t_end && t0 + (HD == 128 ? x >> 1 : x) * 8 + (lane >> 2) >= t_end) vx[x] = make_uint4(0u, 0u, 0u, 0u);   // may hold anything
        // (a byte of 0x7f, sign aside, carries into its top bit)
        nan |= ((vx[x].x & 0x7f7f7f7fu) + 0x01010101u) | ((vx[x].y & 0x7f7f7f7fu) + 0x01010101u) | ((vx[x].z & 0x7f7f7f7fu) + 0x01010101u) |
               ((vx[x].w & 0x7f7f7f7fu) + 0x01010101u);
      }
      if (nan & 0x80808080u) {
        *any_nan = 1;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
          const int key = t0 + (HD == 128 ? x >> 1 : x) * 8 + (lane >> 2), dim = (HD == 128 ? x & 1 : 0) * 64 + (lane & 3) * 16;
          auto clean = [&](uint32_t& w, int d) {
            const uint32_t mask = __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu);
            w &= ~mask;
            for (int e = 0; e < 4; ++e) if (mask >> (8 * e) & 1u) atomicMin(nan_key + d + e, key);
          };
          clean(vx[x].x, dim); clean(vx[x].y, dim + 4); clean(vx[x].z, dim + 8); clean(vx[x].w, dim + 12);
        }
      }
      __syncwarp();
      if (j >= ST && !mbar_wait(bar(KB_V_EMPTY + slot), parity, abort_flag)) { ok = false; if (lane == 0) atomicExch(a.status, 24); break; }
#pragma unroll
      for (int x = 0; x < NX; ++x) put(kt + Geo::KV_BYTES, x, vx[x], scaled, mant_hi, mant_lo);
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(KB_V_FULL + slot));
    }
    if (!ok) *abort_flag = 1;
  } else if (warp == KF_S_WARP || warp == KF_S_WARP + 1) {
    // ------------------------------------------------------------------ issuers of S_t
    const int t = warp - KF_S_WARP;
    const uint32_t idesc = kf_idesc(KF_STEP);
    if (!mbar_wait<false>(bar(KB_Q), 0u, abort_flag)) { ok = false; if (lane == 0) atomicExch(a.status, 25); }
    const uint64_t dq = make_smem_desc(base + t * Geo::Q_BYTES);
    for (int j = 0; j < steps && ok && t < n_mt; ++j) {
      const int slot = j % ST, sb = j & 1;
      // the buffer holds P until the P V of two steps ago is complete
      if (!mbar_wait<false>(bar(KB_K_FULL + slot), (j / ST) & 1u, abort_flag) ||
          (j >= 2 && !mbar_wait<false>(bar(KB_PV_DONE + 2 * t + sb), ((j >> 1) - 1) & 1u, abort_flag))) {
        ok = false;
        if (lane == 0) atomicExch(a.status, 26);
        break;
      }
      tc_fence_after();
      const uint64_t dk = make_smem_desc(base + Geo::OFF_KV + slot * 2 * Geo::KV_BYTES);
      const uint32_t d = tmem_base + KF_S_COL + t * 128 + sb * 64;
#pragma unroll
      for (int k = 0; k < HD / 16; ++k)
        mma_f16_elect(d, dq + (uint64_t)((k >> 2) * (KF_Q_HALF >> 4) + (k & 3) * 2), dk + (uint64_t)((k >> 2) * (KF_KV_HALF >> 4) + (k & 3) * 2), idesc, k > 0 ? 1u : 0u);
      mma_commit_elect(bar(KB_S_FULL + 2 * t + sb));
      mma_commit_elect(bar(KB_K_EMPTY + slot));
    }
    if (!ok) *abort_flag = 1;
  } else if (warp >= KF_PV_WARP) {
    // ------------------------------------------------------------------ issuers of O_t += P_t V
    const int t = warp - KF_PV_WARP;
    const uint32_t idesc = kf_idesc(HD) | (1u << 16), d = tmem_base + KF_O_COL + t * HD;           // B operand MN-major
    for (int j = 0; j < steps && t < n_mt; ++j) {
      const int slot = j % ST, sb = j & 1;
      if (!mbar_wait<false>(bar(KB_V_FULL + slot), (j / ST) & 1u, abort_flag) || !mbar_wait<false>(bar(KB_P_READY + 2 * t + sb), (j >> 1) & 1u, abort_flag)) {
        ok = false;
        if (lane == 0) atomicExch(a.status, 28);
        break;
      }
      tc_fence_after();
      const uint32_t p = tmem_base + KF_S_COL + t * 128 + sb * 64;
      const uint64_t dv = kf_desc_v(base + Geo::OFF_KV + slot * 2 * Geo::KV_BYTES + Geo::KV_BYTES);
#pragma unroll
      for (int k = 0; k < KF_STEP / 16; ++k) kf_mma_ts(d, p + k * 8, dv + (uint64_t)(k * 128), idesc, (j > 0 || k > 0) ? 1u : 0u);   // 16 keys = 2 KB
      mma_commit_elect(bar(KB_PV_DONE + 2 * t + sb));
      mma_commit_elect(bar(KB_V_EMPTY + slot));
    }
    if (!ok) *abort_flag = 1;
  } else {
    // ------------------------------------------------------------------ softmax
    {
      uint4 u[HD / 8];
      float top = 0.f;
      const bf16* const qp = a.q + (size_t)(row0 + rr / G) * a.q_stride + (size_t)(kvh * G + rr % G) * HD;
#pragma unroll
      for (int x = 0; x < HD / 8; ++x) u[x] = row_live ? __ldcg(reinterpret_cast<const uint4*>(qp) + x) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int x = 0; x < HD / 8; ++x) {
        float f[8];
        unpack8(u[x], f);
#pragma unroll
        for (int y = 0; y < 8; ++y) top = fmaxf(top, fabsf(f[y]));
      }
      float up;
      row_f = row_factor<HD>(top, up);
#pragma unroll
      for (int x = 0; x < HD / 8; ++x) {
        float f[8];
        unpack8(u[x], f);
        const uint4 h = make_uint4(pack_f16(f[0] * up, f[1] * up), pack_f16(f[2] * up, f[3] * up), pack_f16(f[4] * up, f[5] * up), pack_f16(f[6] * up, f[7] * up));
        *reinterpret_cast<uint4*>(base_ptr + g * Geo::Q_BYTES + (x >> 3) * KF_Q_HALF + row * 128 + (((x & 7) ^ (row & 7)) << 4)) = h;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(KB_Q));
    }
    const uint32_t lane_base = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_base + KF_S_COL + g * 128, o_addr = lane_base + KF_O_COL + g * HD;
    const int warp_rows = min(rows - g * KF_TILE - (warp & 3) * 32, 32);       // live ones
    const int warp_r0 = r_first + g * KF_TILE + (warp & 3) * 32;
    const int seen_least = seen0 + warp_r0 / G, seen_most = warp_rows > 0 ? seen0 + (warp_r0 + warp_rows - 1) / G : 0;
    // (every turn is taken and passed on once a step, whatever happens; the one before tile 0's first is passed here, tile 1's last one is
    // not passed on)
    float down = 1.f;
    const bool turns = n_mt == 2;
    if (turns && g == 1) turn_pass(warp);
    int j = 0;
    for (; j < steps && g < n_mt; ++j) {
      const int sb = j & 1, k0 = t_begin + j * KF_STEP;
      if (!mbar_wait<false>(bar(KB_S_FULL + 2 * g + sb), (j >> 1) & 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(a.status, 29); break; }
      tc_fence_after();
      const uint32_t addr = s_addr + sb * 64;
      if (k0 >= seen_most) {                          // no row of the warp sees any of these keys
        const uint32_t z[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
        if (turns) {
          turn_wait(warp);
          if (g == 0 || j + 1 < steps) turn_pass(warp);
        }
#pragma unroll
        for (int c = 0; c < 32; c += 8) kf_st8(addr + c, z);
        kf_st_wait();
      } else {
        uint32_t v[64];
        tmem_ld32_nowait(addr, v);
        tmem_ld32_nowait(addr + 32, v + 32);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_regs_ready16(v + 16 * c);
        if (k0 + KF_STEP > seen_least) {              // some row's limit lies in this step
#pragma unroll
          for (int i = 0; i < 64; ++i) if (k0 + i >= seen) v[i] = 0xff800000u;
        }
        // (the converters wrote them before they reported this step's K)
        const float4 kq = *reinterpret_cast<const float4*>(info + (j % KF_INFO) * 8), vq = *reinterpret_cast<const float4*>(info + (j % KF_INFO) * 8 + 4);
        const float f[4] = {fmaxf(row_f * kq.x, KV8_TINY_SCALE), fmaxf(row_f * kq.y, KV8_TINY_SCALE), fmaxf(row_f * kq.z, KV8_TINY_SCALE), fmaxf(row_f * kq.w, KV8_TINY_SCALE)};
        const float ve[4] = {vq.x, vq.y, vq.z, vq.w};
        float mx = -INFINITY, most[4];                // a page's largest score, without its factor
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
          for (int i = 16 * p; i < 16 * p + 16; i += 4) {
            m0 = kf_max3(m0, __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
            m1 = kf_max3(m1, __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
          }
          most[p] = fmaxf(m0, m1);
          mx = fmaxf(mx, most[p] * f[p]);
        }
        float add[4], k[4];                           // weight = 2^(score x factor + add), probability = weight x 2^-k
        auto exponents = [&] {                        // answers the largest weight's
          float top = -INFINITY;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            k[p] = fminf(fmaxf(ve[p] + up_w, -64.f), 126.f);               // (weights 2^-64 below: zeros in fp16, but their probabilities count)
            add[p] = k[p] - m_ref * down;
            top = fmaxf(top, fmaf(most[p], fmaxf(f[p] * down, KV8_TINY_SCALE), add[p]));
          }
          return top;
        };
        auto lowered = [&](float w) {                 // w, if it is no more than what brings the step's largest weight to (2^6, 2^7]
          float top = -INFINITY;
#pragma unroll
          for (int p = 0; p < 4; ++p) top = fmaxf(top, fmaf(most[p], fmaxf(f[p] * down, KV8_TINY_SCALE), -m_ref * down) + ve[p]);
          return fminf(fminf(w, 7.f - ceilf(top)), (float)KV8_MOST_UP);
        };
        if (j == 0) {
          m_ref = mx == -INFINITY ? 0.f : reference(mx);         // (a row that sees a key of the chunk sees its first one)
          down = scale_down(m_ref);
          up_w = lowered(INFINITY);
          exponents();
        } else if (__any_sync(0xffffffffu, (exponents() > KF_MOST || mx - m_ref > KF_RAISE) && row_live)) {
          const float m_new = fmaxf(m_ref, reference(mx)), lift = m_new - m_ref, before = up_w;
          m_ref = m_new;
          down = scale_down(m_ref);
          up_w = lowered(before + floorf(lift));
          exponents();
          const float r = ex2(up_w - before - lift);
          l *= ex2(-lift);
          // every P V up to the step before must be complete
          if (!mbar_wait<false>(bar(KB_PV_DONE + 2 * g + (sb ^ 1)), ((j - 1) >> 1) & 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(a.status, 30); break; }
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < HD; c += 16) {
            uint32_t o[16];
            tmem_ld16(o_addr + c, o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * r);
            kf_st8(o_addr + c, o);
            kf_st8(o_addr + c + 8, o + 8);
          }
        }
        if (turns) turn_wait(warp);
        uint64_t la = 0, lb = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const float fd = fmaxf(f[p] * down, KV8_TINY_SCALE);             // (not zero: a masked score times zero is NaN)
          const float back = __int_as_float((__float_as_int(12582912.f - k[p]) << 23) + 0x3f800000);           // 2^-k
          const uint64_t ff = f2(fd, fd), nm = f2(add[p], add[p]), to_p = f2(back, back);
          uint32_t h[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float x, y;
            un_f2(fma2(f2(__uint_as_float(v[16 * p + 2 * i]), __uint_as_float(v[16 * p + 2 * i + 1])), ff, nm), x, y);
            x = ex2(x);
            y = ex2(y);
            if (i & 1) lb = fma2(f2(x, y), to_p, lb); else la = fma2(f2(x, y), to_p, la);
            h[i] = pack_f16(x, y);
          }
          kf_st8(addr + 8 * p, h);
        }
        if (turns && (g == 0 || j + 1 < steps)) turn_pass(warp);
        float a0, a1, a2, a3;
        un_f2(la, a0, a1);
        un_f2(lb, a2, a3);
        l += (a0 + a1) + (a2 + a3);
        kf_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(KB_P_READY + 2 * g + sb));
    }
    if (!ok) {
      *abort_flag = 1;
      for (; turns && j < steps; ++j) {               // (it gave up before this step's turn)
        turn_wait(warp);
        if (g == 0 || j + 1 < steps) turn_pass(warp);
      }
    }
    if (ok && g < n_mt && !mbar_wait<false>(bar(KB_PV_DONE + 2 * g + ((steps - 1) & 1)), ((steps - 1) >> 1) & 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(a.status, 18); }
    if (!ok) *abort_flag = 1;
  }
  __syncthreads();                                    // (what the converters found is there)
  if (warp < 8 && g < n_mt && ok) {
    // ------------------------------------------------------------------ output: a thread has a row
    tc_fence_after();
    constexpr int PITCH = HD + 4;
    static_assert(8 * 32 * PITCH * 4 <= Geo::OFF_NAN, "staging area");
    const uint32_t o_addr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + KF_O_COL + g * HD;
    const bool nans = *any_nan != 0, direct = seen <= a.chunk, write = row_live && seen > t_begin;
    const size_t qr = (size_t)(row0 + rr / G) * a.Hkv * G + kvh * G + rr % G;
    bf16* const out = a.out + qr * HD;
    const float inv = direct ? 1.f / l : 1.f, back = __int_as_float((127 - (int)up_w) << 23);          // 2^-w
    // Partial results leave through shared memory, which is idle now, row by row: stores of a row by each thread move 32 pieces of 8 bytes (64 tokens
    // at the end of 4096, hd 128 35 us, like this 27).  For final rows, 16 bytes a thread, that would be the slower way (64 / 68 us).
    const uint32_t partials = __ballot_sync(0xffffffffu, write && !direct);
    float* const stage = reinterpret_cast<float*>(base_ptr) + warp * 32 * PITCH;
#pragma unroll 1
    for (int c = 0; c < HD; c += 32) {
      uint32_t o[32];
      tmem_ld32(o_addr + c, o);
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * inv * back);
      if (nans) {
#pragma unroll
        for (int i = 0; i < 32; ++i) if (nan_key[c + i] < seen) o[i] = 0x7fffffffu;
      }
      if (write && direct) {
        if ((reinterpret_cast<uintptr_t>(out) & 15) == 0) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            uint4 w;
            w.x = pack2(__uint_as_float(o[i]), __uint_as_float(o[i + 1])); w.y = pack2(__uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
            w.z = pack2(__uint_as_float(o[i + 4]), __uint_as_float(o[i + 5])); w.w = pack2(__uint_as_float(o[i + 6]), __uint_as_float(o[i + 7]));
            *reinterpret_cast<uint4*>(out + c + i) = w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) out[c + i] = f2bf(__uint_as_float(o[i]));
        }
      } else if (write) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(stage + lane * PITCH + c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
      }
      __syncwarp();
    }
    if (partials != 0) {
      float* const part = a.partial + (qr * a.max_chunks + chunk) * (HD + 2);
#pragma unroll 4
      for (int r = 0; r < 32; ++r) {
        if ((partials >> r & 1u) == 0) continue;
        float* const to = reinterpret_cast<float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(part), r)) + 2 + lane * 2;
#pragma unroll
        for (int k = 0; k < HD; k += 64) __stcg(reinterpret_cast<float2*>(to + k), *reinterpret_cast<const float2*>(stage + r * PITCH + k + lane * 2));
      }
      if (write && !direct) __stcg(reinterpret_cast<float2*>(part), make_float2(m_ref, l));
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == KF_S_WARP) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

template <int HD>
cudaError_t launch_as(const Kv8Attn& a, long long items, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(kv8_flash_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, KfGeo<HD>::SMEM);
  if (e != cudaSuccess) return e;
  return launch_pdl(kv8_flash_kernel<HD>, dim3((unsigned)(items * a.Hkv), (unsigned)a.max_chunks), dim3(KF_THREADS), KfGeo<HD>::SMEM, st, a);
}

}  // namespace

cudaError_t launch_kv8_flash(const Kv8Attn& a, int hd, long long items, cudaStream_t st) { return hd == 128 ? launch_as<128>(a, items, st) : launch_as<64>(a, items, st); }

}  // namespace epara

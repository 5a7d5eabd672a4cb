// Paged KV cache in 8 bits: the append that fills it and the attention that reads it.
//
// A cache layer holds e4m3 codes [page][K|V][kv head][16 tokens][hd] and one fp32 scale for each (page, K|V, kv head): a value
// is code x scale.  The append writes scales that are powers of two: e4m3 is a floating-point format, so a scale only has to
// keep the largest value below 448 and a tighter one would gain no precision; and when a later token of a page needs a larger
// scale, the page's older codes are rescaled without a second rounding (but for values that become subnormal).
#include <algorithm>
#include <cmath>

#include "../../include/epara.h"
#include "common.cuh"
#include "kernels.h"
#include "kv8.cuh"

namespace epara {

namespace {

constexpr int PAGE = EPARA_KV_PAGE;

// ------------------------------------------------------------------------------------------------ append
// A block takes one page of one request, a warp one (K or V, kv head) of it: 16 x hd values in registers, so the maximum, the
// scale and the codes come out of one read.  Bound by HBM: 24 chunks of 65 to 1024 tokens, 8 kv heads, hd 128 14.5 us, floor 12.3 (bf16 in, a byte and
// 1/512 of a scale an element out); one token of each of 64 requests 2.6 us, a launch.
// Blocks: for each request as many as max_q tokens can lie on pages; BY_ROW, where few requests have that many, one for each row of k, which
// takes the page that its row is the first one on (256 requests with one token beside 1024 of another: 39 and 9 us).
constexpr int APPEND_WARPS = 8;

template <int HD, bool BY_ROW>
__global__ void __launch_bounds__(APPEND_WARPS * 32) kv8_append_kernel(const Kv8Append a) {
  constexpr int LPR = HD / 8, TPL = 32 / LPR, NL = PAGE / TPL;    // lanes to a token (8 values each), tokens to a load, loads
  pdl_wait();
  const int b = BY_ROW ? request_of(a.q_rows, a.B, blockIdx.x) : blockIdx.x / a.pages_per_request;
  if (BY_ROW && b >= a.B) return;
  int row, n;
  new_rows(a.q_rows, b, a.T, row, n);
  const int j = BY_ROW ? (int)blockIdx.x - row : blockIdx.x % a.pages_per_request;     // page of the new tokens, or token
  if (BY_ROW && (j < 0 || j >= min(n, a.max_q))) return;
  const int len = a.kv_lens[b];
  if (threadIdx.x == 0 && blockIdx.y == 0 && j == 0) {
    if (n > a.max_q) atomicExch(a.status, ERR_ROWS);
    if (n > 0 && (len < n || len > a.max_len)) atomicExch(a.status, ERR_PAGE_APPEND);
  }
  if (n <= 0 || len < n || len > a.max_len) return;
  const int first = len - n;                       // position of the first new token
  const int end = first + min(n, a.max_q);
  if (BY_ROW && j > 0 && (first + j) % PAGE != 0) return;           // the page is another row's
  const int pg = BY_ROW ? (first + j) / PAGE : first / PAGE + j;
  if (pg * PAGE >= end) return;
  const int lane = threadIdx.x & 31, t0 = lane / LPR, c = lane % LPR;
  const int s0 = max(first - pg * PAGE, 0), s1 = min(end - pg * PAGE, PAGE);   // the page's new slots
  const int t = blockIdx.y * APPEND_WARPS + (threadIdx.x >> 5);
  if (t >= 2 * a.Hkv) return;
  const int kvh = t >> 1, is_v = t & 1, stride = is_v ? a.v_stride : a.k_stride;
  const bf16* const src = (is_v ? a.v : a.k) + (size_t)row * stride + kvh * HD + c * 8;
  const int page = a.tables[(size_t)b * a.table_stride + pg];
  uint4 x[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int s = i * TPL + t0;
    x[i] = make_uint4(0u, 0u, 0u, 0u);
    if (s >= s0 && s < s1) x[i] = __ldcg(reinterpret_cast<const uint4*>(src + (long long)(pg * PAGE + s - first) * stride));
  }
  if (page < 0 || page >= a.kv_pages) {
    if (threadIdx.x == 0 && blockIdx.y == 0) atomicExch(a.status, ERR_PAGE_APPEND);
    return;
  }
  float* const sp = a.scales + ((size_t)page * 2 + is_v) * a.Hkv + kvh;
  const float was = s0 > 0 ? *sp : 0.f;            // (a page that starts afresh had none)
  uint2* const code = reinterpret_cast<uint2*>(a.codes + (((size_t)page * 2 + is_v) * a.Hkv + kvh) * PAGE * HD) + lane;   // [i * 32]: this lane's 8 of token i * TPL + t0
  // largest magnitude, as bf16 bits (which order like the values); from 0x7f80 on it is no number
  uint32_t m2 = 0;
#pragma unroll
  for (int i = 0; i < NL; ++i)
    m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
  uint32_t top = __reduce_max_sync(0xffffffffu, max(m2 & 0xffffu, m2 >> 16));
  if (top >= 0x7f80u) {                            // infinities become NaN, and neither counts for the maximum
    top = 0;
    auto drop = [&](uint32_t& w) {
      const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
      if (lo >= 0x7f80u) w = (w & 0xffff0000u) | 0x7fffu; else top = max(top, lo);
      if (hi >= 0x7f80u) w = (w & 0xffffu) | 0x7fff0000u; else top = max(top, hi);
    };
#pragma unroll
    for (int i = 0; i < NL; ++i) { drop(x[i].x); drop(x[i].y); drop(x[i].z); drop(x[i].w); }
    top = __reduce_max_sync(0xffffffffu, top);
  }
  // 448 = 1.75 x 2^8: the smallest power of two that brings top = 1.m x 2^e to 448 is 2^(e-8) up to m = .75, else 2^(e-7)
  const int ex = (int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);
  float scale = ex >= 1 ? __int_as_float(ex << 23) : KV8_TINY_SCALE;
  if (s0 > 0) {
    if (was >= scale) {
      scale = was;
    } else {
      const float f = was / scale;
      uint2 o[NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) if (i * TPL + t0 < s0) o[i] = code[i * 32];
      auto again = [&](uint32_t w) {
        const float2 l = to_float2(w), h = to_float2(w >> 16);
        return to_e4m3x2(l.x * f, l.y * f) | to_e4m3x2(h.x * f, h.y * f) << 16;
      };
#pragma unroll
      for (int i = 0; i < NL; ++i) if (i * TPL + t0 < s0) code[i * 32] = make_uint2(again(o[i].x), again(o[i].y));
    }
  }
  __syncwarp();                                    // every lane has read the old scale
  if (lane == 0) *sp = scale;
  auto store = [&](auto put) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int s = i * TPL + t0;
      if (s < s0 || s >= s1) continue;
      auto four = [&](uint32_t u, uint32_t v) {
        return to_e4m3x2(put(__uint_as_float(u << 16)), put(__uint_as_float(u & 0xffff0000u))) |
               to_e4m3x2(put(__uint_as_float(v << 16)), put(__uint_as_float(v & 0xffff0000u))) << 16;
      };
      code[i * 32] = make_uint2(four(x[i].x, x[i].y), four(x[i].z, x[i].w));
    }
  };
  if ((__float_as_uint(scale) & 0x007fffffu) == 0) {              // a power of two: its reciprocal is exact
    const float inv = 1.f / scale;
    store([&](float v) { return v * inv; });
  } else {                                         // somebody else's scale
    store([&](float v) { return __fdiv_rn(v, scale); });
  }
}

// ------------------------------------------------------------------------------------------------ attention, few rows
// A block takes a chunk of a request's tokens for one kv head and a tile of 8 NT query rows (row = new token x query head of the
// kv head's group); its four warps take the chunk's pages in turn, with the pages of a ring of their own in flight (16-byte
// asynchronous copies), and are merged at the end.  The products run on mma.sync m16n8k16 in fp16, which holds every e4m3 code
// exactly, with the query rows as the 8 columns: S^T = K Q^T (16 tokens x 8 rows), O^T += V^T P^T (16 dims x 8 rows).  Scales stay
// out of the matrices: a page's K scale multiplies its scores, its V scale the probabilities.  What stands in P is a weight, probability x V scale x c,
// with a power of two c for each row that has brought the largest weight so far to at least 2^6 and lets none pass what fp16 holds: what is 2^-20 of a
// row's largest weight still is a normal fp16, and what a row does not see, or gives no weight, takes no bits from it.  (Relative to the largest V scale
// instead, a page whose V is 2^26 times the others' took all of theirs.)  Which dim a k index of the first product stands for, and which one a row of the
// second, is free, and is chosen so that a lane reads 16 consecutive bytes of K and of V.
// Bound by HBM: 128 requests of 512 to 8192 tokens, 8 kv heads, G 4, hd 128 189 us, 6.0 TB/s (floor 175); two of 100003 and 131072 89 us,
// 5.3 TB/s (72), one round of 536 blocks and the merge; one of a few hundred tokens 6 us, latencies.  On the tensor cores since the
// first form, on FMAs, took 278 us for the first of these: a code and its product are three instructions there.
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t u) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(u));
  return r;
}
__device__ __forceinline__ uint32_t u4(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fffffff); }

// Byte offset of 16-byte piece p of token r in a staged tile; placed so that the reads of a quarter warp (hd 64, V: of half a warp)
// fall into different banks.
template <int HD>
__device__ __forceinline__ int k_piece(int r, int p) {
  return HD == 128 ? r * 128 + ((p ^ ((r & 1) << 2)) << 4) : r * 64 + (p << 4);
}
template <int HD>
__device__ __forceinline__ int v_piece(int r, int p) {
  return HD == 128 ? r * 128 + ((p ^ (((r >> 1) & 3) << 1)) << 4)
                   : (r >> 1) * 128 + ((((r & 1) ^ ((r >> 1) & 1)) << 6) | ((p ^ (((r >> 2) & 1) << 1)) << 4));
}

constexpr int KV8_WARPS = 4;
constexpr int KV8_CLUSTER = 8;                     // most chunks that a cluster merges
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t mapa_cluster(uint32_t addr, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float2 ld_cluster(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
constexpr int kv8_blocks(int hd, int nt) { return nt == 1 ? 4 : hd == 64 ? 3 : 2; }
template <int HD, int NT>
struct Kv8Geo {
  // pages that a warp takes at once (hd 64: what a step costs beside its products is paid for two), steps in its ring, blocks to an SM: for 16 rows of hd 128
  // two, for in the registers of three the loop spills (32 requests of 4096 with 4 tokens each 58 us, three 95; hd 64 three 49, two 49, 64 requests with 8 tokens
  // 128 and 157)
  static constexpr int PAGES = HD == 64 ? 2 : 1, STAGES = NT == 1 ? 3 : 4, BLOCKS = kv8_blocks(HD, NT);
  static constexpr int RING = KV8_WARPS * STAGES * PAGES * 2 * PAGE * HD, MERGE = KV8_WARPS * 8 * NT * HD * 4;
  static constexpr int MERGED = MERGE + 8 * NT * (HD + 2) * 4, SMEM = RING > MERGED ? RING : MERGED;       // ... and the block's own result behind it
};

// CLUSTER: the chunks of a tile are the blocks of a cluster, which merge their results through distributed shared memory; without
// it results of several chunks go to scratch and a second kernel merges them.
template <int HD, int NT, bool CLUSTER>
__global__ void __launch_bounds__(KV8_WARPS * 32, Kv8Geo<HD, NT>::BLOCKS) kv8_attn_kernel(const Kv8Attn a) {
  constexpr int KK = HD / 64, MT = HD / 16;        // 64-wide pieces of a row; m tiles of O^T
  constexpr int TILE = PAGE * HD, ST = Kv8Geo<HD, NT>::STAGES, PP = Kv8Geo<HD, NT>::PAGES, TR = 8 * NT;
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ float sm_m[KV8_WARPS][TR], sm_l[KV8_WARPS][TR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3;
  const int b = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, kvh = blockIdx.y, chunk = blockIdx.z;
  pdl_wait();
  int row0, n;
  new_rows(a.q_rows, b, a.T, row0, n);
  const int G = a.G, len = min(max(a.kv_lens[b], 0), a.max_len);
  const int seen0 = len - n + 1;                   // tokens that new token 0 attends to
  if (n > a.max_q) {
    if (threadIdx.x == 0 && tile == 0 && kvh == 0 && chunk == 0) atomicExch(a.status, ERR_ROWS);
    n = a.max_q;
  }
  const int rows = min(n * G - tile * TR, TR);     // of this tile
  if (rows <= 0 || n > a.max_n) return;
  const int seen_top = seen0 + (tile * TR + rows - 1) / G;
  const int t_begin = chunk * a.chunk, t_end = min(seen_top, t_begin + a.chunk);
  if (!CLUSTER && t_begin >= t_end) return;        // (a block of a cluster goes on with no pages)
  int seen[NT][2];                                 // tokens seen by this thread's rows 8 y + 2 tq + {0, 1}
#pragma unroll
  for (int y = 0; y < NT; ++y)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * y + 2 * tq + e;
      seen[y][e] = r < rows ? seen0 + (tile * TR + r) / G : 0;
    }
  const int seen_least = min(seen0 + tile * TR / G, t_end);        // pages up to here are whole for every row

  // ---- the steps of this warp, PP pages each: lanes hold the ids and scales of 32 pages, and of the 32 after those (by parity)
  const int32_t* const table = a.tables + (size_t)b * a.table_stride;
  const int step0 = t_begin / (PAGE * PP) + warp, pg_end = (t_end + PAGE - 1) / PAGE, step_end = (pg_end + PP - 1) / PP;
  const int n_steps = step0 < step_end ? (step_end - step0 + KV8_WARPS - 1) / KV8_WARPS : 0;
  auto load_id = [&](int batch) {
    const int i = batch * 32 + lane, pg = (step0 + i / PP * KV8_WARPS) * PP + i % PP;
    int id = -1;
    if (pg < pg_end) {
      id = table[pg];
      if (id < 0 || id >= a.kv_pages) { atomicExch(a.status, ERR_PAGE_ATTEND); id = -1; }
    }
    return id;
  };
  auto load_scales = [&](int id) {
    float2 s = make_float2(0.f, 0.f);
    if (id >= 0) {
      const float* p = a.scales + (size_t)id * 2 * a.Hkv + kvh;
      s = make_float2(p[0], p[a.Hkv]);
    }
    return s;
  };
  int id_even = load_id(0), id_odd = load_id(1);
  const uint32_t my_ring = (uint32_t)__cvta_generic_to_shared(ring) + warp * ST * PP * 2 * TILE;
  uint32_t k_dst[TILE / 512], v_dst[TILE / 512];
#pragma unroll
  for (int x = 0; x < TILE / 512; ++x) {
    const int piece = x * 32 + lane, r = piece / (HD / 16), p = piece % (HD / 16);
    k_dst[x] = k_piece<HD>(r, p);
    v_dst[x] = TILE + v_piece<HD>(r, p);
  }
  int fill = 0;                                    // stage of the next step to request
  auto issue = [&](int i) {                        // a step's pages into their stage (one commit group each, empty ones too)
    if (i < n_steps) {
#pragma unroll
      for (int p = 0; p < PP; ++p) {
        const int at = i * PP + p, id = __shfl_sync(0xffffffffu, (at & 32) == 0 ? id_even : id_odd, at & 31);
        if (id >= 0) {
          const uint32_t dst = my_ring + (fill * PP + p) * 2 * TILE;
          const unsigned char* k = a.codes + ((size_t)id * 2 * a.Hkv + kvh) * TILE + lane * 16;
          const unsigned char* v = k + (size_t)a.Hkv * TILE;
#pragma unroll
          for (int x = 0; x < TILE / 512; ++x) cp16(dst + k_dst[x], k + x * 512);
#pragma unroll
          for (int x = 0; x < TILE / 512; ++x) cp16(dst + v_dst[x], v + x * 512);
        }
      }
    }
    cp_commit();
    if (++fill == ST) fill = 0;
  };
#pragma unroll
  for (int i = 0; i < ST - 1; ++i) issue(i);
  float2 sc_even = load_scales(id_even), sc_odd = load_scales(id_odd);

  // ---- Q as the B operand, fp16
  uint32_t q[NT][KK * 4][2];
  float row_f[NT][2];
#pragma unroll
  for (int y = 0; y < NT; ++y) {
    const int r = 8 * y + gq, rr = tile * TR + r;
    uint4 u[KK][2];
    float top = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        u[kk][x] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows)
          u[kk][x] = __ldcg(reinterpret_cast<const uint4*>(a.q + (size_t)(row0 + rr / G) * a.q_stride + (size_t)(kvh * G + rr % G) * HD + kk * 64 + tq * 16 + x * 8));
        float f[8];
        unpack8(u[kk][x], f);
#pragma unroll
        for (int z = 0; z < 8; ++z) top = fmaxf(top, fabsf(f[z]));
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float up;
    const float f = row_factor<HD>(top, up);
#pragma unroll
    for (int e = 0; e < 2; ++e) row_f[y][e] = __shfl_sync(0xffffffffu, f, (2 * tq + e) * 4);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float v[8];
        unpack8(u[kk][x], v);
#pragma unroll
        for (int j = 0; j < 2; ++j) {              // MMA kk * 4 + 2 x + j takes elements 4 j .. 4 j + 3
          q[y][kk * 4 + 2 * x + j][0] = pack_f16(v[4 * j] * up, v[4 * j + 1] * up);
          q[y][kk * 4 + 2 * x + j][1] = pack_f16(v[4 * j + 2] * up, v[4 * j + 3] * up);
        }
      }
  }

  float o[NT][MT][4];
  float m[NT][2], l[NT][2], wc[NT][2];             // a row's maximum so far, sum, and c
#pragma unroll
  for (int y = 0; y < NT; ++y) {
    m[y][0] = m[y][1] = KV8_NONE;
    wc[y][0] = wc[y][1] = 1.f;
    l[y][0] = l[y][1] = 0.f;
#pragma unroll
    for (int j = 0; j < MT; ++j) o[y][j][0] = o[y][j][1] = o[y][j][2] = o[y][j][3] = 0.f;
  }

  int stage = 0;
  for (int i = 0; i < n_steps; ++i) {
    const bool even = (i * PP & 32) == 0;
    if ((i * PP & 31) == 0) {
      if (i > 0) {                                 // the 32 pages after the next ones
        if (even) { id_odd = load_id(i * PP / 32 + 1); sc_odd = load_scales(id_odd); }
        else { id_even = load_id(i * PP / 32 + 1); sc_even = load_scales(id_even); }
      }
    }
    bool there[PP];                                // pages of the pool
    float ks[PP], vs[PP];
#pragma unroll
    for (int p = 0; p < PP; ++p) {
      const int at = (i * PP + p) & 31;
      there[p] = __shfl_sync(0xffffffffu, even ? id_even : id_odd, at) >= 0;
      ks[p] = __shfl_sync(0xffffffffu, even ? sc_even.x : sc_odd.x, at);
      vs[p] = __shfl_sync(0xffffffffu, even ? sc_even.y : sc_odd.y, at);
    }
    issue(i + ST - 1);                             // into the stage that the step before this one has left
    cp_wait<ST - 1>();
    __syncwarp();
    const uint32_t tiles = my_ring + stage * PP * 2 * TILE;
    if (++stage == ST) stage = 0;
    const int t0 = (step0 + i * KV8_WARPS) * PP * PAGE;
    const bool whole = t0 + PP * PAGE <= seen_least && there[0] && there[PP - 1];
    // S^T: rows gq and gq + 8 are tokens t0 + gq and t0 + gq + 8 (page p: 16 more), columns 2 tq + {0, 1} query rows
    float s[PP][NT][4];
#pragma unroll
    for (int p = 0; p < PP; ++p) {
      const uint32_t kt = tiles + p * 2 * TILE;
#pragma unroll
      for (int y = 0; y < NT; ++y) s[p][y][0] = s[p][y][1] = s[p][y][2] = s[p][y][3] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint4 lo = lds16(kt + k_piece<HD>(gq, kk * 4 + tq)), hi = lds16(kt + k_piece<HD>(gq + 8, kk * 4 + tq));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t a0 = to_f16x2(u4(lo, j)), a1 = to_f16x2(u4(hi, j)), a2 = to_f16x2(u4(lo, j) >> 16), a3 = to_f16x2(u4(hi, j) >> 16);
#pragma unroll
          for (int y = 0; y < NT; ++y) mma_f16(s[p][y], a0, a1, a2, a3, q[y][kk * 4 + j][0], q[y][kk * 4 + j][1]);
        }
      }
#pragma unroll
      for (int y = 0; y < NT; ++y) {
        const float f0 = row_f[y][0] * ks[p], f1 = row_f[y][1] * ks[p];
        s[p][y][0] *= f0; s[p][y][1] *= f1; s[p][y][2] *= f0; s[p][y][3] *= f1;          // to the log2 domain
      }
      if (!whole) {                                // (a page that is not there is not attended to, whatever its stage holds)
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
          for (int c = 0; c < 4; ++c) if (!there[p] || t0 + p * PAGE + gq + 8 * (c >> 1) >= seen[y][c & 1]) s[p][y][c] = -INFINITY;
      }
    }
    // Probabilities and weights.  The running maximum and c only change when a weight passes what fp16 holds; a row without a maximum has infinite ones.
    uint32_t pk[PP][NT][2];                        // weights of rows 2 tq + {0, 1}, tokens gq and gq + 8
    float sum[NT][2];
    auto weights = [&] {
      uint32_t most = 0;
#pragma unroll
      for (int y = 0; y < NT; ++y) {
        sum[y][0] = l[y][0];
        sum[y][1] = l[y][1];
#pragma unroll
        for (int p = 0; p < PP; ++p) {
          const float p0 = ex2(s[p][y][0] - m[y][0]), p1 = ex2(s[p][y][1] - m[y][1]), p2 = ex2(s[p][y][2] - m[y][0]), p3 = ex2(s[p][y][3] - m[y][1]);
          const float v0 = fminf(vs[p] * wc[y][0], KV8_MOST_V), v1 = fminf(vs[p] * wc[y][1], KV8_MOST_V);        // (finite: a probability of zero stays one)
          sum[y][0] += p0 + p2;
          sum[y][1] += p1 + p3;
          pk[p][y][0] = pack_f16(p0 * v0, p1 * v1);
          pk[p][y][1] = pack_f16(p2 * v0, p3 * v1);
          most = __vmaxu2(most, __vmaxu2(pk[p][y][0], pk[p][y][1]));
        }
      }
      return ((most + 0x04000400u) & 0x80008000u) != 0u;           // an infinity or NaN among them
    };
    if (__any_sync(0xffffffffu, weights())) {
#pragma unroll
      for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top[PP], to = m[y][e], weight = 0.f;
#pragma unroll
          for (int p = 0; p < PP; ++p) {
            top[p] = fmaxf(s[p][y][e], s[p][y][2 + e]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) top[p] = fmaxf(top[p], __shfl_xor_sync(0xffffffffu, top[p], x));
            to = fmaxf(to, top[p]);
          }
#pragma unroll
          for (int p = 0; p < PP; ++p) weight = fmaxf(weight, ex2(top[p] - to) * vs[p]);
          // c times the largest weight of the step to [2^6, 2^7), unless an earlier one is larger
          const bool first = m[y][e] == KV8_NONE;
          const float lift = to - m[y][e], was = first ? (float)KV8_MOST_UP : (float)((int)(__float_as_uint(wc[y][e]) >> 23) - 127);
          const float now = fminf(fminf(was + floorf(lift), (float)(6 + 127 - (int)(__float_as_uint(weight) >> 23))), (float)KV8_MOST_UP);
          if (to > m[y][e] || (!first && now < was)) {
            const float f = ex2(now - was - lift);
            m[y][e] = to;
            l[y][e] *= ex2(-lift);
            wc[y][e] = __int_as_float((127 + (int)now) << 23);
#pragma unroll
            for (int j = 0; j < MT; ++j) { o[y][j][e] *= f; o[y][j][2 + e] *= f; }
          }
        }
      weights();
    }
#pragma unroll
    for (int y = 0; y < NT; ++y) { l[y][0] = sum[y][0]; l[y][1] = sum[y][1]; }
#pragma unroll
    for (int p = 0; p < PP; ++p) {
      const uint32_t vt = tiles + p * 2 * TILE + TILE;
      uint32_t pt[NT][2];                          // P^T as the B operand
#pragma unroll
      for (int y = 0; y < NT; ++y) { pt[y][0] = transpose_8x8(pk[p][y][0]); pt[y][1] = transpose_8x8(pk[p][y][1]); }
      // V^T as the A operand: bytes of two tokens interleaved, then two codes at a time to fp16; k indices 2 tq + {0, 1} and + 8 are
      // those tokens, rows gq and gq + 8 of m tile j the dims gq HD / 8 + 2 j + {0, 1}
      uint32_t w[4][HD / 32];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int t = 2 * tq + (x & 1) + 8 * (x >> 1);
        if constexpr (HD == 128) {
          const uint4 u = lds16(vt + v_piece<HD>(t, gq));
          w[x][0] = u.x; w[x][1] = u.y; w[x][2] = u.z; w[x][3] = u.w;
        } else {
          const uint2 u = lds8(vt + v_piece<HD>(t, gq >> 1) + (gq & 1) * 8);
          w[x][0] = u.x; w[x][1] = u.y;
        }
      }
      if (!whole) {
        bool odd = false;                          // NaN codes that not every row sees
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (!there[p] || t0 + p * PAGE + 2 * tq + (x & 1) + 8 * (x >> 1) >= t_end) {     // slots behind the last token may hold anything
#pragma unroll
            for (int z = 0; z < HD / 32; ++z) w[x][z] = 0u;
          }
#pragma unroll
          for (int z = 0; z < HD / 32; ++z) odd |= __vcmpeq4(w[x][z] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0u;
        }
        if (__any_sync(0xffffffffu, odd)) {
          // a zero probability times NaN would be NaN: NaN codes are taken out, and the rows that do see one get it from a product
          // of 0/1 matrices
          uint32_t see[NT][2];
#pragma unroll
          for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int t = t0 + p * PAGE + gq + 8 * x;
              see[y][x] = transpose_8x8((t < seen[y][0] ? 0x3c00u : 0u) | (t < seen[y][1] ? 0x3c000000u : 0u));
            }
#pragma unroll
          for (int z = 0; z < HD / 32; ++z) {
            uint32_t bad[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t mask = __vcmpeq4(w[x][z] & 0x7f7f7f7fu, 0x7f7f7f7fu);
              bad[x] = mask & 0x38383838u;         // e4m3 1.0
              w[x][z] &= ~mask;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t b0 = __byte_perm(bad[0], bad[1], h ? 0x7362 : 0x5140), b1 = __byte_perm(bad[2], bad[3], h ? 0x7362 : 0x5140);
#pragma unroll
              for (int y = 0; y < NT; ++y) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(c, to_f16x2(b0), to_f16x2(b0 >> 16), to_f16x2(b1), to_f16x2(b1 >> 16), see[y][0], see[y][1]);
#pragma unroll
                for (int d = 0; d < 4; ++d) if (c[d] > 0.f) o[y][2 * z + h][d] = nan_f();
              }
            }
          }
        }
      }
#pragma unroll
      for (int z = 0; z < HD / 32; ++z)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t b0 = __byte_perm(w[0][z], w[1][z], h ? 0x7362 : 0x5140), b1 = __byte_perm(w[2][z], w[3][z], h ? 0x7362 : 0x5140);
          const uint32_t a0 = to_f16x2(b0), a1 = to_f16x2(b0 >> 16), a2 = to_f16x2(b1), a3 = to_f16x2(b1 >> 16);
#pragma unroll
          for (int y = 0; y < NT; ++y) mma_f16(o[y][2 * z + h], a0, a1, a2, a3, pt[y][0], pt[y][1]);
        }
    }
    __syncwarp();                                  // the stage may be filled again
  }

  // ---- merge of the four warps, in warp order; thread: one row, two dims at a time
  cp_wait<0>();
#pragma unroll
  for (int y = 0; y < NT; ++y)
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[y][e] += __shfl_xor_sync(0xffffffffu, l[y][e], x);
  __syncthreads();
  float* const sm_o = reinterpret_cast<float*>(ring);              // [warp][row][dim]
#pragma unroll
  for (int y = 0; y < NT; ++y)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * y + 2 * tq + e;
      const float back = __int_as_float(0x7f000000 - __float_as_int(wc[y][e]));              // 1 / c
      if (gq == 0) { sm_m[warp][r] = m[y][e] == KV8_NONE ? -INFINITY : m[y][e]; sm_l[warp][r] = l[y][e]; }
#pragma unroll
      for (int j = 0; j < MT; ++j)
        *reinterpret_cast<float2*>(sm_o + (warp * TR + r) * HD + gq * (HD / 8) + 2 * j) = make_float2(o[y][j][e] * back, o[y][j][2 + e] * back);
    }
  __syncthreads();
  float* const own = sm_o + KV8_WARPS * TR * HD;                   // CLUSTER: [row][maximum, sum, dims]
  auto store = [&](size_t qr, int d, float x, float y) {
    bf16* const out = a.out + qr * HD + d;
    if ((reinterpret_cast<uintptr_t>(out) & 3) == 0) {
      *reinterpret_cast<uint32_t*>(out) = pack2(x, y);
    } else {
      out[0] = f2bf(x);
      out[1] = f2bf(y);
    }
  };
  auto q_row = [&](int r) { return (size_t)(row0 + (tile * TR + r) / G) * a.Hkv * G + kvh * G + (tile * TR + r) % G; };
  for (int idx = threadIdx.x; idx < rows * (HD / 2); idx += KV8_WARPS * 32) {
    const int r = idx / (HD / 2), d = idx % (HD / 2) * 2;
    const int sees = seen0 + (tile * TR + r) / G;
    if (!CLUSTER && sees <= t_begin) continue;
    float mm = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < KV8_WARPS; ++w) mm = fmaxf(mm, sm_m[w][r]);
    float ll = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll
    for (int w = 0; w < KV8_WARPS; ++w) {
      // (a warp without a maximum has seen no token of this row, or nothing but NaN)
      const float f = sm_m[w][r] == -INFINITY ? 1.f : ex2(sm_m[w][r] - mm);
      const float2 ow = *reinterpret_cast<const float2*>(sm_o + (w * TR + r) * HD + d);
      ll += sm_l[w][r] * f;
      ox += ow.x * f;
      oy += ow.y * f;
    }
    if (CLUSTER) {
      *reinterpret_cast<float2*>(own + r * (HD + 2) + 2 + d) = make_float2(ox, oy);
      if (d == 0) *reinterpret_cast<float2*>(own + r * (HD + 2)) = make_float2(mm, ll);
    } else if (sees <= a.chunk) {
      store(q_row(r), d, ox / ll, oy / ll);
    } else {
      const size_t at = a.part_tokens ? ((size_t)b * a.part_tokens + (tile * TR + r) / G) * a.Hkv * G + kvh * G + (tile * TR + r) % G : q_row(r);
      float* const part = a.partial + (at * a.max_chunks + chunk) * (HD + 2);
      __stcg(reinterpret_cast<float2*>(part + 2 + d), make_float2(ox, oy));
      if (d == 0) __stcg(reinterpret_cast<float2*>(part), make_float2(mm, ll));
    }
  }
  if constexpr (CLUSTER) {
    cluster_sync_all();
    // rows and dims in turn over the cluster's threads; chunks in order
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(own);
    const int live = (seen_top + a.chunk - 1) / a.chunk;
    for (int idx = chunk * (KV8_WARPS * 32) + threadIdx.x; idx < rows * (HD / 2); idx += (int)gridDim.z * (KV8_WARPS * 32)) {
      const int r = idx / (HD / 2), d = idx % (HD / 2) * 2;
      if (seen0 + (tile * TR + r) / G <= 0) continue;
      float2 ml[KV8_CLUSTER], v[KV8_CLUSTER];
      float mm = -INFINITY, ll = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll
      for (int c = 0; c < KV8_CLUSTER; ++c)
        if (c < live) {
          const uint32_t p = mapa_cluster(base, c) + (uint32_t)r * (HD + 2) * 4;
          ml[c] = ld_cluster(p);
          v[c] = ld_cluster(p + 8 + d * 4);
        }
#pragma unroll
      for (int c = 0; c < KV8_CLUSTER; ++c) if (c < live) mm = fmaxf(mm, ml[c].x);
#pragma unroll
      for (int c = 0; c < KV8_CLUSTER; ++c)
        if (c < live) {
          const float f = ml[c].x == -INFINITY ? 1.f : ex2(ml[c].x - mm);
          ll += ml[c].y * f;
          ox += v[c].x * f;
          oy += v[c].y * f;
        }
      store(q_row(r), d, ox / ll, oy / ll);
    }
    cluster_sync_all();                            // nobody leaves while its results are read
  }
}

// Merge of the chunks of a row: W warps share a (row, query head) and take its chunks in turn.  BY_ROW: a block to a row of q instead of one to
// each of the most rows that a request may have: most of them would have none where one request of many has a long prompt chunk.
constexpr int MERGE_WARPS = 4;
template <int HD, int W, bool BY_ROW>
__global__ void __launch_bounds__(MERGE_WARPS * 32) kv8_merge_kernel(const Kv8Attn a, int tokens) {
  constexpr int E = HD / 32;
  __shared__ float sm_m[MERGE_WARPS], sm_l[MERGE_WARPS], sm_o[MERGE_WARPS][HD];
  const int warp = threadIdx.x / 32 % W, lane = threadIdx.x & 31;
  const int h = blockIdx.y * (MERGE_WARPS / W) + threadIdx.x / (32 * W);
  if (W == 1 && h >= a.Hkv * a.G) return;
  pdl_wait();
  const int b = BY_ROW ? request_of(a.q_rows, a.B, blockIdx.x) : blockIdx.x / tokens;
  if (b >= a.B) return;
  int row0, n;
  new_rows(a.q_rows, b, a.T, row0, n);
  const int i = BY_ROW ? (int)blockIdx.x - row0 : blockIdx.x % tokens, all = n;
  n = min(n, a.max_q);
  if (i < 0 || n < a.min_n || n > a.max_n) return;
  const int sees = min(max(a.kv_lens[b], 0), a.max_len) - all + i + 1;
  if (i >= n || sees <= a.chunk) return;
  const int chunks = (sees + a.chunk - 1) / a.chunk;
  const size_t qr = (size_t)(row0 + i) * a.Hkv * a.G + h;
  const size_t at = a.part_tokens ? ((size_t)b * a.part_tokens + i) * a.Hkv * a.G + h : qr;
  const float* const part = a.partial + at * a.max_chunks * (HD + 2);
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  constexpr int U = 4;                             // chunks in flight
  for (int c0 = warp; c0 < chunks; c0 += W * U) {
    float2 ml[U];
    float2 v[U][E / 2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * W;
      ml[u] = make_float2(-INFINITY, 0.f);
      if (c < chunks) {
        const float* p = part + (size_t)c * (HD + 2);
        ml[u] = __ldcg(reinterpret_cast<const float2*>(p));
#pragma unroll
        for (int e = 0; e < E / 2; ++e) v[u][e] = __ldcg(reinterpret_cast<const float2*>(p + 2 + lane * E + 2 * e));
      }
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);
    if (top > m) {
      const float f = exp2f(m - top);
      m = top;
      l *= f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * W < chunks) {
        const float f = ml[u].x == -INFINITY ? 1.f : exp2f(ml[u].x - m);    // (a chunk of NaN scores has no maximum)
        l += ml[u].y * f;
#pragma unroll
        for (int e = 0; e < E / 2; ++e) { o[2 * e] += v[u][e].x * f; o[2 * e + 1] += v[u][e].y * f; }
      }
  }
  if constexpr (W == 1) {
    const float inv = 1.f / l;
    bf16* const out = a.out + qr * HD + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = f2bf(o[e] * inv);
    return;
  }
  if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) sm_o[warp][lane * E + e] = o[e];
  __syncthreads();
  const int d = threadIdx.x;
  if (d >= HD) return;
  float top = sm_m[0];
#pragma unroll
  for (int w = 1; w < MERGE_WARPS; ++w) top = fmaxf(top, sm_m[w]);
  float ll = 0.f, oo = 0.f;
#pragma unroll
  for (int w = 0; w < MERGE_WARPS; ++w) {
    if (w >= chunks) continue;
    const float f = sm_m[w] == -INFINITY ? 1.f : exp2f(sm_m[w] - top);
    ll += sm_l[w] * f;
    oo += sm_o[w][d] * f;
  }
  a.out[qr * HD + d] = f2bf(oo / ll);
}

// Chunks of the kernel for few rows, `slots` blocks being resident at once.
// Short ones are merged by a cluster of up to eight blocks, all resident: one launch instead of two, which is 2.5 us of the host's time, and
// no longer on the device (one request of 777 tokens, hd 64: 13 chunks and a second kernel 6.2 us, a cluster of seven 6.0; four of
// 1000, hd 128: 9.2 and 8.3; but one of 4000, hd 64: 16 chunks 7.2, a cluster of eight 8.2).
// Otherwise one block a slot for requests as long as the longest one, up to 1.5 where there are many of them, since then they are
// shorter on the average; chunks of at most 2048 tokens when there are more requests than slots.  A block costs its start and its partial
// results; too few of them, or a few more than a wave, leave SMs idle at the end.  Device times by chunk, hd 128: 128 requests of
// 512 to 8192 tokens 1024 198 us, 2048 192, 4096 205; 2 of 100003 and 131072 1024 97, 2432 103, 3456 92, 4096 94; one of 131000 1728 65 (608 blocks for 592 slots), 4096 53; 8 of 4000 to 8192 512
// 28, 640 28, 768 24, 1024 27, 2048 35; 64 of 512 to 1024 512 30, whole 24; hd 64, 32 of 128 to 4096 512 25, 1408 23, 2048 27.
struct Chunks { int tokens, clustered; };
Chunks kv8_chunks(int B, long long items, int slots, int max_len) {
  auto whole64 = [](long long v) { return (int)std::min((v + 63) / 64 * 64, 1ll << 30); };
  const long long len = max_len, in_cluster = std::min<long long>(std::max(slots / items, 1ll), KV8_CLUSTER);
  const int c = whole64((len + in_cluster - 1) / in_cluster);
  if (c <= 256) return {c, c < len};
  const long long n = std::max((long long)(slots * std::min(1.0 + (B - 1) / 32.0, 1.5)) / items, 1ll);
  const long long t = std::max((len + n - 1) / n, std::min(len / 16, 512ll));
  return {whole64(items >= slots ? std::min(t, 2048ll) : t), 0};
}

// ... of the kernel for many rows, one CTA to an SM: as many as fill one round, for a chunk more is partial results to write and merge, and what a
// CTA does around its loop, 9 us, once more.  One request, 512 new tokens after 7680, hd 128, 64 items: one chunk 151 us, two 99, four 121, five
// 149; 1024 new tokens, 128 items: one 154, two 189; 256 after 3840, 32 items: one 83, four 46, five 70.
int kv8_flash_chunk(long long requests, int tiles, int Hkv, int max_len, int sm_count) {
  const long long items = requests * tiles * Hkv, whole = ((long long)max_len + 63) / 64 * 64;
  const long long n = std::max(sm_count / items, 1ll), c = (max_len + n - 1) / n;
  return (int)std::min(std::min(std::max((c + 63) / 64 * 64, 512ll), whole), 1ll << 30);
}

// A call whose requests differ is split where the longest ones are for the kernel for many rows: those of up to few_tokens new tokens go to the
// other one, in a launch of its own.  (256 requests of 1000 to 2000 tokens with one token each beside 1024 of a prompt, hd 128: 1595 us when all go to
// the kernel for many rows; 184 like this, 135 and 31 apart.)
struct AttnPlan {
  int nt, tiles, chunk, chunks, clustered;           // nt 0: the kernel for many rows
  int few_tokens, few_nt, few_tiles, few_chunk, few_chunks, few_clustered;         // few_tokens 0: not split
  int ordered;                                       // see Kv8Attn
  long long many_items;                              // row tiles of the kernel for many rows
};
// Which kernel: up to 16 query rows of a (request, kv head) the one for few rows, with tiles of 8 or 16; beyond them the one whose time is
// estimated to be the shortest.  The figures, in microseconds, were fitted to all three on 850 shapes of 12 to 2048 rows, 1 to 64 requests and 128 to
// 65536 tokens: what was chosen took 1.2 % longer than the best on average, with the kernels as they are now 1.6 %, the estimates being off by 11 %.  The kernel for few rows pays for tiles and for a tile's tokens,
// the one for many for rounds of its CTAs, their steps and, with several chunks, the partial results.
double few_us(int hd, int nt, double items, double tokens) {
  return hd == 128 ? (nt == 1 ? 7.2 + 0.0064 * items + 3.3e-5 * items * tokens : 10.7 + 0.0136 * items + 5.2e-5 * items * tokens)
                   : (nt == 1 ? 5.4 + 0.0041 * items + 2.0e-5 * items * tokens : 7.9 + 0.0099 * items + 2.8e-5 * items * tokens);
}
double many_us(int hd, double r, double steps, bool one_tile, int chunks, double rows) {
  return hd == 128 ? 6.5 + r * (4.1 + steps * (one_tile ? 1.02 : 1.61)) + (chunks > 1 ? 1.0 + 9.0e-5 * rows * chunks : 0.0)
                   : 4.5 + r * (2.5 + steps * (one_tile ? 0.86 : 1.18)) + (chunks > 1 ? 3.6 + 4.7e-5 * rows * chunks : 0.0);
}
AttnPlan attn_plan(int B, int T, int Hq, int Hkv, int hd, int max_q, int max_len, int sm_count) {
  AttnPlan p = {};
  const int G = Hq / Hkv;
  const long long rows = (long long)max_q * G;
  const int requests = std::min(std::max(T / max_q, 1), B);          // ... of that length, if all are alike
  const int many_tiles = (int)((rows + KV8_FLASH_ROWS - 1) / KV8_FLASH_ROWS), many_chunk = kv8_flash_chunk(requests, many_tiles, Hkv, max_len, sm_count);
  if (rows <= 16) {
    p.nt = rows <= 8 || max_len <= 2048 ? 1 : 2;
  } else {
    const double tokens = std::max(max_len - 0.5 * max_q, 1.0);
    auto few_time = [&](int nt) {
      const double tiles = std::min((double)B * ((rows + 8 * nt - 1) / (8 * nt)), (double)T * G / (8 * nt) + B);
      return few_us(hd, nt, tiles * Hkv, tokens);
    };
    const int chunks = (max_len + many_chunk - 1) / many_chunk;
    const double steps = (chunks > 1 ? many_chunk : max_q > max_len / 2 ? tokens : (double)max_len) / 64.0;
    const double many = many_us(hd, std::ceil((double)requests * many_tiles * Hkv * chunks / sm_count), steps, rows <= 128, chunks, (double)rows * requests * Hkv);
    const double eights = few_time(1), sixteens = few_time(2);
    p.nt = many < std::min(eights, sixteens) ? 0 : eights <= sixteens ? 1 : 2;
  }
  const int tile = p.nt ? 8 * p.nt : KV8_FLASH_ROWS;
  p.tiles = (int)((rows + tile - 1) / tile);
  auto few = [&](int nt, long long tiles) { return kv8_chunks(B, (long long)B * tiles * Hkv, kv8_blocks(hd, nt) * sm_count, max_len); };
  if (p.nt) {
    const Chunks c = few(p.nt, p.tiles);
    p.chunk = c.tokens;
    p.clustered = c.clustered;
  } else {
    p.chunk = many_chunk;
    const int few_rows = G <= 16 ? 16 : 32;
    if (G <= few_rows && max_q > few_rows / G && T <= (long long)(B - 1) * max_q + few_rows / G) {             // (else none can be as short)
      p.few_tokens = few_rows / G;
      p.few_nt = G <= 8 ? 1 : 2;
      p.few_tiles = (p.few_tokens * G + 8 * p.few_nt - 1) / (8 * p.few_nt);
      const Chunks c = few(p.few_nt, (G + 8 * p.few_nt - 1) / (8 * p.few_nt));
      p.few_chunk = c.tokens;
      p.few_clustered = c.clustered;
      p.few_chunks = (max_len + p.few_chunk - 1) / p.few_chunk;
    }
    // Every request adds at most one tile to those that the rows fill.  To find a CTA its tile among more requests than KV8_FLASH_SORTED takes longer than it
    // gains, but where the requests are not alike.  (1100 single tokens beside 512 of another request 606 us out of order, 121 in order; 2000 of 64 tokens
    // 1720 and 2190.)
    const long long fill = (long long)T * G / KV8_FLASH_ROWS + std::max(std::min(B, T / (p.few_tokens + 1)), 1);
    p.many_items = (long long)B * p.tiles;
    p.ordered = B <= KV8_FLASH_SORTED || (B <= KV8_FLASH_MOST && 2 * fill < p.many_items);
    if (p.ordered) p.many_items = std::min(p.many_items, fill);
  }
  p.chunks = (max_len + p.chunk - 1) / p.chunk;
  return p;
}
// ... and what it counts fits 32 bits
bool attn_countable(long long B, int Hq, int Hkv, long long max_q) {
  const long long rows = max_q * (Hq / Hkv), tiles = rows / 8 + 1;
  return Hq <= 65535 && rows < (1ll << 31) - 1024 && B * max_q < 1ll << 31 && B * tiles * Hkv < 1ll << 31;
}
size_t many_scratch(const AttnPlan& p, int T, int Hq, int hd) { return p.chunks == 1 || p.clustered ? 0 : (size_t)T * Hq * p.chunks * (hd + 2) * sizeof(float); }
size_t few_scratch(const AttnPlan& p, int B, int Hq, int hd) {
  return p.few_tokens == 0 || p.few_chunks == 1 || p.few_clustered ? 0 : (size_t)B * p.few_tokens * Hq * p.few_chunks * (hd + 2) * sizeof(float);
}

// A warp to a (row, head), or four: 256 new tokens in 2 chunks, hd 128 63 and 70 us with the attention; 32 single tokens x 32 heads in 4 chunks of
// few tokens 71 and 73; one token x 32 heads in 37 chunks 17 and 14.
constexpr int KV8_MERGE_MANY = 2048;
template <int HD, int W, bool BY_ROW>
cudaError_t launch_merge_as(const Kv8Attn& a, unsigned rows, int tokens, cudaStream_t st) {
  const unsigned heads = (unsigned)(a.Hkv * a.G), per = MERGE_WARPS / W;
  return launch_pdl(kv8_merge_kernel<HD, W, BY_ROW>, dim3(rows, (heads + per - 1) / per), dim3(MERGE_WARPS * 32), 0, st, a, tokens);
}
template <int HD>
cudaError_t launch_merge(const Kv8Attn& a, cudaStream_t st) {
  if (a.max_chunks == 1) return cudaSuccess;
  const int tokens = std::min(a.max_q, a.max_n);
  const bool by_row = a.q_rows && a.T < (long long)a.B * tokens;
  const unsigned rows = (unsigned)(by_row ? a.T : a.B * tokens);
  const bool warp_each = (long long)rows * a.Hkv * a.G >= KV8_MERGE_MANY;
  if (by_row) return warp_each ? launch_merge_as<HD, 1, true>(a, rows, tokens, st) : launch_merge_as<HD, MERGE_WARPS, true>(a, rows, tokens, st);
  return warp_each ? launch_merge_as<HD, 1, false>(a, rows, tokens, st) : launch_merge_as<HD, MERGE_WARPS, false>(a, rows, tokens, st);
}

template <int HD, int NT>
cudaError_t launch_few(const Kv8Attn& a, bool clustered, cudaStream_t st) {
  using Geo = Kv8Geo<HD, NT>;
  const auto kernel = clustered ? kv8_attn_kernel<HD, NT, true> : kv8_attn_kernel<HD, NT, false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo::SMEM);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)(a.B * a.tiles), (unsigned)a.Hkv, (unsigned)a.max_chunks);
  if (!clustered) {
    e = launch_pdl(kernel, grid, dim3(KV8_WARPS * 32), Geo::SMEM, st, a);
    return e == cudaSuccess ? launch_merge<HD>(a, st) : e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(KV8_WARPS * 32);
  cfg.dynamicSmemBytes = Geo::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = (unsigned)a.max_chunks;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}
template <int HD>
cudaError_t launch_few(const Kv8Attn& a, int nt, bool clustered, cudaStream_t st) {
  return nt == 1 ? launch_few<HD, 1>(a, clustered, st) : launch_few<HD, 2>(a, clustered, st);
}

template <int HD>
cudaError_t launch_attn(Kv8Attn a, const AttnPlan& p, cudaStream_t st) {
  a.tiles = p.tiles; a.chunk = p.chunk; a.max_chunks = p.chunks;
  a.min_n = 1; a.max_n = a.max_q; a.part_tokens = 0; a.ordered = p.ordered;
  if (p.nt) return launch_few<HD>(a, p.nt, p.clustered, st);
  if (p.few_tokens) {
    Kv8Attn f = a;
    f.tiles = p.few_tiles; f.chunk = p.few_chunk; f.max_chunks = p.few_chunks;
    f.max_n = f.part_tokens = p.few_tokens;
    f.partial = reinterpret_cast<float*>(reinterpret_cast<char*>(a.partial) + many_scratch(p, a.T, a.Hkv * a.G, HD));
    const cudaError_t e = launch_few<HD>(f, p.few_nt, p.few_clustered, st);
    if (e != cudaSuccess) return e;
    a.min_n = p.few_tokens + 1;
  }
  const cudaError_t e = launch_kv8_flash(a, HD, p.many_items, st);
  return e == cudaSuccess ? launch_merge<HD>(a, st) : e;
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// What both calls ask of the cache, the tables and the rows.
int check_cache(const void* codes, const float* scales, long long kv_pages, const int32_t* q_rows, const int32_t* kv_lens, const int32_t* tables,
                int table_stride, int B, int T, int Hkv, int hd, int max_q, int max_len, const int* status) {
  if (!codes || !scales || !kv_lens || !tables || !status || kv_pages <= 0) return EPARA_E_INVALID;
  if (!aligned(codes, 16) || !aligned(scales, 4) || !aligned(q_rows, 4) || !aligned(kv_lens, 4) || !aligned(tables, 4) || !aligned(status, 4)) return EPARA_E_INVALID;
  if (table_stride < ((long long)max_len + PAGE - 1) / PAGE || (!q_rows && max_q != 1) || (!q_rows && T != B)) return EPARA_E_INVALID;
  if ((hd != 64 && hd != 128) || max_len > 1 << 30) return EPARA_E_UNSUPPORTED;
  if (Hkv > 65535) return EPARA_E_UNSUPPORTED;
  return EPARA_OK;
}

}  // namespace
}  // namespace epara

extern "C" {

int epara_kv8_append(int device, void* cuda_stream, const void* k, int k_stride, const void* v, int v_stride, void* kv8_layer, float* kv_scales,
                     long long kv_pages, const int32_t* q_rows, const int32_t* kv_lens, const int32_t* tables, int table_stride, int B, int T,
                     int Hkv, int hd, int max_q, int max_len, int* status) {
  using namespace epara;
  if (B < 0 || T < 0 || Hkv <= 0 || hd <= 0 || max_q <= 0 || max_len <= 0) return EPARA_E_INVALID;
  if (B == 0 || T == 0) return EPARA_OK;           // (whose tensors may have no address)
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16) || k_stride % 8 || v_stride % 8) return EPARA_E_INVALID;
  const int c = check_cache(kv8_layer, kv_scales, kv_pages, q_rows, kv_lens, tables, table_stride, B, T, Hkv, hd, max_q, max_len, status);
  if (c != EPARA_OK) return c;
  if ((long long)k_stride < (long long)Hkv * hd || (long long)v_stride < (long long)Hkv * hd) return EPARA_E_INVALID;
  Kv8Append a;
  a.k = (const bf16*)k; a.v = (const bf16*)v; a.codes = (unsigned char*)kv8_layer; a.scales = kv_scales;
  a.q_rows = q_rows; a.kv_lens = kv_lens; a.tables = tables; a.status = status; a.kv_pages = kv_pages;
  a.k_stride = k_stride; a.v_stride = v_stride; a.table_stride = table_stride; a.T = T; a.Hkv = Hkv; a.max_len = max_len;
  a.max_q = std::min(max_q, T);
  a.B = B;
  a.pages_per_request = (std::min(a.max_q, max_len) + PAGE - 2) / PAGE + 1;
  const long long blocks = (long long)B * a.pages_per_request;
  const bool by_row = q_rows && blocks > 2ll * T;
  if (!by_row && blocks > 0x7fffffffll) return EPARA_E_UNSUPPORTED;
  const DeviceScope scope(device);
  if (!scope.ok) return EPARA_E_CUDA;
  const dim3 grid((unsigned)(by_row ? T : blocks), (unsigned)((2 * Hkv + APPEND_WARPS - 1) / APPEND_WARPS));
  const auto kernel = hd == 128 ? (by_row ? kv8_append_kernel<128, true> : kv8_append_kernel<128, false>)
                                : (by_row ? kv8_append_kernel<64, true> : kv8_append_kernel<64, false>);
  const cudaError_t e = launch_pdl(kernel, grid, dim3(APPEND_WARPS * 32), 0, (cudaStream_t)cuda_stream, a);
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

size_t epara_kv8_attention_scratch_bytes(int device, int B, int T, int Hq, int Hkv, int hd, int max_q, int max_len) {
  using namespace epara;
  if (B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || hd <= 0 || max_q <= 0 || max_len <= 0) return 0;
  max_q = std::min(max_q, T);
  if (!attn_countable(B, Hq, Hkv, max_q) || max_len > 1 << 30) return 0;          // (the call itself is UNSUPPORTED)
  const AttnPlan p = attn_plan(B, T, Hq, Hkv, hd, max_q, max_len, device_sm_count(device));
  return many_scratch(p, T, Hq, hd) + few_scratch(p, B, Hq, hd);
}

int epara_kv8_attention(int device, void* cuda_stream, const void* q, int q_stride, const void* kv8_layer, const float* kv_scales, long long kv_pages,
                        const int32_t* q_rows, const int32_t* kv_lens, const int32_t* tables, int table_stride, void* out, int B, int T, int Hq, int Hkv,
                        int hd, int max_q, int max_len, void* scratch, size_t scratch_bytes, int* status) {
  using namespace epara;
  if (B < 0 || T < 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || hd <= 0 || max_q <= 0 || max_len <= 0) return EPARA_E_INVALID;
  if (B == 0 || T == 0) return EPARA_OK;           // (whose tensors may have no address)
  if (!q || !out || !aligned(q, 16) || q_stride % 8 || !aligned(out, 2)) return EPARA_E_INVALID;
  const int c = check_cache(kv8_layer, kv_scales, kv_pages, q_rows, kv_lens, tables, table_stride, B, T, Hkv, hd, max_q, max_len, status);
  if (c != EPARA_OK) return c;
  if ((long long)q_stride < (long long)Hq * hd) return EPARA_E_INVALID;
  if (!attn_countable(B, Hq, Hkv, std::min(max_q, T))) return EPARA_E_UNSUPPORTED;
  const size_t need = epara_kv8_attention_scratch_bytes(device, B, T, Hq, Hkv, hd, max_q, max_len);
  if (scratch_bytes < need) return EPARA_E_RESOURCE;
  if (need && (!scratch || !aligned(scratch, 16))) return EPARA_E_INVALID;
  Kv8Attn a;
  a.q = (const bf16*)q; a.codes = (const unsigned char*)kv8_layer; a.scales = kv_scales; a.q_rows = q_rows; a.kv_lens = kv_lens; a.tables = tables;
  a.out = (bf16*)out; a.partial = (float*)scratch; a.status = status; a.kv_pages = kv_pages;
  a.q_stride = q_stride; a.table_stride = table_stride; a.B = B; a.T = T; a.Hkv = Hkv; a.G = Hq / Hkv; a.max_q = std::min(max_q, T); a.max_len = max_len;
  const AttnPlan p = attn_plan(B, T, Hq, Hkv, hd, a.max_q, max_len, device_sm_count(device));
  if (p.chunks > 65535 || p.few_chunks > 65535) return EPARA_E_UNSUPPORTED;
  const DeviceScope scope(device);
  if (!scope.ok) return EPARA_E_CUDA;
  const cudaError_t e = hd == 128 ? launch_attn<128>(a, p, (cudaStream_t)cuda_stream) : launch_attn<64>(a, p, (cudaStream_t)cuda_stream);
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

}  // extern "C"

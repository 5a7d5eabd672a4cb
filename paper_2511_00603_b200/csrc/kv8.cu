// Paged KV cache in 8 bits: the append that fills it and the attention that reads it.
//
// A cache layer holds e4m3 codes [page][K|V][kv head][16 tokens][hd] and one fp32 scale for each (page, K|V, kv head): a value
// is code x scale.  The append writes scales that are powers of two: e4m3 is a floating-point format, so a scale only has to
// keep the largest value below 448 and a tighter one would gain no precision; and when a later token of a page needs a larger
// scale, the page's older codes are rescaled without a second rounding (but for values that become subnormal).
#include <algorithm>

#include "../../include/epara.h"
#include "common.cuh"
#include "kernels.h"

namespace epara {

namespace {

constexpr int PAGE = EPARA_KV_PAGE;
constexpr float TINY_SCALE = 1.17549435e-38f;     // 2^-126

// two fp32 -> two e4m3 codes (lo in the low byte), nearest even; what is not finite becomes e4m3's NaN
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  lo = fabsf(lo) <= 3.4028234e38f ? lo : __int_as_float(0x7fffffff);
  hi = fabsf(hi) <= 3.4028234e38f ? hi : __int_as_float(0x7fffffff);
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// two codes (the low 16 bits) -> two fp16, exact
__device__ __forceinline__ uint32_t to_f16x2(uint32_t two_codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two_codes));
  return r;
}
__device__ __forceinline__ float2 to_float2(uint32_t two_codes) {
  const uint32_t h = to_f16x2(two_codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// A request's new rows [row, row + n), from the prefix sums `q_rows` (or one row each); what they say is clamped to the T rows.
__device__ __forceinline__ void new_rows(const int32_t* q_rows, int b, int T, int& row, int& n) {
  if (q_rows == nullptr) { row = b; n = b < T ? 1 : 0; return; }
  row = min(max(q_rows[b], 0), T);
  n = min(max(q_rows[b + 1], row), T) - row;
}

// ------------------------------------------------------------------------------------------------ append
// A block takes one page of one request, a warp one (K or V, kv head) of it: 16 x hd values in registers, so the maximum, the
// scale and the codes come out of one read.
constexpr int APPEND_WARPS = 8;

template <int HD>
__global__ void __launch_bounds__(APPEND_WARPS * 32) kv8_append_kernel(const Kv8Append a) {
  constexpr int E = HD / 32;                       // values of a token in a lane
  pdl_wait();
  const int b = blockIdx.x / a.pages_per_request, j = blockIdx.x % a.pages_per_request;
  int row, n;
  new_rows(a.q_rows, b, a.T, row, n);
  const int len = a.kv_lens[b];
  if (threadIdx.x == 0 && blockIdx.y == 0 && j == 0) {
    if (n > a.max_q) atomicExch(a.status, ERR_ROWS);
    if (n > 0 && (len < n || len > a.max_len)) atomicExch(a.status, ERR_PAGE_APPEND);
  }
  if (n <= 0 || len < n || len > a.max_len) return;
  const int first = len - n;                       // position of the first new token
  const int end = first + min(n, a.max_q);
  const int pg = first / PAGE + j;
  if (pg * PAGE >= end) return;
  const int page = a.tables[(size_t)b * a.table_stride + pg];
  if (page < 0 || page >= a.kv_pages) {
    if (threadIdx.x == 0 && blockIdx.y == 0) atomicExch(a.status, ERR_PAGE_APPEND);
    return;
  }
  const int s0 = max(first - pg * PAGE, 0), s1 = min(end - pg * PAGE, PAGE);   // the page's new slots
  const int lane = threadIdx.x & 31;
  for (int t = blockIdx.y * APPEND_WARPS + (threadIdx.x >> 5); t < 2 * a.Hkv; t += gridDim.y * APPEND_WARPS) {
    const int kvh = t >> 1, is_v = t & 1;
    const bf16* src = is_v ? a.v + (size_t)row * a.v_stride : a.k + (size_t)row * a.k_stride;
    const int stride = is_v ? a.v_stride : a.k_stride;
    src += (long long)(pg * PAGE - first) * stride + kvh * HD + lane * E;
    uint32_t x[PAGE][E / 2];
#pragma unroll
    for (int s = 0; s < PAGE; ++s) {
      const bool is_new = s >= s0 && s < s1;
      if (E == 4) {
        uint2 u = make_uint2(0u, 0u);
        if (is_new) u = __ldcg(reinterpret_cast<const uint2*>(src + (long long)s * stride));
        x[s][0] = u.x; x[s][E / 2 - 1] = u.y;
      } else {
        x[s][0] = is_new ? __ldcg(reinterpret_cast<const uint32_t*>(src + (long long)s * stride)) : 0u;
      }
    }
    // largest finite magnitude, as bf16 bits (which order like the values)
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < PAGE; ++s)
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        const uint32_t lo = x[s][e] & 0x7fffu, hi = (x[s][e] >> 16) & 0x7fffu;
        top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
      }
    top = __reduce_max_sync(0xffffffffu, top);
    // 448 = 1.75 x 2^8: the smallest power of two that brings top = 1.m x 2^e to 448 is 2^(e-8) up to m = .75, else 2^(e-7)
    const int ex = (int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);
    float scale = ex >= 1 ? __int_as_float(ex << 23) : TINY_SCALE;
    float* const sp = a.scales + ((size_t)page * 2 + is_v) * a.Hkv + kvh;
    uint32_t* const code = reinterpret_cast<uint32_t*>(a.codes + (((size_t)page * 2 + is_v) * a.Hkv + kvh) * PAGE * HD);
    if (s0 > 0) {
      const float was = *sp;
      if (was >= scale) {
        scale = was;
      } else {
        const float f = was / scale;
        for (int s = 0; s < s0; ++s) {
          if (E == 4) {
            uint32_t* c = code + s * 32 + lane;
            const uint32_t o = *c;
            const float2 l = to_float2(o), h = to_float2(o >> 16);
            *c = to_e4m3x2(l.x * f, l.y * f) | to_e4m3x2(h.x * f, h.y * f) << 16;
          } else {
            uint16_t* c = reinterpret_cast<uint16_t*>(code) + s * 32 + lane;
            const float2 l = to_float2(*c);
            *c = (uint16_t)to_e4m3x2(l.x * f, l.y * f);
          }
        }
      }
    }
    __syncwarp();                                  // every lane has read the old scale
    if (lane == 0) *sp = scale;
    const bool pow2 = (__float_as_uint(scale) & 0x007fffffu) == 0;
    const float inv = 1.f / scale;                 // exact for a power of two; a caller's other scales are divided by
    auto put = [&](float v) { return pow2 ? v * inv : __fdiv_rn(v, scale); };
#pragma unroll
    for (int s = 0; s < PAGE; ++s) {
      if (s < s0 || s >= s1) continue;
      const uint32_t lo = to_e4m3x2(put(__uint_as_float(x[s][0] << 16)), put(__uint_as_float(x[s][0] & 0xffff0000u)));
      if (E == 4) {
        const uint32_t hi = to_e4m3x2(put(__uint_as_float(x[s][E / 2 - 1] << 16)), put(__uint_as_float(x[s][E / 2 - 1] & 0xffff0000u)));
        code[s * 32 + lane] = lo | hi << 16;
      } else {
        reinterpret_cast<uint16_t*>(code)[s * 32 + lane] = (uint16_t)lo;
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ attention, few rows
// A block takes a chunk of a request's tokens for one kv head and a tile of 16 query rows (row = new token x query head of the
// kv head's group); its four warps take the chunk's pages in turn, with the pages of a ring of their own in flight (16-byte
// asynchronous copies), and are merged at the end.  The products run on mma.sync m16n8k16 in fp16, which holds every e4m3 code
// exactly: S = Q K^T with the query rows as M, O += P V.  Scales stay out of the matrices: a page's K scale multiplies its
// scores, its V scale the probabilities, relative to the largest V scale so far so that fp16 holds them.  Which token an
// MMA column or k index stands for is free as long as both sides agree, and is chosen so that a lane reads 16 consecutive
// bytes of K and of V and no value moves between lanes.
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void mma_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t u4(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fffffff); }

// Byte offset of 16-byte piece p of token r in a staged tile; placed so that the reads of a quarter warp fall into different banks.
template <int HD>
__device__ __forceinline__ int k_piece(int r, int p) {
  return HD == 128 ? r * 128 + ((p ^ ((r & 1) << 2)) << 4) : r * 64 + (p << 4);
}
template <int HD>
__device__ __forceinline__ int v_piece(int r, int p) {
  return HD == 128 ? r * 128 + ((p ^ (((r >> 2) & 3) << 1)) << 4)
                   : (r >> 1) * 128 + ((((r & 1) ^ ((r >> 2) & 1)) << 6) | ((p ^ (((r >> 3) & 1) << 1)) << 4));
}

constexpr int KV8_WARPS = 4;
constexpr int KV8_STAGES = 4;

template <int HD>
constexpr int kv8_smem() {
  return std::max(KV8_WARPS * KV8_STAGES * 2 * PAGE * HD, KV8_WARPS * 16 * HD * 4);
}

template <int HD>
__global__ void __launch_bounds__(KV8_WARPS * 32, 3) kv8_attn_kernel(const Kv8Attn a) {
  constexpr float LOG2E = 1.4426950408889634f;
  constexpr int KK = HD / 64, NT = HD / 8;         // 64-wide pieces of a row; n tiles of O
  constexpr int TILE = PAGE * HD;
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ float sm_m[KV8_WARPS][16], sm_l[KV8_WARPS][16];
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
  const int rows = min(n * G - tile * 16, 16);     // of this tile
  if (rows <= 0) return;
  const int seen_top = seen0 + (tile * 16 + rows - 1) / G;
  const int t_begin = chunk * a.chunk, t_end = min(seen_top, t_begin + a.chunk);
  if (t_begin >= t_end) return;
  int seen[2];                                     // of this thread's rows gq and gq + 8
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = gq + 8 * e;
    seen[e] = r < rows ? seen0 + (tile * 16 + r) / G : 0;
  }
  const int seen_least = seen0 + tile * 16 / G;    // pages up to here are whole for every row

  // ---- the pages of this warp: lanes hold the ids and scales of 32 of them, and of the 32 after those
  const int32_t* const table = a.tables + (size_t)b * a.table_stride;
  const int pg0 = t_begin / PAGE + warp, pg_end = (t_end + PAGE - 1) / PAGE;
  const int n_pages = pg0 < pg_end ? (pg_end - pg0 + KV8_WARPS - 1) / KV8_WARPS : 0;
  auto load_id = [&](int batch) {
    const int i = batch * 32 + lane;
    int id = -1;
    if (i < n_pages) {
      id = table[pg0 + i * KV8_WARPS];
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
  int id_cur = load_id(0), id_next = load_id(1);
  const uint32_t my_ring = (uint32_t)__cvta_generic_to_shared(ring) + warp * KV8_STAGES * 2 * TILE;
  auto issue = [&](int i) {                        // page i of this warp into its stage (one commit group each, empty ones too)
    if (i < n_pages) {
      const int id = __shfl_sync(0xffffffffu, (i & 32) == 0 ? id_cur : id_next, i & 31);
      if (id >= 0) {
        const uint32_t dst = my_ring + (i % KV8_STAGES) * 2 * TILE;
        const unsigned char* k = a.codes + ((size_t)id * 2 * a.Hkv + kvh) * TILE;
        const unsigned char* v = k + (size_t)a.Hkv * TILE;
#pragma unroll
        for (int x = 0; x < TILE / 512; ++x) {
          const int piece = x * 32 + lane, r = piece / (HD / 16), p = piece % (HD / 16);
          cp16(dst + k_piece<HD>(r, p), k + piece * 16);
        }
#pragma unroll
        for (int x = 0; x < TILE / 512; ++x) {
          const int piece = x * 32 + lane, r = piece / (HD / 16), p = piece % (HD / 16);
          cp16(dst + TILE + v_piece<HD>(r, p), v + piece * 16);
        }
      }
    }
    cp_commit();
  };
  // (ids by position: batch x is in id_cur or id_next by the parity of x, see the end of the loop)
#pragma unroll
  for (int i = 0; i < KV8_STAGES - 1; ++i) issue(i);
  float2 sc_cur = load_scales(id_cur), sc_next = load_scales(id_next);

  // ---- Q: fp16, a row's largest value brought to [2^14, 2^15) by a power of two that joins the score's factor
  uint32_t q[KK * 4][4];
  float row_f[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = gq + 8 * e, rr = tile * 16 + r;
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
        for (int y = 0; y < 8; ++y) top = fmaxf(top, fabsf(f[y]));
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int ex = min(max((int)(__float_as_uint(top) >> 23), 15), 254);     // biased exponent
    const float up = __uint_as_float((uint32_t)(254 + 14 - ex < 254 ? 254 + 14 - ex : 254) << 23);   // 2^(14 - (ex - 127))
    row_f[e] = LOG2E * rsqrtf((float)HD) / up;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float f[8];
        unpack8(u[kk][x], f);
#pragma unroll
        for (int j = 0; j < 2; ++j) {              // MMA kk * 4 + 2 x + j takes elements 4 j .. 4 j + 3
          q[kk * 4 + 2 * x + j][e] = pack_f16(f[4 * j] * up, f[4 * j + 1] * up);
          q[kk * 4 + 2 * x + j][2 + e] = pack_f16(f[4 * j + 2] * up, f[4 * j + 3] * up);
        }
      }
  }

  float o[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, v_ref = TINY_SCALE;

  for (int i = 0; i < n_pages; ++i) {
    if ((i & 31) == 0) {
      if (i > 0) {                                 // the next 32 pages
        if (i & 32) { id_cur = load_id(i / 32 + 1); sc_cur = load_scales(id_cur); }
        else { id_next = load_id(i / 32 + 1); sc_next = load_scales(id_next); }
      }
      float top = (i & 32) == 0 ? sc_cur.y : sc_next.y;
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      if (top > v_ref) {
        const float f = v_ref / top;
#pragma unroll
        for (int j = 0; j < NT; ++j) { o[j][0] *= f; o[j][1] *= f; o[j][2] *= f; o[j][3] *= f; }
        v_ref = top;
      }
    }
    const int id = __shfl_sync(0xffffffffu, (i & 32) == 0 ? id_cur : id_next, i & 31);
    const float ks = __shfl_sync(0xffffffffu, (i & 32) == 0 ? sc_cur.x : sc_next.x, i & 31);
    const float vs = __shfl_sync(0xffffffffu, (i & 32) == 0 ? sc_cur.y : sc_next.y, i & 31);
    issue(i + KV8_STAGES - 1);                     // into the stage that the page before this one has left
    cp_wait<KV8_STAGES - 1>();
    __syncwarp();
    if (id >= 0) {
      const uint32_t kt = my_ring + (i % KV8_STAGES) * 2 * TILE, vt = kt + TILE;
      const int t0 = (pg0 + i * KV8_WARPS) * PAGE;
      float s[2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
        const int r = 4 * (gq >> 1) + 2 * x + (gq & 1);            // token of column gq of n tile x
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const uint4 u = lds16(kt + k_piece<HD>(r, kk * 4 + tq));
#pragma unroll
          for (int j = 0; j < 4; ++j) mma_f16(s[x], q[kk * 4 + j], to_f16x2(u4(u, j)), to_f16x2(u4(u, j) >> 16));
        }
      }
      // scores to the log2 domain, masked; a thread has tokens t0 + 4 tq + 2 x + {0, 1} of rows gq and gq + 8
      const float f0 = row_f[0] * ks, f1 = row_f[1] * ks;
      const bool whole = t0 + PAGE <= min(seen_least, t_end);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[x][c] *= c < 2 ? f0 : f1;
          if (!whole && t0 + 4 * tq + 2 * x + (c & 1) >= seen[c >> 1]) s[x][c] = -INFINITY;
        }
      // the running maximum is only raised when a score passes it by more than 2^8
      const float top0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
      const float top1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
      if (__any_sync(0xffffffffu, top0 > m[0] + 8.f || top1 > m[1] + 8.f)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = e ? top1 : top0;
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          if (top > m[e]) {
            const float f = exp2f(m[e] - top);
            m[e] = top;
            l[e] *= f;
#pragma unroll
            for (int j = 0; j < NT; ++j) { o[j][2 * e] *= f; o[j][2 * e + 1] *= f; }
          }
        }
      }
      const float m0 = m[0] == -INFINITY ? 0.f : m[0], m1 = m[1] == -INFINITY ? 0.f : m[1];
      const float vf = vs / v_ref;
      uint32_t p[4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float p0 = exp2f(s[x][0] - m0), p1 = exp2f(s[x][1] - m0), p2 = exp2f(s[x][2] - m1), p3 = exp2f(s[x][3] - m1);
        l[0] += p0 + p1;
        l[1] += p2 + p3;
        p[2 * x] = pack_f16(p0 * vf, p1 * vf);
        p[2 * x + 1] = pack_f16(p2 * vf, p3 * vf);
      }
      // V: bytes of two tokens interleaved, then two codes at a time to fp16; k index 2 tq + {0, 1} and + 8 stand for
      // tokens 4 tq + {0, 1} and + 2, column gq of n tile j for dim gq * NT + j
      uint32_t w[4][HD / 32];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if constexpr (HD == 128) {
          const uint4 u = lds16(vt + v_piece<HD>(4 * tq + y, gq));
          w[y][0] = u.x; w[y][1] = u.y; w[y][2] = u.z; w[y][3] = u.w;
        } else {
          const uint2 u = lds8(vt + v_piece<HD>(4 * tq + y, gq >> 1) + (gq & 1) * 8);
          w[y][0] = u.x; w[y][1] = u.y;
        }
      }
      bool odd = false;                            // NaN codes that not every row sees
      if (!whole) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int t = t0 + 4 * tq + y;
          if (t >= t_end) {                        // slots behind the last token may hold anything
#pragma unroll
            for (int z = 0; z < HD / 32; ++z) w[y][z] = 0u;
          }
#pragma unroll
          for (int z = 0; z < HD / 32; ++z) odd |= __vcmpeq4(w[y][z] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0u;
        }
      }
      if (__any_sync(0xffffffffu, odd)) {
        // a zero probability times NaN would be NaN: NaN codes are taken out and the rows that do see one get it here, by a
        // product of 0/1 matrices
        uint32_t see[4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            see[2 * x + e] = (t0 + 4 * tq + 2 * x < seen[e] ? 0x3c00u : 0u) | (t0 + 4 * tq + 2 * x + 1 < seen[e] ? 0x3c000000u : 0u);
#pragma unroll
        for (int z = 0; z < HD / 32; ++z) {
          uint32_t bad[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const uint32_t mask = __vcmpeq4(w[y][z] & 0x7f7f7f7fu, 0x7f7f7f7fu);
            bad[y] = mask & 0x38383838u;           // e4m3 1.0
            w[y][z] &= ~mask;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t a0 = __byte_perm(bad[0], bad[1], h ? 0x7362 : 0x5140), a1 = __byte_perm(bad[2], bad[3], h ? 0x7362 : 0x5140);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float c[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(c, see, to_f16x2(a0 >> (16 * y)), to_f16x2(a1 >> (16 * y)));
#pragma unroll
              for (int d = 0; d < 4; ++d) if (c[d] > 0.f) o[z * 4 + h * 2 + y][d] = nan_f();
            }
          }
        }
      }
#pragma unroll
      for (int z = 0; z < HD / 32; ++z)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t a0 = __byte_perm(w[0][z], w[1][z], h ? 0x7362 : 0x5140), a1 = __byte_perm(w[2][z], w[3][z], h ? 0x7362 : 0x5140);
          mma_f16(o[z * 4 + h * 2], p, to_f16x2(a0), to_f16x2(a1));
          mma_f16(o[z * 4 + h * 2 + 1], p, to_f16x2(a0 >> 16), to_f16x2(a1 >> 16));
        }
    }
    __syncwarp();                                  // the stage may be filled again
  }

  // ---- merge of the four warps, in warp order; thread: one row, a run of dims
  cp_wait<0>();
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
  }
  __syncthreads();
  float* const sm_o = reinterpret_cast<float*>(ring);              // [warp][row][dim]
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = gq + 8 * e;
    if (tq == 0) { sm_m[warp][r] = m[e]; sm_l[warp][r] = l[e]; }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < NT; ++j) sm_o[(warp * 16 + r) * HD + (2 * tq + c) * NT + j] = o[j][2 * e + c] * v_ref;
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < rows * (HD / 2); idx += KV8_WARPS * 32) {
    const int r = idx / (HD / 2), d = idx % (HD / 2) * 2, rr = tile * 16 + r;
    const int sees = seen0 + rr / G;
    if (sees <= t_begin) continue;
    float mm = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < KV8_WARPS; ++w) mm = fmaxf(mm, sm_m[w][r]);
    float ll = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll
    for (int w = 0; w < KV8_WARPS; ++w) {
      const float f = sm_m[w][r] == -INFINITY ? 0.f : exp2f(sm_m[w][r] - mm);
      const float2 ow = *reinterpret_cast<const float2*>(sm_o + (w * 16 + r) * HD + d);
      ll += sm_l[w][r] * f;
      // (a warp without a token of this row has zeros, or what other rows' products left: not its business)
      ox += sm_m[w][r] == -INFINITY && sm_l[w][r] == 0.f ? 0.f : ow.x * f;
      oy += sm_m[w][r] == -INFINITY && sm_l[w][r] == 0.f ? 0.f : ow.y * f;
    }
    const size_t qr = (size_t)(row0 + rr / G) * a.Hkv * G + kvh * G + rr % G;
    if (sees <= a.chunk) {
      bf16* const out = a.out + qr * HD + d;
      if ((reinterpret_cast<uintptr_t>(out) & 3) == 0) {
        *reinterpret_cast<uint32_t*>(out) = pack2(ox / ll, oy / ll);
      } else {
        out[0] = f2bf(ox / ll);
        out[1] = f2bf(oy / ll);
      }
    } else {
      float* const part = a.partial + (qr * a.max_chunks + chunk) * (HD + 2);
      __stcg(reinterpret_cast<float2*>(part + 2 + d), make_float2(ox, oy));
      if (d == 0) __stcg(reinterpret_cast<float2*>(part), make_float2(mm, ll));
    }
  }
}

// Merge of the chunks of a row, one block per (row, query head): warps take chunks in turn.
constexpr int MERGE_WARPS = 4;
template <int HD>
__global__ void __launch_bounds__(MERGE_WARPS * 32) kv8_merge_kernel(const Kv8Attn a) {
  constexpr int E = HD / 32;
  __shared__ float sm_m[MERGE_WARPS], sm_l[MERGE_WARPS], sm_o[MERGE_WARPS][HD];
  const int i = blockIdx.x % a.max_q, b = blockIdx.x / a.max_q, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  int row0, n;
  new_rows(a.q_rows, b, a.T, row0, n);
  const int sees = min(max(a.kv_lens[b], 0), a.max_len) - n + i + 1;
  if (i >= n || sees <= a.chunk) return;
  const int chunks = (sees + a.chunk - 1) / a.chunk;
  const size_t qr = (size_t)(row0 + i) * a.Hkv * a.G + h;
  const float* const part = a.partial + qr * a.max_chunks * (HD + 2);
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  constexpr int U = 4;                             // chunks in flight
  for (int c0 = warp; c0 < chunks; c0 += MERGE_WARPS * U) {
    float2 ml[U];
    float2 v[U][E / 2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * MERGE_WARPS;
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
      if (c0 + u * MERGE_WARPS < chunks) {
        const float f = ml[u].x == -INFINITY ? 1.f : exp2f(ml[u].x - m);    // (a chunk of NaN scores has no maximum)
        l += ml[u].y * f;
#pragma unroll
        for (int e = 0; e < E / 2; ++e) { o[2 * e] += v[u][e].x * f; o[2 * e + 1] += v[u][e].y * f; }
      }
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

// Tokens of a chunk: enough blocks for some waves of three per SM, chunks of 64 to 1024 tokens.
int kv8_chunk(long long B, int tiles, int Hkv, int max_len, int sm_count) {
  const long long blocks = 12ll * sm_count, items = B * tiles * Hkv, whole = ((long long)max_len + 63) / 64 * 64;
  if (items >= blocks) return (int)std::min<long long>(whole, 1 << 30);
  const long long c = ((long long)max_len * items + blocks - 1) / blocks;
  return (int)std::min(std::min(std::max((c + 63) / 64 * 64, 64ll), 1024ll), whole);
}

struct AttnPlan { int tiles, chunk, chunks; };
AttnPlan attn_plan(int B, int Hq, int Hkv, int max_q, int max_len, int sm_count) {
  AttnPlan p;
  p.tiles = (int)(((long long)max_q * (Hq / Hkv) + 15) / 16);
  p.chunk = kv8_chunk(B, p.tiles, Hkv, max_len, sm_count);
  p.chunks = (max_len + p.chunk - 1) / p.chunk;
  return p;
}

template <int HD>
cudaError_t launch_attn(const Kv8Attn& a, int B, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(kv8_attn_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kv8_smem<HD>());
  if (e != cudaSuccess) return e;
  e = launch_pdl(kv8_attn_kernel<HD>, dim3((unsigned)(B * a.tiles), (unsigned)a.Hkv, (unsigned)a.max_chunks), dim3(KV8_WARPS * 32), kv8_smem<HD>(), st, a);
  if (e != cudaSuccess || a.max_chunks == 1) return e;
  return launch_pdl(kv8_merge_kernel<HD>, dim3((unsigned)(B * a.max_q), (unsigned)(a.Hkv * a.G)), dim3(MERGE_WARPS * 32), 0, st, a);
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// What both calls ask of the cache, the tables and the rows.
int check_cache(const void* codes, const float* scales, long long kv_pages, const int32_t* q_rows, const int32_t* kv_lens, const int32_t* tables,
                int table_stride, int B, int T, int Hkv, int hd, int max_q, int max_len, const int* status) {
  if (!codes || !scales || !kv_lens || !tables || !status || kv_pages <= 0 || B < 0 || T < 0 || Hkv <= 0 || hd <= 0 || max_q <= 0 || max_len <= 0) return EPARA_E_INVALID;
  if (!aligned(codes, 16) || !aligned(scales, 4) || !aligned(q_rows, 4) || !aligned(kv_lens, 4) || !aligned(tables, 4) || !aligned(status, 4)) return EPARA_E_INVALID;
  if (table_stride < ((long long)max_len + PAGE - 1) / PAGE || (!q_rows && max_q != 1) || (!q_rows && T != B)) return EPARA_E_INVALID;
  if (hd != 64 && hd != 128) return EPARA_E_UNSUPPORTED;
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
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16) || k_stride % 8 || v_stride % 8) return EPARA_E_INVALID;
  const int c = check_cache(kv8_layer, kv_scales, kv_pages, q_rows, kv_lens, tables, table_stride, B, T, Hkv, hd, max_q, max_len, status);
  if (c != EPARA_OK) return c;
  if ((long long)k_stride < (long long)Hkv * hd || (long long)v_stride < (long long)Hkv * hd) return EPARA_E_INVALID;
  if (B == 0 || T == 0) return EPARA_OK;
  Kv8Append a;
  a.k = (const bf16*)k; a.v = (const bf16*)v; a.codes = (unsigned char*)kv8_layer; a.scales = kv_scales;
  a.q_rows = q_rows; a.kv_lens = kv_lens; a.tables = tables; a.status = status; a.kv_pages = kv_pages;
  a.k_stride = k_stride; a.v_stride = v_stride; a.table_stride = table_stride; a.T = T; a.Hkv = Hkv; a.max_len = max_len;
  a.max_q = std::min(max_q, T);
  a.pages_per_request = (std::min(a.max_q, max_len) + PAGE - 2) / PAGE + 1;
  if ((long long)B * a.pages_per_request > 0x7fffffffll) return EPARA_E_UNSUPPORTED;
  if (cudaSetDevice(device) != cudaSuccess) return EPARA_E_CUDA;
  const dim3 grid((unsigned)(B * a.pages_per_request), (unsigned)((2 * Hkv + APPEND_WARPS - 1) / APPEND_WARPS));
  const cudaError_t e = hd == 128 ? launch_pdl(kv8_append_kernel<128>, grid, dim3(APPEND_WARPS * 32), 0, (cudaStream_t)cuda_stream, a)
                                  : launch_pdl(kv8_append_kernel<64>, grid, dim3(APPEND_WARPS * 32), 0, (cudaStream_t)cuda_stream, a);
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

size_t epara_kv8_attention_scratch_bytes(int device, int B, int T, int Hq, int Hkv, int hd, int max_q, int max_len) {
  using namespace epara;
  if (B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || hd <= 0 || max_q <= 0 || max_len <= 0) return 0;
  const AttnPlan p = attn_plan(B, Hq, Hkv, std::min(max_q, T), max_len, device_sm_count(device));
  return p.chunks == 1 ? 0 : (size_t)T * Hq * p.chunks * (hd + 2) * sizeof(float);
}

int epara_kv8_attention(int device, void* cuda_stream, const void* q, int q_stride, const void* kv8_layer, const float* kv_scales, long long kv_pages,
                        const int32_t* q_rows, const int32_t* kv_lens, const int32_t* tables, int table_stride, void* out, int B, int T, int Hq, int Hkv,
                        int hd, int max_q, int max_len, void* scratch, size_t scratch_bytes, int* status) {
  using namespace epara;
  if (!q || !out || Hq <= 0 || Hkv <= 0 || Hq % Hkv || !aligned(q, 16) || q_stride % 8 || !aligned(out, 2)) return EPARA_E_INVALID;
  const int c = check_cache(kv8_layer, kv_scales, kv_pages, q_rows, kv_lens, tables, table_stride, B, T, Hkv, hd, max_q, max_len, status);
  if (c != EPARA_OK) return c;
  if ((long long)q_stride < (long long)Hq * hd) return EPARA_E_INVALID;
  if (B == 0 || T == 0) return EPARA_OK;
  if (Hq > 65535) return EPARA_E_UNSUPPORTED;
  const size_t need = epara_kv8_attention_scratch_bytes(device, B, T, Hq, Hkv, hd, max_q, max_len);
  if (scratch_bytes < need) return EPARA_E_RESOURCE;
  if (need && (!scratch || !aligned(scratch, 16))) return EPARA_E_INVALID;
  Kv8Attn a;
  a.q = (const bf16*)q; a.codes = (const unsigned char*)kv8_layer; a.scales = kv_scales; a.q_rows = q_rows; a.kv_lens = kv_lens; a.tables = tables;
  a.out = (bf16*)out; a.partial = (float*)scratch; a.status = status; a.kv_pages = kv_pages;
  a.q_stride = q_stride; a.table_stride = table_stride; a.T = T; a.Hkv = Hkv; a.G = Hq / Hkv; a.max_q = std::min(max_q, T); a.max_len = max_len;
  const AttnPlan p = attn_plan(B, Hq, Hkv, a.max_q, max_len, device_sm_count(device));
  a.tiles = p.tiles; a.chunk = p.chunk; a.max_chunks = p.chunks;
  if ((long long)B * a.tiles > 0x7fffffffll || (long long)B * a.max_q > 0x7fffffffll || a.max_chunks > 65535) return EPARA_E_UNSUPPORTED;
  if (cudaSetDevice(device) != cudaSuccess) return EPARA_E_CUDA;
  const cudaError_t e = hd == 128 ? launch_attn<128>(a, B, (cudaStream_t)cuda_stream) : launch_attn<64>(a, B, (cudaStream_t)cuda_stream);
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

}  // extern "C"

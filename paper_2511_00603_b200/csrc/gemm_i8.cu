// int8 matrix product with a scale per token and per channel, C = epi((A W^T) a_scale[m] w_scale[n] + bias): int8 operands, exact
// int32 sums (the order of K never shows), the scales applied in fp32 in the epilogue.
//
// Two kernels, as for the bf16 products and for the same reasons: rows of 128 bytes are 128 values here instead of 64, so a
// k-block moves the same bytes and the tensor core does twice the work on them.
//   swap    few rows, bound by reading W once or by latency: a tile of 128 rows of W is the MMA's M and 16 to 256 batch rows its N, K
//           in ranges over a cluster whose partial sums meet in distributed shared memory;
//   pair    256-row tiles on pairs of CTAs, persistent, two accumulators.
// (A third one for up to 16 rows on mma.sync, as for bf16, was slower here: 1 x 32000 x 4096 35 us, swapped operands 23;
// 16 x 6144 x 4096 11.4 and 8.8; 1 x 6144 x 4096 9.0 and 8.5.)
// Few rows are bound by HBM or, below 30 MB of W, by the latencies of a launch and a first tile: 1 x 6144 x 4096 8.5 us with W cold, 6.6 with
// W in L2 (floor 3.8), 96 x 28672 x 4096 27 us, 4.4 TB/s (18.4).  Many by the tensor cores: 8192 x 4096 x 14336 332 us at the full clock, 2900 TOP/s, 87 % of twice what
// cuBLAS does in bf16; 390 in calls that keep the GPU at its power limit, where the clock falls from 1965 to 1290 MHz (on zeros 263).
// Operands come by plain TMA (columns past K and rows past the matrix arrive as zeros), products run as tcgen05.mma kind::i8,
// sums are in tensor memory.  Every wait is bounded; a kernel that gives up leaves a code in *status.
#include <algorithm>

#include "../../include/epara.h"
#include "common.cuh"
#include "kernels.h"
#include "tcgen05.cuh"

namespace epara {

namespace {

using namespace tc;

struct alignas(64) I8Args {
  CUtensorMap tmA, tmW;
  const float* a_scale;
  const float* w_scale;
  const bf16* bias;
  void* C;
  int* status;
  int M, N, K, ldc, epi;
  int bn;                // swap: batch rows of a tile; pair: columns
  int tiles_m, tiles_n;
  int vec;               // rows of C start on 16 bytes (swap: on four elements)
};

constexpr int KB = 128;                            // bytes of a k-block's row

// int8 x int8 -> int32, both operands signed and K-major
__device__ __forceinline__ uint32_t make_idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_i8_elect(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_i8_pair_elect(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}

// The roundings are spelled out: an output has the same bits whichever kernel its batch runs on.
__device__ __forceinline__ float scaled(int sum, float a, float w) { return __fmul_rn(__fmul_rn((float)sum, a), w); }

// GELU of two values, x Phi(x) = max(x, 0) - |x| Q(|x|) with Q(u) = erfc(u / sqrt 2) / 2 = 2^P(u): P is a polynomial of degree 9 fitted over [0, 13.6],
// where 2^P is within 3e-5 of Q, 7e-5 with the roundings of fp32, relative to Q itself.  So the result is as good as its bf16 in the tail too, where
// 1 + tanh or 1 + erf cancels: by the form of the bf16 products, whose error is relative to x, GELU(-4) has no correct digit.  (2^(P + 16) x 2^-16: ex2 flushes
// what is below 2^-126.)  Two fp32 operations an instruction, one special function an element as there.
__device__ __forceinline__ void gelu_tail2(float& a, float& b) {
  float ua = fminf(fabsf(a), 13.6f), ub = fminf(fabsf(b), 13.6f);
  const float sa = a >= 0.f ? 1.f : 0.f, sb = b >= 0.f ? 1.f : 0.f;          // (0 for a NaN, which a 0 keeps)
  asm("{\n\t.reg .b64 u, p;\n\t.reg .f32 p0, p1;\n\tmov.b64 u, {%0, %1};\n\t"
      "fma.rn.f32x2 p, u, %2, %3;\n\tfma.rn.f32x2 p, p, u, %4;\n\tfma.rn.f32x2 p, p, u, %5;\n\tfma.rn.f32x2 p, p, u, %6;\n\tfma.rn.f32x2 p, p, u, %7;\n\t"
      "fma.rn.f32x2 p, p, u, %8;\n\tfma.rn.f32x2 p, p, u, %9;\n\tfma.rn.f32x2 p, p, u, %10;\n\tfma.rn.f32x2 p, p, u, %11;\n\t"
      "mov.b64 {p0, p1}, p;\n\tex2.approx.ftz.f32 p0, p0;\n\tex2.approx.ftz.f32 p1, p1;\n\tmov.b64 p, {p0, p1};\n\t"
      "mul.rn.f32x2 u, u, %12;\n\tmul.rn.f32x2 u, u, p;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "+f"(ua), "+f"(ub)
      : "l"(pair_of(-1.7544811159e-9f)), "l"(pair_of(1.3074171077e-7f)), "l"(pair_of(-4.2764518187e-6f)), "l"(pair_of(8.1234662503e-5f)),
        "l"(pair_of(-1.0029386031e-3f)), "l"(pair_of(8.5882926360e-3f)), "l"(pair_of(-5.3763829172e-2f)), "l"(pair_of(-4.5902839303e-1f)),
        "l"(pair_of(-1.1508688927f)), "l"(pair_of(14.9999616086f)), "l"(pair_of(-1.52587890625e-5f)));
  a = fmaf(a, sa, ua);
  b = fmaf(b, sb, ub);
}

// ------------------------------------------------------------------------------------------------ swap
constexpr int SW_BM = 128, SW_W_BYTES = SW_BM * KB;                // 16 KB
constexpr int SW_RING_1 = 192 * 1024, SW_RING_2 = 104 * 1024;      // one or two CTAs per SM
constexpr int SW_TILE_ROWS = 256;
static_assert(SW_TILE_ROWS * SW_BM * 4 <= SW_RING_1 && 128 * SW_BM * 4 <= SW_RING_2, "exchange buffer");
constexpr int SW_STAGES_MAX = 10;
constexpr int SW_EPI_WARPS = 8, SW_A_WARP = 2 + SW_EPI_WARPS, SW_THREADS = 32 * (SW_A_WARP + 1);
constexpr int SW_BAR_BYTES = 512;
inline size_t sw_smem(int ring) { return 1024 + (size_t)ring + SW_BAR_BYTES; }

// D[n, m] = sum_k W[n, k] A[m, k]: the accumulator holds C transposed, TMEM lane = output column, TMEM column = batch row.  A
// cluster of S CTAs takes a tile, a k range each; after the last MMAs every CTA sends the slices of its sums to the batch rows'
// owners and an owner adds them up, a warp per row.
template <int S>
__global__ void __launch_bounds__(SW_THREADS, 2) gemm_i8_swap_kernel(const __grid_constant__ I8Args g, int ring_bytes) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bars = base + ring_bytes;
  auto wfull = [&](int s) { return bars + 8u * s; };
  auto wempty = [&](int s) { return bars + 8u * (SW_STAGES_MAX + s); };
  auto afull = [&](int s) { return bars + 8u * (2 * SW_STAGES_MAX + s); };
  auto aempty = [&](int s) { return bars + 8u * (3 * SW_STAGES_MAX + s); };
  const uint32_t tfull = bars + 8u * (4 * SW_STAGES_MAX);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + ring_bytes + 8 * (4 * SW_STAGES_MAX + 1));
  static_assert(8 * (4 * SW_STAGES_MAX + 1) + 16 <= SW_BAR_BYTES, "barrier area");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = S == 1 ? 0 : (int)cluster_ctarank();
  const int item = blockIdx.x / S, nb = g.bn;
  const int n0 = (item / g.tiles_m) * SW_BM, m0 = (item % g.tiles_m) * nb;   // the row tiles of one W tile are neighbours and share it through L2
  const int rows = min(nb, g.M - m0);
  const int kblocks = (g.K + KB - 1) / KB, per = (kblocks + S - 1) / S;
  const int kb0 = rank * per, kb1 = min(kblocks, kb0 + per);
  const bool empty = kb0 >= kb1;
  const int a_bytes = nb * KB;
  const int a_stages = ring_bytes < SW_RING_1 ? (nb > 64 ? 2 : 4) : nb > 128 ? 3 : nb > 64 ? 4 : nb > 32 ? 6 : 8;
  const int w_stages = min(SW_STAGES_MAX, (ring_bytes - a_stages * a_bytes) / SW_W_BYTES);
  const uint32_t w_base = base + a_stages * a_bytes;                // (nb is a multiple of 16: 2 KB steps)
  const uint32_t tmem_cols = nb > 128 ? 256u : nb > 64 ? 128u : 64u;

  if (threadIdx.x == 0) {
    for (int s = 0; s < w_stages; ++s) { mbar_init(wfull(s), 1); mbar_init(wempty(s), 1); }
    for (int s = 0; s < a_stages; ++s) { mbar_init(afull(s), 1); mbar_init(aempty(s), 1); }
    mbar_init(tfull, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == 0) tensormap_prefetch_elect(&g.tmW);
  if (warp == SW_A_WARP) tensormap_prefetch_elect(&g.tmA);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // (W may be what the kernel before this one wrote: it, too, is read after the wait)
  pdl_wait();
  bool acc_ok = true;
  if (warp == 0) {
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (kb - kb0 >= w_stages && !mbar_wait(wempty(stage), phase ^ 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, 51); break; }
      mbar_expect_tx_elect(wfull(stage), (uint32_t)SW_W_BYTES);
      tma_load_2d_elect(w_base + stage * SW_W_BYTES, &g.tmW, kb * KB, n0, wfull(stage));
      if (++stage == w_stages) { stage = 0; phase ^= 1u; }
    }
    if (!ok) { *abort_flag = 1; drain_sleep(200000ull); }
  } else if (warp == SW_A_WARP) {
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (kb - kb0 >= a_stages && !mbar_wait(aempty(stage), phase ^ 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, 52); break; }
      mbar_expect_tx_elect(afull(stage), (uint32_t)a_bytes);
      tma_load_2d_elect(base + stage * a_bytes, &g.tmA, kb * KB, m0, afull(stage));
      if (++stage == a_stages) { stage = 0; phase ^= 1u; }
    }
    if (!ok) { *abort_flag = 1; drain_sleep(200000ull); }
  } else if (warp == 1) {
    const uint32_t idesc = make_idesc_i8(SW_BM, nb);
    int ws = 0, as = 0;
    uint32_t wphase = 0, aphase = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_both(afull(as), aphase, wfull(ws), wphase, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, 53); break; }
      const uint64_t dw = make_smem_desc(w_base + ws * SW_W_BYTES), da = make_smem_desc(base + as * a_bytes);
#pragma unroll
      for (int k = 0; k < KB / 32; ++k)
        mma_i8_elect(tmem_base, dw + (uint64_t)(k * 2), da + (uint64_t)(k * 2), idesc, (kb > kb0 || k > 0) ? 1u : 0u);
      mma_commit_elect(wempty(ws));
      mma_commit_elect(aempty(as));
      if (++ws == w_stages) { ws = 0; wphase ^= 1u; }
      if (++as == a_stages) { as = 0; aphase ^= 1u; }
    }
    if (!ok) *abort_flag = 1;
    else if (!empty) mma_commit_elect(tfull);
  } else {
    acc_ok = empty || mbar_wait(tfull, 0u, abort_flag);
    if (!acc_ok) {
      if (lane == 0) atomicExch(g.status, 54);
      *abort_flag = 1;
    }
  }
  // The slices go over the owners' operand rings, which must be idle: every CTA of the cluster is past its last MMA first.
  __syncthreads();
  if (S > 1) cluster_sync_relaxed();
  const int rp = ((nb + S - 1) / S + 3) & ~3;       // batch rows per owner
  if (warp >= 2 && warp < SW_A_WARP) {
    const int quarter = warp & 3, alt = (warp - 2) >> 2;
    const uint32_t col_off = (uint32_t)(quarter * 32 + lane) * 4u;
    tc_fence_after();
    const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t plane = (uint32_t)(rank * rp) * (SW_BM * 4u) + col_off;
    for (int c = alt * 16; c < rows; c += 32) {
      uint32_t r[16];
      if (empty || !acc_ok) {
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = 0u;
      } else {
        tmem_ld16(taddr + (uint32_t)c, r);
      }
      // (rp is a multiple of four, so four rows go to one owner; rows past the live ones are sent along with them)
#pragma unroll
      for (int j4 = 0; j4 < 16; j4 += 4) {
        const int owner = S == 1 ? 0 : (c + j4) / rp;
        const uint32_t dst = (S == 1 ? base : mapa_shared(base, (uint32_t)owner)) + plane + (uint32_t)(c + j4 - owner * rp) * (SW_BM * 4u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (S == 1) asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + (uint32_t)j * (SW_BM * 4u)), "r"(r[j4 + j]) : "memory");
          else asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(dst + (uint32_t)j * (SW_BM * 4u)), "r"(r[j4 + j]) : "memory");
        }
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (S > 1) cluster_sync_all();                     // every slice has reached its owner

  if (warp >= 2 && warp < SW_A_WARP) {
    const int epi = g.epi, N = g.N, ldc = g.ldc, col = lane * 4, n = n0 + col;
    const bool full = n + 4 <= N && g.vec, resid = (epi & EPI_RESID_F32) != 0;
    const int live = min(4, N - n);                  // live columns of this lane
    float ws[4] = {0.f, 0.f, 0.f, 0.f}, bias[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < live) {
        ws[j] = g.w_scale[n + j];
        if (epi & EPI_BIAS) bias[j] = bf2f(g.bias[n + j]);
      }
    constexpr int U = 4;
    const int r0 = rank * rp, nrows = min(rp, rows - r0);
    const int* const red = reinterpret_cast<const int*>(base_ptr);
#pragma unroll 1
    for (int l0 = warp - 2; l0 < nrows; l0 += SW_EPI_WARPS * U) {
      float4 old[U];
      float v[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int l = l0 + u * SW_EPI_WARPS;
        old[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (resid && l < nrows && live > 0) {
          const float* cf = static_cast<const float*>(g.C) + (size_t)(m0 + r0 + l) * ldc + n;
          if (full) old[u] = *reinterpret_cast<const float4*>(cf);
          else { old[u].x = cf[0]; if (live > 1) old[u].y = cf[1]; if (live > 2) old[u].z = cf[2]; if (live > 3) old[u].w = cf[3]; }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int l = min(l0 + u * SW_EPI_WARPS, nrows - 1);
        int4 s = *reinterpret_cast<const int4*>(red + l * SW_BM + col);
#pragma unroll
        for (int q = 1; q < S; ++q) {
          const int4 p = *reinterpret_cast<const int4*>(red + (q * rp + l) * SW_BM + col);
          s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
        }
        const float as = __ldcg(g.a_scale + m0 + r0 + l);
        v[u][0] = scaled(s.x, as, ws[0]); v[u][1] = scaled(s.y, as, ws[1]); v[u][2] = scaled(s.z, as, ws[2]); v[u][3] = scaled(s.w, as, ws[3]);
        if (epi & EPI_BIAS) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[u][j] = __fadd_rn(v[u][j], bias[j]);
        }
        if (epi & EPI_GELU) {
#pragma unroll
          for (int j = 0; j < 4; j += 2) gelu_tail2(v[u][j], v[u][j + 1]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int l = l0 + u * SW_EPI_WARPS;
        if (l >= nrows || live <= 0) continue;
        const size_t row = (size_t)(m0 + r0 + l) * ldc;
        if (epi & EPI_SWIGLU) {                      // gate and up are adjacent columns
          bf16* cb = static_cast<bf16*>(g.C) + row + (n >> 1);
          const float x = silu_f(v[u][0]) * v[u][1], y = silu_f(v[u][2]) * v[u][3];
          if (full) *reinterpret_cast<uint32_t*>(cb) = pack2(x, y);
          else { cb[0] = f2bf(x); if (live > 2) cb[1] = f2bf(y); }
        } else if (resid) {
          float* cf = static_cast<float*>(g.C) + row + n;
          const float4 z = make_float4(__fadd_rn(old[u].x, v[u][0]), __fadd_rn(old[u].y, v[u][1]), __fadd_rn(old[u].z, v[u][2]), __fadd_rn(old[u].w, v[u][3]));
          if (full) *reinterpret_cast<float4*>(cf) = z;
          else { cf[0] = z.x; if (live > 1) cf[1] = z.y; if (live > 2) cf[2] = z.z; if (live > 3) cf[3] = z.w; }
        } else {
          bf16* cb = static_cast<bf16*>(g.C) + row + n;
          if (full) *reinterpret_cast<uint2*>(cb) = make_uint2(pack2(v[u][0], v[u][1]), pack2(v[u][2], v[u][3]));
          else { cb[0] = f2bf(v[u][0]); if (live > 1) cb[1] = f2bf(v[u][1]); if (live > 2) cb[2] = f2bf(v[u][2]); if (live > 3) cb[3] = f2bf(v[u][3]); }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(tmem_cols) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ pair
constexpr int PR_A_BYTES = 128 * KB;                // 16 KB: this CTA's 128 rows of A
constexpr int PR_STAGES = 6, PR_STAGE_BYTES = 2 * PR_A_BYTES, PR_RING = PR_STAGES * PR_STAGE_BYTES;
constexpr int PR_EPI_WARPS = 16, PR_W_WARP = 2 + PR_EPI_WARPS, PR_THREADS = 32 * (PR_W_WARP + 1);
constexpr int PR_STAGE_OUT = PR_EPI_WARPS * 2048;   // epilogue staging: 32 rows x 64 bytes a warp
constexpr size_t PR_SMEM = 1024 + (size_t)PR_RING + PR_STAGE_OUT + 256;
constexpr int PR_ACC_COLS = 256;

// Outputs of one warp for one tile: 32 rows (lane = row) x the part-th 64 of the tile's columns (32 of a tile 128 wide).  A chunk's values are parked in
// the warp's staging area and leave it as 16-byte pieces of 64-byte row segments (MODE 2: additions at L2), or one by one where
// rows of C do not start on 16 bytes or the matrix ends.  MODE: 0 bf16, 1 SwiGLU, 2 fp32 residual.
// Additions at L2 take subnormals for zeros, before and after.  With 2^-100 or more to add that cannot show: a subnormal C is lost in the rounding anyway, and
// what is left of two that cancel is a multiple of 2^-123.  Pieces with less are added here.  (All of them read ahead of a chunk's sums and
// added here: 16384 x 4096 x 512 160 to 176 us, like this 140 to 155; 2048 x 4096 x 1024 22 to 30 and 21 to 23.)
template <int MODE>
__device__ __forceinline__ void i8_epilogue(const I8Args& g, int m_base, int n0, uint32_t taddr, unsigned char* wst, int part, int lane, float as, uint32_t tempty) {
  constexpr int CW = MODE == 2 ? 16 : 32;           // accumulator columns of a chunk
  const int cols = g.bn > 128 ? 64 : 32, c_begin = part * cols, c_end = min(min(c_begin + cols, g.bn), g.N - n0);
  if (c_begin >= c_end) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive_cluster(tempty);
    return;
  }
#pragma unroll 1
  for (int c = c_begin; c < c_end; c += CW) {
    const int n = n0 + c;
    uint32_t r[CW];
    if (MODE == 2) tmem_ld16(taddr + (uint32_t)c, r); else tmem_ld32(taddr + (uint32_t)c, r);
    if (c + CW >= c_end) {                          // that was this warp's last read of the accumulator
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(tempty);
    }
    float v[CW];
    if (n + CW <= g.N) {
#pragma unroll
      for (int j = 0; j < CW; j += 4) {
        const float4 w = *reinterpret_cast<const float4*>(g.w_scale + n + j);
        v[j] = scaled((int)r[j], as, w.x); v[j + 1] = scaled((int)r[j + 1], as, w.y);
        v[j + 2] = scaled((int)r[j + 2], as, w.z); v[j + 3] = scaled((int)r[j + 3], as, w.w);
      }
      if (g.epi & EPI_BIAS) {
#pragma unroll
        for (int j = 0; j < CW; j += 8) {
          const uint4 b = *reinterpret_cast<const uint4*>(g.bias + n + j);
          add_bias2(v[j], v[j + 1], b.x); add_bias2(v[j + 2], v[j + 3], b.y);
          add_bias2(v[j + 4], v[j + 5], b.z); add_bias2(v[j + 6], v[j + 7], b.w);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < CW; ++j) {
        v[j] = n + j < g.N ? scaled((int)r[j], as, g.w_scale[n + j]) : 0.f;
        if ((g.epi & EPI_BIAS) && n + j < g.N) v[j] = __fadd_rn(v[j], bf2f(g.bias[n + j]));
      }
    }
    if (g.epi & EPI_GELU) {
#pragma unroll
      for (int j = 0; j < CW; j += 2) gelu_tail2(v[j], v[j + 1]);
    }
    // row segments: 64 bytes (SwiGLU 32), 16-byte pieces swizzled against bank conflicts
    constexpr int PIECES = MODE == 1 ? 2 : 4;
    __syncwarp();                                   // the chunk before has left the staging area
    {
      unsigned char* srow = wst + lane * (PIECES * 16);
      const int sw = PIECES == 2 ? (lane >> 2) & 1 : (lane >> 1) & 3;
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        uint4 o;
        if (MODE == 2) {
          o = make_uint4(__float_as_uint(v[4 * k]), __float_as_uint(v[4 * k + 1]), __float_as_uint(v[4 * k + 2]), __float_as_uint(v[4 * k + 3]));
        } else if (MODE == 1) {
          o.x = pack2(silu_f(v[16 * k]) * v[16 * k + 1], silu_f(v[16 * k + 2]) * v[16 * k + 3]);
          o.y = pack2(silu_f(v[16 * k + 4]) * v[16 * k + 5], silu_f(v[16 * k + 6]) * v[16 * k + 7]);
          o.z = pack2(silu_f(v[16 * k + 8]) * v[16 * k + 9], silu_f(v[16 * k + 10]) * v[16 * k + 11]);
          o.w = pack2(silu_f(v[16 * k + 12]) * v[16 * k + 13], silu_f(v[16 * k + 14]) * v[16 * k + 15]);
        } else {
          o.x = pack2(v[8 * k], v[8 * k + 1]); o.y = pack2(v[8 * k + 2], v[8 * k + 3]);
          o.z = pack2(v[8 * k + 4], v[8 * k + 5]); o.w = pack2(v[8 * k + 6], v[8 * k + 7]);
        }
        *reinterpret_cast<uint4*>(srow + ((k ^ sw) << 4)) = o;
      }
    }
    __syncwarp();
    constexpr int PER = MODE == 2 ? 4 : 8;          // outputs of a piece
    const int out_n = MODE == 1 ? n >> 1 : n, out_N = MODE == 1 ? g.N >> 1 : g.N;
#pragma unroll
    for (int x = 0; x < PIECES; ++x) {
      const int piece = x * 32 + lane, row = piece / PIECES, k = piece % PIECES;
      const int sw = PIECES == 2 ? (row >> 2) & 1 : (row >> 1) & 3;
      const uint4 o = *reinterpret_cast<const uint4*>(wst + row * (PIECES * 16) + ((k ^ sw) << 4));
      const int m = m_base + row, col = out_n + k * PER;
      if (m >= g.M || col >= out_N) continue;
      if (g.vec && col + PER <= out_N) {
        if (MODE == 2) {
          constexpr float LEAST = 7.8886091e-31f;   // 2^-100
          if (!(fminf(fminf(fabsf(__uint_as_float(o.x)), fabsf(__uint_as_float(o.y))), fminf(fabsf(__uint_as_float(o.z)), fabsf(__uint_as_float(o.w)))) >= LEAST)) {
            float4* const p = reinterpret_cast<float4*>(static_cast<float*>(g.C) + (size_t)m * g.ldc + col);
            const float4 c = *p;
            *p = make_float4(__fadd_rn(c.x, __uint_as_float(o.x)), __fadd_rn(c.y, __uint_as_float(o.y)), __fadd_rn(c.z, __uint_as_float(o.z)),
                             __fadd_rn(c.w, __uint_as_float(o.w)));
            continue;
          }
          float* p = static_cast<float*>(g.C) + (size_t)m * g.ldc + col;
          asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(o.x)), "f"(__uint_as_float(o.y)),
                       "f"(__uint_as_float(o.z)), "f"(__uint_as_float(o.w)) : "memory");
        } else {
          *reinterpret_cast<uint4*>(static_cast<bf16*>(g.C) + (size_t)m * g.ldc + col) = o;
        }
      } else {
        const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          if (col + e >= out_N) break;
          if (MODE == 2) static_cast<float*>(g.C)[(size_t)m * g.ldc + col + e] += __uint_as_float(w[e & 3]);
          else static_cast<unsigned short*>(g.C)[(size_t)m * g.ldc + col + e] = (unsigned short)(w[(e >> 1) & 3] >> (16 * (e & 1)));
        }
      }
    }
  }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PR_THREADS, 1) gemm_i8_pair_kernel(const __grid_constant__ I8Args g) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  unsigned char* stage_out = base_ptr + PR_RING;
  const uint32_t bars = base + PR_RING + PR_STAGE_OUT;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (PR_STAGES + s); };
  auto tfull = [&](int a) { return bars + 8u * (2 * PR_STAGES + a); };
  auto tempty = [&](int a) { return bars + 8u * (2 * PR_STAGES + 2 + a); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + PR_RING + PR_STAGE_OUT + 8 * (2 * PR_STAGES + 4));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1, total = g.tiles_m * g.tiles_n;
  if (threadIdx.x == 0) {
    for (int s = 0; s < PR_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull(a), 1); mbar_init(tempty(a), 2 * PR_EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2u * PR_ACC_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (warp == 0) tensormap_prefetch_elect(&g.tmA);
  if (warp == PR_W_WARP) tensormap_prefetch_elect(&g.tmW);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                        // the peer's barriers exist before anything is reported to them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  const int kblocks = (g.K + KB - 1) / KB, bn = g.bn;
  // items run down the rows first: the pairs at work share the columns of few W tiles and the rows of A through L2
  auto item_m = [&](int item) { return (item % g.tiles_m) * 256; };
  auto item_n = [&](int item) { return (item / g.tiles_m) * bn; };

  if (warp == 0 || warp == PR_W_WARP) {
    // ------------------------------------------------------------ TMA producers: A (this CTA's 128 rows), W (half of the tile's)
    const bool is_a = warp == 0;
    int stage = 0, used = 0;
    uint32_t phase = 0;
    bool ok = true;
    const uint32_t bytes = 2u * (PR_A_BYTES + (uint32_t)(bn >> 1) * KB);   // both CTAs' boxes of a k-block
    for (int item = pair; item < total && ok; item += n_pairs) {
      const int y = is_a ? item_m(item) + rank * 128 : item_n(item) + rank * (bn >> 1);
      for (int kb = 0; kb < kblocks; ++kb) {
        if (++used > PR_STAGES && !mbar_wait(empty(stage), phase ^ 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, is_a ? 55 : 56); break; }
        if (is_a && rank == 0) mbar_expect_tx_elect(full(stage), bytes);
        tma_load_2d_pair_elect(base + stage * PR_STAGE_BYTES + (is_a ? 0 : PR_A_BYTES), is_a ? &g.tmA : &g.tmW, kb * KB, y, mapa_shared(full(stage), 0));
        if (++stage == PR_STAGES) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) { *abort_flag = 1; drain_sleep(200000ull); }
  } else if (warp == 1) {
    if (rank == 0) {
      // ---------------------------------------------------------- MMA issuer of the pair
      const uint32_t idesc = make_idesc_i8(256, bn);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true, ready = false;
      for (int item = pair; item < total && ok; item += n_pairs) {
        if (!mbar_wait(tempty(acc), acc_phase ^ 1u, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, 57); break; }
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)(acc * PR_ACC_COLS);
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!ready && !mbar_wait<false>(full(stage), phase, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, 58); break; }
          const uint32_t sa = base + stage * PR_STAGE_BYTES;
          const uint64_t da = make_smem_desc(sa), db = make_smem_desc(sa + PR_A_BYTES);
          const uint32_t used = empty(stage);
          if (++stage == PR_STAGES) { stage = 0; phase ^= 1u; }
          ready = mbar_test(full(stage), phase);
#pragma unroll
          for (int k = 0; k < KB / 32; ++k)
            mma_i8_pair_elect(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (kb > 0 || k > 0) ? 1u : 0u);
          mma_commit_pair_elect(used);
        }
        if (!ok) break;
        mma_commit_pair_elect(tfull(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok) *abort_flag = 1;
    }
  } else {
    // ------------------------------------------------------------ epilogue (16 warps of both CTAs)
    const int ew = warp - 2, quarter = warp & 3, part = ew >> 2;
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    unsigned char* wst = stage_out + ew * 2048;
    for (int item = pair; item < total && ok; item += n_pairs) {
      const int m_base = item_m(item) + rank * 128 + quarter * 32, n0 = item_n(item);
      const float as = m_base + lane < g.M ? __ldcg(g.a_scale + m_base + lane) : 0.f;
      if (!mbar_wait(tfull(acc), acc_phase, abort_flag)) { ok = false; if (lane == 0) atomicExch(g.status, 59); break; }
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * PR_ACC_COLS);
      const uint32_t te = mapa_shared(tempty(acc), 0);
      if (g.epi & EPI_RESID_F32) i8_epilogue<2>(g, m_base, n0, taddr, wst, part, lane, as, te);
      else if (g.epi & EPI_SWIGLU) i8_epilogue<1>(g, m_base, n0, taddr, wst, part, lane, as, te);
      else i8_epilogue<0>(g, m_base, n0, taddr, wst, part, lane, as, te);
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
    if (!ok) *abort_flag = 1;
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                        // neither CTA leaves while the other may still read its operands or signal it
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2u * PR_ACC_COLS) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ host
// Bytes [rows, cols] with a row stride of ld, in boxes of 128 bytes x box_rows, 128-byte swizzle.
bool make_i8_map(CUtensorMap* tm, const void* p, long long rows, long long cols, long long ld, int box_rows) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  const Encode fn = reinterpret_cast<Encode>(tensor_map_encoder());
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {(cuuint32_t)KB, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

enum { I8_SWAP, I8_PAIR };
struct I8Plan { int kernel, bn, split; };

inline int swap_ring(int bn, long long ctas, int split, int sm_count) { return bn <= 32 || (bn <= 128 && (ctas > sm_count || split == 8)) ? SW_RING_2 : SW_RING_1; }

// The kernel and its tile by an estimate of the time in microseconds, whose terms are: a launch and its set-up; what an SM takes in, 105 KB a
// microsecond, against what HBM delivers of W, 8 MB a microsecond (4.6 where two CTAs with wide tiles share an SM: their rings are short), and a
// tenth of the smaller one; for swapped operands 0.8 for every 32 rows that a CTA writes out and the exchange, which two CTAs on an SM slow down by 0.3;
// for pairs what a k-block takes, and 0.3 a tile more.  The figures were fitted to the times of 120 shapes of up to 700 rows, each with every
// kernel and split: what is chosen takes 0.7 % longer than the best on average, 9 % at most.  Calls in a row with W cold, measured (estimate),
// swapped operands: 1 x 6144 x 4096 one range 9.6 (9.4), two 8.5 (7.5), four 8.6 (8.0); 1 x 4096 x 4096 two 7.7 (7.0), four 6.7 (6.4); 32 x 4096 x
// 14336 two 17.3 (15.7), four 14.7 (12.4); 128 x 4096 x 14336 four 16.0 (15.8), two 18.9 (24.2); 256 x 3000 x 3000 tiles of 96 rows with two
// 9.3 (9.3), with four 15.5 (10.2), pairs, 128 columns 9.3 (10.0); 256 x 6144 x 4096 tiles of 96 rows 12.6 (14.0), pairs 11.6 (11.9); 96 x 28672 x
// 4096 31, pairs, 256 columns 28, 224 27; 768 x 4096 x 14336 on pairs, 128 / 192 / 256 columns 52 / 35 / 41.
I8Plan i8_plan(long long M, int N, int K, int sm_count) {
  const int kblocks = (K + KB - 1) / KB;
  const double w_mb = (double)N * K * 1e-6;
  I8Plan p = {I8_PAIR, 256, 1};
  double best = 1e30;
  for (int bn = 128; bn <= 256; bn += 32) {
    const long long tiles = (M + 255) / 256 * ((N + bn - 1) / bn), pairs = sm_count / 2, rounds = (tiles + pairs - 1) / pairs;
    const double t = 4.1 + std::max((double)rounds * kblocks * (0.117 + 0.001 * bn), w_mb / 5.5) + 0.3 * (double)(rounds - 1);
    if (t < best) { best = t; p.bn = bn; }
  }
  if (M > 1024) return p;
  const int tiles_n = (N + SW_BM - 1) / SW_BM;
  for (int tiles_m = (int)((M + SW_TILE_ROWS - 1) / SW_TILE_ROWS); tiles_m <= 32; ++tiles_m) {
    const int bn = (int)(((M + tiles_m - 1) / tiles_m + 15) / 16 * 16);
    if (tiles_m > 1 && bn < 32) break;
    for (int s = 1; s <= 8 && s <= kblocks; s *= 2) {
      const long long ctas = (long long)tiles_n * ((M + bn - 1) / bn) * s, per_sm = (ctas + sm_count - 1) / sm_count;
      const bool two = swap_ring(bn, ctas, s, sm_count) == SW_RING_2;
      const double main = (double)per_sm * ((kblocks + s - 1) / s) * (16.0 + bn / 8.0) / 105.0, hbm = w_mb / (two && bn > 64 ? 4.6 : 8.0);
      const double out = 0.8 * ((bn + 32 * s - 1) / (32 * s)) + (s > 1 ? 0.23 + 0.028 * bn * (s - 1) / s : 0.0) + (s == 8 ? 0.6 : 0.0);
      const double turns = two ? (double)((per_sm + 1) / 2) * (per_sm % 2 ? 1.0 : 1.3) : (double)per_sm;
      const double t = 2.8 + std::max(main, hbm) + 0.1 * std::min(main, hbm) + out * turns;
      if (t < best) { best = t; p.kernel = I8_SWAP; p.bn = bn; p.split = s; }
    }
  }
  return p;
}

template <int S>
cudaError_t launch_i8_swap(const I8Args& g, int sm_count, cudaStream_t st) {
  const int tiles = g.tiles_m * g.tiles_n;
  const int ring = swap_ring(g.bn, (long long)tiles * S, S, sm_count);
  cudaError_t e = cudaFuncSetAttribute(gemm_i8_swap_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sw_smem(SW_RING_1));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * S));
  cfg.blockDim = dim3(SW_THREADS);
  cfg.dynamicSmemBytes = sw_smem(ring);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = S;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, gemm_i8_swap_kernel<S>, g, ring);
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace
}  // namespace epara

extern "C" int epara_gemm_i8(int device, void* cuda_stream, const epara_gemm_i8_problem* p, int* status) {
  using namespace epara;
  if (!p || !status || !aligned(status, 4)) return EPARA_E_INVALID;
  const epara_gemm_i8_problem& q = *p;
  if (q.M < 0 || q.N <= 0 || q.K <= 0) return EPARA_E_INVALID;
  if (q.M == 0) return EPARA_OK;                   // (whose tensors may have no address)
  if (!q.A || !q.W || !q.C || !q.a_scale || !q.w_scale) return EPARA_E_INVALID;
  if (q.K > EPARA_GEMM_I8_MAX_K || q.M > 1 << 30 || q.N > 1 << 30 || ((long long)q.M + 127) / 128 * (((long long)q.N + 127) / 128) > 1 << 30) return EPARA_E_UNSUPPORTED;
  if (q.lda % 16 || q.ldw % 16 || q.lda < q.K || q.ldw < q.K) return EPARA_E_INVALID;
  const bool f32 = (q.epilogue & EPARA_EPI_RESID_F32) != 0, swi = (q.epilogue & EPARA_EPI_SWIGLU) != 0;
  if (!aligned(q.A, 16) || !aligned(q.W, 16) || !aligned(q.C, 16) || !aligned(q.a_scale, 16) || !aligned(q.w_scale, 16)) return EPARA_E_INVALID;
  if ((q.epilogue & EPARA_EPI_BIAS) && (!q.bias || !aligned(q.bias, 16))) return EPARA_E_INVALID;
  if ((q.epilogue & ~(EPARA_EPI_BIAS | EPARA_EPI_GELU | EPARA_EPI_SWIGLU | EPARA_EPI_RESID_F32)) || (swi && (q.N % 2 || f32))) return EPARA_E_INVALID;
  if (q.ldc < (swi ? q.N / 2 : q.N)) return EPARA_E_INVALID;
  const DeviceScope scope(device);
  if (!scope.ok) return EPARA_E_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const int sm = device_sm_count(device);
  const I8Plan plan = i8_plan(q.M, q.N, q.K, sm);
  I8Args g;
  g.a_scale = q.a_scale; g.w_scale = q.w_scale; g.bias = (const bf16*)q.bias; g.C = q.C; g.status = status;
  g.M = q.M; g.N = q.N; g.K = q.K; g.ldc = q.ldc; g.epi = q.epilogue;
  g.bn = plan.bn; g.tiles_m = g.tiles_n = 1; g.vec = 0;
  cudaError_t e;
  if (plan.kernel == I8_SWAP) {
    g.tiles_m = (q.M + g.bn - 1) / g.bn;
    g.tiles_n = (q.N + SW_BM - 1) / SW_BM;
    g.vec = q.ldc % (swi ? 2 : 4) == 0;
    if (!make_i8_map(&g.tmA, q.A, q.M, q.K, q.lda, g.bn) || !make_i8_map(&g.tmW, q.W, q.N, q.K, q.ldw, SW_BM)) return EPARA_E_CUDA;
    e = plan.split == 1 ? launch_i8_swap<1>(g, sm, st) : plan.split == 2 ? launch_i8_swap<2>(g, sm, st) : plan.split == 4 ? launch_i8_swap<4>(g, sm, st) : launch_i8_swap<8>(g, sm, st);
  } else {
    g.tiles_m = (q.M + 255) / 256;
    g.tiles_n = (q.N + g.bn - 1) / g.bn;
    g.vec = q.ldc % (f32 ? 4 : 8) == 0;
    if (!make_i8_map(&g.tmA, q.A, q.M, q.K, q.lda, 128) || !make_i8_map(&g.tmW, q.W, q.N, q.K, q.ldw, g.bn / 2)) return EPARA_E_CUDA;
    e = cudaFuncSetAttribute(gemm_i8_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PR_SMEM);
    const int pairs = std::min(g.tiles_m * g.tiles_n, sm / 2);
    if (e == cudaSuccess) e = launch_pdl(gemm_i8_pair_kernel, dim3((unsigned)(2 * pairs)), dim3(PR_THREADS), PR_SMEM, st, g);
  }
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

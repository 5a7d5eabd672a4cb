// Root-mean-square norm with the residual's addition, quantised to int8 with a scale per row:
//   h = resid + x,  y = (h g) / sqrt(mean(h^2) + eps),  s = max(max|y| / 127, 2^-126),  q = rn(y / s)
// (without g: y = h).  One pass: the row stays in registers between its two uses, and since y = (h g) r with one r for the row,
// max|y| = r max|h g| comes out of the same reduction as the sum of squares.  All arithmetic is fp32; the sum h is kept in
// fp32 like the rest of the residual stream.  A row with a NaN or infinity (or whose squares overflow fp32) gets a NaN scale and
// zero codes, so that its products are NaN too.
// Bound by HBM: 11 bytes an element with a bf16 x and both residuals.
#include "../../include/epara.h"
#include "common.cuh"
#include "kernels.h"

namespace epara {

namespace {

constexpr float FLT_LARGEST = 3.4028234e38f;
constexpr float TINY_SCALE = 1.17549435e-38f;     // 2^-126: codes of a row of zeros need no case of their own

struct NormI8 {
  const void* x;
  const float* resid;
  float* resid_out;
  const bf16* gain;
  int8_t* q;
  float* scales;
  long long x_stride, resid_stride, out_stride, q_stride;
  int rows, d;
  float eps;
};

// V consecutive values
template <int V, bool F32>
__device__ __forceinline__ void load_x(const void* p, size_t i, float* f) {
  if constexpr (V == 1) {
    f[0] = F32 ? __ldcs(static_cast<const float*>(p) + i) : __uint_as_float((uint32_t)__ldcs(static_cast<const unsigned short*>(p) + i) << 16);
  } else if constexpr (F32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = __ldcs(q), b = __ldcs(q + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    unpack8(__ldcs(reinterpret_cast<const uint4*>(static_cast<const bf16*>(p) + i)), f);
  }
}

// TPR threads of a block share a row; each has NV groups of V values (V 8: vectors; V 1: any alignment).
constexpr int MOST_THREADS = 512;                  // where a thread holds the most: 128 registers
constexpr int most_groups(int v) { return v == 8 ? 4 : 16; }
template <int V, int NV, bool F32>
__global__ void __launch_bounds__(NV == most_groups(V) ? MOST_THREADS : 1024) rms_norm_i8_kernel(const NormI8 a, int tpr) {
  __shared__ float2 red[32];
  pdl_wait();
  const int t = threadIdx.x % tpr, sub = threadIdx.x / tpr;
  const long long row = (long long)blockIdx.x * (blockDim.x / tpr) + sub;
  const bool live = row < a.rows;
  float h[NV][V];
  float ss = 0.f, top = 0.f;
  if (live) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * tpr) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = 0.f;
      if (c < a.d) load_x<V, F32>(a.x, row * a.x_stride + c, h[i]);
    }
    if (a.resid != nullptr) {
      float r[NV][V];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + i * tpr) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) r[i][e] = 0.f;
        if (c < a.d) load_x<V, true>(a.resid, row * a.resid_stride + c, r[i]);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + i * tpr) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) h[i][e] += r[i][e];
        if (c < a.d && a.resid_out != nullptr) {
          float* o = a.resid_out + row * a.out_stride + c;
          if constexpr (V == 8) {
            *reinterpret_cast<float4*>(o) = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
            *reinterpret_cast<float4*>(o + 4) = make_float4(h[i][4], h[i][5], h[i][6], h[i][7]);
          } else {
            o[0] = h[i][0];
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * tpr) * V;
      if (a.gain != nullptr && c < a.d) {
        float g[V];
        if constexpr (V == 8) unpack8(*reinterpret_cast<const uint4*>(a.gain + c), g);
        else g[0] = bf2f(a.gain[c]);
#pragma unroll
        for (int e = 0; e < V; ++e) { ss = fmaf(h[i][e], h[i][e], ss); h[i][e] *= g[e]; }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float m = fabsf(h[i][e]);
        top = fmaxf(top, m <= FLT_LARGEST ? m : INFINITY);
      }
    }
  }
  ss = warp_sum(ss);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (tpr > 32) {                                  // (tpr is a multiple of 32, the same for the whole block)
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(ss, top);
    __syncthreads();
    const int w0 = sub * (tpr >> 5), lane = threadIdx.x & 31;
    const float2 v = lane < (tpr >> 5) ? red[w0 + lane] : make_float2(0.f, 0.f);
    ss = warp_sum(v.x);
    top = v.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if (!live) return;
  float r = 1.f;
  bool fine = true;
  if (a.gain != nullptr) {
    r = 1.f / sqrtf(ss / (float)a.d + a.eps);
    fine = ss <= FLT_LARGEST && r <= FLT_LARGEST;
  }
  top *= r;
  fine = fine && top <= FLT_LARGEST;
  const float scale = fmaxf(top / 127.f, TINY_SCALE);
  if (t == 0) a.scales[row] = fine ? scale : __int_as_float(0x7fffffff);
  const float f = 1.f / scale;
  // y f + 1.5 x 2^23 has rn(y f) in its low bits
  constexpr float MAGIC = 12582912.f;
  int8_t* const q = a.q + row * a.q_stride;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * tpr) * V;
    if (c >= a.d) continue;
    uint32_t b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) b[e] = fine ? __float_as_uint(fmaf(h[i][e] * r, f, MAGIC)) : 0u;
    if constexpr (V == 8) {
      uint2 o;
      o.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
      o.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
      *reinterpret_cast<uint2*>(q + c) = o;
    } else {
      q[c] = (int8_t)(b[0] & 0xffu);
    }
  }
}

// Rows too long for registers: the row is read twice (its second time through the caches).  With resid and no resid_out the sum
// is formed twice.
template <bool F32>
__global__ void __launch_bounds__(1024) rms_norm_i8_long_kernel(const NormI8 a) {
  __shared__ float2 red[32];
  pdl_wait();
  const long long row = blockIdx.x;
  float ss = 0.f, top = 0.f;
  auto value = [&](int c) {
    float v;
    load_x<1, F32>(a.x, row * a.x_stride + c, &v);
    if (a.resid != nullptr) v += a.resid[row * a.resid_stride + c];
    return v;
  };
  const bool in_place = a.resid != nullptr && a.resid_out != nullptr;
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    float h = value(c);
    if (in_place) a.resid_out[row * a.out_stride + c] = h;
    if (a.gain != nullptr) { ss = fmaf(h, h, ss); h *= bf2f(a.gain[c]); }
    const float m = fabsf(h);
    top = fmaxf(top, m <= FLT_LARGEST ? m : INFINITY);
  }
  ss = warp_sum(ss);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(ss, top);
  __syncthreads();
  const float2 v = red[threadIdx.x & 31];
  ss = warp_sum(v.x);
  top = v.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float r = 1.f;
  bool fine = true;
  if (a.gain != nullptr) {
    r = 1.f / sqrtf(ss / (float)a.d + a.eps);
    fine = ss <= FLT_LARGEST && r <= FLT_LARGEST;
  }
  top *= r;
  fine = fine && top <= FLT_LARGEST;
  const float scale = fmaxf(top / 127.f, TINY_SCALE), f = 1.f / scale;
  if (threadIdx.x == 0) a.scales[row] = fine ? scale : __int_as_float(0x7fffffff);
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    float h = in_place ? a.resid_out[row * a.out_stride + c] : value(c);     // (each thread reads what it wrote itself)
    if (a.gain != nullptr) h *= bf2f(a.gain[c]);
    a.q[row * a.q_stride + c] = fine ? (int8_t)__float2int_rn(h * r * f) : (int8_t)0;
  }
}

template <int V, bool F32>
cudaError_t launch_norm_i8(const NormI8& a, int sm_count, cudaStream_t st) {
  const int groups = (a.d + V - 1) / V;
  constexpr int MOST = most_groups(V);             // groups a thread can hold
  if (groups > MOST * MOST_THREADS) return launch_pdl(rms_norm_i8_long_kernel<F32>, dim3((unsigned)a.rows), dim3(1024), 0, st, a);
  auto threads = [&](int nv) { return ((groups + nv - 1) / nv + 31) / 32 * 32; };
  // with no more rows than SMs a row is spread over as many threads as it has vectors, one load of each operand deep
  constexpr int FEW = V == 8 ? 1 : 4, MID = V == 8 ? 2 : 8;
  int nv = a.rows <= sm_count ? (threads(FEW) <= 1024 ? FEW : threads(MID) <= 1024 ? MID : MOST) : groups <= 32 * FEW ? FEW : groups <= 32 * MID ? MID : MOST;
  const int tpr = threads(nv);
  const int per_block = a.rows <= sm_count ? 1 : tpr >= 128 ? 1 : 128 / tpr;
  const dim3 grid((unsigned)((a.rows + per_block - 1) / per_block)), block((unsigned)(tpr * per_block));
  if (nv == FEW) return launch_pdl(rms_norm_i8_kernel<V, FEW, F32>, grid, block, 0, st, a, tpr);
  if (nv == MID) return launch_pdl(rms_norm_i8_kernel<V, MID, F32>, grid, block, 0, st, a, tpr);
  return launch_pdl(rms_norm_i8_kernel<V, MOST, F32>, grid, block, 0, st, a, tpr);
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace
}  // namespace epara

extern "C" int epara_rms_norm_i8(int device, void* cuda_stream, const void* x, int x_type, long long x_stride, const float* resid,
                                 long long resid_stride, float* resid_out, long long resid_out_stride, const void* gain, float eps,
                                 signed char* q, long long q_stride, float* scales, int rows, int d) {
  using namespace epara;
  if (!x || !q || !scales || rows < 0 || d <= 0 || (x_type != EPARA_T_BF16 && x_type != EPARA_T_F32)) return EPARA_E_INVALID;
  if (x_stride < d || q_stride < d || (resid && resid_stride < d) || (resid_out && (!resid || resid_out_stride < d))) return EPARA_E_INVALID;
  const bool f32 = x_type == EPARA_T_F32;
  if (!aligned(x, f32 ? 4 : 2) || !aligned(scales, 4) || !aligned(resid, 4) || !aligned(resid_out, 4) || !aligned(gain, 2)) return EPARA_E_INVALID;
  if (!(eps >= 0.f)) return EPARA_E_INVALID;
  if (rows == 0) return EPARA_OK;
  if (cudaSetDevice(device) != cudaSuccess) return EPARA_E_CUDA;
  NormI8 a;
  a.x = x; a.resid = resid; a.resid_out = resid_out; a.gain = (const bf16*)gain; a.q = (int8_t*)q; a.scales = scales;
  a.x_stride = x_stride; a.resid_stride = resid_stride; a.out_stride = resid_out_stride; a.q_stride = q_stride;
  a.rows = rows; a.d = d; a.eps = eps;
  const bool vec = d % 8 == 0 && aligned(x, 16) && x_stride % (f32 ? 4 : 8) == 0 && aligned(resid, 16) && aligned(resid_out, 16) &&
                   (!resid || resid_stride % 4 == 0) && (!resid_out || resid_out_stride % 4 == 0) && aligned(gain, 16) && aligned(q, 8) && q_stride % 8 == 0;
  const int sm = device_sm_count(device);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e = vec ? (f32 ? launch_norm_i8<8, true>(a, sm, st) : launch_norm_i8<8, false>(a, sm, st))
                      : (f32 ? launch_norm_i8<1, true>(a, sm, st) : launch_norm_i8<1, false>(a, sm, st));
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

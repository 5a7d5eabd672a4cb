// Root-mean-square norm with the residual's addition, quantised to int8 with a scale per row:
//   h = resid + x,  y = (h g) / sqrt(mean(h^2) + eps),  s = max(max|y| / 127, 2^-126),  q = rn(y / s)
// (without g: y = h).  One pass: the row stays in registers between its two uses, and since y = (h g) r with one r for the row,
// max|y| = r max|h g| comes out of the same reduction as the sum of squares.  All arithmetic is fp32; the sum h is kept in
// fp32 like the rest of the residual stream.  A row with a NaN or infinity (or whose squares overflow fp32) gets a NaN scale and
// zero codes, so that its products are NaN too.
// Bound by HBM: 11 bytes an element with a bf16 x and both residuals, 114 us for 16384 rows of 4096, floor 113; x in fp32 alone 54, floor 51; one row 2.6 us, a launch.
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

// V consecutive values as they are in memory, and as fp32 (bf16 values stay packed until they are used: a thread holds four groups)
template <int V, bool F32>
struct Raw {
  uint32_t w[F32 ? V : (V + 1) / 2];
  __device__ __forceinline__ void load(const void* p, long long i) {
    if constexpr (F32) {
      const float* q = static_cast<const float*>(p) + i;
      if constexpr (V == 1) {
        w[0] = __float_as_uint(__ldcs(q));
      } else {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          const uint4 a = __ldcs(reinterpret_cast<const uint4*>(q + e));
          w[e] = a.x; w[e + 1] = a.y; w[e + 2] = a.z; w[e + 3] = a.w;
        }
      }
    } else {
      const unsigned short* q = static_cast<const unsigned short*>(p) + i;
      if constexpr (V == 1) {
        w[0] = __ldcs(q);
      } else if constexpr (V == 4) {
        const uint2 u = __ldcs(reinterpret_cast<const uint2*>(q));
        w[0] = u.x; w[1] = u.y;
      } else {
        const uint4 u = __ldcs(reinterpret_cast<const uint4*>(q));
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < (F32 ? V : (V + 1) / 2); ++e) w[e] = 0u;
  }
  __device__ __forceinline__ float value(int e) const {
    if constexpr (F32) return __uint_as_float(w[e]);
    return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
  }
};
template <int V>
__device__ __forceinline__ void load_gain(const bf16* p, float* g) {
  if constexpr (V == 1) {
    g[0] = bf2f(*p);
  } else if constexpr (V == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    g[0] = __uint_as_float(u.x << 16); g[1] = __uint_as_float(u.x & 0xffff0000u); g[2] = __uint_as_float(u.y << 16); g[3] = __uint_as_float(u.y & 0xffff0000u);
  } else {
    unpack8(*reinterpret_cast<const uint4*>(p), g);
  }
}

// gain[c .. c + 3] for c = 4 n - shift, out of the two aligned groups that hold them; zeros outside [0, d)
__device__ __forceinline__ void load_gain_shifted(const bf16* gain, int c, int shift, int d, float* g) {
  const int n4 = c + shift;
  const unsigned long long hi = n4 < d ? *reinterpret_cast<const unsigned long long*>(gain + n4) : 0ull;
  const unsigned long long lo = shift && n4 > 0 ? *reinterpret_cast<const unsigned long long*>(gain + n4 - 4) : 0ull;
  const int s = 16 * (4 - shift);
  const unsigned long long v = shift ? lo >> s | hi << (64 - s) : hi;
#pragma unroll
  for (int e = 0; e < 4; ++e) g[e] = c + e >= 0 && c + e < d ? __uint_as_float((uint32_t)(v >> (16 * e)) << 16) : 0.f;
}

// The row's sum of squares (without gain 0; NaN when an element is not finite) and largest magnitude to its scale and the factor of its
// codes (0 when the row is not finite).  Answers what elements are to be multiplied by before the factor: 1, but for a row so close to zero that the two
// have to go one after the other.
__device__ __forceinline__ float row_scale(const NormI8& a, float ss, float top, float& scale, float& factor) {
  float r = 1.f;
  bool fine = ss <= FLT_LARGEST;
  if (a.gain != nullptr) {
    r = 1.f / sqrtf(ss / (float)a.d + a.eps);
    fine = fine && r <= FLT_LARGEST;
  }
  const float y = top * r;
  fine = fine && y <= FLT_LARGEST;
  scale = fine ? fmaxf(y / 127.f, TINY_SCALE) : __int_as_float(0x7fffffff);
  // (r / scale with one rounding instead of four: a code whose y / scale lies next to a border is wrong less often)
  factor = !fine ? 0.f : scale > TINY_SCALE ? 127.f / top : r / scale;
  if (!(factor > FLT_LARGEST)) return 1.f;
  factor = 1.f / scale;
  return r;
}
// y f + 1.5 x 2^23 has rn(y f) in its low bits.  The product is rounded first: values in bf16 often lie on a border exactly, as half of the
// largest one does, and there the rounded product is on it, too, and goes to the even code, where the factor's own error would decide otherwise.
// (A NaN times a factor of 0 is one still: a row that is not finite has its codes masked.)
__device__ __forceinline__ uint32_t code_of(float y, float factor) { return __float_as_uint(__fadd_rn(__fmul_rn(y, factor), 12582912.f)); }

// TPR threads of a block share a row; each has NV groups of V values.
// PHASE: rows of any length and place, V = 4.  All tensors have the same row stride, so that groups of four that are aligned in one are in
// all of them; the row's first and last group may be cut, and only the gains are not aligned with them.
constexpr int MOST_THREADS = 512;                  // where a thread holds the most: 128 registers
template <int V, int NV, bool F32, bool RESID, bool PHASE>
__global__ void __launch_bounds__(NV * V >= 32 || NV * V == 16 && V == 1 ? MOST_THREADS : 1024, NV * V >= 32 && !(F32 && RESID) ? 2 : 1)
rms_norm_i8_kernel(const NormI8 a, int tpr) {
  __shared__ float red[2][32];
  pdl_wait();
  const int t = threadIdx.x % tpr, sub = threadIdx.x / tpr, lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * (blockDim.x / tpr) + sub;
  const bool live = row < a.rows;
  const int shift = PHASE ? (int)(row * a.x_stride & 3) : 0;         // elements that the first group has before the row
  Raw<V, F32> x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * tpr) * V - shift;
    x[i].zero();
    if (live && c < a.d) x[i].load(a.x, row * a.x_stride + c);
  }
  float h[NV][V];
  if constexpr (RESID) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * tpr) * V - shift;
      Raw<V, true> r;
      r.zero();
      if (live && c < a.d) r.load(a.resid, row * a.resid_stride + c);
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = r.value(e);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * tpr) * V - shift;
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] += x[i].value(e);
      if (live && c < a.d && a.resid_out != nullptr) {
        float* o = a.resid_out + row * a.out_stride + c;
        if (PHASE && (c < 0 || c + V > a.d)) {
#pragma unroll
          for (int e = 0; e < V; ++e) if (c + e >= 0 && c + e < a.d) o[e] = h[i][e];
        } else if constexpr (V == 1) {
          o[0] = h[i][0];
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(o + e) = make_float4(h[i][e], h[i][e + 1], h[i][e + 2], h[i][e + 3]);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = x[i].value(e);
  }
  float ss = 0.f, top = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * tpr) * V - shift;
    if (PHASE && (c < 0 || c + V > a.d)) {
#pragma unroll
      for (int e = 0; e < V; ++e) if (c + e < 0 || c + e >= a.d) h[i][e] = 0.f;     // a neighbour's
    }
    if (a.gain != nullptr && c < a.d) {
      float g[V];
      if constexpr (PHASE) load_gain_shifted(a.gain, c, shift, a.d, g);
      else load_gain<V>(a.gain + c, g);
#pragma unroll
      for (int e = 0; e < V; ++e) { ss = fmaf(h[i][e], h[i][e], ss); h[i][e] *= g[e]; }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      top = fmaxf(top, fabsf(h[i][e]));          // (drops a NaN ...
      ss = fmaf(h[i][e], 0.f, ss);               // ... which the sum keeps, infinities too)
    }
  }
  for (int o = min(tpr, 32) >> 1; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if (tpr > 32) {                                // (8, 16 or a multiple of 32, the same for the whole block)
    float* const r = red[0];
    if (lane == 0) { r[threadIdx.x >> 5] = ss; r[32 + (threadIdx.x >> 5)] = top; }
    __syncthreads();
    const int w0 = sub * (tpr >> 5), warps = tpr >> 5;
    if (warps <= 8) {
      ss = top = 0.f;
      for (int w = 0; w < warps; ++w) { ss += r[w0 + w]; top = fmaxf(top, r[32 + w0 + w]); }
    } else {
      ss = warp_sum(lane < warps ? r[w0 + lane] : 0.f);
      top = lane < warps ? r[32 + w0 + lane] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
  }
  float scale, factor;
  const float before = row_scale(a, ss, top, scale, factor);
  if (before != 1.f) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] *= before;
  }
  if (live && t == 0) a.scales[row] = scale;
  const uint32_t keep = factor != 0.f ? 0xffffffffu : 0u;
  int8_t* const q = a.q + row * a.q_stride;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * tpr) * V - shift;
    if (!live || c >= a.d) continue;
    uint32_t b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) b[e] = code_of(h[i][e], factor);
    auto four = [&](int e) { return __byte_perm(__byte_perm(b[e], b[e + 1], 0x0040), __byte_perm(b[e + 2], b[e + 3], 0x0040), 0x5410) & keep; };
    if constexpr (V == 8) {
      *reinterpret_cast<uint2*>(q + c) = make_uint2(four(0), four(4));
    } else if constexpr (V == 4) {
      if (PHASE && (c < 0 || c + V > a.d)) {
#pragma unroll
        for (int e = 0; e < V; ++e) if (c + e >= 0 && c + e < a.d) q[c + e] = (int8_t)(b[e] & keep & 0xffu);
      } else {
        *reinterpret_cast<uint32_t*>(q + c) = four(0);
      }
    } else {
      q[c] = (int8_t)(b[0] & keep & 0xffu);
    }
  }
}

// Rows too long for registers: the row is read twice (its second time through the caches).  With resid and no resid_out the sum
// is formed twice.  A thread adds up to 2^20 squares: 32 at a time in fp32, these sums in 64 bits (in fp32 alone a row of 2^23 like values was off by
// 1.3e-5, and the error grows with the row).
template <bool F32>
__global__ void __launch_bounds__(1024) rms_norm_i8_long_kernel(const NormI8 a) {
  __shared__ float red[2][32];
  pdl_wait();
  const long long row = blockIdx.x;
  float ss = 0.f, top = 0.f;
  double sum = 0.;
  int pending = 0;
  auto value = [&](int c) {
    Raw<1, F32> x;
    x.load(a.x, row * a.x_stride + c);
    float v = x.value(0);
    if (a.resid != nullptr) v += a.resid[row * a.resid_stride + c];
    return v;
  };
  const bool in_place = a.resid != nullptr && a.resid_out != nullptr;
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    float h = value(c);
    if (in_place) a.resid_out[row * a.out_stride + c] = h;
    if (a.gain != nullptr) { ss = fmaf(h, h, ss); h *= bf2f(a.gain[c]); }
    top = fmaxf(top, fabsf(h));
    ss = fmaf(h, 0.f, ss);
    if (++pending == 32) { sum += ss; ss = 0.f; pending = 0; }
  }
  ss = warp_sum((float)(sum + ss));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (lane == 0) { red[0][w] = ss; red[1][w] = top; }
  __syncthreads();
  ss = warp_sum(red[0][lane]);
  top = red[1][lane];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float scale, factor;
  const float first = row_scale(a, ss, top, scale, factor);
  if (threadIdx.x == 0) a.scales[row] = scale;
  const uint32_t keep = factor != 0.f ? 0xffu : 0u;
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    float h = in_place ? a.resid_out[row * a.out_stride + c] : value(c);     // (each thread reads what it wrote itself)
    if (a.gain != nullptr) h *= bf2f(a.gain[c]);
    a.q[row * a.q_stride + c] = (int8_t)(code_of(h * first, factor) & keep);
  }
}

template <int V, int NV, bool F32, bool PHASE>
cudaError_t launch_as(const NormI8& a, int tpr, int per_block, cudaStream_t st) {
  const dim3 grid((unsigned)(((long long)a.rows + per_block - 1) / per_block)), block((unsigned)(tpr * per_block));
  return a.resid != nullptr ? launch_pdl(rms_norm_i8_kernel<V, NV, F32, true, PHASE>, grid, block, 0, st, a, tpr)
                            : launch_pdl(rms_norm_i8_kernel<V, NV, F32, false, PHASE>, grid, block, 0, st, a, tpr);
}

// Threads to a row: with no more rows than SMs as many as it has groups, one load of each operand deep; otherwise one to four groups a
// thread, whichever leaves the fewest idle, more groups ahead, the more so the fewer bytes a group is.  Short rows share a warp.
// Bytes a second on a B200, rows of 4096: x in fp32 with a residual 6.7 TB/s, in bf16 6.4; bf16 alone 4.1 (49 us for 16384 rows, 40 without
// gains, floor 31: some 20 instructions an element); 65536 rows of 64 5.9 with a residual (2.1 before short rows shared a warp); 16384 rows of 4095
// 5.0, element by element 2.4; 6000 of 11000 5.6.  Tried for bf16 alone: 8 groups a thread 56, values packed until they are used 69, rows in turn
// with the next ones on their way through shared memory 63, two values an instruction 49 (and slower for 14336 wide).
template <int V, bool F32, bool PHASE>
cudaError_t launch_norm_i8(const NormI8& a, int sm_count, cudaStream_t st) {
  const int groups = (a.d + V - 1) / V + (PHASE ? 1 : 0);            // (PHASE: a row may touch one more)
  constexpr int A = V == 8 ? 1 : V == 4 ? 2 : 4;   // groups a thread: A, 2 A, 3 A, 4 A
  auto threads = [&](int k) {
    const int t = (groups + k * A - 1) / (k * A);
    return t <= 8 ? 8 : t <= 16 ? 16 : (t + 31) / 32 * 32;
  };
  int k = 0;
  if (a.rows <= sm_count) {
    while (++k < 4 && threads(k) > 1024) {}
  } else {
    int best = 1 << 30;
    for (int j = 4; j >= 1; --j) {
      const int cost = threads(j) * j * (!F32 && a.resid == nullptr ? 20 - 3 * j : 14 - j);
      if (j == 4 && F32 && a.resid != nullptr && threads(j) > 192) continue;         // (92 registers a thread: two long rows an SM at a time)
      if (cost < best && threads(j) <= (j == 4 ? MOST_THREADS : 1024)) { best = cost; k = j; }
    }
  }
  if (k == 0 || threads(k) > (k == 4 ? MOST_THREADS : 1024)) return launch_pdl(rms_norm_i8_long_kernel<F32>, dim3((unsigned)a.rows), dim3(1024), 0, st, a);
  const int tpr = threads(k), per_block = a.rows <= sm_count || tpr >= 128 ? 1 : 128 / tpr;
  if (k == 1) return launch_as<V, A, F32, PHASE>(a, tpr, per_block, st);
  if (k == 2) return launch_as<V, 2 * A, F32, PHASE>(a, tpr, per_block, st);
  if (k == 3) return launch_as<V, 3 * A, F32, PHASE>(a, tpr, per_block, st);
  return launch_as<V, 4 * A, F32, PHASE>(a, tpr, per_block, st);
}

template <bool F32>
cudaError_t launch_norm_i8(const NormI8& a, int width, int sm_count, cudaStream_t st) {
  if (width == 8) return launch_norm_i8<8, F32, false>(a, sm_count, st);
  if (width == 4) return launch_norm_i8<4, F32, false>(a, sm_count, st);
  if (width == -4) return launch_norm_i8<4, F32, true>(a, sm_count, st);
  return launch_norm_i8<1, F32, false>(a, sm_count, st);
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace
}  // namespace epara

extern "C" int epara_rms_norm_i8(int device, void* cuda_stream, const void* x, int x_type, long long x_stride, const float* resid,
                                 long long resid_stride, float* resid_out, long long resid_out_stride, const void* gain, float eps,
                                 signed char* q, long long q_stride, float* scales, int rows, int d) {
  using namespace epara;
  if (rows < 0 || d <= 0 || (x_type != EPARA_T_BF16 && x_type != EPARA_T_F32) || !(eps >= 0.f)) return EPARA_E_INVALID;
  if (d > 1 << 30) return EPARA_E_UNSUPPORTED;
  if (rows == 0) return EPARA_OK;                  // (whose tensors may have no address)
  if (!x || !q || !scales) return EPARA_E_INVALID;
  if (x_stride < d || q_stride < d || (resid && resid_stride < d) || (resid_out && (!resid || resid_out_stride < d))) return EPARA_E_INVALID;
  const bool f32 = x_type == EPARA_T_F32;
  if (!aligned(x, f32 ? 4 : 2) || !aligned(scales, 4) || !aligned(resid, 4) || !aligned(resid_out, 4) || !aligned(gain, 2)) return EPARA_E_INVALID;
  const DeviceScope scope(device);
  if (!scope.ok) return EPARA_E_CUDA;
  NormI8 a;
  a.x = x; a.resid = resid; a.resid_out = resid_out; a.gain = (const bf16*)gain; a.q = (int8_t*)q; a.scales = scales;
  a.x_stride = x_stride; a.resid_stride = resid_stride; a.out_stride = resid_out_stride; a.q_stride = q_stride;
  a.rows = rows; a.d = d; a.eps = eps;
  // groups of `v` values are aligned in every tensor of a row / of all rows taken as one
  auto bases = [&](int v) {
    const size_t f = v == 8 ? 16 : 4 * v;
    return aligned(x, f32 ? f : 2 * v) && aligned(resid, f) && aligned(resid_out, f) && aligned(q, v);
  };
  auto strides = [&](int v) { return d % v == 0 && x_stride % v == 0 && q_stride % v == 0 && (!resid || resid_stride % v == 0) && (!resid_out || resid_out_stride % v == 0); };
  int width = 1;
  if (bases(8) && strides(8) && aligned(gain, 16)) width = 8;
  else if (bases(4) && strides(4) && aligned(gain, 8)) width = 4;
  else if (bases(4) && aligned(gain, 8) && q_stride == x_stride && (!resid || resid_stride == x_stride) && (!resid_out || resid_out_stride == x_stride)) width = -4;
  const int sm = device_sm_count(device);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = f32 ? launch_norm_i8<true>(a, width, sm, st) : launch_norm_i8<false>(a, width, sm, st);
  return e == cudaSuccess ? EPARA_OK : EPARA_E_CUDA;
}

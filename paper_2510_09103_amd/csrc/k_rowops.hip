// Row-wise operators of a model's end: dropout whose mask is never stored, and the root-mean-square norm with the residual's
// addition (and that dropout) in front of it, forward and backward.
//
//   keep(r, c) = bits16(philox4x32-10(counter = (c / 8, r, offset), key = seed), c % 8) >= thr
//   h = round(residual + keep x s),  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd g
//   n = h rstd;  dh' = dh + rstd (g dy - n mean(g dy n));  dx = keep s dh';  dg = sum_r dy n
//
// All of them are bound by memory: every tensor is read once and written once, a row stays in the registers of the wavefront or
// workgroup that works on it between the sums over it and what they are needed for.
#include "ew_math.h"
#include "ops_plan.h"

namespace adapm {

namespace {

// 16 bytes at the alignment of their elements: rows may start anywhere
typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef float f32x4_e4 __attribute__((ext_vector_type(4), aligned(4), may_alias));
typedef uint32_t u32x2_e1 __attribute__((ext_vector_type(2), aligned(1), may_alias));

struct V8 {
  float v[8];
};

// element type: float, or uint16_t for bf16
template <class T>
__device__ __forceinline__ float load1(const T* p);
template <>
__device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load1<uint16_t>(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }

// elements p[0 .. n) of a group of eight, n >= 8: all of them; zeros behind the end
__device__ __forceinline__ V8 load8(const float* p, int n) {
  V8 r;
  if (n >= 8) {
    const f32x4_e4 a = *reinterpret_cast<const f32x4_e4*>(p), b = *reinterpret_cast<const f32x4_e4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.v[i] = a[i]; r.v[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < n ? p[i] : 0.f;
  }
  return r;
}
__device__ __forceinline__ V8 load8(const uint16_t* p, int n) {
  V8 r;
  if (n >= 8) {
    const u32x4_e2 a = *reinterpret_cast<const u32x4_e2*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.v[2 * i] = bf16lo(a[i]); r.v[2 * i + 1] = bf16hi(a[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < n ? load1(p + i) : 0.f;
  }
  return r;
}
__device__ __forceinline__ void store8(float* p, const V8& r, int n) {
  if (n >= 8) {
    f32x4_e4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = r.v[i]; b[i] = r.v[4 + i]; }
    *reinterpret_cast<f32x4_e4*>(p) = a;
    *reinterpret_cast<f32x4_e4*>(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = r.v[i];
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const V8& r, int n) {
  u32x4_e2 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = pack_bf16x2(r.v[2 * i], r.v[2 * i + 1]);
  if (n >= 8) {
    *reinterpret_cast<u32x4_e2*>(p) = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint16_t)(a[i / 2] >> (16 * (i & 1)));
  }
}
// the value that a store in the type T keeps
__device__ __forceinline__ void round8(V8&, const float*) {}
__device__ __forceinline__ void round8(V8& r, const uint16_t*) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = pack_bf16x2(r.v[2 * i], r.v[2 * i + 1]);
    r.v[2 * i] = bf16lo(w);
    r.v[2 * i + 1] = bf16hi(w);
  }
}
__device__ __forceinline__ V8 load8_as(const void* p, int bf16, int64_t at, int n) {
  return bf16 ? load8(reinterpret_cast<const uint16_t*>(p) + at, n) : load8(reinterpret_cast<const float*>(p) + at, n);
}

// Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011).  One counter
// serves eight elements with 16 bits each: the generator's 20 wide multiplications for eight elements cost about 15 lane-cycles
// an element, below the time that memory needs for the element; one word an element would be twice that and above it.
__device__ __forceinline__ void philox8(const DropDev& d, uint64_t offset, uint32_t group, uint32_t row, uint32_t (&w)[4]) {
  uint32_t c0 = group, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32), k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}
// what is dropped becomes zero whatever it was (infinities and NaN among it)
__device__ __forceinline__ void drop8(V8& r, const DropDev& d, uint64_t offset, uint32_t group, uint32_t row) {
  uint32_t w[4];
  philox8(d, offset, group, row, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t bits = (i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
    r.v[i] = bits >= d.thr ? r.v[i] * d.scale : 0.f;
  }
}
__device__ __forceinline__ uint64_t drop_offset(const DropDev& d) { return d.offset + (d.offset_dev ? *d.offset_dev : 0ull); }

// ---- dropout ---------------------------------------------------------------------------------------------------------
template <class T, class I>
__global__ __launch_bounds__(256) void dropout_kernel(Rows y, Rows x, Rows residual, I total, uint32_t groups, int64_t cols, DropDev d) {
  const uint64_t offset = drop_offset(d);
  for (I i = (I)blockIdx.x * 256 + threadIdx.x; i < total; i += (I)gridDim.x * 256) {
    const I row = i / groups;
    const uint32_t g = (uint32_t)(i - row * groups);
    const int64_t c = (int64_t)g * 8;
    const int n = (int)(cols - c < 8 ? cols - c : 8);
    V8 v = load8(reinterpret_cast<const T*>(x.p) + (int64_t)row * x.stride + c, n);
    V8 r;
    if (residual.p) r = load8(reinterpret_cast<const T*>(residual.p) + (int64_t)row * residual.stride + c, n);
    if (d.thr) drop8(v, d, offset, g, (uint32_t)row);
    if (residual.p) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v.v[k] += r.v[k];
    }
    store8(reinterpret_cast<T*>(y.p) + (int64_t)row * y.stride + c, v, n);
  }
}

// ---- norm ------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
// A row belongs to TPR threads: one of the four wavefronts of a workgroup (TPR = 64), or a workgroup of two or four.
constexpr int threads_of(int tpr) { return tpr == 64 ? 256 : tpr; }

// Over the threads of a row.  `red` is used by one sum only until the next barrier but one: two of them in turn need no second barrier.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float* red) {
  x = wave_sum(x);
  if (TPR == 64) return x;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return TPR == 128 ? red[0] + red[1] : (red[0] + red[1]) + (red[2] + red[3]);
}
template <int TPR>
__device__ __forceinline__ float row_max(float x, float* red) {
  x = wave_max(x);
  if (TPR == 64) return x;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return TPR == 128 ? fmaxf(red[0], red[1]) : fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

template <class T, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void norm_forward_kernel(NormDev a) {
  __shared__ float red[2][4];
  const int t = threadIdx.x % TPR;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (threads_of(TPR) / TPR) + threadIdx.x / TPR;
  if (row >= a.rows) return;         // whole wavefronts where TPR = 64, whole workgroups where one is a row
  const uint64_t offset = a.drop.thr ? drop_offset(a.drop) : 0;
  V8 h[NV];
  float sq = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + t) * 8, n = a.cols - c;
    if (n > 0) h[k] = load8(reinterpret_cast<const T*>(a.x.p) + row * a.x.stride + c, n);
  }
  if (a.h.p) {
    V8 r[NV];
    if (a.residual.p) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + t) * 8, n = a.cols - c;
        if (n > 0) r[k] = load8(reinterpret_cast<const T*>(a.residual.p) + row * a.residual.stride + c, n);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + t) * 8, n = a.cols - c;
      if (n > 0) {
        if (a.drop.thr) drop8(h[k], a.drop, offset, (uint32_t)c / 8, (uint32_t)row);
        if (a.residual.p) {
#pragma unroll
          for (int i = 0; i < 8; ++i) h[k].v[i] += r[k].v[i];
        }
        // the norm is of the residual stream as it is kept: the backward pass reads the same values
        round8(h[k], (const T*)nullptr);
        store8(reinterpret_cast<T*>(a.h.p) + row * a.h.stride + c, h[k], n);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if ((k * TPR + t) * 8 < a.cols) {      // behind the row's end the last group holds zeros
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = fmaf(h[k].v[i], (k * TPR + t) * 8 + i < a.cols ? h[k].v[i] : 0.f, sq);
    }
  const float rstd = rsqrtf(row_sum<TPR>(sq, red[0]) / (float)a.cols + a.eps);
  if (t == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + t) * 8, n = a.cols - c;
    if (n > 0) {
      const V8 g = load8_as(a.weight, a.w_bf16, c, n);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[k].v[i] = h[k].v[i] * rstd * g.v[i];
      if (!a.out8) store8(reinterpret_cast<T*>(a.y.p) + row * a.y.stride + c, h[k], n);
    }
  }
  if (!a.out8) return;
  // e4m3 with one scale a row: the row's largest value becomes the type's largest, 448.  The scale is a normal number: below 2^-126 the
  // quotient would lose digits, 1 / scale would be infinite and the row's zeros NaN.  Such a row keeps values of 2^-126 times the type's.
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if ((k * TPR + t) * 8 < a.cols) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((k * TPR + t) * 8 + i < a.cols) top = fmaxf(top, fabsf(h[k].v[i]));
    }
  top = row_max<TPR>(top, red[1]);
  const float scale = top > 0.f ? fmaxf(top / 448.f, 0x1p-126f) : 1.f, inv = 1.f / scale;
  if (t == 0) a.y_scale[row] = scale;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + t) * 8, n = a.cols - c;
    if (n > 0) {
      uint32_t q[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // a value that the product with 1 / scale takes past 448 stays 448, NaN stays NaN
        float z[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = h[k].v[4 * i + j] * inv;
          z[j] = v != v ? v : __builtin_amdgcn_fmed3f(v, -448.f, 448.f);
        }
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
        q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], w, true);
      }
      uint8_t* p = reinterpret_cast<uint8_t*>(a.y.p) + row * a.y.stride + c;
      if (n >= 8) {
        u32x2_e1 w;
        w[0] = q[0]; w[1] = q[1];
        *reinterpret_cast<u32x2_e1*>(p) = w;
      } else {
        for (int i = 0; i < n; ++i) p[i] = (uint8_t)(q[i / 4] >> (8 * (i & 3)));
      }
    }
  }
}

// Each workgroup takes every gridDim-th set of rows and keeps its share of dweight in registers on the way (fp32); the sums of the
// workgroups are added by norm_dweight_kernel in a fixed order.
template <class T, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void norm_backward_kernel(NormDev a) {
  constexpr int RPB = threads_of(TPR) / TPR;
  __shared__ float red[2][4];
  int turn = 0;
  const int t = threadIdx.x % TPR;
  const uint64_t offset = a.drop.thr ? drop_offset(a.drop) : 0;
  V8 dg[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[k].v[i] = 0.f;
  for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < a.rows; row += (int64_t)gridDim.x * RPB) {
    const float rstd = a.rstd[row];
    V8 dy[NV], h[NV], up[NV];
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + t) * 8, n = a.cols - c;
      if (n > 0) {
        dy[k] = load8(reinterpret_cast<const T*>(a.dy.p) + row * a.dy.stride + c, n);
        h[k] = load8(reinterpret_cast<const T*>(a.h.p) + row * a.h.stride + c, n);
        if (a.dh.p) up[k] = load8(reinterpret_cast<const T*>(a.dh.p) + row * a.dh.stride + c, n);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + t) * 8, n = a.cols - c;
      if (n > 0) {
        const V8 g = load8_as(a.weight, a.w_bf16, c, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[k].v[i] *= rstd;                                   // n
          dg[k].v[i] = fmaf(dy[k].v[i], h[k].v[i], dg[k].v[i]);
          dy[k].v[i] *= g.v[i];
          dot = fmaf(dy[k].v[i], h[k].v[i], dot);              // zeros behind the row's end
        }
      }
    }
    const float mean = row_sum<TPR>(dot, red[turn]) / (float)a.cols;
    turn ^= 1;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + t) * 8, n = a.cols - c;
      if (n > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dy[k].v[i] = rstd * fmaf(-h[k].v[i], mean, dy[k].v[i]);
          if (a.dh.p) dy[k].v[i] += up[k].v[i];
        }
        if (a.dres.p) store8(reinterpret_cast<T*>(a.dres.p) + row * a.dres.stride + c, dy[k], n);
        if (a.drop.thr) drop8(dy[k], a.drop, offset, (uint32_t)c / 8, (uint32_t)row);
        store8(reinterpret_cast<T*>(a.dx.p) + row * a.dx.stride + c, dy[k], n);
      }
    }
  }
  float* out = a.partial + (int64_t)blockIdx.x * a.cols;
  if (TPR > 64) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + t) * 8, n = a.cols - c;
      if (n > 0) store8(out + c, dg[k], n);
    }
  } else {
    // the four wavefronts of the workgroup, one after the other
    __shared__ float sum[TPR == 64 ? NV * 512 : 1];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if ((int)(threadIdx.x >> 6) == w) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int at = (k * 8 + i) * 64 + t;
            sum[at] = w ? sum[at] + dg[k].v[i] : dg[k].v[i];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const int k = c / 512, u = (c / 8) % 64, i = c % 8;
      out[c] = sum[(k * 8 + i) * 64 + u];
    }
  }
}

// dweight[c] = sum over the workgroups' partial sums: 16 columns x 64 slices of the workgroups, joined in a fixed order.  (64 columns x 16
// slices: 20.8 us for 1024 x 2048 partial sums on 32 workgroups.)
__global__ __launch_bounds__(1024) void norm_dweight_kernel(const float* __restrict__ partial, int groups, int cols, void* out, int bf16) {
  __shared__ float red[64][17];
  const int l = threadIdx.x & 15, sl = threadIdx.x >> 4, c = blockIdx.x * 16 + l;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 4
    for (int g = sl; g < groups; g += 64) s += partial[(int64_t)g * cols + c];
  }
  red[sl][l] = s;
  __syncthreads();
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    if (sl < o) red[sl][l] += red[sl + o][l];
    __syncthreads();
  }
  if (sl == 0 && c < cols) {
    const float v = red[0][l];
    if (bf16) store1(reinterpret_cast<uint16_t*>(out) + c, v);
    else reinterpret_cast<float*>(out)[c] = v;
  }
}

// Threads of a row and groups of eight elements of each thread: as many threads as the row has groups, up to a workgroup of 256, so that a
// thread needs few registers and a compute unit holds many rows.  Backward of 16384 x 2048 with one wavefront a row, four groups a thread
// and 204 registers 110 us, with four wavefronts and 83 registers 74 (4.5 TB/s); forward of 8192 x 1600 with dropout 24.2 and 21.1 (5.0).
struct Shape {
  int tpr, nv;
};
Shape shape_of(int64_t cols) {
  if (cols <= 512) return {64, 1};
  if (cols <= 1024) return {128, 1};
  if (cols <= 2048) return {256, 1};
  if (cols <= 4096) return {256, 2};
  if (cols <= 8192) return {256, 4};
  return {256, 8};
}

template <class T>
void norm_forward(const NormDev& n, hipStream_t s) {
  const Shape f = shape_of(n.cols);
  const int rpb = threads_of(f.tpr) / f.tpr;
  // a dimension of the grid holds less than 2^32 threads
  const int64_t groups = (n.rows + rpb - 1) / rpb, wide = groups < (1 << 20) ? groups : 1 << 20;
  const dim3 grid((unsigned)wide, (unsigned)((groups + wide - 1) / wide)), block((unsigned)threads_of(f.tpr));
  if (f.tpr == 64) hipLaunchKernelGGL((norm_forward_kernel<T, 64, 1>), grid, block, 0, s, n);
  else if (f.tpr == 128) hipLaunchKernelGGL((norm_forward_kernel<T, 128, 1>), grid, block, 0, s, n);
  else if (f.nv == 1) hipLaunchKernelGGL((norm_forward_kernel<T, 256, 1>), grid, block, 0, s, n);
  else if (f.nv == 2) hipLaunchKernelGGL((norm_forward_kernel<T, 256, 2>), grid, block, 0, s, n);
  else if (f.nv == 4) hipLaunchKernelGGL((norm_forward_kernel<T, 256, 4>), grid, block, 0, s, n);
  else hipLaunchKernelGGL((norm_forward_kernel<T, 256, 8>), grid, block, 0, s, n);
}

template <class T>
void norm_backward(const NormDev& n, hipStream_t s) {
  const Shape f = shape_of(n.cols);
  const int groups = norm_backward_groups(n.rows, n.cols);
  const dim3 grid((unsigned)groups), block((unsigned)threads_of(f.tpr));
  if (f.tpr == 64) hipLaunchKernelGGL((norm_backward_kernel<T, 64, 1>), grid, block, 0, s, n);
  else if (f.tpr == 128) hipLaunchKernelGGL((norm_backward_kernel<T, 128, 1>), grid, block, 0, s, n);
  else if (f.nv == 1) hipLaunchKernelGGL((norm_backward_kernel<T, 256, 1>), grid, block, 0, s, n);
  else if (f.nv == 2) hipLaunchKernelGGL((norm_backward_kernel<T, 256, 2>), grid, block, 0, s, n);
  else if (f.nv == 4) hipLaunchKernelGGL((norm_backward_kernel<T, 256, 4>), grid, block, 0, s, n);
  else hipLaunchKernelGGL((norm_backward_kernel<T, 256, 8>), grid, block, 0, s, n);
  hipLaunchKernelGGL(norm_dweight_kernel, dim3((unsigned)((n.cols + 15) / 16)), dim3(1024), 0, s, n.partial, groups, n.cols, n.dweight, n.g_bf16);
}

template <class T>
void dropout(Rows y, Rows x, Rows residual, int64_t rows, int64_t cols, const DropDev& d, hipStream_t s) {
  const int64_t groups = (cols + 7) / 8, total = rows * groups;
  const int64_t wanted = (total + 255) / 256;
  const dim3 grid((unsigned)(wanted < 16384 ? wanted : 16384)), block(256);
  // 32-bit places, whose division by the groups of a row is cheap, wherever the loop's last step stays inside them
  if (total <= 0xffffffffll - 16384 * 256)
    hipLaunchKernelGGL((dropout_kernel<T, uint32_t>), grid, block, 0, s, y, x, residual, (uint32_t)total, (uint32_t)groups, cols, d);
  else
    hipLaunchKernelGGL((dropout_kernel<T, uint64_t>), grid, block, 0, s, y, x, residual, (uint64_t)total, (uint32_t)groups, cols, d);
}

}  // namespace

void launch_dropout(bool bf16, Rows y, Rows x, Rows residual, int64_t rows, int64_t cols, const DropDev& d, hipStream_t s) {
  if (bf16) dropout<uint16_t>(y, x, residual, rows, cols, d, s);
  else dropout<float>(y, x, residual, rows, cols, d, s);
}

void launch_norm_forward(bool bf16, const NormDev& n, hipStream_t s) {
  if (bf16) norm_forward<uint16_t>(n, s);
  else norm_forward<float>(n, s);
}

int norm_backward_groups(int64_t rows, int64_t cols) {
  const int tpr = shape_of(cols).tpr, rpb = threads_of(tpr) / tpr;
  const int64_t g = (rows + rpb - 1) / rpb;
  return (int)(g < 1 ? 1 : g < 1024 ? g : 1024);
}

void launch_norm_backward(bool bf16, const NormDev& n, hipStream_t s) {
  if (bf16) norm_backward<uint16_t>(n, s);
  else norm_backward<float>(n, s);
}

}  // namespace adapm

// gradclip.hip -- the norm of a list of gradients and its clipping.
//   norm = sqrt(sum of g^2 over all of them),  c = 1 if norm <= max_norm, else max_norm / norm
//   out = c g
// The list is laid out once as chunks in device memory.  Squares are summed in
// 64 bits, which no gradient's square leaves in either direction: a fixed
// number of workgroups, each over its own chunks, one partial sum each.  The
// second launch adds the partial sums in every workgroup alike and scales.
// Few chunks stay in one workgroup's registers between sum and scaling: one launch.
#include "kernels.hpp"
#include "launch.hpp"

namespace lora {

__global__ __launch_bounds__(64) void grad_layout_kernel(GradEntries es, int count, int chunk, GradChunk *out) {
  const int i = blockIdx.x;
  if (i >= count) return;
  const GradEntry e = es.e[i];
  const int64_t n = (e.n + chunk - 1) / chunk;
  for (int64_t k = threadIdx.x; k < n; k += 64) {
    GradChunk c;
    c.g = (const char *)e.g + k * chunk * ((e.flags & 1) ? 4 : 2);
    c.out = e.out ? (char *)e.out + k * chunk * ((e.flags & 2) ? 4 : 2) : nullptr;
    c.n = (int)min((int64_t)chunk, e.n - k * chunk);
    c.flags = e.flags;
    out[e.first + k] = c;
  }
}

// The 392 gradients of a 28-layer stack (194 MB fp32): norm 29 us (6.7 TB/s), scaling 69 (389 MB, 5.7
// TB/s, a copy's rate).  Reading twice is what the norm asks for; on the chip there is room
// for the half of it at most.
constexpr int GN_NT = 256;

__device__ __forceinline__ float grad_at(const GradChunk &c, int i) {
  return (c.flags & 1) ? ((const float *)c.g)[i] : BF16::to_float(((const uint16_t *)c.g)[i]);
}

template <typename E>
__device__ __forceinline__ double square_sum(const GradChunk &c) {
  double s = 0.0;
  const int nv = c.n / E::VEC;
  for (int i = threadIdx.x; i < nv; i += GN_NT) {
    float f[E::VEC];
    unpack_vec(E(), ((const u32x4 *)c.g)[i], f);
#pragma unroll
    for (int e = 0; e < E::VEC; ++e) s += (double)f[e] * (double)f[e];
  }
  const int i = nv * E::VEC + threadIdx.x;
  if (i < c.n) {
    const double x = grad_at(c, i);
    s += x * x;
  }
  return s;
}

__device__ __forceinline__ double grad_block_sum(double x, double *red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < GN_NT / 64; ++w) x += red[w];
  return x;
}

__global__ __launch_bounds__(GN_NT) void grad_norm_kernel(const GradChunk *chunks, int nchunk, double *part) {
  __shared__ double red[GN_NT / 64];
  double s = 0.0;
  for (int k = blockIdx.x; k < nchunk; k += gridDim.x) {
    const GradChunk c = chunks[k];
    s += (c.flags & 1) ? square_sum<F32>(c) : square_sum<BF16>(c);
  }
  s = grad_block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// (an unordered norm is not at most max_norm: the factor is NaN)
__device__ __forceinline__ float clip_factor(double norm, float max_norm) {
  return norm <= (double)max_norm ? 1.0f : (float)((double)max_norm / norm);
}

// The norm from the partial sums, in every workgroup alike.
__device__ __forceinline__ double total_norm(const double *part, int parts, double *red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += GN_NT) s += part[i];
  return sqrt(grad_block_sum(s, red));
}

__global__ __launch_bounds__(GN_NT) void grad_total_kernel(const double *part, int parts, float *norm) {
  __shared__ double red[GN_NT / 64];
  const double x = total_norm(part, parts, red);
  if (threadIdx.x == 0) norm[0] = (float)x;
}

// (stores past the last-level cache, where the gradients are read a second time: 97 us for
// both launches over 194 MB in fp32, else 106; more vectors in flight a thread or larger
// chunks change neither launch)
template <typename EI, typename EO>
__device__ __forceinline__ void scale_chunk(const GradChunk &c, float k) {
  // whole groups of 8 elements as vectors, the rest one by one
  const int n8 = c.n / 8;
  for (int i = threadIdx.x; i < n8; i += GN_NT) {
    float f[8];
#pragma unroll
    for (int q = 0; q < 8 / EI::VEC; ++q) unpack_vec(EI(), ((const u32x4 *)c.g)[i * (8 / EI::VEC) + q], f + q * EI::VEC);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= k;
#pragma unroll
    for (int q = 0; q < 8 / EO::VEC; ++q)
      __builtin_nontemporal_store(pack_vec(EO(), f + q * EO::VEC), (u32x4 *)c.out + i * (8 / EO::VEC) + q);
  }
  const int i = n8 * 8 + threadIdx.x;
  if (i < c.n) ((typename EO::T *)c.out)[i] = EO::from_float(grad_at(c, i) * k);
}

__global__ __launch_bounds__(GN_NT) void grad_scale_kernel(const GradChunk *chunks, int nchunk, const double *part, int parts,
                                                           float max_norm, float *norm) {
  __shared__ double red[GN_NT / 64];
  const double x = total_norm(part, parts, red);
  const float k = clip_factor(x, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    norm[0] = (float)x;
    norm[1] = k;
  }
  for (int i = blockIdx.x; i < nchunk; i += gridDim.x) {
    const GradChunk c = chunks[i];
    if (c.out == c.g && k == 1.0f) continue;  // in place and unclipped: nothing changes
    if (c.flags & 1) {
      if (c.flags & 2) scale_chunk<F32, F32>(c, k);
      else scale_chunk<F32, BF16>(c, k);
    } else {
      if (c.flags & 2) scale_chunk<BF16, F32>(c, k);
      else scale_chunk<BF16, BF16>(c, k);
    }
  }
}

// ---- few chunks: one workgroup ---------------------------------------------------------
// Two gradients of 2048 elements: 3.5 us, 5.0 a call, where two launches took 8.6.
constexpr int GS_NT = 1024;
__device__ __forceinline__ f32x4 grad4(const GradChunk &c, int i) {
  if (i + 4 <= c.n) {
    if (c.flags & 1) return *(const f32x4 *)((const float *)c.g + i);
    const uint2 x = *(const uint2 *)((const uint16_t *)c.g + i);
    return f32x4{__builtin_bit_cast(float, x.x << 16), __builtin_bit_cast(float, x.x & 0xffff0000u),
                 __builtin_bit_cast(float, x.y << 16), __builtin_bit_cast(float, x.y & 0xffff0000u)};
  }
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < c.n) x[e] = grad_at(c, i + e);
  return x;
}
__device__ __forceinline__ void put4(const GradChunk &c, int i, f32x4 x) {
  if (i + 4 <= c.n) {
    if (c.flags & 2) *(f32x4 *)((float *)c.out + i) = x;
    else *(uint2 *)((uint16_t *)c.out + i) = uint2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < c.n) {
      if (c.flags & 2) ((float *)c.out)[i + e] = x[e];
      else ((uint16_t *)c.out)[i + e] = BF16::from_float(x[e]);
    }
}
// (chunks of at most 4 GS_NT elements)
__global__ __launch_bounds__(GS_NT) void grad_few_kernel(const GradChunk *chunks, int nchunk, bool clip, float max_norm,
                                                         float *norm) {
  __shared__ double red[GS_NT / 64];
  const int i = 4 * threadIdx.x;
  f32x4 x[GRAD_FEW];
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < GRAD_FEW; ++k)
    x[k] = k < nchunk ? grad4(chunks[k], i) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < GRAD_FEW; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) s += (double)x[k][e] * (double)x[k][e];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = red[0];
#pragma unroll
  for (int w = 1; w < GS_NT / 64; ++w) s += red[w];
  s = sqrt(s);
  const float c = clip_factor(s, max_norm);
  if (threadIdx.x == 0) {
    norm[0] = (float)s;
    if (clip) norm[1] = c;
  }
  if (!clip) return;
#pragma unroll
  for (int k = 0; k < GRAD_FEW; ++k)
    if (k < nchunk) put4(chunks[k], i, x[k] * c);
}

hipError_t launch_grad_layout(const GradEntries &e, int count, int chunk, GradChunk *out, hipStream_t st) {
  hipLaunchKernelGGL(grad_layout_kernel, dim3(count), dim3(64), 0, st, e, count, chunk, out);
  return hipGetLastError();
}

hipError_t launch_grad_few(const GradChunk *c, int nchunk, bool clip, float max_norm, float *norm, hipStream_t st) {
  hipLaunchKernelGGL(grad_few_kernel, dim3(1), dim3(GS_NT), 0, st, c, nchunk, clip, max_norm, norm);
  return hipGetLastError();
}

static int grad_wgs(int nchunk) { return nchunk < 1 ? 1 : nchunk < GRAD_PARTS ? nchunk : GRAD_PARTS; }

hipError_t launch_grad_norm(const GradChunk *c, int nchunk, double *part, float *norm, hipStream_t st) {
  const int parts = grad_wgs(nchunk);
  hipLaunchKernelGGL(grad_norm_kernel, dim3(parts), dim3(GN_NT), 0, st, c, nchunk, part);
  if (norm) hipLaunchKernelGGL(grad_total_kernel, dim3(1), dim3(GN_NT), 0, st, part, parts, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradChunk *c, int nchunk, double *part, float max_norm, float *norm, hipStream_t st) {
  const int parts = grad_wgs(nchunk);
  hipLaunchKernelGGL(grad_scale_kernel, dim3(parts), dim3(GN_NT), 0, st, c, nchunk, part, parts, max_norm, norm);
  return hipGetLastError();
}

}  // namespace lora

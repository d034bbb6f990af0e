// gradclip.hip -- the norm of a list of gradients and its clipping.
//   norm = sqrt(sum of g^2 over all of them),  c = 1 if norm <= max_norm, else max_norm / norm
//   out = c g
// The list is laid out once as chunks in device memory.  Squares are summed in
// 64 bits, which no gradient's square leaves in either direction: a fixed
// number of workgroups, each over its own chunks, one partial sum each.
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
    for (int q = 0; q < 8 / EO::VEC; ++q) ((u32x4 *)c.out)[i * (8 / EO::VEC) + q] = pack_vec(EO(), f + q * EO::VEC);
  }
  const int i = n8 * 8 + threadIdx.x;
  if (i < c.n) ((typename EO::T *)c.out)[i] = EO::from_float(grad_at(c, i) * k);
}

__global__ __launch_bounds__(GN_NT) void grad_scale_kernel(const GradChunk *chunks, int nchunk, const double *part, int parts,
                                                           float max_norm, float *norm) {
  __shared__ double red[GN_NT / 64];
  const double x = total_norm(part, parts, red);
  const float k = x <= (double)max_norm ? 1.0f : (float)((double)max_norm / x);
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

hipError_t launch_grad_layout(const GradEntries &e, int count, int chunk, GradChunk *out, hipStream_t st) {
  hipLaunchKernelGGL(grad_layout_kernel, dim3(count), dim3(64), 0, st, e, count, chunk, out);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const GradChunk *c, int nchunk, double *part, float *norm, hipStream_t st) {
  const int parts = nchunk < 1 ? 1 : nchunk < GRAD_PARTS ? nchunk : GRAD_PARTS;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(parts), dim3(GN_NT), 0, st, c, nchunk, part);
  if (norm) hipLaunchKernelGGL(grad_total_kernel, dim3(1), dim3(GN_NT), 0, st, part, parts, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradChunk *c, int nchunk, double *part, float max_norm, float *norm, hipStream_t st) {
  const int parts = nchunk < 1 ? 1 : nchunk < GRAD_PARTS ? nchunk : GRAD_PARTS;
  hipLaunchKernelGGL(grad_scale_kernel, dim3(parts), dim3(GN_NT), 0, st, c, nchunk, part, parts, max_norm, norm);
  return hipGetLastError();
}

}  // namespace lora

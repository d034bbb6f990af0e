// x8prod.hip -- the rank-r products of the LoRA backward whose input x is kept in
// 8 bits (act8.hpp): u = x A^T where it is not saved, and the token reductions
//   dA = du^T x,  dB = s dy^T u.
// Codes are whole numbers up to 127, exact in bf16, so a product on the matrix
// cores takes them as they are; a scale belongs to a row and 128 columns of x and goes
// to the other side of the product: in u to the group's sum, in dA to du.  du and u
// are fp32 and stay so: v as the sum of three bf16, which hold its 24 bits.  (Two leave
// 2^-18 of it, 2e-6 of the gradient's norm; one 2^-9.  The third product is in the noise of the 29.5 us
// of 8192 -> 3072 at 4096 tokens.)
#include <algorithm>

#include "act8.hpp"
#include "launch.hpp"
#include "meet_flags.hpp"

namespace lora {

// 8 codes as a matrix-core operand of bf16 (whole numbers up to 127: no rounding).
__device__ __forceinline__ u32x4 x8_operand(uint2 q) {
  float f[8];
  act8_floats(q, f);
  u32x4 r;
#pragma unroll
  for (int d = 0; d < 4; ++d) r[d] = pack_bf16x2(f[2 * d], f[2 * d + 1]);
  return r;
}

// ---- u = x A^T -----------------------------------------------------------------------
// A workgroup of 8 waves takes 16 tokens, 16 JB ranks and a range of groups; each wave every
// eighth group.  The wave loads a group of x and of A in whole lines, a step ahead, in
// the one of two register sets that the step does not use, and turns it into operands (row or rank
// l % 16, 8 columns l / 16 on) through LDS of its own.  Loads go through buffer resources:
// tokens, columns and ranks past the end read zeros.
// What bounds it is how many lines its loads touch: loads in the operands' layout, 16 rows
// an instruction and no two neighbouring lanes in one, took 8.4 us at 4096 x 3072 codes and r =
// 16 (10.1 at r = 32) in the place of 6.3 (9.4).  32 tokens a workgroup, which read A half as often, and two
// ranges took as long (6.3, 8.5) and left sums of u to be added, 2.5 more.
constexpr int X8D_NW = 8;

template <int JB>
__global__ __launch_bounds__(64 * X8D_NW) void x8_down_kernel(X8Down a, int groups_per) {
  constexpr uint32_t OOB = 0x80000000u;
  constexpr int LD = JB * 16 + 1, ROWS = 16, RB = 16 * JB, TX = ACT8_G + 16, TA = 2 * ACT8_G + 16;  // bytes of a row
  constexpr int TURN = ROWS * TX + RB * TA + ROWS * 4;
  static_assert(ROWS * LD * 4 <= TURN, "a wave's sums take its LDS over");
  __shared__ __align__(16) char lds[X8D_NW][TURN];
  const int lane = threadIdx.x & 63, c = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char *const turn_x = lds[wave], *const turn_a = turn_x + ROWS * TX;
  float *const turn_s = (float *)(turn_a + RB * TA);
  const int ng = (a.K + ACT8_G - 1) / ACT8_G;
  const int g1 = min(ng, ((int)blockIdx.y + 1) * groups_per);
  const int t0 = blockIdx.x * ROWS, rows = min(ROWS, a.T - t0), j0 = blockIdx.z * RB;
  const __amdgpu_buffer_rsrc_t rx =
      __builtin_amdgcn_make_buffer_rsrc((void *)(a.x.codes + (int64_t)t0 * a.K), (short)0, rows * a.K, 0x00020000);
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void *)(a.x.scale + (int64_t)t0 * ng), (short)0, rows * ng * 4, 0x00020000);
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void *)a.A, (short)0, a.r * a.K * 2, 0x00020000);
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  struct Step {
    u32x2 x[4];  // rows 4 i + q4, columns 8 c on
    u32x4 w[4 * JB];
    float s;
  };
  const bool scale_lane = lane < ROWS;
  // (offsets added to one choice: a choice for each load became a branch around it, with its own wait)
  auto load = [&](int g, Step &st) {
    const int col = g * ACT8_G + 8 * c;
    const uint32_t at = g < g1 && col < a.K ? (uint32_t)col : OOB;
    const uint32_t at_a = at == OOB ? OOB : 2 * at;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      st.x[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, at + (uint32_t)((4 * i + q4) * a.K), 0, 0));
#pragma unroll
    for (int i = 0; i < 4 * JB; ++i)
      st.w[i] = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, at_a + (uint32_t)((j0 + 4 * i + q4) * a.K * 2), 0, 0));
    st.s = __builtin_bit_cast(
        float, __builtin_amdgcn_raw_buffer_load_b32(rs, g < g1 && scale_lane ? (uint32_t)((lane * ng + g) * 4) : OOB, 0, 0));
    __builtin_amdgcn_sched_barrier(0);
  };
  f32x4 tot[JB];
#pragma unroll
  for (int j = 0; j < JB; ++j) tot[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](const Step &st) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *(u32x2 *)(turn_x + (4 * i + q4) * TX + 8 * c) = st.x[i];
#pragma unroll
    for (int i = 0; i < 4 * JB; ++i) *(u32x4 *)(turn_a + (4 * i + q4) * TA + 16 * c) = st.w[i];
    if (scale_lane) turn_s[lane] = st.s;
    u32x4 w[JB][4];
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) w[j][k] = *(const u32x4 *)(turn_a + (16 * j + c) * TA + 64 * k + 16 * q4);
    u32x4 xb[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) xb[k] = x8_operand(*(const uint2 *)(turn_x + c * TX + 32 * k + 8 * q4));
    const f32x4 s = *(const f32x4 *)(turn_s + 4 * q4);
    f32x4 acc[JB];
#pragma unroll
    for (int j = 0; j < JB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < JB; ++j) mma16(BF16(), acc[j], xb[k], w[j][k]);
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) tot[j][i] = __builtin_fmaf(s[i], acc[j][i], tot[j][i]);
  };
  {
    Step st[2];
    int g = blockIdx.y * groups_per + wave;
    load(g, st[0]);
    for (; g < g1; g += 2 * X8D_NW) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        load(g + (k + 1) * X8D_NW, st[k ^ 1]);
        if (g + k * X8D_NW < g1) compute(st[k]);
      }
    }
  }
  // the waves' sums, each in its LDS: element i of a lane is token 4 q4 + i, rank 16 j + c
  float *const red = (float *)lds[wave];
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[(4 * q4 + i) * LD + 16 * j + c] = tot[j][i];
  __syncthreads();
  float *u = a.u + ((int64_t)blockIdx.y * a.T + t0) * a.r;
  for (int e = threadIdx.x; e < ROWS * RB; e += 64 * X8D_NW) {
    const int t = e / RB, k = e % RB;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < X8D_NW; ++w) v += ((const float *)lds[w])[t * LD + k];
    if (t < rows && j0 + k < a.r) u[(int64_t)t * a.r + j0 + k] = v;
  }
}

struct X8DownSplit {
  int blocks, parts, groups;
};
static X8DownSplit x8_down_split(int64_t T, int64_t K) {
  const int64_t ng = (K + ACT8_G - 1) / ACT8_G, blocks = (T + 15) / 16;
  // as many ranges as give each CU a workgroup, each of a group a wave at least
  const int64_t p = std::max<int64_t>(1, std::min<int64_t>({4, 256 / blocks, ng / X8D_NW}));
  const int64_t groups = (ng + p - 1) / p;
  return {(int)blocks, (int)((ng + groups - 1) / groups), (int)groups};
}
int x8_down_parts(int64_t T, int64_t K) { return x8_down_split(T, K).parts; }

hipError_t launch_x8_down(const X8Down &a, hipStream_t st) {
  if (a.r < 1 || a.r > 128) return hipErrorInvalidValue;
  const X8DownSplit s = x8_down_split(a.T, a.K);
  const int jb = a.r <= 16 ? 1 : 2;
  const dim3 grid(s.blocks, s.parts, (a.r + 16 * jb - 1) / (16 * jb)), block(64 * X8D_NW);
  if (jb == 1) hipLaunchKernelGGL((x8_down_kernel<1>), grid, block, 0, st, a, s.groups);
  else hipLaunchKernelGGL((x8_down_kernel<2>), grid, block, 0, st, a, s.groups);
  return hipGetLastError();
}

// ---- dA = du^T x, dB = s dy^T u ------------------------------------------------------
// An item is 128 columns of x (a group: one scale a token) or 64 of dy, 128 bytes of a row
// either way, by 16 JB ranks, over a range of tokens.  Its waves take steps of 32 tokens in turn:
// lane (c = l % 16, g = l / 16) loads Q = 8 (4) columns of tokens 8 g .. 8 g + 7, and the 8
// tokens of one of its columns are an operand whose reduction axis is the token axis;
// product q takes column Q c + q of every c.  The waves' tiles are summed in LDS.
// 8192 -> 3072 at 4096 tokens, r = 32: 28 us, of which 7 are the sums, the meeting and the stores, 11
// a step's arithmetic and turns (V in three terms, turned for each 128 bytes of a row), and the rest
// loads that these do not hide; the 59 MB alone would be 11.  Loads are a step ahead: two steps
// ahead, and none left out at the end, took as long there and 6.3 us for 4.5 where a wave has a step or
// two (256 tokens, 3072 -> 3072, r = 16).
constexpr int X8P_NW = 8, X8P_ROWS = 32;
constexpr int X8_SC1 = 16;  // cache policy of the device scope

struct X8Unit {
  const void *X;
  const float *scale, *V;
  float *out;
  int L, ng, t0, t1, cb, jg;
  float mult;
};

// A buffer resource of scalars (the compiler moves their sums to vector registers in a loop, and then
// loads lane by lane).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t x8_resource(const void *p, int bytes) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), (short)0, __builtin_amdgcn_readfirstlane(bytes),
                                           0x00020000);
}

// LDS floats in which a wave turns a step's V around: 32 tokens of up to 16 JB ranks, 16 floats
// more after each 8 tokens (the four quarters of a wave then read different banks), and the scales.
constexpr int x8_turn(int jb) { return X8P_ROWS * 16 * jb + 3 * 16 + X8P_ROWS; }
// And those of its tile: 16 JB ranks of up to 128 columns, 4 floats behind each.
constexpr int x8_tile(int jb) { return 16 * jb * (ACT8_G + 4); }
constexpr int X8P_SLOT(int jb) { return ACT8_G * 16 * jb; }  // floats of an item's sums in the workspace

enum { V_FLAT = 0, V_ROWS = 1, V_EACH = 2 };
template <int JB, int VK, bool X8>
__device__ __forceinline__ void x8_item(const X8Prod &a, const X8Unit &n, int item, int part, int parts, float *lds) {
  constexpr uint32_t OOB = 0x80000000u;
  constexpr int ES = X8 ? 1 : 2, Q = 8 / ES, COLS = 16 * Q, RB = 16 * JB, TILE = COLS * RB, NT = 64 * X8P_NW;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float *const turn = lds + wave * x8_turn(JB), *const turn_s = turn + X8P_ROWS * RB + 48;
  const int col = n.cb * COLS + Q * c, r = a.r;
  const int row = VK == V_FLAT ? r : RB;  // of V in `turn`
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  struct StepX {
    u32x2 x[8];
  };
  struct StepV {
    f32x4 v[2 * JB];
    float s;
  };
  // Loads go through buffer resources based at the step's first token: tokens past the range,
  // columns past L and ranks past r read zeros.
  uint32_t off_x[8];  // (added to one choice: a choice for each load became a branch around it)
#pragma unroll
  for (int i = 0; i < 8; ++i) off_x[i] = (col < n.L ? (uint32_t)(col * ES) : OOB) + (uint32_t)((8 * g + i) * n.L * ES);
  auto load_x = [&](int tb, StepX &st) {
    const int rows = max(0, min(X8P_ROWS, n.t1 - tb));
    const __amdgpu_buffer_rsrc_t rx = x8_resource((const char *)n.X + (int64_t)tb * n.L * ES, rows * n.L * ES);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      st.x[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, off_x[i], 0, 0));
  };
  auto load_v = [&](int tb, StepV &st) {
    const int rows = max(0, min(X8P_ROWS, n.t1 - tb));
    if constexpr (X8) {
      const __amdgpu_buffer_rsrc_t rs = x8_resource(n.scale + (int64_t)tb * n.ng, rows * n.ng * 4);
      st.s = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, ((lane & 31) * n.ng + n.cb) * 4, 0, 0));
    }
    const __amdgpu_buffer_rsrc_t rv = x8_resource(n.V + (int64_t)tb * r, rows * r * 4);
#pragma unroll
    for (int k = 0; k < 2 * JB; ++k) {
      if constexpr (VK == V_FLAT) {
        st.v[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, (k * 64 + lane) * 16, 0, 0));
      } else if constexpr (VK == V_ROWS) {
        const int f = (k * 64 + lane) * 4, t = f / RB, j = n.jg + f % RB;
        st.v[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, j < r ? (uint32_t)((t * r + j) * 4) : OOB, 0, 0));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int f = (4 * k + e) * 64 + lane, t = f / RB, j = n.jg + f % RB;
          st.v[k][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rv, j < r ? (uint32_t)((t * r + j) * 4) : OOB, 0, 0));
        }
      }
    }
  };
  // A step's V from the order of its loads to an operand's: ranks 16 j + c of tokens 8 g .. 8 g + 7, times
  // their scales.  (A wave's own LDS: its accesses are in order.)
  auto turned = [&](const StepV &st, float (&v)[JB][8]) {
    if constexpr (VK != V_EACH) {
#pragma unroll
      for (int k = 0; k < 2 * JB; ++k) {
        const int f = (k * 64 + lane) * 4, q = (f >= 8 * row) + (f >= 16 * row) + (f >= 24 * row);
        *(f32x4 *)(turn + f + 16 * q) = st.v[k];  // (zeros behind the rows where r is less than the item's ranks)
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2 * JB; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int f = (4 * k + e) * 64 + lane;
          turn[f + 16 * (f / (8 * RB))] = st.v[k][e];
        }
    }
    if (X8) turn_s[lane & 31] = st.s;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = X8 ? turn_s[8 * g + i] : 1.0f;
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (past the last rank whatever follows: it comes into sums of ranks that are not stored)
        const float x = turn[(8 * g + i) * row + 16 * g + 16 * j + c];
        v[j][i] = X8 ? x * s[i] : x;
      }
  };
  f32x4 acc[Q][JB];
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int j = 0; j < JB; ++j) acc[q][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](const StepX &sx, const StepV &sv) {
    u32x4 vb[JB][3];
    float vs[JB][8];
    turned(sv, vs);
#pragma unroll
    for (int j = 0; j < JB; ++j) {
      float(&v)[8] = vs[j];
#pragma unroll
      for (int p = 0; p < 3; ++p) {  // each the next bits of what is left
#pragma unroll
        for (int d = 0; d < 4; ++d) vb[j][p][d] = pack_bf16x2(v[2 * d], v[2 * d + 1]);
        if (p == 2) break;
        float h[8];
        unpack_vec(BF16(), vb[j][p], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= h[i];
      }
    }
    // Four columns at a time: a product into a sum comes 4 JB products after the one before it.
#pragma unroll
    for (int q0 = 0; q0 < Q; q0 += 4) {
      u32x4 xt[4];  // columns of the 8 tokens
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (X8) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(sx.x[i][q0 / 4] >> (8 * q));
#pragma unroll
          for (int d = 0; d < 4; ++d) xt[q][d] = pack_bf16x2(f[2 * d], f[2 * d + 1]);
        } else {
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t lo = sx.x[2 * d][q >> 1], hi = sx.x[2 * d + 1][q >> 1];
            xt[q][d] = q & 1 ? (lo >> 16 | (hi & 0xffff0000u)) : ((lo & 0xffffu) | hi << 16);
          }
        }
      }
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int j = 0; j < JB; ++j) mma16(BF16(), acc[q0 + q][j], xt[q], vb[j][p]);
    }
  };
  {
    // Two steps' registers in turn, by name: a copy of one would wait for its loads.
    constexpr int STEP = X8P_NW * X8P_ROWS;
    StepX x[2];
    StepV v[2];
    int tb = n.t0 + wave * X8P_ROWS;
    auto load = [&](int at, int k) {
      load_x(at, x[k]);
      load_v(at, v[k]);
      __builtin_amdgcn_sched_barrier(0);  // (a wait for one step's loads is none for the next one's)
    };
    load(min(tb, n.t1), 0);
    for (; tb + 2 * STEP < n.t1; tb += 2 * STEP) {
      load(tb + STEP, 1);
      compute(x[0], v[0]);
      load(tb + 2 * STEP, 0);
      compute(x[1], v[1]);
    }
    if (tb < n.t1) {
      const bool two = tb + STEP < n.t1;
      if (two) load(tb + STEP, 1);
      compute(x[0], v[0]);
      if (two) compute(x[1], v[1]);
    }
  }
  // acc[q][j] element i: column (4 g + i) Q + q, rank 16 j + c.  The waves' tiles side by side in LDS,
  // columns of a rank together, and every thread the sums of some of its places: four columns of a
  // rank, in the order of the output, dA [rank][column], dB [column][rank].  (A pairwise
  // tree had seven barriers in the place of two.)
  __syncthreads();
  float *const tile = lds + wave * x8_tile(JB);
  constexpr int LD = COLS + 4;
#pragma unroll
  for (int j = 0; j < JB; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < Q; q += 4)
        *(f32x4 *)(tile + (16 * j + c) * LD + (4 * g + i) * Q + q) =
            f32x4{acc[q][j][i], acc[q + 1][j][i], acc[q + 2][j][i], acc[q + 3][j][i]};
  __syncthreads();
  constexpr int PER = (TILE / 4 + NT - 1) / NT;
  static_assert(TILE / 4 % NT == 0 || TILE / 4 < NT, "whole rounds of threads");
  const bool mine = (int)threadIdx.x < TILE / 4;
  auto place = [&](int y, int *l, int *k) {
    const int e = y * NT + (mine ? (int)threadIdx.x : 0);
    *l = 4 * (X8 ? e % (COLS / 4) : e / RB);
    *k = X8 ? e / (COLS / 4) : e % RB;
  };
  f32x4 sum[PER];
#pragma unroll
  for (int y = 0; y < PER; ++y) {
    int l, k;
    place(y, &l, &k);
    sum[y] = *(const f32x4 *)(lds + k * LD + l);
#pragma unroll
    for (int w = 1; w < X8P_NW; ++w) sum[y] += *(const f32x4 *)(lds + w * x8_tile(JB) + k * LD + l);
  }
  if (parts > 1) {
    // The parts of an item meet (meet.hpp): each leaves its sums in memory, and the one that comes last adds
    // them in ascending order.  Sums and flags are written and read at device scope.
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(a.slots + (int64_t)item * parts * X8P_SLOT(JB)), (short)0, parts * X8P_SLOT(JB) * 4, 0x00020000);
    const uint32_t off = mine ? threadIdx.x * 16 : OOB;  // (threads without a place store and load nothing)
#pragma unroll
    for (int y = 0; y < PER; ++y)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sum[y]), rs, off + (part * X8P_SLOT(JB) + y * NT * 4) * 4, 0, X8_SC1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int *all = (int *)lds;
    if (wave == 0) {
      MeetFlags flags{a.sync + (int64_t)item * parts, lane};
      const bool up = meet_arrive(flags, part, parts, a.gen);
      if (up) meet_lower(flags, parts);
      if (lane == 0) *all = up;
    }
    __syncthreads();
    if (!*all) return;  // (two may see all: they store the same sums)
    for (int p = 0; p < parts; p += 4) {  // four parts' loads at once
      f32x4 v[4][PER];
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < PER; ++y)
          v[x][y] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                  rs, off + (min(p + x, parts - 1) * X8P_SLOT(JB) + y * NT * 4) * 4, 0, X8_SC1));
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < PER; ++y)
          if (p + x < parts) sum[y] = p + x == 0 ? v[x][y] : sum[y] + v[x][y];
    }
  }
  if (!mine) return;
#pragma unroll
  for (int y = 0; y < PER; ++y) {
    int l, k;
    place(y, &l, &k);
    if (k >= r - n.jg || n.cb * COLS + l >= n.L) continue;  // (columns are in whole eights)
    if constexpr (X8) {
      *(f32x4 *)(n.out + (int64_t)(n.jg + k) * n.L + n.cb * COLS + l) = sum[y] * n.mult;
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) n.out[(int64_t)(n.cb * COLS + l + x) * r + n.jg + k] = sum[y][x] * n.mult;
    }
  }
}

// Workgroups: the items of dB, then those of dA, each in `parts` ranges of tokens.  An item has all r
// ranks (V_FLAT: V's rows of a step are one run of memory, read in whole vectors), or some
// of them (V_ROWS: vectors of each row, r a multiple of 4; V_EACH: a value each).
template <int JB, int VK>
__global__ __launch_bounds__(64 * X8P_NW) void x8_prod_kernel(X8Prod a, int parts, int chunk, int items_b) {
  constexpr int TILES = X8P_NW * x8_tile(JB), TURN = X8P_NW * x8_turn(JB);
  __shared__ __align__(16) float lds[TILES > TURN ? TILES : TURN];
  const int nz = (a.r + 16 * JB - 1) / (16 * JB);
  const int unit = blockIdx.x, part = unit % parts, item = unit / parts;
  const bool dB = item < items_b;
  const int own = dB ? item : item - items_b;
  X8Unit n;
  n.cb = own / nz;
  n.jg = own % nz * 16 * JB;
  n.t0 = part * chunk;
  n.t1 = min(a.T, n.t0 + chunk);
  n.X = dB ? a.dy : (const void *)a.x.codes;
  n.scale = a.x.scale;
  n.V = dB ? a.u : a.du;
  n.L = dB ? a.N : a.K;
  n.ng = (a.K + ACT8_G - 1) / ACT8_G;
  n.mult = dB ? a.scale : a.du_scale;
  n.out = dB ? a.dB : a.dA;
  if (dB) x8_item<JB, VK, false>(a, n, item, part, parts, lds);
  else x8_item<JB, VK, true>(a, n, item, part, parts, lds);
}

// du and u as one sum each, in place, of the partial sums that they came in: ascending, so the product
// kernel's loads stay free of sums, which would wait for them.
__global__ __launch_bounds__(256) void x8_join_kernel(float *du, int du_parts, float *u, int u_parts, int64_t n) {
  float *const x = blockIdx.y == 0 ? du : u;
  const int parts = blockIdx.y == 0 ? du_parts : u_parts;
  if (parts == 1) return;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float v[MAX_SPLIT];  // all parts' loads at once
#pragma unroll
    for (int p = 0; p < MAX_SPLIT; ++p) v[p] = x[min(p, parts - 1) * n + i];
    float s = v[0];
#pragma unroll
    for (int p = 1; p < MAX_SPLIT; ++p) s = p < parts ? s + v[p] : s;
    x[i] = s;
  }
}

static int x8_jb(int64_t r) { return r <= 16 ? 1 : 2; }
static int64_t x8_items(int64_t L, int64_t cols, int64_t r) {
  return (L + cols - 1) / cols * ((r + 16 * x8_jb(r) - 1) / (16 * x8_jb(r)));
}

// Ranges of tokens: those that take the least time, in units of a step of a workgroup's waves (256
// tokens, 1.4 us with 16 ranks and 2.6 with 32).  A workgroup has a CU for itself, and spends about as much as
// X8_FIXED steps on its first loads, the sums of its waves and the stores (3 us), X8_MEET more on a
// meeting (2.7 us).
constexpr int X8_FIXED = 2, X8_MEET = 2;
X8Plan x8_plan(int64_t T, int64_t K, int64_t N, int64_t r) {
  constexpr int64_t STEP = X8P_NW * X8P_ROWS;
  const int64_t items = x8_items(K, ACT8_G, r) + x8_items(N, ACT8_G / 2, r), steps = (T + STEP - 1) / STEP;
  int64_t best = 0, parts = 1, per = steps;
  for (int64_t p = 1; p <= std::min<int64_t>(steps, 16); ++p) {
    const int64_t n = (steps + p - 1) / p;  // steps of a range
    if ((steps + n - 1) / n != p) continue;
    const int64_t t = (items * p + 255) / 256 * (n + X8_FIXED + (p > 1 ? X8_MEET : 0));
    if (p == 1 || t < best) best = t, parts = p, per = n;
  }
  X8Plan q{(int)parts, (int)(per * STEP), 0, 0};
  if (parts > 1) {
    q.sync_bytes = (size_t)(items * parts) * sizeof(meet_word);
    q.slot_bytes = (size_t)(items * parts) * X8P_SLOT(x8_jb(r)) * 4;
  }
  return q;
}

hipError_t launch_x8_prod(const X8Prod &a, hipStream_t st) {
  const X8Plan p = x8_plan(a.T, a.K, a.N, a.r);
  const int items_b = (int)x8_items(a.N, ACT8_G / 2, a.r), items = items_b + (int)x8_items(a.K, ACT8_G, a.r);
  const dim3 grid(items * p.parts), block(64 * X8P_NW);
  if (a.du_parts > MAX_SPLIT || a.u_parts > MAX_SPLIT) return hipErrorInvalidValue;
  if (p.parts > 64 || (p.parts > 1 && (!a.sync || !a.slots || a.gen == 0))) return hipErrorInvalidValue;
  if (a.du_parts > 1 || a.u_parts > 1) {
    const int64_t n = (int64_t)a.T * a.r;
    const dim3 g((unsigned)std::min<int64_t>((n + 255) / 256, 1024), a.u_parts > 1 ? 2 : 1);
    hipLaunchKernelGGL(x8_join_kernel, g, dim3(256), 0, st, a.du, a.du_parts, a.u_parts > 1 ? const_cast<float *>(a.u) : nullptr,
                       a.u_parts, n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
#define PROD(JB, VK) hipLaunchKernelGGL((x8_prod_kernel<JB, VK>), grid, block, 0, st, a, p.parts, p.chunk, items_b)
  if (a.r <= 16) PROD(1, V_FLAT);
  else if (a.r <= 32) PROD(2, V_FLAT);
  else if (a.r % 4 == 0) PROD(2, V_ROWS);
  else PROD(2, V_EACH);
#undef PROD
  return hipGetLastError();
}

}  // namespace lora

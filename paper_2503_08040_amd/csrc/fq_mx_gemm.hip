// Products of microscaled 4-bit matrices: C[i, j] = sum over the groups g of 2^(sa + sb) * (codes of a . codes of b).
//
// The matrix instruction takes the scales itself: one 16 x 16 x 128 step has, per lane, 32 codes of a row or column
// and the byte of their scale, and adds the exact products in binary32.  So a product here is a plain matrix loop on
// 17/32 byte an element.  The storage order (fq.h) makes 1 KiB of codes one operand, lane by lane, and a dword of
// scales the four operands of 64 rows, told apart by the instruction's byte select.
#include <type_traits>

#include "fq_device.h"
#include "fq_kernels.h"

namespace fq {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr int kOperand = 1024;    // 16 rows x 128
constexpr int kScaleBlock = 256;  // scales of 64 rows x 128
constexpr int kFp4 = 4;           // the instruction's format code of E2M1

// acc += a b with byte kSa of sa, kSb of sb: rows of `a` go to registers, rows of `b` to lanes, so with C's columns
// as `a` a lane has 4 consecutive columns of one row of C.
template <int kSa, int kSb>
__device__ __forceinline__ v4f mfma(const v4i& a, const v4i& b, const v4f& acc, int sa, int sb) {
  const v8i wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, acc, kFp4, kFp4, kSa, sa, kSb, sb);
}

__device__ __forceinline__ v4f mfma_select(const v4i& a, const v4i& b, const v4f& acc, int ia, int sa, int ib, int sb) {
  switch (4 * (ia & 3) + (ib & 3)) {
#define FQ_CASE(x, y) case 4 * x + y: return mfma<x, y>(a, b, acc, sa, sb);
    FQ_CASE(0, 0) FQ_CASE(0, 1) FQ_CASE(0, 2) FQ_CASE(0, 3) FQ_CASE(1, 0) FQ_CASE(1, 1) FQ_CASE(1, 2) FQ_CASE(1, 3)
    FQ_CASE(2, 0) FQ_CASE(2, 1) FQ_CASE(2, 2) FQ_CASE(2, 3) FQ_CASE(3, 0) FQ_CASE(3, 1) FQ_CASE(3, 2)
    default: return mfma<3, 3>(a, b, acc, sa, sb);
#undef FQ_CASE
  }
}

// 4 consecutive values of a row of C
__device__ __forceinline__ void store4(const MxGemmParams& p, const v4f& v, int row, int col) {
  if (row >= p.M || col >= p.N) return;
  const int64_t o = (int64_t)row * p.ldc + col;
  const bool whole = p.vec_ok && col + 4 <= p.N;
  if (p.out_bf16) {
    uint16_t* dst = static_cast<uint16_t*>(p.c) + o;
    const v2f lo = {v[0], v[1]}, hi = {v[2], v[3]};
    const v2u b = {__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, v2bf)),
                   __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, v2bf))};
    if (whole) {
      *reinterpret_cast<v2u*>(dst) = b;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < p.N) dst[e] = (uint16_t)(b[e >> 1] >> (16 * (e & 1)));
    }
  } else {
    float* dst = static_cast<float*>(p.c) + o;
    if (whole) {
      *reinterpret_cast<v4f*>(dst) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < p.N) dst[e] = v[e];
    }
  }
}

// ---- small outputs: a workgroup per tile of kM x kN strips, the contraction split over its kW wavefronts -----------
// Operands go straight from memory to registers, kU blocks of 128 at a time; the wavefronts' sums are joined through
// LDS in a fixed order.
template <int kM, int kN, int kW, int kU>
__global__ __launch_bounds__(64 * kW) void mx_gemm_split_kernel(MxGemmParams p, int tiles_j) {
  static_assert(4 % kM == 0 && 4 % kN == 0, "the strips of a tile share their scale dwords");
  __shared__ v4f part[kW][kM * kN][64];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ti = blockIdx.x / tiles_j, tj = blockIdx.x % tiles_j;
  const int i0 = ti * kM, j0 = tj * kN, nkb = p.a.nkb;
  // strips behind the last one repeat it: their results are not stored
  const uint8_t *ap[kM], *bp[kN];
#pragma unroll
  for (int i = 0; i < kM; ++i) ap[i] = p.a.codes + (int64_t)min(i0 + i, p.a.strips - 1) * nkb * kOperand + lane * 16;
#pragma unroll
  for (int j = 0; j < kN; ++j) bp[j] = p.b.codes + (int64_t)min(j0 + j, p.b.strips - 1) * nkb * kOperand + lane * 16;
  const uint8_t* const as = p.a.scales + (int64_t)(i0 >> 2) * nkb * kScaleBlock + lane * 4;
  const uint8_t* const bs = p.b.scales + (int64_t)(j0 >> 2) * nkb * kScaleBlock + lane * 4;
  const int ash = 8 * (i0 & 3), bsh = 8 * (j0 & 3);
  v4f acc[kM][kN];
#pragma unroll
  for (int i = 0; i < kM; ++i)
#pragma unroll
    for (int j = 0; j < kN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  auto blocks = [&](int kb, auto n_c) {
    constexpr int n = decltype(n_c)::value;
    v4i a[n][kM], b[n][kN];
    uint32_t sa[n], sb[n];
#pragma unroll
    for (int u = 0; u < n; ++u) {
      const int64_t k = kb + u * kW;
#pragma unroll
      for (int i = 0; i < kM; ++i) a[u][i] = *reinterpret_cast<const v4i*>(ap[i] + k * kOperand);
#pragma unroll
      for (int j = 0; j < kN; ++j) b[u][j] = *reinterpret_cast<const v4i*>(bp[j] + k * kOperand);
      sa[u] = *reinterpret_cast<const uint32_t*>(as + k * kScaleBlock) >> ash;
      sb[u] = *reinterpret_cast<const uint32_t*>(bs + k * kScaleBlock) >> bsh;
    }
#pragma unroll
    for (int u = 0; u < n; ++u)
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int j = 0; j < kN; ++j) acc[i][j] = mfma_select(b[u][j], a[u][i], acc[i][j], j, (int)sb[u], i, (int)sa[u]);
  };
  int kb = w;
  for (; kb + (kU - 1) * kW < nkb; kb += kU * kW) blocks(kb, std::integral_constant<int, kU>{});
  for (; kb < nkb; kb += kW) blocks(kb, std::integral_constant<int, 1>{});

#pragma unroll
  for (int i = 0; i < kM; ++i)
#pragma unroll
    for (int j = 0; j < kN; ++j) part[w][i * kN + j][lane] = acc[i][j];
  __syncthreads();
  for (int s = w; s < kM * kN; s += kW) {
    v4f v = part[0][s][lane];
#pragma unroll
    for (int k = 1; k < kW; ++k) v += part[k][s][lane];
    store4(p, v, (i0 + s / kN) * 16 + (lane & 15), (j0 + s % kN) * 16 + 4 * (lane >> 4));
  }
}

template <int kM, int kN, int kW, int kU>
void split(const MxGemmParams& p, hipStream_t st) {
  const int ti = (p.a.strips + kM - 1) / kM, tj = (p.b.strips + kN - 1) / kN;
  hipLaunchKernelGGL((mx_gemm_split_kernel<kM, kN, kW, kU>), dim3(ti * tj), dim3(64 * kW), 0, st, p, tj);
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmParams& p, hipStream_t st) {
  split<4, 4, 4, 2>(p, st);
  return hipGetLastError();
}

}  // namespace fq

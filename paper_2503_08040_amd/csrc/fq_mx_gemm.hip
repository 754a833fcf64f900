// Products of microscaled 4-bit matrices: C[i, j] = sum over the groups g of 2^(sa + sb) * (codes of a . codes of b).
//
// The matrix instruction takes the scales itself: one 16 x 16 x 128 step has, per lane, 32 codes of a row or column
// and the byte of their scale, and adds the exact products in binary32.  So a product here is a plain matrix loop on
// 17/32 byte an element.  The storage order (fq.h) makes 1 KiB of codes one operand, lane by lane, and a dword of
// scales the four operands of 64 rows, told apart by the instruction's byte select.
//
// Measured, bf16 outputs: 8192 x 8192 over 8192 224 to 237 us by card (4.6 to 4.9 PFLOP/s), 4096 x 4096 over 11008 79 us
// (4.7), 4096 x 11008 over 4096 89 us (4.1, the third round of tiles is two thirds full), 2048 x 2048 over 2048 9.0 us,
// 512 x 512 over 512 2.8 us (a launch is about 2.5), one token 4096 -> 11008 6.2 us (3.9 TB/s of W).  This instruction alone does
// 7.3 PFLOP/s on random codes and 9.8 on zeros: power bounds the large ones.  A block of a 256 x 256 tile takes 0.54 us
// on 64 compute units (1308 cycles at 2.4 GHz; its products are 1024) and 0.83 us on all 256.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fq_device.h"
#include "fq_gemm_unit.h"
#include "fq_kernels.h"
#include "fq_mx_device.h"

namespace fq {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));

constexpr int kMaxDevices = 64;   // per-device host-side caches
constexpr int kMaxBlocks = 1 << 21;   // blocks of a contraction whose codes' offsets fit 31 bits
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

__device__ __forceinline__ v2u pack_bf16(const v4f& v) {
  const v2f lo = {v[0], v[1]}, hi = {v[2], v[3]};
  return v2u{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, v2bf)),
             __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, v2bf))};
}

// 4 consecutive values of a row of C
__device__ __forceinline__ void store4(const MxGemmParams& p, const v4f& v, int row, int col) {
  if (row >= p.M || col >= p.N) return;
  const int64_t o = (int64_t)row * p.ldc + col;
  const bool whole = col + 4 <= p.N;
  if (p.out_bf16) {
    uint16_t* dst = static_cast<uint16_t*>(p.c) + o;
    const v2u b = pack_bf16(v);
    if (whole) {
      *reinterpret_cast<v2u_at2*>(dst) = b;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < p.N) dst[e] = (uint16_t)(b[e >> 1] >> (16 * (e & 1)));
    }
  } else {
    float* dst = static_cast<float*>(p.c) + o;
    if (whole) {
      *reinterpret_cast<v4f_at4*>(dst) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < p.N) dst[e] = v[e];
    }
  }
}

// 32 values of a bf16 row, from column `col` on, as packed pairs; of a row that is not there zeros.  A group that ends
// behind the row's end is read as its last 32 values, so that nothing waits here; drop_read puts it right when it is used.
__device__ __forceinline__ void load_group(const MxGemmParams& p, int row, int col, v4u (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = v4u{0u, 0u, 0u, 0u};
  if (row >= p.M) return;
  const uint16_t* const src = p.x + row * p.ld;
  if (p.K >= 32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const v4u_at2*>(src + min(col, p.K - 32) + 8 * i);
  } else if (col == 0) {
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i >> 3][(i >> 1) & 3] |= (i < p.K ? (uint32_t)src[min(i, p.K - 1)] : 0u) << (16 * (i & 1));
  }
}

// Takes away the first n values of 32 that a group does not have.
__device__ __forceinline__ void drop_read(int n, v4u (&x)[4]) {
  const v4u zero = {0u, 0u, 0u, 0u};
  if (n >= 32) x[0] = x[1] = x[2] = x[3] = zero;
  if (n & 16) {
    x[0] = x[2];
    x[1] = x[3];
    x[2] = x[3] = zero;
  }
  if (n & 8) {
    x[0] = x[1];
    x[1] = x[2];
    x[2] = x[3];
    x[3] = zero;
  }
  // up to 7 values more: 2 dwords, 1 dword, half a dword
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const v4u next = i < 3 ? x[(i + 1) & 3] : zero;
    const uint32_t w[8] = {x[i][0], x[i][1], x[i][2], x[i][3], next[0], next[1], next[2], next[3]};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t a = n & 4 ? w[d + 2] : w[d], b = n & 4 ? w[d + 3] : w[d + 1], c = n & 4 ? w[d + 4] : w[d + 2];
      const uint32_t lo = n & 2 ? b : a, hi = n & 2 ? c : b;
      x[i][d] = n & 1 ? lo >> 16 | hi << 16 : lo;
    }
  }
}

// Codes and scale byte of a group, the same as mx_quantize_kernel's.
__device__ __forceinline__ uint32_t quantize_group(const v4u (&x)[4], int bias, v4i& codes) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = pk_max(m, x[i >> 2][i & 3] & 0x7FFF7FFFu);
  const uint32_t byte = scale_byte(max(m >> 16, m & 0xFFFFu), bias);
  const float s = scale_value(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c = 0;
#pragma unroll
    for (int d = 0; d < 4; ++d) c = cvt_fp4(c, x[i][d], s, d);
    codes[i] = byte == 255u ? 0 : (int)c;
  }
  return byte;
}

// ---- small outputs: a workgroup per tile of kM x kN strips, the contraction split over its kW wavefronts -----------
// Operands go straight from memory to registers, kU blocks of 128 at a time; the wavefronts' sums are joined through
// LDS in a fixed order.  kFused: A is bf16 and every workgroup quantizes the rows of its tile as it goes.  Such products
// are latency and, for few rows, the read of B: 33 x 4096 over 11008 7.9 us (3.0 TB/s), 777 x 2201 over 1544 7.3 us.
// Tiles of 64 x 64 gain nothing from 8 wavefronts over 4.
template <int kM, int kN, int kW, int kU, bool kFused>
__global__ __launch_bounds__(64 * kW) void mx_gemm_split_kernel(MxGemmParams p, int tiles_i, int tiles) {
  static_assert(4 % kM == 0 && 4 % kN == 0, "the strips of a tile share their scale dwords");
  __shared__ v4f part[kW][kM * kN][64];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // An XCD takes a run of tiles down the columns, so that its L2 holds few columns' B (777 x 2201 over 1544 in 13 x 35
  // tiles 8.65 -> 7.3 us, 131 x 1544 over 2200 in 5 x 49 4.5 -> 3.4).
  const unsigned place = xcd_run(blockIdx.x, tiles);
  const int tj = place / (unsigned)tiles_i, ti = place % (unsigned)tiles_i;
  const int i0 = ti * kM, j0 = tj * kN, nkb = p.b.nkb;
  // strips behind the last one repeat it: their results are not stored
  const uint8_t *ap[kM], *bp[kN];
#pragma unroll
  for (int i = 0; i < kM; ++i)
    ap[i] = kFused ? nullptr : p.a.codes + (int64_t)min(i0 + i, p.a.strips - 1) * nkb * kOperand + lane * 16;
#pragma unroll
  for (int j = 0; j < kN; ++j) bp[j] = p.b.codes + (int64_t)min(j0 + j, p.b.strips - 1) * nkb * kOperand + lane * 16;
  const uint8_t* const as = kFused ? nullptr : p.a.scales + (int64_t)(i0 >> 2) * nkb * kScaleBlock + lane * 4;
  const uint8_t* const bs = p.b.scales + (int64_t)(j0 >> 2) * nkb * kScaleBlock + lane * 4;
  const int ash = 8 * (i0 & 3), bsh = 8 * (j0 & 3);
  v4f acc[kM][kN];
#pragma unroll
  for (int i = 0; i < kM; ++i)
#pragma unroll
    for (int j = 0; j < kN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  // kU blocks' operands are requested while those of the kU before are multiplied
  struct Set {
    v4i a[kU][kM], b[kU][kN];
    v4u x[kU][kM][4];
    uint32_t sa[kU], sb[kU];
  };
  auto request = [&](Set& s, int kb) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int k = kb + u * kW;
      if (k >= nkb) break;
#pragma unroll
      for (int j = 0; j < kN; ++j) s.b[u][j] = *reinterpret_cast<const v4i*>(bp[j] + (int64_t)k * kOperand);
      s.sb[u] = *reinterpret_cast<const uint32_t*>(bs + (int64_t)k * kScaleBlock) >> bsh;
      if constexpr (kFused) {
#pragma unroll
        for (int i = 0; i < kM; ++i)
          load_group(p, (i0 + i) * 16 + (lane & 15), k * 128 + 32 * (lane >> 4), s.x[u][i]);
      } else {
#pragma unroll
        for (int i = 0; i < kM; ++i) s.a[u][i] = *reinterpret_cast<const v4i*>(ap[i] + (int64_t)k * kOperand);
        s.sa[u] = *reinterpret_cast<const uint32_t*>(as + (int64_t)k * kScaleBlock) >> ash;
      }
    }
  };
  auto multiply = [&](Set& s, int kb) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (kb + u * kW >= nkb) break;
      if constexpr (kFused) {
        s.sa[u] = 0;
        const int missing = (kb + u * kW) * 128 + 32 * (lane >> 4) - (p.K - 32);
#pragma unroll
        for (int i = 0; i < kM; ++i) {
          if (missing > 0 && p.K >= 32) drop_read(missing, s.x[u][i]);
          s.sa[u] |= quantize_group(s.x[u][i], p.bias, s.a[u][i]) << (8 * i);
        }
      }
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int j = 0; j < kN; ++j)
          acc[i][j] = mfma_select(s.b[u][j], s.a[u][i], acc[i][j], j, (int)s.sb[u], i, (int)s.sa[u]);
    }
  };
  Set even, odd;
  request(even, w);
  for (int kb = w; kb < nkb; kb += 2 * kU * kW) {
    request(odd, kb + kU * kW);
    multiply(even, kb);
    request(even, kb + 2 * kU * kW);
    multiply(odd, kb + kU * kW);
  }

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

// The same instruction in place and in order.  With half of the registers as accumulators the compiler's allocation of its
// own form moves them about in the loop.  What follows a matrix instruction and reads acc other than as another's
// accumulator has to wait by itself.
template <int kSa, int kSb>
__device__ __forceinline__ void mfma_in_place(v4f& acc, const v4i& a, const v4i& b, int sa, int sb) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:4 blgp:4"
               : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(kSa & 1), "n"(kSb & 1), "n"(kSa >> 1), "n"(kSb >> 1));
}

__device__ __forceinline__ void mfma_in_place_select(v4f& acc, const v4i& a, const v4i& b, int ia, int sa, int ib, int sb) {
  switch (4 * (ia & 3) + (ib & 3)) {
#define FQ_CASE(x, y) case 4 * x + y: return mfma_in_place<x, y>(acc, a, b, sa, sb);
    FQ_CASE(0, 0) FQ_CASE(0, 1) FQ_CASE(0, 2) FQ_CASE(0, 3) FQ_CASE(1, 0) FQ_CASE(1, 1) FQ_CASE(1, 2) FQ_CASE(1, 3)
    FQ_CASE(2, 0) FQ_CASE(2, 1) FQ_CASE(2, 2) FQ_CASE(2, 3) FQ_CASE(3, 0) FQ_CASE(3, 1) FQ_CASE(3, 2)
    default: return mfma_in_place<3, 3>(acc, a, b, sa, sb);
#undef FQ_CASE
  }
}

// ---- large outputs: 2 x kWC wavefronts of 16 kR x 16 kC, operands through LDS ----------------------------------------
// A stage is one block of 128 of the contraction: codes of the tile's strips, then their scales, brought by direct
// global -> LDS loads.  There are kStages of them: while a block is multiplied out of registers, the next one's operands
// are fetched from LDS and up to three more blocks are under way.  A workgroup walks over several tiles and the ring of
// stages runs on from one to the next, so that only the first tile waits for its operands.
// 128 x 256 takes 8 wavefronts of 64 x 64, 256 x 256 8 of 128 x 64: 4 of 128 x 128 read a third less from LDS but leave one
// on a SIMD, 1408 cycles a block instead of 1306, and twice the time for C (2 to 3 % slower).  128 x 128 takes two
// workgroups of 4; a ring of 8 stages was slower.
template <int kR_, int kC_, int kWC_, int kOcc_, int kStages_>
struct LdsGeo {
  static constexpr int kR = kR_, kC = kC_, kWC = kWC_, kOcc = kOcc_;        // strips of a wavefront; workgroups of a CU
  static constexpr int kWaves = 2 * kWC, kThreads = 64 * kWaves;
  static constexpr int kStages = kStages_;
  static constexpr int kStripsI = 2 * kR, kStripsJ = kC * kWC, kStrips = kStripsI + kStripsJ;      // of the tile
  static constexpr int kQuadsI = kStripsI / 4, kQuads = kStrips / 4;        // 64 rows' scales
  static constexpr int kLoads = kStrips / kWaves;                           // strips that a wavefront loads, and one of the quads
  static constexpr int kCodes = kStrips * kOperand;                         // bytes of a stage
  static constexpr int kStage = kCodes + kQuads * kScaleBlock;
  static constexpr int kPatchRow = 128, kPatch = 16 * kPatchRow;            // a wavefront's patch for C
  static constexpr int kLds = kStages * kStage + kWaves * kPatch;
  static_assert(kR % 4 == 0 && kC % 4 == 0 && kLoads * kWaves == kStrips && kQuads <= kWaves && kOcc * kLds <= 160 * 1024);
};

// 16 rows of kChunks 16-byte chunks from a patch in LDS to C at (row0, col0); chunk c of row r lies at c ^ r.
template <int kChunks, class T>
__device__ __forceinline__ void store_patch(const MxGemmParams& p, const int8_t* patch, int row0, int col0, int lane) {
  constexpr int kPer = 16 / (int)sizeof(T), kStep = 64 / kChunks;      // elements of a chunk, rows of a store
  const int c = lane % kChunks, col = col0 + c * kPer, r0 = lane / kChunks;
  T* const dst = static_cast<T*>(p.c) + (int64_t)(row0 + r0) * p.ldc + col;
  auto from = [&](int i) { return patch + (r0 + i * kStep) * kChunks * 16 + ((c ^ (r0 + i * kStep)) & (kChunks - 1)) * 16; };
  if (row0 + 16 <= p.M && col0 + kChunks * kPer <= p.N) {
#pragma unroll
    for (int i = 0; i < 16 / kStep; ++i)
      *reinterpret_cast<v4u_at2*>(dst + i * kStep * p.ldc) = *reinterpret_cast<const v4u*>(from(i));
  } else {
    const int valid = min(p.N - col, kPer);
#pragma unroll 1
    for (int i = 0; i < 16 / kStep; ++i) {
      if (row0 + r0 + i * kStep >= p.M) break;
      const T* const v = reinterpret_cast<const T*>(from(i));
      if (valid == kPer) {
        *reinterpret_cast<v4u_at2*>(dst + i * kStep * p.ldc) = *reinterpret_cast<const v4u*>(v);
      } else {
#pragma unroll 1
        for (int e = 0; e < valid; ++e) dst[i * kStep * p.ldc + e] = v[e];
      }
    }
  }
}

template <class G, class T>
__global__ __launch_bounds__(G::kThreads, G::kOcc * G::kWaves / 4) void mx_gemm_lds_kernel(MxGemmParams p, int tiles_i, int tiles_j) {
  extern __shared__ __attribute__((aligned(1024))) int8_t lds[];
  constexpr int kR = G::kR, kC = G::kC, kLoads = G::kLoads, kAllLoads = kLoads + 1;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / G::kWC, wc = w % G::kWC;
  const int nkb = p.a.nkb, tiles = tiles_i * tiles_j;
  const uint32_t lds0 = lds_address(lds);
  // First strips of tile b: groups of 4 tile columns, walked row by row.  Everything up to the first loads is short, as a
  // small product waits for the fetch of its code.
  auto tile_of = [&](int b, int& i0, int& j0) {
    const unsigned place = xcd_run(b, tiles), group = 4u * tiles_i, g = place / group, within = place - g * group;
    const unsigned across = min(4u, tiles_j - 4 * g);
    const unsigned by = across == 4 ? 0x40000000u : across == 3 ? 0x55555556u : 0x80000000u;
    const unsigned ti = across == 1 ? within : __umulhi(within, by);      // within / across, exact below 2^30
    i0 = ti * G::kStripsI;
    j0 = (4 * g + within - ti * across) * G::kStripsJ;
  };

  // The loader's side.  What this wavefront loads of a tile: kLoads of the strips, A's before B's, and 64 rows' scales;
  // behind the end the last ones again.
  const unsigned row_codes = (unsigned)nkb * kOperand, row_scales = (unsigned)nkb * kScaleBlock;      // nkb < kMaxBlocks
  const int quad_of = min(w, G::kQuads - 1);
  const int8_t *strip[kLoads], *quad;
  auto aim = [&](int b) {
    int i0, j0;
    tile_of(b, i0, j0);
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int s = w * kLoads + n;
      const bool of_b = G::kStripsI % kLoads == 0 ? w >= G::kStripsI / kLoads : s >= G::kStripsI;
      const MxSide& side = of_b ? p.b : p.a;
      strip[n] = reinterpret_cast<const int8_t*>(side.codes) +
                 (uint64_t)(unsigned)min(s + (of_b ? j0 - G::kStripsI : i0), side.strips - 1) * row_codes;
    }
    const bool of_b = quad_of >= G::kQuadsI;
    const MxSide& side = of_b ? p.b : p.a;
    quad = reinterpret_cast<const int8_t*>(side.scales) +
           (uint64_t)(unsigned)min(quad_of + ((of_b ? j0 - G::kStripsI : i0) >> 2), side.quads - 1) * row_scales;
  };
  int aimed = blockIdx.x, ahead = 0;      // tile and block to load next
  unsigned code_off = lane * 16u, scale_off = lane * 4u;
  uint32_t stage_at = lds0;
  aim(aimed);
  auto load = [&](int n) {
    if (n < kLoads) load_lds_at(strip[n], code_off, stage_at + (w * kLoads + n) * kOperand);
    else load_lds_dword(quad, scale_off, stage_at + G::kCodes + quad_of * kScaleBlock);
  };
  // the block behind: of the next tile, or behind the last tile the last block again, into a stage that nobody reads
  auto advance = [&]() {
    stage_at = stage_at == lds0 + (G::kStages - 1) * G::kStage ? lds0 : stage_at + G::kStage;
    code_off += kOperand;
    scale_off += kScaleBlock;
    if (__builtin_expect(++ahead < nkb, 1)) return;
    if (aimed + (int)gridDim.x < tiles) {
      aimed += gridDim.x;
      aim(aimed);
      code_off -= row_codes;
      scale_off -= row_scales;
      ahead = 0;
    } else {
      --ahead;
      code_off -= kOperand;
      scale_off -= kScaleBlock;
    }
  };
  // until at most n stages are under way; lgkmcnt(0)
  auto wait_stages = [](auto n_c) {
    constexpr int n = decltype(n_c)::value * kAllLoads;
    static_assert(n < 64);
    __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 0x0070);
  };

  // The multiplier's side.
  v4f acc[kR][kC];
  struct Operands {
    v4i a[kR], b[kC];
    int sa[kR / 4], sb[kC / 4];
  } f[2];
  const int aoff = wr * kR * kOperand + lane * 16, boff = (G::kStripsI + wc * kC) * kOperand + lane * 16;
  const int saoff = G::kCodes + wr * (kR / 4) * kScaleBlock + lane * 4;
  const int sboff = G::kCodes + (G::kQuadsI + wc * (kC / 4)) * kScaleBlock + lane * 4;
  const int8_t* rd = lds;      // stage of the operands to fetch
  // A block's fetches and a stage's loads, spread over the products of a block.  With few of them the loads go first, as
  // early as their stage is free: 2048 x 2048 over 4096 in tiles of 128 x 128 14.0 -> 13.2 us (tiles of 256 x 256: no
  // order was measurably better).
  constexpr int kFetch = kR + kC + kR / 4 + kC / 4, kProducts = kR * kC;
  constexpr bool kLoadsFirst = kProducts <= 16;
  constexpr int kFetchStep = kProducts >= 2 * kFetch ? 2 : 1, kLoadStep = kLoadsFirst ? 1 : kProducts / kAllLoads;
  constexpr int kFetch0 = kLoadsFirst ? kAllLoads : 0;
  static_assert(kFetch0 + kFetch * kFetchStep <= kProducts && kLoadStep > 0);
  auto fetch = [&](Operands& o, int n) {
    if (n < kC) o.b[n] = *reinterpret_cast<const v4i*>(rd + boff + n * kOperand);
    else if (n < kC + kR) o.a[n - kC] = *reinterpret_cast<const v4i*>(rd + aoff + (n - kC) * kOperand);
    else if (n < kC + kR + kC / 4) o.sb[n - kC - kR] = *reinterpret_cast<const int*>(rd + sboff + (n - kC - kR) * kScaleBlock);
    else if (n < kFetch)
      o.sa[n - kC - kR - kC / 4] = *reinterpret_cast<const int*>(rd + saoff + (n - kC - kR - kC / 4) * kScaleBlock);
  };
  auto next_stage = [&]() { rd = rd == lds + (G::kStages - 1) * G::kStage ? lds : rd + G::kStage; };
  // a block out of `o`, the next one into `other`
  auto block = [&](const Operands& o, Operands& other) {
    // the next block is there, and everybody has this one's operands in registers, so its stage is free
    wait_stages(std::integral_constant<int, G::kStages - 2>{});
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        // every other row backwards, so that successive products share an operand: less power, 8192 x 8192 over 8192
        // 228 -> 224.5 us, 4096 x 11008 over 4096 90 -> 88.5
        const int n = i * kC + j, at = i & 1 ? kC - 1 - j : j;
        mfma_in_place_select(acc[i][at], o.b[at], o.a[i], at, o.sb[at >> 2], i, o.sa[i >> 2]);
        if (n >= kFetch0 && (n - kFetch0) % kFetchStep == 0) fetch(other, (n - kFetch0) / kFetchStep);
        if (n % kLoadStep == 0 && n / kLoadStep < kAllLoads) load(n / kLoadStep);
        __builtin_amdgcn_sched_barrier(0);
      }
    advance();
    next_stage();
  };

#pragma unroll 1
  for (int k = 0; k < G::kStages; ++k) {
#pragma unroll
    for (int n = 0; n < kAllLoads; ++n) load(n);
    advance();
  }
  wait_stages(std::integral_constant<int, G::kStages - 1>{});
  asm volatile("s_barrier" ::: "memory");
#pragma unroll
  for (int n = 0; n < kFetch; ++n) fetch(f[0], n);
  next_stage();

#pragma unroll 1
  for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int j = 0; j < kC; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    int left = nkb;
#pragma unroll 1
    for (; left > 1; left -= 2) {
      block(f[0], f[1]);
      block(f[1], f[0]);
    }
    if (left) {
      block(f[0], f[1]);
      const Operands o = f[0];
      f[0] = f[1];
      f[1] = o;
    }
    // 32 wait states for the last products, more than any matrix instruction of 4 passes needs before its result is read
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    int i0, j0;
    tile_of(t, i0, j0);
    // C leaves strip by strip through a patch of the wavefront's own, so that rows are stored in pieces of kPatchRow bytes.
    constexpr int kChunks = G::kPatchRow / 16, kPass = G::kPatchRow / (16 * (int)sizeof(T));
    int8_t* const patch = lds + G::kStages * G::kStage + w * G::kPatch;
    const int r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int jj = 0; jj < kC; jj += kPass) {
#pragma unroll
        for (int j = 0; j < kPass; ++j) {
          asm volatile("" : "+a"(acc[i][jj + j]));      // read here and not before
          const int at = (16 * j + 4 * q) * (int)sizeof(T);
          int8_t* const dst = patch + r * G::kPatchRow + (((at >> 4) ^ r) & (kChunks - 1)) * 16 + (at & 15);
          if constexpr (sizeof(T) == 2) *reinterpret_cast<v2u*>(dst) = pack_bf16(acc[i][jj + j]);
          else *reinterpret_cast<v4f*>(dst) = acc[i][jj + j];
        }
        // lanes read what others of the wavefront wrote: LDS serves a wavefront in order, the compiler is told to
        asm volatile("" ::: "memory");
        store_patch<kChunks, T>(p, patch, (i0 + wr * kR + i) * 16, (j0 + wc * kC + jj) * 16, lane);
        asm volatile("" ::: "memory");
      }
  }
  wait_stages(std::integral_constant<int, 0>{});      // nothing may be under way into LDS when the workgroup ends
}

template <class G, class T>
hipError_t through_lds(const MxGemmParams& p, int cus, hipStream_t st) {
  // the kernel needs more dynamic LDS than the default limit: raise it once per device
  static std::atomic<bool> attr_set[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(mx_gemm_lds_kernel<G, T>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds);
    if (e != hipSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  const int ti = (p.a.strips + G::kStripsI - 1) / G::kStripsI, tj = (p.b.strips + G::kStripsJ - 1) / G::kStripsJ;
  const int grid = std::min(ti * tj, G::kOcc * cus);
  hipLaunchKernelGGL((mx_gemm_lds_kernel<G, T>), dim3(grid), dim3(G::kThreads), G::kLds, st, p, ti, tj);
  return hipGetLastError();
}

template <class G>
hipError_t through_lds(const MxGemmParams& p, int cus, hipStream_t st) {
  return p.out_bf16 ? through_lds<G, uint16_t>(p, cus, st) : through_lds<G, float>(p, cus, st);
}

template <int kM, int kN, int kW, int kU, bool kFused>
hipError_t split(const MxGemmParams& p, hipStream_t st) {
  const int ti = (p.a.strips + kM - 1) / kM, tj = (p.b.strips + kN - 1) / kN;
  hipLaunchKernelGGL((mx_gemm_split_kernel<kM, kN, kW, kU, kFused>), dim3(ti * tj), dim3(64 * kW), 0, st, p, ti, ti * tj);
  return hipGetLastError();
}

int64_t tiles_of(int64_t M, int64_t N, int rows, int cols) { return ((M + rows - 1) / rows) * ((N + cols - 1) / cols); }

// Microseconds that the tiles of 256 x 256 (one workgroup per compute unit), of 128 x 256 (one) and of 128 x 128 (two)
// take, fitted to measurements of outputs from 1024 x 2048 to 8192 x 8192 and contractions from 256 to 11008 on 256
// compute units; the model is within 15 % of them where the two are close.  Other numbers of units take the same
// constants, unmeasured.  A full round of 256 x 256 tiles takes 5 + 0.82 per block of the contraction (power holds the
// clock down), a part of a round less; of 128 x 128 tiles, a quarter of that output a tile, 2.3 + 0.52 per block, half
// a round or less 1 + 0.11 to 0.29; of 128 x 256 tiles, one to a compute unit, 2.7 + 0.46.
// Measured, 128 x 128, 128 x 256 and 256 x 256: 2048 x 4096 over 4096 22.5, 21.7 and 27.7 us, over 11008 51.1, 47.1 and 59.0,
// 2048 x 11008 over 4096 58.9, 53.2 and 55.3, 512 x 11008 19.4, 18.4 and 25.4, 4096 x 4096 38.9, 38.1 and 34.7,
// 1024 x 4096 12.8, 16.8 and 24.1, 1100 x 8192 over 2048 17.8, 20.3 and 18.1.
double time_256(int64_t n, int nkb, int cus) {
  const int64_t full = n / cus;
  const double f = (double)(n % cus) / cus;
  return 5 + full * (5 + 0.82 * nkb) + (f > 0 ? 2 + 3 * f + (0.52 + 0.3 * f * f) * nkb : 0);
}
double time_128x256(int64_t n, int nkb, int cus) {
  const int64_t full = n / cus;
  const double f = (double)(n % cus) / cus;
  return 4 + full * (2.7 + 0.46 * nkb) + (f > 0 ? 1.8 + (0.28 + 0.17 * f) * nkb : 0);
}
double time_128(int64_t n, int nkb, int cus) {
  const int64_t full = n / (2 * cus);
  const double f = (double)(n % (2 * cus)) / (2 * cus);
  return 4 + full * (2.3 + 0.52 * nkb) + (f > 0.5 ? 1.5 + 0.5 * nkb : f > 0 ? 1 + (0.11 + 0.35 * f) * nkb : 0);
}

}  // namespace

// The largest tiles of which there are more than half as many as compute units: fewer leave the chip idle, more move
// more bytes per product.  1024 x 2048 outputs (128 tiles of 128 x 128, 512 of 64 x 64) take the same time either way,
// 256 x 11008 (172, 688) 11.6 and 17.9 us at a contraction of 4096, 1024 x 1024 (64, 256) 10.6 and 8.4;
// 256 x 1024 (64 tiles of 64 x 64, 256 of 32 x 32) 7.2 and 4.9.  While two workgroups of 64 x 64 tiles per compute unit
// hold them all and the contraction is short, those are faster where the edges waste larger ones: 300 x 6000 over 1000
// (141, 470) 6.6 and 5.5, 777 x 2432 (133, 494) over 1544 7.2 and 7.0, but over 4096 11.1 and 11.9.  A tile more than
// twice as high or wide as the output is for nothing.
MxForm mx_form(int M, int N, int nkb, int cus) {
  const int narrow = std::min(M, N);
  const int64_t n128 = tiles_of(M, N, 128, 128), n64 = tiles_of(M, N, 64, 64);
  const bool at_once = n64 <= 2 * cus && nkb <= 16;
  if (narrow > 64 && 2 * n128 > cus && !at_once && nkb > 0 && nkb < kMaxBlocks) {
    const double t128 = time_128(n128, nkb, cus), t128x256 = time_128x256(tiles_of(M, N, 128, 256), nkb, cus);
    const double least = N > 128 ? std::min(t128, t128x256) : t128;
    if (narrow > 128 && time_256(tiles_of(M, N, 256, 256), nkb, cus) < least) return MxForm::k256x256;
    return least < t128 ? MxForm::k128x256 : MxForm::k128x128;
  }
  if (narrow > 32 && 2 * n64 > cus) return MxForm::k64x64;
  if (N > 32 && 2 * tiles_of(M, N, 32, 64) > cus) return MxForm::k32x64;
  return MxForm::k32x32;
}

// The forward of a linear layer quantizes X inside its product where that is the faster way.  A workgroup then reads
// its 16 rows of X in bf16, four times their codes, and with more workgroups than compute units that is repeated:
// 1 x 4096 -> 11008 takes 6.7 us instead of 9.6, 128 x 2048 -> 2048 (256 workgroups) 5.7 instead of 6.6, 16 x 11008 -> 4096
// 15.3 instead of 10.9, 200 x 500 -> 2000 (416) 4.5 instead of 6.6, 200 x 2000 -> 2000 8.1 instead of 7.8,
// 32 x 1000 -> 30000 (938) 9.9 instead of 10.4, 32 x 512 -> 60000 (1876) 14.7 instead of 13.1; 16 x 4096 -> 32000 (500) the
// same, -> 128000 65 instead of 57.
// Rows that do not begin at dwords are read at a third of the rate: 128 x 1999 -> 2048 8.5 instead of 7.3, 16 x 1023 -> 4096
// 5.9 instead of 7.4.  The sums are those of the stored codes' product: 8 wavefronts share a contraction.
bool mx_linear_fused(int M, int N, int K, int cus, bool unaligned) {
  const MxForm form = mx_form(M, N, (K + 127) / 128, cus);
  if (form != MxForm::k32x32 && form != MxForm::k32x64) return false;
  const int64_t n = tiles_of(M, N, 16, 64), k = (unaligned ? 3 : 1) * (int64_t)K;
  if (M <= 16) return M * k <= (n <= 2 * cus ? 65536 : 32768);
  return n <= cus ? k <= 4096 : n <= 4 * cus && k <= 1024;
}

hipError_t launch_mx_gemm(const MxGemmParams& p, hipStream_t st) {
  if (p.x) return split<1, 4, 8, 1, true>(p, st);
  const int cus = mx_plan_units(compute_units());
  if (cus <= 0) return hipErrorInvalidDevice;
  switch (mx_form(p.M, p.N, p.a.nkb, cus)) {
    case MxForm::k32x32: return split<2, 2, 8, 2, false>(p, st);
    case MxForm::k32x64: return split<2, 4, 8, 2, false>(p, st);
    case MxForm::k64x64: return split<4, 4, 4, 2, false>(p, st);
    case MxForm::k128x128: return through_lds<LdsGeo<4, 4, 2, 2, 4>>(p, cus, st);
    case MxForm::k128x256: return through_lds<LdsGeo<4, 4, 4, 1, 4>>(p, cus, st);
    case MxForm::k256x256: return through_lds<LdsGeo<8, 4, 4, 1, 4>>(p, cus, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace fq

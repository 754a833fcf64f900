// Microscaled 4-bit matrices: quantization along the rows, the columns or both in one launch, and the way back.
//
// A group of 32 values shares 2^s; s comes from the exponent of the group's largest magnitude, which is an integer
// maximum over the bf16 bits without the sign (so infinities and NaNs come out largest), and the codes from the
// conversion instructions, which divide by a power of two and round to E2M1 to nearest even.  Both kernels stream:
// 2 bytes an element on the bf16 side, 17/32 per side on the other.  Memory bounds them: 4096 x 11008 is quantized
// along the rows in 22.6 us (5.0 TB/s), along both in 27.6 us (5.0) and read back in 25 us (4.5), where a copy of 1 GiB
// reaches 4.7 TB/s.  Stochastic rounding is bound by the vector unit (one Philox block per 8 elements, two conversions per
// pair and side): both sides 34.5 us.  Below a million elements a call is latency: 3.1 us for 131 x 2200.
//
// A wavefront has 32 rows x 128 columns, a lane 8 x 8 of them: 16 lanes read 256 bytes of a row, four lanes next to
// each other hold a row's group, the four lanes 16 apart a column's.  So either maximum is taken in registers with
// two exchanges, and neither side needs the elements transposed through LDS; only the finished codes pass through it,
// to leave in 16-byte stores.  (The dword writes of the codes meet in 8 of the 64 banks; in addresses exchanged so that
// they do not, 4096 x 11008 takes the same 27.7 us.)
#include "fq_device.h"
#include "fq_kernels.h"
#include "fq_mx_device.h"

namespace fq {

namespace {

typedef float v2f __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kTile = 128;        // rows and columns of a workgroup: whole operands along either axis
constexpr int kWaveRows = 32;     // of a wavefront: one group along the columns

// bf16 half k of a dword as binary32, or random bits in the upper half of a word
__device__ __forceinline__ uint32_t upper(uint32_t w, int k) { return k ? w & 0xFFFF0000u : w << 16; }

// Stochastic codes of two values, in byte 0.  The conversion adds its random word, as a fraction of a step, to the value
// and cuts; for the second value it takes the word one bit up.  Either value has 16 bits of its own, so both are
// converted with the word of one, and the nibbles that were made with the right word are put together.
__device__ __forceinline__ uint32_t cvt_sr(uint32_t x0, uint32_t x1, uint32_t u0, uint32_t u1, float scale) {
  const v2f v = {__uint_as_float(x0), __uint_as_float(x1)};
  const uint32_t first = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, v, u0, scale, 0);
  const uint32_t second = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, v, u1 >> 1, scale, 0);
  return (first & 0x0Fu) | (second & ~0x0Fu);
}
// byte 0 of each
__device__ __forceinline__ uint32_t bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

struct Random8 { uint32_t w[4]; };

// 8 values, the first n (1 to 7) of them dropped.
__device__ __forceinline__ v4u drop_first(const v4u& v, int n) {
  const uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
  const int s = 16 * (n & 3);
  const uint64_t a = lo >> s | (hi << 1) << (63 - s), b = hi >> s;
  const uint64_t l = n & 4 ? b : a, h = n & 4 ? 0 : b;
  return v4u{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}

// The 8 x 8 values at (row0, col0), packed pairs; what is not there reads as 0.  All loads are requested before one of
// them is used.  Behind the edges a lane reads the last row and the last group of 8 columns.  That group may end behind
// its row, in what follows there; of the last row, which nothing follows, the last 8 values are read instead.  What a small
// matrix pays for edges is the fetch of their code: 300 x 1020 with every row shifted 4.4 us, so 3.4, 300 x 1024 3.0.
__device__ __forceinline__ void load_rows(const MxQuantParams& p, int row0, int col0, v4u (&x)[8]) {
  if (p.cols < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = v4u{0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (row0 + i < p.rows && col0 + e < p.cols) x[i][e >> 1] |= (uint32_t)p.x[(row0 + i) * p.ld + col0 + e] << (16 * (e & 1));
    }
    return;
  }
  const int last = p.rows - 1, col = min(col0, (p.cols - 1) & ~7), col_last = min(col, p.cols - 8);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = *reinterpret_cast<const v4u_at2*>(p.x + min(row0 + i, last) * p.ld + (row0 + i < last ? col : col_last));
  const int valid = p.cols - col0;
  if (valid < 8) {
    if (valid > 0 && row0 == (last & ~7)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i == (last & 7)) x[i] = drop_first(x[i], 8 - valid);
    }
    v4u mask;
#pragma unroll
    for (int d = 0; d < 4; ++d) mask[d] = valid >= 2 * d + 2 ? 0xFFFFFFFFu : valid == 2 * d + 1 ? 0xFFFFu : 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] &= mask;
  }
  if (row0 + 8 > p.rows) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row0 + i >= p.rows) x[i] = v4u{0u, 0u, 0u, 0u};
  }
}

template <bool kRows, bool kCols, bool kSr>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(MxQuantParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t codes_lds[4][2][2 * kOperand];   // wavefront, side
  __shared__ __attribute__((aligned(16))) uint8_t scales_lds[2][2][kScaleBlock];   // side, half of the tile
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int h = lane >> 4, q = lane & 15;
  const int nbc = p.r.nkb;                               // tiles across
  const int tile = kRows && kCols ? blockIdx.x >> p.apart : blockIdx.x;
  const int bi = tile / nbc, bk = tile % nbc;
  const bool rows = kRows && !(kCols && p.apart && (blockIdx.x & 1)), cols = kCols && !(kRows && p.apart && !(blockIdx.x & 1));
  const int row0 = bi * kTile + w * kWaveRows + 8 * h, col0 = bk * kTile + 8 * q;

  v4u x[8];
  load_rows(p, row0, col0, x);
  Random8 rnd[kSr ? 8 : 1];
  if constexpr (kSr) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      philox4x32_10((uint32_t)(col0 >> 3), (uint32_t)(row0 + i), (uint32_t)p.seed, (uint32_t)(p.seed >> 32), rnd[i].w);
  }
  constexpr uint32_t kMag = 0x7FFF7FFFu;

  if (rows) {
    uint8_t* const lds = codes_lds[w][0];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      // rows i and i + 1: their maxima in the two halves of a dword
      uint32_t m2[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        m2[k] = pk_max(pk_max(x[i + k][0] & kMag, x[i + k][1] & kMag), pk_max(x[i + k][2] & kMag, x[i + k][3] & kMag));
      const uint32_t m = quad_max(pk_max(__builtin_amdgcn_perm(m2[1], m2[0], 0x05040100u),
                                         __builtin_amdgcn_perm(m2[1], m2[0], 0x07060302u)));
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t byte = scale_byte(k ? m >> 16 : m & 0xFFFFu, p.bias);
        const float s = scale_value(byte);
        uint32_t c = 0;
        if constexpr (kSr) {
          uint32_t n[4];
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t v = x[i + k][d], u = rnd[i + k].w[d];
            n[d] = cvt_sr(upper(v, 0), upper(v, 1), upper(u, 0), upper(u, 1), s);
          }
          c = bytes(n[0], n[1], n[2], n[3]);
        } else {
#pragma unroll
          for (int d = 0; d < 4; ++d) c = cvt_fp4(c, x[i + k][d], s, d);
        }
        if (byte == 255u) c = 0;
        const int r = 8 * h + i + k;                     // of the 32
        *reinterpret_cast<uint32_t*>(lds + (r >> 4) * kOperand + ((r & 15) + 16 * (q >> 2)) * 16 + 4 * (q & 3)) = c;
        if ((q & 3) == 0)
          scales_lds[0][w >> 1][((r & 15) + 16 * (q >> 2)) * 4 + 2 * (w & 1) + (r >> 4)] = (uint8_t)byte;
      }
    }
  }
  if (cols) {
    uint8_t* const lds = codes_lds[w][1];
#pragma unroll
    for (int d = 0; d < 4; ++d) {                        // columns 2 d and 2 d + 1 of the lane's 8
      uint32_t m = x[0][d] & kMag;
#pragma unroll
      for (int i = 1; i < 8; ++i) m = pk_max(m, x[i][d] & kMag);
      m = row_max(m);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t byte = scale_byte(k ? m >> 16 : m & 0xFFFFu, p.bias);
        const float s = scale_value(byte);
        uint32_t c = 0;
        if constexpr (kSr) {
          uint32_t n[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            n[i] = cvt_sr(upper(x[2 * i][d], k), upper(x[2 * i + 1][d], k), upper(rnd[2 * i].w[d], k),
                          upper(rnd[2 * i + 1].w[d], k), s);
          c = bytes(n[0], n[1], n[2], n[3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            c = cvt_fp4(c, __builtin_amdgcn_perm(x[2 * i + 1][d], x[2 * i][d], k ? 0x07060302u : 0x05040100u), s, i);
        }
        if (byte == 255u) c = 0;
        const int col = 8 * q + 2 * d + k;               // of the tile's 128
        *reinterpret_cast<uint32_t*>(lds + col * 16 + 4 * h) = c;
        if (h == 0) scales_lds[1][col >> 6][((col & 15) + 16 * w) * 4 + ((col >> 4) & 3)] = (uint8_t)byte;
      }
    }
  }
  __syncthreads();

#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (rows) {
      const int strip = bi * 8 + w * 2 + u;
      if (strip < p.r.strips)
        *reinterpret_cast<v4u*>(p.r.codes + ((int64_t)strip * p.r.nkb + bk) * kOperand + lane * 16) =
            *reinterpret_cast<const v4u*>(codes_lds[w][0] + u * kOperand + lane * 16);
    }
    if (cols) {
      const int c = lane + 64 * u, strip = bk * 8 + (c >> 4);
      if (strip < p.t.strips)
        *reinterpret_cast<v4u*>(p.t.codes + ((int64_t)strip * p.t.nkb + bi) * kOperand + w * 256 + (c & 15) * 16) =
            *reinterpret_cast<const v4u*>(codes_lds[w][1] + c * 16);
    }
  }
  const int half = w & 1;
  if (rows && w < 2 && 2 * bi + half < p.r.quads)
    *reinterpret_cast<uint32_t*>(p.r.scales + ((int64_t)(2 * bi + half) * p.r.nkb + bk) * kScaleBlock + lane * 4) =
        *reinterpret_cast<const uint32_t*>(&scales_lds[0][half][lane * 4]);
  if (cols && w >= 2 && 2 * bk + half < p.t.quads)
    *reinterpret_cast<uint32_t*>(p.t.scales + ((int64_t)(2 * bk + half) * p.t.nkb + bi) * kScaleBlock + lane * 4) =
        *reinterpret_cast<const uint32_t*>(&scales_lds[1][half][lane * 4]);
}

__device__ __forceinline__ uint32_t cvt_bf16(uint32_t codes, float scale, int sel) {
  v2bf v;
  switch (sel) {
    case 0: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0); break;
    case 1: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1); break;
    case 2: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2); break;
    default: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3); break;
  }
  return __builtin_bit_cast(uint32_t, v);
}

// Byte k of 8 dwords, 16-byte aligned.
__device__ __forceinline__ void load_bytes(const uint8_t* src, int k, uint32_t (&byte)[8]) {
  const v4u lo = reinterpret_cast<const v4u*>(src)[0], hi = reinterpret_cast<const v4u*>(src)[1];
#pragma unroll
  for (int i = 0; i < 8; ++i) byte[i] = (i < 4 ? lo[i & 3] : hi[i & 3]) >> (8 * k) & 255u;
}

// Dword k of lane row h (16 lanes each) becomes dword h of lane row k.
__device__ __forceinline__ void transpose_rows(v4u& v) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const v2u s = __builtin_amdgcn_permlane32_swap(v[k], v[k + 2], false, false);
    v[k] = s[0];
    v[k + 2] = s[1];
  }
#pragma unroll
  for (int k = 0; k < 4; k += 2) {
    const v2u s = __builtin_amdgcn_permlane16_swap(v[k], v[k + 1], false, false);
    v[k] = s[0];
    v[k + 1] = s[1];
  }
}

// The same split of a tile the other way: a lane takes 8 dwords of codes (8 values each) and has 8 x 8 values.
template <bool kCols, bool kBf16>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(MxDequantParams p) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int h = lane >> 4, q = lane & 15;
  const int nbc = (p.cols + kTile - 1) / kTile;
  const int bi = blockIdx.x / nbc, bk = blockIdx.x % nbc;
  const int row0 = bi * kTile + w * kWaveRows + 8 * h, col0 = bk * kTile + 8 * q;
  // the columns' side exchanges dwords between the rows of a wavefront: those lanes stay together
  if (col0 >= p.cols || (kCols ? bi * kTile + w * kWaveRows : row0) >= p.rows) return;
  constexpr uint32_t kNan = 0x7FC07FC0u;
  uint32_t y[8][4];          // bf16 pairs
  if constexpr (!kCols) {
    const int strip = row0 >> 4, r = row0 & 15;          // the lane's 8 rows lie in one strip
    const int64_t at = (int64_t)strip * p.s.nkb + bk;
    const int64_t sat = (int64_t)(strip >> 2) * p.s.nkb + bk;
    uint32_t c[8], byte[8];
    const uint8_t* const src = p.s.codes + at * kOperand + (r + 16 * (q >> 2)) * 16 + 4 * (q & 3);
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = *reinterpret_cast<const uint32_t*>(src + i * 16);
    load_bytes(p.s.scales + sat * kScaleBlock + (r + 16 * (q >> 2)) * 4, strip & 3, byte);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int d = 0; d < 4; ++d) y[i][d] = byte[i] == 255u ? kNan : cvt_bf16(c[i], scale_value(byte[i]), d);
  } else {
    const int strip = col0 >> 4, r = col0 & 15;
    const int64_t at = (int64_t)strip * p.s.nkb + bi;
    const int64_t sat = (int64_t)(strip >> 2) * p.s.nkb + bi;
    // the four lanes 16 apart need 8 columns' 16 bytes: each loads two of them, then dword h of all goes to lane h
    uint32_t c[8], byte[8];
    const v4u* const src = reinterpret_cast<const v4u*>(p.s.codes + at * kOperand + (r + 16 * w) * 16) + 2 * h;
    v4u a = src[0], b = src[1];
    load_bytes(p.s.scales + sat * kScaleBlock + (r + 16 * w) * 4, strip & 3, byte);
    transpose_rows(a);
    transpose_rows(b);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[2 * j] = a[j];
      c[2 * j + 1] = b[j];
    }
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // rows 2 i and 2 i + 1 of columns 2 d and 2 d + 1
        uint32_t v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          v[k] = byte[2 * d + k] == 255u ? kNan : cvt_bf16(c[2 * d + k], scale_value(byte[2 * d + k]), i);
        y[2 * i][d] = __builtin_amdgcn_perm(v[1], v[0], 0x05040100u);
        y[2 * i + 1][d] = __builtin_amdgcn_perm(v[1], v[0], 0x07060302u);
      }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (row0 + i >= p.rows) break;
    const int64_t o = (row0 + i) * p.ldo + col0;
    const bool whole = col0 + 8 <= p.cols;
    if constexpr (kBf16) {
      uint16_t* dst = static_cast<uint16_t*>(p.out) + o;
      if (whole) {
        *reinterpret_cast<v4u_at2*>(dst) = v4u{y[i][0], y[i][1], y[i][2], y[i][3]};
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col0 + e < p.cols) dst[e] = (uint16_t)(y[i][e >> 1] >> (16 * (e & 1)));
      }
    } else {
      uint32_t* dst = static_cast<uint32_t*>(p.out) + o;
      if (whole) {
#pragma unroll
        for (int d = 0; d < 2; ++d)
          *reinterpret_cast<v4u_at2*>(dst + 4 * d) = v4u{y[i][2 * d] << 16, y[i][2 * d] & 0xFFFF0000u, y[i][2 * d + 1] << 16,
                                               y[i][2 * d + 1] & 0xFFFF0000u};
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col0 + e < p.cols) dst[e] = (e & 1) ? y[i][e >> 1] & 0xFFFF0000u : y[i][e >> 1] << 16;
      }
    }
  }
}

int tiles(int rows, int cols) { return ((rows + kTile - 1) / kTile) * ((cols + kTile - 1) / kTile); }

template <bool kSr>
void quantize_sides(const MxQuantParams& p, dim3 grid, hipStream_t st) {
  if (p.r.codes && p.t.codes) hipLaunchKernelGGL((mx_quantize_kernel<true, true, kSr>), grid, dim3(kThreads), 0, st, p);
  else if (p.r.codes) hipLaunchKernelGGL((mx_quantize_kernel<true, false, kSr>), grid, dim3(kThreads), 0, st, p);
  else hipLaunchKernelGGL((mx_quantize_kernel<false, true, kSr>), grid, dim3(kThreads), 0, st, p);
}

}  // namespace

// Few tiles are quantized along either axis by a workgroup each: what counts then is how long one takes (131 x 2200
// stochastic 6.0 -> 5.0 us).  From more than 128 tiles on they would not all run at once and read x twice (1536 x 2048
// 5.5 us instead of 4.9).
hipError_t launch_mx_quantize(const MxQuantParams& given, hipStream_t st) {
  MxQuantParams p = given;
  const int n = tiles(p.rows, p.cols);
  p.apart = p.r.codes && p.t.codes && n <= 128 ? 1 : 0;
  const dim3 grid(n << p.apart);
  if (p.stochastic) quantize_sides<true>(p, grid, st);
  else quantize_sides<false>(p, grid, st);
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(const MxDequantParams& p, hipStream_t st) {
  const dim3 grid(tiles(p.rows, p.cols)), block(kThreads);
  if (p.columns) {
    if (p.out_bf16) hipLaunchKernelGGL((mx_dequantize_kernel<true, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((mx_dequantize_kernel<true, false>), grid, block, 0, st, p);
  } else {
    if (p.out_bf16) hipLaunchKernelGGL((mx_dequantize_kernel<false, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((mx_dequantize_kernel<false, false>), grid, block, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace fq

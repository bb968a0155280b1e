// Linears in 4 bits with group scales: quantizer, packing, and the product with fp16 activations on the matrix cores.
//
// A weight is (q - z) s with a code q of 4 bits and, per row and group of g columns, a scale s (fp16) and a zero point z.
// The product keeps the integers apart from the scales: per row and group the matrix cores sum (q - z) x, whose factors
// are exact in fp16 and whose products (16 bits) are exact in the fp32 accumulation, and the sum is multiplied by s once,
// in fp32. Nothing is rounded to fewer bits before the result.
#include <cstring>

#include "fluxbin_device.h"
#include "fluxbin_quant_internal.h"

namespace fluxbin {

namespace {

typedef _Float16 w4_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 w4_h8 __attribute__((ext_vector_type(8)));
typedef float w4_f4 __attribute__((ext_vector_type(4)));
typedef unsigned int w4_u2 __attribute__((ext_vector_type(2)));
typedef unsigned int w4_u4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------------------------------
// Quantizer. A lane takes 8 consecutive columns of a row, a wavefront 512. Groups of 32 to 512 columns (powers of two) are
// 4 to 64 neighbouring lanes, reduced by shuffles (SPLIT = false); any other group is one wavefront's, which goes over it
// twice (SPLIT = true).
// ---------------------------------------------------------------------------------------------------------------------

template <bool FP32>
__device__ __forceinline__ void load8(const void* W, int64_t row_off, int c, int N, float (&v)[8]) {
  if (c + 8 <= N) {
    if (FP32) {
      const float* p = static_cast<const float*>(W) + row_off + c;
      __builtin_memcpy(v, p, 32);
    } else {
      w4_h8 h;
      __builtin_memcpy(&h, static_cast<const _Float16*>(W) + row_off + c, 16);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = float(h[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = c + i >= N ? 0.f
                        : (FP32 ? static_cast<const float*>(W)[row_off + c + i]
                                : float(static_cast<const _Float16*>(W)[row_off + c + i]));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {   // not a number: 0; the rest to what fp16 holds
    v[i] = v[i] == v[i] ? v[i] : 0.f;
    v[i] = fminf(fmaxf(v[i], -65504.f), 65504.f);
  }
}

struct W4Quant {
  const void* W;
  uint32_t* codes;
  uint16_t* scales;
  uint8_t* zeros;
  uint16_t* values;
  int64_t ldw, ldv, tasks;
  int32_t M, N, g, G, Wn, per_row;   // Wn: code words per row; per_row: tasks per row
};

template <bool ASYM>
__device__ __forceinline__ void store8(const W4Quant& a, int row, int c, const float (&v)[8], float s, float inv, float z) {
  uint32_t word = 0;
  uint16_t out[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float q = __builtin_rintf(v[i] * inv);
    q = ASYM ? fminf(fmaxf(q + z, 0.f), 15.f) : fminf(fmaxf(q, -8.f), 7.f) + 8.f;
    if (c + i < a.N) word |= uint32_t(q) << (4 * i);
    out[i] = f2h(fminf(fmaxf((q - z) * s, -65504.f), 65504.f));
  }
  if (c >= a.N) return;
  a.codes[int64_t(row) * a.Wn + (c >> 3)] = word;
  if (!a.values) return;
  uint16_t* p = a.values + int64_t(row) * a.ldv + c;
  if (c + 8 <= a.N) {
    __builtin_memcpy(p, out, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < a.N) p[i] = out[i];
  }
}

template <bool FP32, bool ASYM, bool SPLIT>
__global__ void __launch_bounds__(256) k_w4_quantize(W4Quant a) {
  const int64_t task = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (task >= a.tasks) return;
  const int lane = int(threadIdx.x) & 63;
  const int row = int(task / a.per_row), part = int(task % a.per_row);
  const int64_t off = int64_t(row) * a.ldw;
  const int c0 = SPLIT ? part * a.g : part * 512, c1 = SPLIT ? (c0 + a.g < a.N ? c0 + a.g : a.N) : a.N;
  const int span = SPLIT ? 64 : a.g / 8;   // lanes that share a group
  float v[8], lo = 0.f, hi = 0.f;
  for (int c = c0 + 8 * lane; c < c1; c += 512) {
    load8<FP32>(a.W, off, c, SPLIT ? c1 : a.N, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = fminf(lo, v[i]);
      hi = fmaxf(hi, v[i]);
    }
    if (!SPLIT) break;
  }
  for (int o = 1; o < span; o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o));
    hi = fmaxf(hi, __shfl_xor(hi, o));
  }
  const _Float16 sh = _Float16(fabsf(ASYM ? (hi - lo) * (1.f / 15.f) : fmaxf(hi, -lo) * (1.f / 7.f)));   // no -0
  const float s = float(sh), inv = s > 0.f ? 1.f / s : 0.f;
  const float z = ASYM ? fminf(fmaxf(__builtin_rintf(-lo * inv), 0.f), 15.f) : 8.f;
  const int c = c0 + 8 * lane;
  if (lane % span == 0 && c < a.N) {
    const int64_t at = int64_t(row) * a.G + (SPLIT ? part : c / a.g);
    a.scales[at] = __builtin_bit_cast(uint16_t, sh);
    if (ASYM) a.zeros[at] = uint8_t(z);
  }
  if (!SPLIT) {
    if (c < a.N) store8<ASYM>(a, row, c, v, s, inv, z);
  } else {
    for (int k = c; k < c1; k += 512) {
      load8<FP32>(a.W, off, k, c1, v);
      store8<ASYM>(a, row, k, v, s, inv, z);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Packing: [row tile][chunk][lane][16 bytes]. Lane (row m = lane & 15 of the tile, k group q = lane >> 4) holds the operands
// of four matrix instructions: word j is columns 128 chunk + 32 j + 8 q + e, e = 0..7, its nibble t the column
// e = 2 t (t < 4) or 2 (t - 4) + 1, so that one mask takes a pair of neighbours into the halves of a register.
// ---------------------------------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(256) k_w4_pack(const uint32_t* codes, uint8_t* out, int32_t M, int32_t Wn, int32_t Nc,
                                                 int64_t blocks) {
  const int64_t blk = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (blk >= blocks) return;
  const int lane = int(threadIdx.x) & 63, tile = int(blk / Nc), chunk = int(blk % Nc);
  const int64_t row = int64_t(tile) * 16 + (lane & 15);
  w4_u4 o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int w = chunk * 16 + 4 * j + (lane >> 4);
    const uint32_t c = row < M && w < Wn ? codes[row * Wn + w] : 0u;
    uint32_t r = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      r |= ((c >> (8 * t)) & 15u) << (4 * t);
      r |= ((c >> (8 * t + 4)) & 15u) << (16 + 4 * t);
    }
    o[j] = r;
  }
  *reinterpret_cast<w4_u4*>(out + blk * 1024 + lane * 16) = o;
}

// Scale quads [row tile][quad][16 rows][4] fp16, zero points [row tile][quad][16 rows][4] bytes: slot 4 quad + i is part
// slot % gc of chunk slot / gc. Rows and columns past the end: scale 0, zero point 8.
__global__ void __launch_bounds__(256) k_w4_pack_scales(const uint16_t* scales, const uint8_t* zeros, uint16_t* out_s,
                                                        uint8_t* out_z, int32_t M, int32_t N, int64_t g, int32_t G,
                                                        int32_t gc, int32_t Nq, int64_t n) {
  const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (e >= n) return;
  const int i = int(e & 3), m = int(e >> 2) & 15;
  const int64_t tq = e >> 6;
  const int quad = int(tq % Nq);
  const int64_t row = tq / Nq * 16 + m;
  const int64_t col = int64_t(4 * quad + i) * (kChunk / gc);
  const bool in = row < M && col < N;
  const int64_t at = in ? row * G + col / g : 0;
  out_s[e] = in ? scales[at] : uint16_t(0);
  if (out_z) out_z[e] = in ? uint8_t(zeros[at] & 15) : uint8_t(8);
}

// ---------------------------------------------------------------------------------------------------------------------
// Product. A workgroup takes RT row tiles x 16 BT batch rows and a part of the columns; its wavefronts take steps of four
// chunks in turn and add their sums in LDS in wavefront order. With parts > 1 a second kernel adds the parts' sums in part
// order. Activations are operand A (lane: batch row lane & 15), weights operand B (lane: row lane & 15), so a lane's
// results, codes and scales are all of one row of W.
// ---------------------------------------------------------------------------------------------------------------------

// Activation operand of word j: x[b][c .. c + 7], zero past N or B.
__device__ __forceinline__ w4_h8 load_x(const uint16_t* x, bool in, int c, int N) {
  w4_h8 v = {};
  if (!in) return v;
  if (c + 8 <= N) {
    __builtin_memcpy(&v, x + c, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < N) v[i] = __builtin_bit_cast(_Float16, x[c + i]);
  }
  return v;
}

// The eight q - z of a word as fp16: a nibble put into the low bits of 1024 (or, four bits up, of 64 after a division by
// 16) is that number plus q; the sums below are exact.
__device__ __forceinline__ w4_h8 decode8(uint32_t w, w4_h2 lo, w4_h2 hi) {
  const uint32_t m = 0x000F000Fu, mh = 0x00F000F0u, k = 0x64006400u;
  const w4_h2 sixteenth = {_Float16(0.0625f), _Float16(0.0625f)};
  const uint32_t v = w >> 8;
  const w4_h2 a = __builtin_bit_cast(w4_h2, (w & m) | k) + lo;
  const w4_h2 b = __builtin_elementwise_fma(__builtin_bit_cast(w4_h2, (w & mh) | k), sixteenth, hi);
  const w4_h2 c = __builtin_bit_cast(w4_h2, (v & m) | k) + lo;
  const w4_h2 d = __builtin_elementwise_fma(__builtin_bit_cast(w4_h2, (v & mh) | k), sixteenth, hi);
  return w4_h8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// -(1024 + z) and -(64 + z) in both halves.
__device__ __forceinline__ w4_h2 zero_lo(uint32_t z) { return __builtin_bit_cast(w4_h2, (0xE400u | z) * 0x10001u); }
__device__ __forceinline__ w4_h2 zero_hi(uint32_t z) { return __builtin_bit_cast(w4_h2, (0xD400u | (z << 4)) * 0x10001u); }

constexpr int kW4Waves = 8;

template <int BT, int RT, int GC, bool ZERO>
__global__ void __launch_bounds__(64 * kW4Waves) k_w4_gemm(W4Args a) {
  __shared__ __attribute__((aligned(16))) w4_f4 red[kW4Waves][RT * BT][64];
  const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int tile0 = int(blockIdx.x) * RT, b0 = int(blockIdx.z) * 16 * BT;
  const int steps = (a.Nc + 3) / 4;
  const int s0 = int(int64_t(steps) * blockIdx.y / a.parts), s1 = int(int64_t(steps) * (blockIdx.y + 1) / a.parts);

  const uint8_t* codes[RT];
  const uint8_t* scales[RT];
  const uint8_t* zeros[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int64_t t = tile0 + r < a.Mt ? tile0 + r : a.Mt - 1;   // tiles past the end: never stored
    codes[r] = a.codes + t * a.Nc * 1024 + lane * 16;
    scales[r] = a.scales + t * a.Nq * 128 + m * 8;
    zeros[r] = ZERO ? a.zeros + t * a.Nq * 64 + m * 4 : nullptr;
  }
  const uint16_t* x[BT];
  bool in[BT];
#pragma unroll
  for (int t = 0; t < BT; ++t) {
    const int b = b0 + 16 * t + m;
    in[t] = b < a.B;
    x[t] = a.x + int64_t(in[t] ? b : 0) * a.ldx + 8 * q;
  }
  w4_f4 acc[RT][BT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < BT; ++t) acc[r][t] = w4_f4{0.f, 0.f, 0.f, 0.f};

  for (int s = s0 + wave; s < s1; s += kW4Waves) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = 4 * s + k;
      if (c >= a.Nc) break;
      w4_h8 xv[BT][4];
#pragma unroll
      for (int t = 0; t < BT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[t][j] = load_x(x[t], in[t], kChunk * c + 32 * j, a.N - 8 * q);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const w4_u4 w = *reinterpret_cast<const w4_u4*>(codes[r] + int64_t(c) * 1024);
        w4_f4 d[BT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = c * GC + j * GC / 4;
          const uint32_t z = ZERO ? zeros[r][int64_t(slot >> 2) * 64 + (slot & 3)] : 8u;
          const w4_h8 wv = decode8(w[j], zero_lo(z), zero_hi(z));
#pragma unroll
          for (int t = 0; t < BT; ++t) {
            if (j % (4 / GC) == 0) d[t] = w4_f4{0.f, 0.f, 0.f, 0.f};
            d[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[t][j], wv, d[t], 0, 0, 0);
          }
          if ((j + 1) % (4 / GC) == 0) {
            const float sc = h2f(*reinterpret_cast<const uint16_t*>(scales[r] + int64_t(slot >> 2) * 128 + (slot & 3) * 2));
#pragma unroll
            for (int t = 0; t < BT; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[r][t][i] = __builtin_fmaf(sc, d[t][i], acc[r][t][i]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < BT; ++t) red[wave][r * BT + t][lane] = acc[r][t];
  __syncthreads();
  for (int e = int(threadIdx.x); e < RT * BT * 64; e += 64 * kW4Waves) {
    const int rt = e >> 6, l = e & 63;
    w4_f4 sum = red[0][rt][l];
#pragma unroll
    for (int w = 1; w < kW4Waves; ++w) sum += red[w][rt][l];
    const int row = (tile0 + rt / BT) * 16 + (l & 15);
    if (row >= a.M) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = b0 + 16 * (rt % BT) + 4 * (l >> 4) + i;
      if (b >= a.B) continue;
      if (a.parts > 1)
        a.partials[(int64_t(blockIdx.y) * a.B + b) * a.M + row] = sum[i];
      else if (a.y_fp32)
        static_cast<float*>(a.y)[b * a.ldy + row] = sum[i];
      else
        static_cast<uint16_t*>(a.y)[b * a.ldy + row] = f2h(sum[i]);
    }
  }
}

__global__ void __launch_bounds__(256) k_w4_reduce(W4Args a) {
  const int row = int(blockIdx.x) * 256 + int(threadIdx.x), b = int(blockIdx.y);
  if (row >= a.M) return;
  float sum = 0.f;
  for (int p = 0; p < a.parts; ++p) sum += a.partials[(int64_t(p) * a.B + b) * a.M + row];
  if (a.y_fp32)
    static_cast<float*>(a.y)[b * a.ldy + row] = sum;
  else
    static_cast<uint16_t*>(a.y)[b * a.ldy + row] = f2h(sum);
}

template <int BT, int RT>
void launch_gemm_gz(const W4Args& a, int gc, dim3 grid, hipStream_t stream) {
  const dim3 block(64 * kW4Waves);
#define W4_LAUNCH(GC)                                                                     \
  if (a.zeros)                                                                            \
    hipLaunchKernelGGL((k_w4_gemm<BT, RT, GC, true>), grid, block, 0, stream, a);         \
  else                                                                                    \
    hipLaunchKernelGGL((k_w4_gemm<BT, RT, GC, false>), grid, block, 0, stream, a)
  if (gc == 1) {
    W4_LAUNCH(1);
  } else if (gc == 2) {
    W4_LAUNCH(2);
  } else {
    W4_LAUNCH(4);
  }
#undef W4_LAUNCH
}

}  // namespace

W4Plan w4_plan(const fluxbin_w4_shape& s, int B, int cus) {
  const W4Derived d = w4_derive(s);
  W4Plan p{};
  p.bt = B <= 16 ? 1 : B <= 32 ? 2 : 4;
  p.rt = 1;
  const int64_t wgs = ceil_div(d.Mt, p.rt) * ceil_div(B, 16 * p.bt), steps = ceil_div(d.Nc, 4);
  int64_t parts = cus / wgs;
  if (parts > steps / kW4Waves) parts = steps / kW4Waves;
  p.parts = int(parts < 1 ? 1 : parts);
  p.ws_bytes = p.parts > 1 ? uint64_t(p.parts) * uint64_t(B) * uint64_t(s.M) * 4u : 0u;
  return p;
}

uint64_t w4_workspace(const fluxbin_w4_shape& s, int B, int cus) {
  uint64_t most = 0;
  for (int b = 1; b <= B; ++b) {
    const uint64_t n = w4_plan(s, b, cus).ws_bytes;
    most = n > most ? n : most;
  }
  return round_up256(most);
}

fluxbin_status launch_w4_gemm(const W4Args& a, const W4Plan& p, int gc, hipStream_t stream) {
  const dim3 grid(unsigned(ceil_div(a.Mt, p.rt)), unsigned(p.parts), unsigned(ceil_div(a.B, 16 * p.bt)));
  if (p.bt == 1)
    launch_gemm_gz<1, 1>(a, gc, grid, stream);
  else if (p.bt == 2)
    launch_gemm_gz<2, 1>(a, gc, grid, stream);
  else
    launch_gemm_gz<4, 1>(a, gc, grid, stream);
  if (p.parts > 1)
    hipLaunchKernelGGL(k_w4_reduce, dim3(unsigned(ceil_div(a.M, 256)), unsigned(a.B)), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the 4-bit product");
}

fluxbin_status launch_w4_pack(const fluxbin_w4_shape& s, const uint32_t* d_codes, const uint16_t* d_scales,
                              const uint8_t* d_zeros, void* d_packed, hipStream_t stream) {
  const W4Derived d = w4_derive(s);
  uint8_t* base = static_cast<uint8_t*>(d_packed);
  const int64_t blocks = d.Mt * d.Nc, n = d.Mt * d.Nq * 64;
  hipLaunchKernelGGL(k_w4_pack, dim3(unsigned(ceil_div(blocks, 4))), dim3(256), 0, stream, d_codes, base, int32_t(s.M),
                     int32_t(ceil_div(s.N, 8)), int32_t(d.Nc), blocks);
  hipLaunchKernelGGL(k_w4_pack_scales, dim3(unsigned(ceil_div(n, 256))), dim3(256), 0, stream, d_scales, d_zeros,
                     reinterpret_cast<uint16_t*>(base + d.off_scales), s.has_zeros ? base + d.off_zeros : nullptr,
                     int32_t(s.M), int32_t(s.N), s.g, int32_t(d.G), d.gc, int32_t(d.Nq), n);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the 4-bit packing");
}

template <bool FP32>
static void quantize_launch(const W4Quant& a, bool asym, bool split, hipStream_t stream) {
  const dim3 grid(unsigned(ceil_div(a.tasks, 4))), block(256);
  if (asym && split)
    hipLaunchKernelGGL((k_w4_quantize<FP32, true, true>), grid, block, 0, stream, a);
  else if (asym)
    hipLaunchKernelGGL((k_w4_quantize<FP32, true, false>), grid, block, 0, stream, a);
  else if (split)
    hipLaunchKernelGGL((k_w4_quantize<FP32, false, true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((k_w4_quantize<FP32, false, false>), grid, block, 0, stream, a);
}

fluxbin_status launch_w4_quantize(const void* d_W, int w_is_fp32, int64_t ldw, const fluxbin_w4_shape& s,
                                  uint32_t* d_codes, uint16_t* d_scales, uint8_t* d_zeros, uint16_t* d_values,
                                  int64_t ldv, hipStream_t stream) {
  const W4Derived d = w4_derive(s);
  const int64_t g = s.g < s.N ? s.g : s.N;
  const bool split = s.g < 32 || s.g > 512 || (s.g & (s.g - 1)) != 0;   // s.g >= N may be any number
  W4Quant a{};
  a.W = d_W;
  a.codes = d_codes;
  a.scales = d_scales;
  a.zeros = d_zeros;
  a.values = d_values;
  a.ldw = ldw;
  a.ldv = ldv;
  a.M = int32_t(s.M);
  a.N = int32_t(s.N);
  a.g = int32_t(split ? g : s.g);
  a.G = int32_t(d.G);
  a.Wn = int32_t(ceil_div(s.N, 8));
  a.per_row = int32_t(split ? d.G : ceil_div(s.N, 512));
  a.tasks = s.M * a.per_row;
  if (w_is_fp32)
    quantize_launch<true>(a, s.has_zeros != 0, split, stream);
  else
    quantize_launch<false>(a, s.has_zeros != 0, split, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the 4-bit quantizer");
}

}  // namespace fluxbin

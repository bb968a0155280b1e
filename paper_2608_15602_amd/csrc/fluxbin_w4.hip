// Linears in 4 bits with group scales: quantizer, packing, and the product with fp16 activations on the matrix cores.
//
// A weight is (q - z) s with a code q of 4 bits and, per row and group of g columns, a scale s (fp16) and a zero point z.
// The product keeps the integers apart from the scales: per row and group the matrix cores sum (q - z) x, whose factors
// are exact in fp16 and whose products (16 bits) are exact in the fp32 accumulation, and the sum is multiplied by s once,
// in fp32. Nothing is rounded to fewer bits before the result.
#include <type_traits>

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
// twice (SPLIT = true). Bound by memory: 11008x4096 from fp16 with the values 47 us, 4.3 of the 5.1 TB/s of a copy.
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
  float sf = fabsf(ASYM ? (hi - lo) * (1.f / 15.f) : fmaxf(hi, -lo) * (1.f / 7.f));   // no -0
  asm("" : "+v"(sf));   // rounded to fp32 first: the product is not to be taken into the conversion's rounding
  const _Float16 sh = _Float16(sf);
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
// Product of few batch rows. A workgroup takes RT row tiles x 16 BT batch rows and a part of the columns; its NW wavefronts
// take steps of four whole chunks in turn, then the chunks that are left, and add their sums in LDS in wavefront order. With
// parts > 1 a second kernel adds the parts' sums in part order. Activations are operand A (lane: batch row lane & 15),
// weights operand B (lane: row lane & 15), so a lane's results, codes and scales are all of one row of W. Batch rows and row
// tiles past the end repeat others and are not stored: a result row depends on its own operand row only.
//
// Bound by the stream of codes. Every chunk's registers are loaded again for the next step as soon as it has been used, so
// a wavefront keeps a step (4 RT KB) of requests ahead. Activations go through the wavefront's own LDS: a request takes
// four whole row pieces of 256 bytes (XR requests a chunk), and lanes pick their operands from there: straight from memory
// an operand is 64 bytes of each of 16 rows, and such requests took 2.5 times as long and bound the kernel (8192x28672 at
// B = 16: 65 us with them). 28672x8192 with zero points per group of 128 at B = 1: 29 us (122 MB, 4.2 TB/s; the kernel
// under the profiler 24.9); 8192x28672 at B = 16: 37 us; 4096x4096 at B = 1: 5 us.
// Activations are handed over inside a wavefront: its LDS operations happen in the order in which they are issued, and the
// compiler keeps a store and a load that may meet in order. No fences: with one on either side of each store 28672x8192 at
// B = 1 took 36.6 us (8192x28672 at B = 16: 33.6).
// ---------------------------------------------------------------------------------------------------------------------

// Eight activations from column c of a row, zero past its end: the requests go out together, past the end for the last
// column, without branches between them.
__device__ __forceinline__ w4_h8 load_x8(const uint16_t* row, int c, int N) {
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = row[c + i < N ? c + i : N - 1];
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = c + i < N ? h[i] : 0u;
  return __builtin_bit_cast(w4_h8, w4_u4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16});
}

// The eight q - z of a word as fp16: a nibble put into the low bits of 1024 (or, four bits up, of 64 after a division by
// 16) is that number plus q; the sums below are exact.
__device__ __forceinline__ w4_h8 decode8(uint32_t w, w4_h2 lo, w4_h2 hi) {
  const uint32_t m = 0x000F000Fu, mh = 0x00F000F0u;
  uint32_t k = 0x64006400u;
  asm("" : "+v"(k));   // in a register: with two literals the mask and the or would be two instructions
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

template <int NW, int BT, int XR, int RT, int GC, bool ZERO>
__global__ void __launch_bounds__(64 * NW) k_w4_gemm(W4Args a) {
  // activations: [wavefront][buffer][4 XR rows][16 pieces of 16 bytes], piece p of row r at p ^ (r & 15), so that both the
  // writes (16 pieces of a row) and the reads (a piece of 16 rows) touch all banks; at the end the wavefronts' sums
  constexpr int kXs = 4 * XR * 16, kRed = RT * BT * 64;
  __shared__ __attribute__((aligned(16))) w4_f4 lds[NW * (2 * kXs > kRed ? 2 * kXs : kRed)];
  const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int tile0 = int(blockIdx.x) * RT, b0 = int(blockIdx.z) * 16 * BT;
  const int steps = a.N / (4 * kChunk);   // of four whole chunks
  const int s0 = int(int64_t(steps) * blockIdx.y / a.parts), s1 = int(int64_t(steps) * (blockIdx.y + 1) / a.parts);
  const int rows = a.B - b0 < 16 * BT ? a.B - b0 : 16 * BT;

  int64_t tiles[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) tiles[r] = tile0 + r < a.Mt ? tile0 + r : a.Mt - 1;
  w4_f4 acc[RT][BT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < BT; ++t) acc[r][t] = w4_f4{0.f, 0.f, 0.f, 0.f};

  // acc[r] += scales * (codes - zero points) xv of a chunk: its words, and the scales and zero points of slots first ..
  auto chunk = [&](const w4_h8 (&xv)[BT][4], const w4_u4& w, const w4_u2 (&sc)[GC], const uint32_t (&zp)[GC], int first,
                   w4_f4 (&sum)[BT]) __attribute__((always_inline)) {
    w4_f4 d[BT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = first + j * GC / 4;
      const uint32_t z = ZERO ? (zp[slot >> 2] >> (8 * (slot & 3))) & 255u : 8u;
      const w4_h8 wv = decode8(w[j], zero_lo(z), zero_hi(z));
#pragma unroll
      for (int t = 0; t < BT; ++t) {
        if (j % (4 / GC) == 0) d[t] = w4_f4{0.f, 0.f, 0.f, 0.f};
        d[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[t][j], wv, d[t], 0, 0, 0);
      }
      if ((j + 1) % (4 / GC) == 0) {
        const float f = h2f(uint16_t(sc[slot >> 2][(slot & 3) >> 1] >> (16 * (slot & 1))));
#pragma unroll
        for (int t = 0; t < BT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[t][i] = __builtin_fmaf(f, d[t][i], sum[t][i]);
      }
    }
  };

  int s = s0 + wave;
  if (s < s1) {
    w4_f4* xs = lds + wave * 2 * kXs;
    const uint8_t* codes[RT];
    const uint8_t* scales[RT];
    const uint8_t* zeros[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      codes[r] = a.codes + (tiles[r] * a.Nc + 4 * int64_t(s)) * 1024 + lane * 16;
      scales[r] = a.scales + (tiles[r] * a.Nq + int64_t(s) * GC) * 128 + m * 8;
      zeros[r] = ZERO ? a.zeros + (tiles[r] * a.Nq + int64_t(s) * GC) * 64 + m * 4 : nullptr;
    }
    const uint16_t* x[XR];
    int put[XR], take[BT];
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      const int r = 4 * i + q;
      x[i] = a.x + int64_t(b0 + (r < rows ? r : rows - 1)) * a.ldx + int64_t(s) * 4 * kChunk + 8 * m;
      put[i] = r * 16 + (m ^ (r & 15));
    }
#pragma unroll
    for (int t = 0; t < BT; ++t) take[t] = 16 * t + m < 4 * XR ? 16 * t + m : 0;   // its row, or row 0

    w4_u4 w[4][RT];
    w4_h8 xr[XR];   // the next chunk's, on their way
    w4_u2 sc[RT][GC];
    uint32_t zp[RT][GC];
    auto load_scales = [&](w4_u2 (&v)[RT][GC], uint32_t (&z)[RT][GC]) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < GC; ++i) {
          v[r][i] = *reinterpret_cast<const w4_u2*>(scales[r] + i * 128);
          z[r][i] = ZERO ? *reinterpret_cast<const uint32_t*>(zeros[r] + i * 64) : 0u;
        }
    };
    auto load_codes = [&](int k) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) w[k][r] = *reinterpret_cast<const w4_u4*>(codes[r] + k * 1024);
    };
    auto load_x = [&](int k) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < XR; ++i) __builtin_memcpy(&xr[i], x[i] + k * kChunk, 16);
    };
    auto put_x = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < XR; ++i) *reinterpret_cast<w4_h8*>(xs + buf * kXs + put[i]) = xr[i];
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) load_codes(k);
    load_scales(sc, zp);
    load_x(0);
    put_x(0);
    load_x(1);
    for (;;) {
      // The next step's pointers; the last step's requests repeat it.
      const int64_t on = s + NW < s1 ? NW : 0;
      w4_u2 scn[RT][GC];
      uint32_t zpn[RT][GC];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        codes[r] += on * 4096;
        scales[r] += on * GC * 128;
        if (ZERO) zeros[r] += on * GC * 64;
      }
      load_scales(scn, zpn);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        put_x((k + 1) & 1);
        if (k == 2) {
#pragma unroll
          for (int i = 0; i < XR; ++i) x[i] += on * 4 * kChunk;
        }
        load_x((k + 2) & 3);
        w4_h8 xv[BT][4];
#pragma unroll
        for (int t = 0; t < BT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            xv[t][j] = *reinterpret_cast<const w4_h8*>(xs + (k & 1) * kXs + take[t] * 16 + ((4 * j + q) ^ (take[t] & 15)));
#pragma unroll
        for (int r = 0; r < RT; ++r) chunk(xv, w[k][r], sc[r], zp[r], k * GC, acc[r]);
        load_codes(k);
      }
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < GC; ++i) {
          sc[r][i] = scn[r][i];
          zp[r][i] = zpn[r][i];
        }
      if (on == 0) break;
      s += NW;
    }
  }
  // the chunks after the last whole step, one at a time
  if (int(blockIdx.y) == a.parts - 1) {
    for (int c = 4 * steps + (wave + NW - steps % NW) % NW; c < a.Nc; c += NW) {
      w4_h8 xv[BT][4];
#pragma unroll
      for (int t = 0; t < BT; ++t) {
        const uint16_t* row = a.x + int64_t(b0 + (16 * t + m < rows ? 16 * t + m : 0)) * a.ldx;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = kChunk * c + 32 * j + 8 * q;
          xv[t][j] = load_x8(row, col, a.N);
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const w4_u4 w = *reinterpret_cast<const w4_u4*>(a.codes + (tiles[r] * a.Nc + c) * 1024 + lane * 16);
        w4_u2 sc[GC];
        uint32_t zp[GC];
        const int64_t quad = tiles[r] * a.Nq + c * GC / 4;
        sc[0] = *reinterpret_cast<const w4_u2*>(a.scales + quad * 128 + m * 8);
        zp[0] = ZERO ? *reinterpret_cast<const uint32_t*>(a.zeros + quad * 64 + m * 4) : 0u;
        const int first = c * GC & 3;   // this chunk's slots to the front
        if (first) {
          const uint64_t v = ((uint64_t(sc[0].y) << 32) | sc[0].x) >> (16 * first);
          sc[0] = w4_u2{uint32_t(v), uint32_t(v >> 32)};
          zp[0] >>= 8 * first;
        }
        chunk(xv, w, sc, zp, 0, acc[r]);
      }
    }
  }
  __syncthreads();   // everyone is done with the activations
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < BT; ++t) lds[wave * kRed + (r * BT + t) * 64 + lane] = acc[r][t];
  __syncthreads();
  for (int e = int(threadIdx.x); e < RT * BT * 64; e += 64 * NW) {
    const int rt = e >> 6, l = e & 63;
    w4_f4 sum = lds[e];
#pragma unroll
    for (int v = 1; v < NW; ++v) sum += lds[v * kRed + e];
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

// ---------------------------------------------------------------------------------------------------------------------
// Product of many batch rows. A workgroup of eight wavefronts takes 256 rows x 16 NB batch rows and a part of the chunks,
// four wavefronts the part's even chunks and four its odd ones; a wavefront owns 64 rows and all the batch rows, so that a
// decoded weight serves 16 NB of them (decoding 8 weights takes 13 vector instructions, the matrix instructions of a
// 16-row block NB times 16 cycles). The activations of two chunks are staged in LDS for all, two chunks ahead; codes and
// scales come as far ahead into registers. At the end the halves' sums are added in LDS; with more parts a second kernel
// adds the parts' sums. Bound by the vector work and the matrix cores beside it about equally (8192x8192 at B = 512:
// 39% and 31% of the time, the rest waits), so two wavefronts share a SIMD. 11008x4096 with groups of 64 at B = 256: 50 us,
// 460 TFLOP/s on 172 workgroups for 256 CUs; 28672x8192 at B = 512: 313 us, 770 TFLOP/s; 8192x8192 at B = 2048: 886.
// ---------------------------------------------------------------------------------------------------------------------

template <int NB, int GC, bool ZERO>
__global__ void __launch_bounds__(512, 2) k_w4_gemm_many(W4Args a) {
  constexpr int kXs = 16 * NB * 16;   // 16-byte pieces of a chunk's activations, piece p of row r at p ^ (r & 15)
  __shared__ __attribute__((aligned(16))) w4_h8 xs[2][2][kXs];   // [half][buffer]
  const int tid = int(threadIdx.x) & 255, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6) & 3, half = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 8);
  const int m = lane & 15, q = lane >> 4;
  const int row0 = int(blockIdx.x) * 256 + 64 * wave, b0 = int(blockIdx.z) * 16 * NB;
  const int c0 = int(int64_t(a.Nc) * blockIdx.y / a.parts), c1 = int(int64_t(a.Nc) * (blockIdx.y + 1) / a.parts);

  const uint16_t* x[NB];   // this thread's pieces: row 16 i + (tid >> 4), piece tid & 15
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int b = b0 + 16 * i + (tid >> 4);
    x[i] = a.x + int64_t(b < a.B ? b : a.B - 1) * a.ldx + 8 * (tid & 15);
  }
  const int put = (tid >> 4) * 16 + ((tid & 15) ^ (tid >> 4));

  w4_f4 acc[4][NB];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < NB; ++t) acc[r][t] = w4_f4{0.f, 0.f, 0.f, 0.f};

  typedef typename std::conditional<GC == 4, uint64_t, uint32_t>::type Scales;
  struct Chunk {
    w4_u4 w[4];
    Scales sc[4];     // GC of 16 bits
    uint32_t zp[4];   // GC of 8 bits
  };
  auto load = [&](int c, Chunk& v) __attribute__((always_inline)) {
    const int slot = c * GC;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t t = row0 / 16 + r < a.Mt ? row0 / 16 + r : a.Mt - 1;   // row tiles past the end: never stored
      const uint8_t* w = a.codes + (t * a.Nc + c) * 1024;
      const uint8_t* s = a.scales + (t * a.Nq + (slot >> 2)) * 128 + (slot & 3) * 2;
      const uint8_t* z = ZERO ? a.zeros + (t * a.Nq + (slot >> 2)) * 64 + (slot & 3) : nullptr;
      v.w[r] = *reinterpret_cast<const w4_u4*>(w + uint32_t(lane * 16));
      if (GC == 1) {
        v.sc[r] = *reinterpret_cast<const uint16_t*>(s + uint32_t(m * 8));
        v.zp[r] = ZERO ? z[uint32_t(m * 4)] : 0u;
      } else if (GC == 2) {
        v.sc[r] = *reinterpret_cast<const uint32_t*>(s + uint32_t(m * 8));
        v.zp[r] = ZERO ? *reinterpret_cast<const uint16_t*>(z + uint32_t(m * 4)) : 0u;
      } else {
        v.sc[r] = *reinterpret_cast<const uint64_t*>(s + uint32_t(m * 8));
        v.zp[r] = ZERO ? *reinterpret_cast<const uint32_t*>(z + uint32_t(m * 4)) : 0u;
      }
    }
  };
  w4_h8 xr[NB];
  auto load_x = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) __builtin_memcpy(&xr[i], x[i] + int64_t(c) * kChunk, 16);
  };
  auto put_x = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) xs[half][buf][256 * i + put] = xr[i];
  };
  // A barrier for LDS only: loads from memory stay on their way.
  auto sync = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  };
  auto multiply = [&](const w4_h8 (&xv)[NB][4], const Chunk& cur) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      w4_f4 d[NB];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int part = j * GC / 4;
        const uint32_t z = ZERO ? (cur.zp[r] >> (8 * part)) & 255u : 8u;
        const w4_h8 wv = decode8(cur.w[r][j], zero_lo(z), zero_hi(z));
#pragma unroll
        for (int t = 0; t < NB; ++t) {
          if (j % (4 / GC) == 0) d[t] = w4_f4{0.f, 0.f, 0.f, 0.f};
          d[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[t][j], wv, d[t], 0, 0, 0);
        }
        if ((j + 1) % (4 / GC) == 0) {
          const float f = h2f(uint16_t(cur.sc[r] >> (16 * part)));
#pragma unroll
          for (int t = 0; t < NB; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][t][i] = __builtin_fmaf(f, d[t][i], acc[r][t][i]);
        }
      }
    }
  };
  auto take = [&](int buf, w4_h8 (&xv)[NB][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) xv[t][j] = xs[half][buf][(16 * t + m) * 16 + ((4 * j + q) ^ m)];
  };

  const int whole = a.N / kChunk, last = c1 < whole ? c1 : whole;   // whole chunks of this part: c0 .. last - 1
  const int pairs = (last - c0 + 1) / 2;
  if (pairs > 0) {
    // this half's chunk of pair i; requests past its last chunk repeat the part's last one
    auto at = [&](int i) __attribute__((always_inline)) {
      const int c = c0 + 2 * i + half;
      return c < last ? c : last - 1;
    };
    Chunk one, two;
    load(at(0), one);
    load_x(at(0));
    put_x(0);
    load_x(at(1));
    // pair i: its codes in `cur`, its activations in buffer b when everyone has passed the barrier
    auto step = [&](int i, int b, const Chunk& cur, Chunk& next) __attribute__((always_inline)) {
      sync();
      w4_h8 xv[NB][4];
      take(b, xv);
      put_x(b ^ 1);
      load(at(i + 1), next);
      load_x(at(i + 2));
      if (c0 + 2 * i + half < last) multiply(xv, cur);
    };
    int i = 0;
    for (; i + 1 < pairs; i += 2) {
      step(i, 0, one, two);
      step(i + 1, 1, two, one);
    }
    if (i < pairs) step(i, 0, one, two);
  }
  if (c1 > last) {   // the last chunk, not whole: the first half's
    const int col = last * kChunk + 8 * (tid & 15);
    sync();
    if (half == 0) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int b = b0 + 16 * i + (tid >> 4);
        xr[i] = load_x8(a.x + int64_t(b < a.B ? b : a.B - 1) * a.ldx, col, a.N);
      }
      put_x(0);
    }
    sync();
    if (half == 0) {
      Chunk one;
      load(last, one);
      w4_h8 xv[NB][4];
      take(0, xv);
      multiply(xv, one);
    }
  }
  // the second half's sums to the first, through the activations' LDS
  w4_f4* sums = reinterpret_cast<w4_f4*>(&xs[0][0][0]);
  static_assert(sizeof(xs) >= sizeof(w4_f4) * 4 * NB * 256, "room for the sums");
  sync();
  if (half == 1) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NB; ++t) sums[(r * NB + t) * 256 + tid] = acc[r][t];
  }
  sync();
  if (half == 1) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < NB; ++t) acc[r][t] += sums[(r * NB + t) * 256 + tid];
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = b0 + 16 * t + 4 * q + i;
      if (b >= a.B) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = row0 + 16 * r + m;
        if (row >= a.M) continue;
        if (a.parts > 1)
          a.partials[(int64_t(blockIdx.y) * a.B + b) * a.M + row] = acc[r][t][i];
        else if (a.y_fp32)
          static_cast<float*>(a.y)[b * a.ldy + row] = acc[r][t][i];
        else
          static_cast<uint16_t*>(a.y)[b * a.ldy + row] = f2h(acc[r][t][i]);
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

template <int NB>
void launch_many(const W4Args& a, int gc, dim3 grid, hipStream_t stream) {
#define W4_LAUNCH(GC)                                                                     \
  if (a.zeros)                                                                            \
    hipLaunchKernelGGL((k_w4_gemm_many<NB, GC, true>), grid, dim3(512), 0, stream, a);    \
  else                                                                                    \
    hipLaunchKernelGGL((k_w4_gemm_many<NB, GC, false>), grid, dim3(512), 0, stream, a)
  if (gc == 1) {
    W4_LAUNCH(1);
  } else if (gc == 2) {
    W4_LAUNCH(2);
  } else {
    W4_LAUNCH(4);
  }
#undef W4_LAUNCH
}

template <int NW, int BT, int XR, int RT>
void launch_gemm_gz(const W4Args& a, int gc, dim3 grid, hipStream_t stream) {
  const dim3 block(64 * NW);
#define W4_LAUNCH(GC)                                                                     \
  if (a.zeros)                                                                            \
    hipLaunchKernelGGL((k_w4_gemm<NW, BT, XR, RT, GC, true>), grid, block, 0, stream, a);         \
  else                                                                                    \
    hipLaunchKernelGGL((k_w4_gemm<NW, BT, XR, RT, GC, false>), grid, block, 0, stream, a)
  if (gc == 1) {
    W4_LAUNCH(1);
  } else if (gc == 2) {
    W4_LAUNCH(2);
  } else if constexpr (BT == 1 || RT == 1) {   // the plan has no two row tiles there
    W4_LAUNCH(4);
  }
#undef W4_LAUNCH
}

}  // namespace

// Times in us on a 256-CU device, as far as the choice between the kernels needs them (B > 32).
static double few_us(const fluxbin_w4_shape& s, int B, const W4Plan& p, int cus) {
  const double blocks = double(ceil_div(B, 32)), waves = double(ceil_div(s.M, 16 * p.rt)) * blocks * p.nw;
  const double stream = 0.15e-6 * double(s.M) * double(s.N) * blocks, rounds = 5.0 * double(int64_t(waves / (8 * cus)) + 1);
  const double rows = s.N % 8 ? 1.8 : 1;   // activation rows that are not 16-byte aligned (3001x1999 at B = 256: 47 us)
  return 3 + rows * (stream > rounds ? stream : rounds) + 1.5 * double(s.N / 512) / (p.nw * p.parts) + (p.parts > 1 ? 3 : 0);
}

static double many_us(const fluxbin_w4_shape& s, int B, int nb, int parts, int cus) {
  const int64_t wgs = ceil_div(s.M, 256) * ceil_div(B, 16 * nb) * parts;
  const int64_t pairs = ceil_div(ceil_div(ceil_div(s.N, kChunk), parts), 2);
  const double join = parts > 1 ? 3 + double(parts) * B * double(s.M) * 8 / 4.5e6 : 0;
  return 6 + double(ceil_div(wgs, cus)) * (double(pairs) * (nb == 3 ? 2.3 : 2.75) + 1.5) + join;
}

W4Plan w4_plan(const fluxbin_w4_shape& s, int B, int cus) {
  const W4Derived d = w4_derive(s);
  const int64_t steps = s.N / 512;
  W4Plan p{};
  p.bt = B <= 16 ? 1 : 2;
  p.parts = 1;
  // Wavefronts of a workgroup: as many as keep up to `limit` of them on every CU, one step each at least.
  auto waves = [&](int64_t groups, int64_t limit, int most) {
    int nw = 2;
    while (nw < most && nw * 2 * groups <= limit * cus && nw < steps) nw *= 2;
    return nw;
  };
  if (B > 4 && d.Mt >= 2 * cus && !(d.gc == 4 && B > 16)) {   // (more registers than there are)
    // two row tiles share the activations' way through LDS: 28672x8192 at B = 16 36 us, 43 with one; at B = 4 31 and 29
    p.rt = 2;
    p.nw = waves(ceil_div(d.Mt, 2), 8, 8);
  } else if (B > 4) {
    p.rt = 1;
    p.nw = waves(d.Mt, 16, 8);
  } else {
    // six wavefronts per CU, and more while each has six steps: at B = 1 28672x8192 30.4 us with 4 in a workgroup, 35.4 with 2,
    // 38 with 16; 8192x28672 28 with 16, 31 with 4; 14336x4096 11.0 with 2, 11.4 with 8; 8192x8192 11.4 with 4, 12.6 with 16
    p.rt = 1;
    p.nw = 2;
    while (p.nw < 16 && p.nw < steps && (d.Mt * p.nw < 6 * cus || steps >= 6 * p.nw)) p.nw *= 2;
  }
  if (p.rt == 1) {
    // few rows and many columns: 512x28672 at B = 1 11.5 us, 8.8 with 4 parts; 512x4096 3.9 and 6.0
    const int64_t room = 2 * cus / (d.Mt * ceil_div(B, 32));
    int64_t parts = steps / p.nw < room ? steps / p.nw : room;
    if (parts > 8) parts = 8;
    if (parts >= 3) p.parts = int(parts);
  }
  if (B > 32) {
    double best = few_us(s, B, p, cus);
    for (int nb = 3; nb <= 4; ++nb)
      for (int parts = 1; parts <= 8 && 2 * parts <= d.Nc + 1; ++parts) {
        const double us = many_us(s, B, nb, parts, cus);
        if (us >= best) continue;
        best = us;
        p.many = true;
        p.bt = nb;
        p.parts = parts;
      }
  }
  p.ws_bytes = p.parts > 1 ? uint64_t(p.parts) * uint64_t(B) * uint64_t(s.M) * 4u : 0u;
  return p;
}

// At least what the plan of any batch up to B needs. Up to 32 rows there are three plans. Past that the times that plans are
// chosen by change where 32, 48 or 64 more rows begin and, in between, grow with the rows by the parts that are joined: from
// the first to the last row of such a stretch plans go from more parts to fewer, or to the few-row kernel's.
uint64_t w4_workspace(const fluxbin_w4_shape& s, int B, int cus) {
  uint64_t most = 0;
  auto stretch = [&](int first, int last) {
    const int a = w4_plan(s, first, cus).parts, b = w4_plan(s, last, cus).parts, parts = a > b ? a : b;
    const uint64_t n = parts > 1 ? uint64_t(parts) * uint64_t(last) * uint64_t(s.M) * 4u : 0u;
    most = n > most ? n : most;
  };
  for (int first = 1; first <= B;) {
    int last = first <= 4 ? 4 : first <= 16 ? 16 : 32;
    if (first > 32) {
      const int to32 = int(ceil_div(first, 32)) * 32, to48 = int(ceil_div(first, 48)) * 48;
      last = to32 < to48 ? to32 : to48;
    }
    if (last > B) last = B;
    stretch(first, last);
    first = last + 1;
  }
  return round_up256(most);
}

template <int NW, int RT>
static void launch_few(const W4Args& a, const W4Plan& p, int gc, hipStream_t stream) {
  const dim3 grid(unsigned(ceil_div(a.Mt, RT)), unsigned(p.parts), unsigned(ceil_div(a.B, 16 * p.bt)));
  if (p.bt == 1 && a.B > 4)
    launch_gemm_gz<NW, 1, 4, RT>(a, gc, grid, stream);
  else if (p.bt == 1)
    launch_gemm_gz<NW, 1, 1, 1>(a, gc, grid, stream);   // one row tile: see the plan
  else
    launch_gemm_gz<NW, 2, 8, RT>(a, gc, grid, stream);
}

fluxbin_status launch_w4_gemm(const W4Args& a, const W4Plan& p, int gc, hipStream_t stream) {
  if (p.many) {
    const dim3 grid(unsigned(ceil_div(a.Mt, 16)), unsigned(p.parts), unsigned(ceil_div(a.B, 16 * p.bt)));
    if (p.bt == 3)
      launch_many<3>(a, gc, grid, stream);
    else
      launch_many<4>(a, gc, grid, stream);
  } else if (p.nw == 16) {   // B <= 4
    launch_gemm_gz<16, 1, 1, 1>(a, gc, dim3(unsigned(a.Mt), unsigned(p.parts), 1), stream);
  } else if (p.rt == 1) {
    if (p.nw == 2)
      launch_few<2, 1>(a, p, gc, stream);
    else if (p.nw == 4)
      launch_few<4, 1>(a, p, gc, stream);
    else
      launch_few<8, 1>(a, p, gc, stream);
  } else {
    if (p.nw == 2)
      launch_few<2, 2>(a, p, gc, stream);
    else if (p.nw == 4)
      launch_few<4, 2>(a, p, gc, stream);
    else
      launch_few<8, 2>(a, p, gc, stream);
  }
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
                     int32_t(s.M), int32_t(s.N), d.g, int32_t(d.G), d.gc, int32_t(d.Nq), n);
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
  a.g = int32_t(split ? d.g : s.g);
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

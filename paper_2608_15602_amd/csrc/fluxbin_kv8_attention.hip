// Attention over the paged 8-bit key/value cache on the matrix cores.
//
// For a cached head, the query rows that share it (the new tokens times the query heads of the group) are columns of
//   S^T = K Q^T          (16 tokens x 16 columns an instruction, 32 elements deep),   O^T += V^T P^T.
// Codes are exact in fp16, so K and V enter as codes and the scales, one per page and head, stay apart: the key's multiplies
// the score in fp32; the value's is added to the score as its logarithm, p = 2^(s + log2 sv - m), so that O sums p * code
// and the softmax sum is that of p / sv. With m the running maximum of s + log2 sv no p leaves fp16's range, however the
// scales of the pages differ. p is fed as the sum of two fp16 numbers (22 bits).
// The results of the first product have the layout that the second takes (a lane holds tokens 4 q + i of one column), and
// the cache stores values in that order: neither p nor the codes cross lanes.
#include "fluxbin_kv8_device.h"

namespace fluxbin {

namespace {

constexpr int kTile = 64;      // tokens of a step of a wavefront
constexpr int kWaves = 4;
constexpr float kLeast = 9.094947e-13f;   // 2^-40 stands for the scale of values that are all zero
constexpr float kShift = 8.f, kSlack = 6.f;   // p is at most 2^(kShift + kSlack), below fp16's 2^16

// The eight codes of two words as fp16: a byte in the low bits of 1024 is that number plus the byte.
__device__ __forceinline__ kv_h8 codes8(uint32_t a, uint32_t b) {
  const kv_h2 off = {_Float16(-1152.f), _Float16(-1152.f)};
  const uint32_t k = 0x64646464u;
  const kv_h2 x = __builtin_bit_cast(kv_h2, __builtin_amdgcn_perm(k, a, 0x04010400u)) + off;
  const kv_h2 y = __builtin_bit_cast(kv_h2, __builtin_amdgcn_perm(k, a, 0x04030402u)) + off;
  const kv_h2 z = __builtin_bit_cast(kv_h2, __builtin_amdgcn_perm(k, b, 0x04010400u)) + off;
  const kv_h2 w = __builtin_bit_cast(kv_h2, __builtin_amdgcn_perm(k, b, 0x04030402u)) + off;
  return kv_h8{x.x, x.y, y.x, y.y, z.x, z.y, w.x, w.y};
}

// Work of a sequence: column tiles (16 columns: row i of the sequence and head g of the group are column i G + g), and
// token tiles that some row of it attends.
struct Seq {
  int start, n, ctx, end;   // first row, rows, tokens, attendable tokens
  int qt, t0, nt;           // column tiles, first token tile, token tiles
};

__device__ __forceinline__ Seq seq_of(const Kv8AttnArgs& a, int b) {
  Seq s;
  const int o0 = a.c.offsets[b], o1 = a.c.offsets[b + 1];
  s.start = o0;
  s.n = o0 >= 0 && o1 <= a.c.T && o1 > o0 ? o1 - o0 : 0;
  s.ctx = kv_context(a.c, b);
  const int cap = a.c.max_blocks << a.c.pshift;
  s.end = s.ctx < cap ? s.ctx : cap;
  int begin = 0;
  if (a.window > 0 && s.ctx - s.n + 1 > a.window) begin = s.ctx - s.n + 1 - a.window;
  if (begin > s.end) begin = s.end;
  s.qt = (s.n * a.G + 15) >> 4;
  s.t0 = begin / kTile;
  s.nt = (s.end + kTile - 1) / kTile - s.t0;
  if (s.nt < 1) s.nt = 1;   // nothing to attend: one tile, all of it masked
  return s;
}

__device__ __forceinline__ int64_t units_of(const Kv8AttnArgs& a, const Seq& s) {
  return int64_t(s.qt) * a.c.Hkv * s.nt;
}

// Inclusive sum over the lanes below and of this one.
__device__ __forceinline__ int64_t wave_scan(int64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uint64_t(v)))));
  const uint32_t hi = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uint64_t(v) >> 32))));
  return int64_t((uint64_t(hi) << 32) | lo);
}

// Units of all sequences.
__device__ int64_t total_units(const Kv8AttnArgs& a, int lane) {
  int64_t sum = 0;
  for (int b = lane; b < a.c.B; b += 64) sum += units_of(a, seq_of(a, b));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  return uniform64(sum);
}

// The sequence that holds unit u (u < total), and its first unit.
__device__ int find_unit(const Kv8AttnArgs& a, int lane, int64_t u, int64_t& first) {
  int64_t before = 0;
  for (int b0 = 0; b0 < a.c.B; b0 += 64) {
    const int b = b0 + lane;
    const int64_t mine = b < a.c.B ? units_of(a, seq_of(a, b)) : 0;
    const int64_t upto = before + wave_scan(mine, lane);
    const uint64_t hit = __ballot(upto > u);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      first = uniform64(__shfl(upto - mine, l));
      return b0 + l;
    }
    before = uniform64(__shfl(upto, 63));
  }
  first = before;
  return a.c.B;
}

// Units per workgroup: an even share, at least one step for each wavefront.
__device__ __forceinline__ int64_t quota_of(int64_t total, int wgs) {
  const int64_t q = (total + wgs - 1) / wgs;
  return q < kWaves ? kWaves : q;
}

// Floats of a partial result: 16 columns x D, then their maxima and sums.
template <int D>
constexpr int part_floats() { return 16 * D + 32; }

// Stores a column's element run, if there is such a column.
template <int D>
__device__ __forceinline__ void store_out(const Kv8AttnArgs& a, const Seq& s, int head, int col, int d, float v) {
  const int i = col / a.G, g = col - i * a.G;
  if (i < s.n) a.out[int64_t(s.start + i) * a.ots + int64_t(head * a.G + g) * a.ohs + d] = f2h(v);
}

template <int D>
__global__ void __launch_bounds__(64 * kWaves) k_kv8_attention(Kv8AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float lds_o[kWaves][16][D + 4];
  __shared__ float lds_m[kWaves][16], lds_l[kWaves][16];
  const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int m16 = lane & 15, q4 = lane >> 4;
  const int64_t total = total_units(a, lane), quota = quota_of(total, a.wgs);
  const int64_t u0 = quota * blockIdx.x;
  int64_t u1 = u0 + quota;
  if (u1 > total) u1 = total;
  if (u0 >= u1) return;
  int64_t first;
  int b = find_unit(a, lane, u0, first);
  Seq s = seq_of(a, b);
  int64_t u = u0;
  while (u < u1) {
    while (u - first >= units_of(a, s)) {   // the next sequence with rows
      first += units_of(a, s);
      if (++b >= a.c.B) return;
      s = seq_of(a, b);
    }
    const int64_t rel = u - first;
    const int item = int(rel / s.nt), ta = int(rel - int64_t(item) * s.nt);   // item: column tile, head
    const int64_t room = u1 - u;
    const int tb = room < s.nt - ta ? ta + int(room) : s.nt;
    const int head = item % a.c.Hkv, ct = item / a.c.Hkv;

    const int col = ct * 16 + m16, ci = col / a.G, cg = col - ci * a.G;   // this lane's column
    const bool has = ci < s.n;
    const int pos = s.ctx - s.n + ci;
    const int hi = has ? (a.causal && pos + 1 < s.end ? pos + 1 : s.end) : 0;
    const int lo = a.window > 0 && pos + 1 > a.window ? pos + 1 - a.window : 0;

    kv_h8 qf[D / 32];
    {
      const uint16_t* p = a.q + int64_t(s.start + (has ? ci : 0)) * a.qts + int64_t(head * a.G + (has ? cg : 0)) * a.qhs;
#pragma unroll
      for (int f = 0; f < D / 32; ++f) {
        kv_h8 v = {};
        if (has) __builtin_memcpy(&v, p + 32 * f + 8 * q4, 16);
        qf[f] = v;
      }
    }
    kv_f4 o[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = kv_f4{0.f, 0.f, 0.f, 0.f};
    float mx = -__builtin_inff(), sum = 0.f;

    for (int t = ta + wave; t < tb; t += kWaves) {
      const int tok = (s.t0 + t) * kTile;
      kv_u4 kw[4][D / 64], vw[4][D / 64];
      float ks[4], vs[4];
      bool ok[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = tok + 16 * j;
        int page = at < s.end ? kv_page(a.c, b, at) : -1;
        ok[j] = page >= 0;
        page = page < 0 ? 0 : page;
        const int64_t ph = int64_t(page) * a.c.Hkv + head;
        const int64_t off =
            kv_page_offset<D>(a.c, page, head) + int64_t((at & ((1 << a.c.pshift) - 1)) >> 4) * 16 * D + lane * 16;
#pragma unroll
        for (int k = 0; k < D / 64; ++k) {
          kw[j][k] = *reinterpret_cast<const kv_u4*>(a.c.k + off + k * 1024);
          vw[j][k] = *reinterpret_cast<const kv_u4*>(a.c.v + off + k * 1024);
        }
        ks[j] = a.c.ks[ph];
        vs[j] = a.c.vs[ph];
      }
      kv_f4 sc[4];
      float top = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kv_f4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < D / 64; ++k) {
          d = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kw[j][k].x, kw[j][k].y), qf[2 * k], d, 0, 0, 0);
          d = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kw[j][k].z, kw[j][k].w), qf[2 * k + 1], d, 0, 0, 0);
        }
        vs[j] = ok[j] && vs[j] > kLeast ? vs[j] : kLeast;
        const float f = ks[j] * a.scale2, lv = __builtin_amdgcn_logf(vs[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = tok + 16 * j + 4 * q4 + i;
          const float v = d[i] * f + lv;
          sc[j][i] = ok[j] && at < hi && at >= lo ? v : -__builtin_inff();
          top = fmaxf(top, sc[j][i]);
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > mx + kSlack)) {   // also the first scores of a column
        const float now = fmaxf(mx, top), r = now == mx ? 1.f : __builtin_amdgcn_exp2f(mx - now);
        sum *= r;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d] *= r;
        mx = now;
      }
      const float base = mx == -__builtin_inff() ? 0.f : mx - kShift;
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        kv_h8 ph, pl;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float iv = __builtin_amdgcn_rcpf(vs[j + h]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(sc[j + h][i] - base);
            sum = __builtin_fmaf(p, iv, sum);
            const _Float16 up = _Float16(p);
            ph[4 * h + i] = up;
            pl[4 * h + i] = _Float16(p - float(up));
          }
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const kv_h8 v = codes8(vw[j][d / 4][d % 4], vw[j + 1][d / 4][d % 4]);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph, o[d], 0, 0, 0);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl, o[d], 0, 0, 0);
        }
      }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (q4 == 0) {
      lds_m[wave][m16] = mx;
      lds_l[wave][m16] = sum;
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<kv_f4*>(&lds_o[wave][m16][16 * d + 4 * q4]) = o[d];
    __syncthreads();
    const bool whole = ta == 0 && tb == s.nt;
    float* part = a.part + (int64_t(blockIdx.x) * 2 + (u == u0 ? 0 : 1)) * part_floats<D>();
    for (int e = int(threadIdx.x); e < 16 * D / 4; e += 64 * kWaves) {
      const int c = e / (D / 4), d = e % (D / 4) * 4;
      float top = lds_m[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds_m[w][c]);
      kv_f4 v = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = lds_m[w][c], r = mw == top ? 1.f : __builtin_amdgcn_exp2f(mw - top);   // no scores: both -inf, v 0
        l = __builtin_fmaf(lds_l[w][c], r, l);
        const kv_f4 x = *reinterpret_cast<const kv_f4*>(&lds_o[w][c][d]);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(x[i], r, v[i]);
      }
      if (whole) {
        const float il = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 4; ++i) store_out<D>(a, s, head, ct * 16 + c, d + i, v[i] * il);
      } else {
        *reinterpret_cast<kv_f4*>(part + c * D + d) = v;
        if (d == 0) {
          part[16 * D + c] = top;
          part[16 * D + 16 + c] = l;
        }
      }
    }
    u += tb - ta;
    __syncthreads();   // lds of the next item
  }
}

// Adds the partial results of an item (sequence, column tile, head) that several workgroups have worked on, in their order.
template <int D>
__global__ void __launch_bounds__(256) k_kv8_join(Kv8AttnArgs a) {
  const int lane = int(threadIdx.x) & 63;
  const int64_t total = total_units(a, lane), quota = quota_of(total, a.wgs);
  // an item that is split crosses a border between two workgroups: the one that crosses this border as its first
  const int64_t border = quota * (int64_t(blockIdx.x) + 1);
  if (border >= total) return;
  int64_t first;
  const int b = find_unit(a, lane, border, first);
  const Seq s = seq_of(a, b);
  const int item = int((border - first) / s.nt);
  const int64_t i0 = first + int64_t(item) * s.nt, i1 = i0 + s.nt;
  if (i0 >= border || i0 < border - quota) return;   // starts at the border, or crosses an earlier one
  const int w0 = int(blockIdx.x), w1 = int((i1 - 1) / quota);
  const int head = item % a.c.Hkv, ct = item / a.c.Hkv;
  const int slot0 = i0 == border - quota ? 0 : 1;   // the first workgroup's first or last item; the others' first
  for (int e = int(threadIdx.x); e < 16 * D / 4; e += 256) {
    const int c = e / (D / 4), d = e % (D / 4) * 4;
    float top = -__builtin_inff(), l = 0.f;
    kv_f4 v = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0; w <= w1; ++w) {
      const float* part = a.part + (int64_t(w) * 2 + (w == w0 ? slot0 : 0)) * part_floats<D>();
      const float mw = part[16 * D + c], lw = part[16 * D + 16 + c];
      const kv_f4 x = *reinterpret_cast<const kv_f4*>(part + c * D + d);
      const float now = fmaxf(top, mw);
      const float r = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now), k = mw == now ? 1.f : __builtin_amdgcn_exp2f(mw - now);
      l = l * r + lw * k;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = v[i] * r + x[i] * k;
      top = now;
    }
    const float il = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < 4; ++i) store_out<D>(a, s, head, ct * 16 + c, d + i, v[i] * il);
  }
}

int attention_wgs(int cus) { return 2 * cus; }

template <int D>
void attention_launch(const Kv8AttnArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_kv8_attention<D>, dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  hipLaunchKernelGGL(k_kv8_join<D>, dim3(unsigned(a.wgs - 1)), dim3(256), 0, stream, a);
}

}  // namespace

uint64_t kv8_workspace(int32_t D, int cus) {
  return round_up256(uint64_t(attention_wgs(cus)) * 2u * uint64_t(16 * D + 32) * 4u);
}

fluxbin_status launch_kv8_attention(Kv8AttnArgs a, int D, int cus, hipStream_t stream) {
  a.wgs = attention_wgs(cus);
  if (D == 64)
    attention_launch<64>(a, stream);
  else if (D == 128)
    attention_launch<128>(a, stream);
  else
    attention_launch<256>(a, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the attention");
}

}  // namespace fluxbin

// Attention over the paged 8-bit key/value cache on the matrix cores.
//
// For a cached head, the query rows that share it (the new tokens times the query heads of the group) are columns of
//   S^T = K Q^T          (16 tokens x 16 columns an instruction, 32 elements deep),   O^T += V^T P^T.
// Codes are exact in fp16, so K and V enter as codes and the scales, one per page and head, stay apart: the key's multiplies
// the score in fp32; the value's is added to the score as its logarithm, p = 2^(s + log2 sv - m), so that O sums p * code
// and the softmax sum is that of p / sv. With m the running maximum of s + log2 sv no p leaves fp16's range, however the
// scales of the pages differ. p is fed as the sum of two fp16 numbers, 21 bits or more where it is above 2^-3; numbers below
// are multiples of 2^-24, 2^-32 of the largest p (one number, 11 bits, put the results of ordinary prompts 0.00028 of their norm
// off 64 bits, against 0.00021 by the final rounding alone).
// The results of the first product have the layout that the second takes (a lane holds tokens 4 q + i of one column), and
// the cache stores values in that order: neither p nor the codes cross lanes.
#include "fluxbin_kv8_walk.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

// Floats of a partial result: 16 columns x D, then their maxima and sums. The workspace holds two for each workgroup (its
// first and its last item), then a record for each.
template <int D>
constexpr int part_floats() { return 16 * D + 32; }

// Workgroup (share of the units; a unit is a token tile of a sequence's column tile and head, in that order, or with a.whole
// all of them): goes over the
// items of its share; its wavefronts split an item's tiles and join their results in LDS. Items that it has only a part
// of go to the workspace.
//
// Bound by the stream of codes. A step's keys are requested when the last step's have been used and before its softmax, its
// values when the last step's have been used, so that a wavefront always has 8 KB or more on their way (D = 128); page
// numbers and scales come for 64 blocks of 16 tokens at a time, one per lane (a request for each block's page, and its wait
// before the codes' requests, cost a quarter of the time). Two contexts of 50000 and 65536 tokens, 8 cached heads of 128:
// 50 us, 4.7 TB/s, 6 of them the join; 32 of 256 to 8192 tokens: 43 us, 3.6 TB/s, where a workgroup's share is 18 steps of
// one or two items and every item's start (lengths, pages, codes, one after another) is seen.
// ONCE: every code is read by one workgroup only (one column tile), past the caches' ordinary order.
// TREE: rows attend what is before their sequence's first, and of its rows those that their masks name.
template <int D, bool ONCE, bool TREE>
__global__ void __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) k_kv8_attention(Kv8AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float lds_o[kWaves][16][D + 4];
  __shared__ float lds_m[kWaves][16], lds_l[kWaves][16];
  const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int m16 = lane & 15, q4 = lane >> 4;
  Walk<TREE> walk(a);
  const int64_t total = walk.total(), quota = quota_of(a, total);
  const int64_t u0 = quota * blockIdx.x;
  const int64_t u1 = u0 + quota < total ? u0 + quota : total;
  Joint joint = {};
  for (int64_t u = u0; u < u1;) {
    int64_t first;
    const Seq s = walk.find(u, first);
    if (s.n == 0) break;
    const int64_t rel = u - first;
    const int item = a.whole ? int(rel) : int(quotient(rel, s.nt));   // column tile, head
    const int ta = a.whole ? 0 : int(rel - int64_t(item) * s.nt);
    const int64_t room = a.whole ? s.nt : u1 - u;
    const int tb = room < s.nt - ta ? ta + int(room) : s.nt;
    const int ct = item / a.c.Hkv, head = item - ct * a.c.Hkv;

    const int col = ct * 16 + m16, ci = col / a.G, cg = col - ci * a.G;   // this lane's column
    const bool has = ci < s.n;
    const int pos = s.ctx - s.n + ci, fresh = s.ctx - s.n;   // position of the sequence's first row
    const uint64_t* mask = TREE ? a.masks + int64_t(s.start + (has ? ci : 0)) * a.words : nullptr;
    const int hi = has ? (a.causal && pos + 1 < s.end ? pos + 1 : s.end) : 0;
    const int lo = TREE ? tree_low(a, mask, fresh, s.n) : a.window > 0 && pos + 1 > a.window ? pos + 1 - a.window : 0;
    // tokens that all of the tile's columns attend
    const int i0 = ct * 16 / a.G, i1 = (ct * 16 + 15) / a.G, il = i1 < s.n ? i1 : s.n - 1;
    int all_hi = a.causal && s.ctx - s.n + i0 + 1 < s.end ? s.ctx - s.n + i0 + 1 : s.end;
    int all_lo = a.window > 0 && s.ctx - s.n + il + 1 > a.window ? s.ctx - s.n + il + 1 - a.window : 0;
    if (TREE) {
      all_hi = fresh < s.end ? fresh : s.end;
      all_lo = lo;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        const int other = __shfl_xor(all_lo, o);
        all_lo = other > all_lo ? other : all_lo;
      }
      all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    }

    kv_f4 o[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = kv_f4{0.f, 0.f, 0.f, 0.f};
    float mx = -__builtin_inff(), sum = 0.f;

    const int per = (tb - ta + kWaves - 1) / kWaves, w0 = ta + wave * per;
    const int w1 = w0 + per < tb ? w0 + per : tb;
    if (w0 < w1) {
      kv_h8 qf[D / 32];
      {
        const uint16_t* p = a.q + int64_t(s.start + (has ? ci : 0)) * a.qts + int64_t(head * a.G + (has ? cg : 0)) * a.qhs;
#pragma unroll
        for (int f = 0; f < D / 32; ++f) __builtin_memcpy(&qf[f], p + 32 * f + 8 * q4, 16);   // no such column: never stored
      }
      // blocks of 16 tokens 4 (t0 + w) + lane .. of 16 steps: page, key scale with the softmax's, value scale's logarithm
      // and reciprocal; blocks without a page as bits, which are masked as positions are
      int page;
      bool held;
      uint64_t holes;
      float kf, lv, iv;
      auto look = [&](int w) __attribute__((always_inline)) {   // requests; kf and iv hold what is in the cache
        const int tok = (s.t0 + w) * kTile + 16 * lane;
        page = tok < s.end && 16 * lane < (w1 - w) * kTile ? kv_page(a.c, s.b, tok) : -1;
        held = page >= 0;
        page = held ? page : 0;
        const int64_t at = int64_t(page) * a.c.Hkv + head;
        kf = a.c.ks[at];
        iv = a.c.vs[at];
      };
      auto scales = [&]() __attribute__((always_inline)) {
        const float v = iv > kLeast ? iv : kLeast;
        holes = __ballot(!held);
        kf = held ? kf * a.scale2 : 0.f;
        lv = __builtin_amdgcn_logf(v);
        iv = __builtin_amdgcn_rcpf(v);
      };
      auto offset = [&](int w, int j) __attribute__((always_inline)) {   // of block j of step w in the codes
        const int p = __builtin_amdgcn_readlane(page, ((w - w0) & 15) * 4 + j);
        const int tok = (s.t0 + w) * kTile + 16 * j;
        return kv_page_offset<D>(a.c, p, head) + int64_t((tok & ((1 << a.c.pshift) - 1)) >> 4) * 16 * D;
      };
      auto number = [&](float v, int l) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
      };
      kv_u4 kw[4][D / 64], vw[4][D / 64];
      int64_t off[4];
      auto load = [&](const uint8_t* base, kv_u4 (&v)[4][D / 64]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
            const kv_u4* p = reinterpret_cast<const kv_u4*>(base + off[j] + k * 1024 + uint32_t(lane * 16));
            v[j][k] = ONCE ? __builtin_nontemporal_load(p) : *p;
          }
      };
      look(w0);
#pragma unroll
      for (int j = 0; j < 4; ++j) off[j] = offset(w0, j);
      load(a.c.k, kw);
      load(a.c.v, vw);
      scales();
      for (int w = w0; w < w1; ++w) {
        const int tok = (s.t0 + w) * kTile;
        float kj[4], lj[4], rj[4];
        const uint32_t gone = uint32_t(holes >> (((w - w0) & 15) * 4)) & 15u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int l = ((w - w0) & 15) * 4 + j;
          kj[j] = number(kf, l);
          lj[j] = number(lv, l);
          rj[j] = number(iv, l);
        }
        kv_f4 sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          kv_f4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kw[j][k].x, kw[j][k].y), qf[2 * k], d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kw[j][k].z, kw[j][k].w), qf[2 * k + 1], d, 0, 0, 0);
          }
          sc[j] = d;
        }
        const int wn = w + 1 < w1 ? w + 1 : w;   // the last step's requests repeat it: without branches around them
        if (wn > w && ((wn - w0) & 15) == 0) {
          look(wn);
          scales();
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) off[j] = offset(wn, j);
        load(a.c.k, kw);
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[j][i] = __builtin_fmaf(sc[j][i], kj[j], lj[j]);
        if (tok < all_lo || tok + kTile > all_hi || gone != 0) {
          const uint64_t seen = TREE ? tree_bits(mask, a.words, tok - fresh, s.n) : 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int at = tok + 16 * j + 4 * q4 + i;
              bool in = at < hi && at >= lo && !(gone >> j & 1);
              if (TREE) in = in && (seen >> (16 * j + 4 * q4 + i) & 1);
              sc[j][i] = in ? sc[j][i] : -__builtin_inff();
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[j][i]);
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
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = __builtin_amdgcn_exp2f(sc[j + h][i] - base);
              sum = __builtin_fmaf(p, rj[j + h], sum);
              const _Float16 up = _Float16(p);
              ph[4 * h + i] = up;
              pl[4 * h + i] = _Float16(__builtin_fmaf(float(up), -1.f, p));
            }
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            const kv_h8 v = codes8(vw[j][d / 4][d % 4], vw[j + 1][d / 4][d % 4]);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph, o[d], 0, 0, 0);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl, o[d], 0, 0, 0);
          }
        }
        load(a.c.v, vw);
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
    const int cols = s.n * a.G - ct * 16;   // columns of this tile, 16 or more if it is full
    float* part = a.part + (int64_t(blockIdx.x) * 2 + (u == u0 ? 0 : 1)) * part_floats<D>();
    for (int e = int(threadIdx.x); e < 16 * D / 4; e += 64 * kWaves) {
      const int c = e / (D / 4), d = e % (D / 4) * 4;
      if (c >= cols) break;
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
        const float r = l == 0.f ? 0.f : 1.f / l;
        store_out(a, s, head, ct * 16 + c, d, v * r);
      } else {
        *reinterpret_cast<kv_f4*>(part + c * D + d) = v;
        if (d == 0) {
          part[16 * D + c] = top;
          part[16 * D + 16 + c] = l;
        }
      }
    }
    if (ta == 0 && tb < s.nt) joint = Joint{int(quotient(u + s.nt - 1, int(quota))), u == u0 ? 0 : 1, s.start, s.n, ct, head, {0, 0}};
    u += a.whole ? 1 : tb - ta;
    __syncthreads();   // lds of the next item
  }
  if (threadIdx.x == 0) reinterpret_cast<Joint*>(a.part + int64_t(a.wgs) * 2 * part_floats<D>())[blockIdx.x] = joint;
}

// Adds the partial results of an item (sequence, column tile, head) that several workgroups have worked on, in their order.
// A workgroup takes four columns of the item that a workgroup of the first kernel began and did not end; its threads are
// the columns' elements four at a time, times slices of the contributions, whose sums are added in LDS.
template <int D>
__global__ void __launch_bounds__(512) k_kv8_join(Kv8AttnArgs a) {
  constexpr int kSlices = 512 / D;
  __shared__ kv_f4 sums[512];
  __shared__ float tops[512], ls[512];
  const Joint it = reinterpret_cast<const Joint*>(a.part + int64_t(a.wgs) * 2 * part_floats<D>())[blockIdx.x];
  if (it.last == 0 || it.last >= a.wgs) return;
  const int tid = int(threadIdx.x), slice = tid / D, c = int(blockIdx.y) * 4 + tid % D / (D / 4), d = tid % (D / 4) * 4;
  const int w0 = int(blockIdx.x);
  const float* parts = a.part + int64_t(w0) * 2 * part_floats<D>();
  auto at = [&](int w) __attribute__((always_inline)) {   // contribution w of the item
    return parts + int64_t(2 * w + (w == 0 ? it.slot : 0)) * part_floats<D>();
  };
  float top = -__builtin_inff(), l = 0.f;
  kv_f4 v = {0.f, 0.f, 0.f, 0.f};
  const bool has = c < it.n * a.G - it.ct * 16;
  if (has) {
    for (int w = slice; w <= it.last - w0; w += 4 * kSlices) {
      float m[4], s[4];
      kv_f4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // contributions past the last repeat it, with no weight
        const int wi = w + i * kSlices;
        const float* p = at(wi <= it.last - w0 ? wi : it.last - w0);
        m[i] = p[16 * D + c];
        s[i] = p[16 * D + 16 + c];
        x[i] = *reinterpret_cast<const kv_f4*>(p + c * D + d);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (w + i * kSlices > it.last - w0) break;
        const float now = fmaxf(top, m[i]);
        const float r = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now), k = m[i] == now ? 1.f : __builtin_amdgcn_exp2f(m[i] - now);
        l = l * r + s[i] * k;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = v[e] * r + x[i][e] * k;
        top = now;
      }
    }
  }
  tops[tid] = top;
  ls[tid] = l;
  sums[tid] = v;
  __syncthreads();
  if (slice > 0 || !has) return;
  float most = top;
#pragma unroll
  for (int i = 1; i < kSlices; ++i) most = fmaxf(most, tops[tid + i * D]);
  v = kv_f4{0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    const float mi = tops[tid + i * D], r = mi == most ? 1.f : __builtin_amdgcn_exp2f(mi - most);
    const kv_f4 x = sums[tid + i * D];
    l = __builtin_fmaf(ls[tid + i * D], r, l);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(x[e], r, v[e]);
  }
  Seq q;
  q.start = it.start;
  q.n = it.n;
  store_out(a, q, it.head, it.ct * 16 + c, d, v * (l == 0.f ? 0.f : 1.f / l));
}

// ---------------------------------------------------------------------------------------------------------------------
// Prompt chunks. A workgroup takes 16 CT columns for each of its four wavefronts, of one sequence and head, and goes over all
// the tokens that they attend. A tile of 64 tokens is decoded once for all wavefronts: each turns a part of its codes into
// fp16 in LDS, in operand order, a tile ahead of its use, its requests two tiles ahead. Two sequences with 1024 and 700 new
// rows on 4096 and 1500 tokens, 64 heads of 128 over 8: 292 us, 500 TFLOP/s, the launches for sequences of few rows among
// them (a large fp16 matrix product: 1144; with p as one fp16 number, half of the second product's matrix work, 243 us); 4096
// rows on 8192 tokens 716. Counters: matrix cores 30%, vector instructions 38% of the SIMDs' time, wavefronts wait 21% of
// theirs and fill 59% of their places: the rest is uneven ends.
// ---------------------------------------------------------------------------------------------------------------------

// D = 256: 128 KB of LDS, one workgroup per CU; otherwise two.
template <int D, int CT>
__global__ void __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) k_kv8_chunk(Kv8AttnArgs a) {
  constexpr int kCols = 16 * CT * kWaves, kF = D / 32, kE = D / 16, kU = D / 64;
  static_assert(kWaves * 16 == kTile, "a block of 16 tokens for each wavefront to decode");
  __shared__ __attribute__((aligned(16))) kv_h8 lk[2][4 * kF * 64], lv[2][2 * kE * 64];   // [block][f][lane], [pair][e][lane]
  const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int m16 = lane & 15, q4 = lane >> 4, head = int(blockIdx.y);

  // the sequence and column block of this workgroup
  int b = 0, cb = int(blockIdx.x);
  for (;; b += 64) {
    if (b >= a.c.B) return;
    const int mine_b = b + lane;
    int nb = 0;
    if (mine_b < a.c.B) {
      const int o0 = a.c.offsets[mine_b], o1 = a.c.offsets[mine_b + 1];
      if (o0 >= 0 && o1 <= a.c.T && o1 > o0 && (o1 - o0) * a.G >= a.chunk_from) nb = ((o1 - o0) * a.G + kCols - 1) / kCols;
    }
    int upto = nb;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(upto, o);
      if (lane >= o) upto += u;
    }
    const uint64_t hit = __ballot(upto > cb);
    if (hit) {
      const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
      cb = __builtin_amdgcn_readlane(upto, l) - 1 - cb;   // the last rows, which attend the most tokens, first
      b += l;
      break;
    }
    cb -= __builtin_amdgcn_readlane(upto, 63);
  }
  const Seq s = seq_of<false>(a, b);
  const int first_pos = s.ctx - s.n;
  const int i_lo = cb * kCols / a.G, i_hi0 = (cb * kCols + kCols - 1) / a.G, i_hi = i_hi0 < s.n ? i_hi0 : s.n - 1;
  int end = a.causal && first_pos + i_hi + 1 < s.end ? first_pos + i_hi + 1 : s.end;
  end = end < 0 ? 0 : end;
  const int begin = a.window > 0 && first_pos + i_lo + 1 > a.window ? first_pos + i_lo + 1 - a.window : 0;
  const int t0 = begin / kTile, t1 = begin < end ? (end + kTile - 1) / kTile : t0;

  int hi[CT], lo[CT];
  kv_h8 qf[CT][kF];
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const int col = cb * kCols + (wave * CT + t) * 16 + m16, ci = col / a.G, cg = col - ci * a.G, pos = first_pos + ci;
    const bool has = ci < s.n;
    hi[t] = has ? (a.causal && pos + 1 < s.end ? pos + 1 : s.end) : 0;
    lo[t] = a.window > 0 && pos + 1 > a.window ? pos + 1 - a.window : 0;
    const uint16_t* p = a.q + int64_t(s.start + (has ? ci : 0)) * a.qts + int64_t(head * a.G + (has ? cg : 0)) * a.qhs;
#pragma unroll
    for (int f = 0; f < kF; ++f) __builtin_memcpy(&qf[t][f], p + 32 * f + 8 * q4, 16);   // no such column: never stored
  }
  // this wavefront's rows: tokens that all of them attend, and that some of them may
  const int c_lo = cb * kCols + wave * CT * 16, r_lo = c_lo / a.G, r_hi0 = (c_lo + CT * 16 - 1) / a.G;
  const int r_hi = r_hi0 < s.n ? r_hi0 : s.n - 1;
  const int all_hi = a.causal && first_pos + r_lo + 1 < s.end ? first_pos + r_lo + 1 : s.end;
  const int all_lo = a.window > 0 && first_pos + r_hi + 1 > a.window ? first_pos + r_hi + 1 - a.window : 0;
  const int any_hi = r_lo >= s.n ? 0 : (a.causal && first_pos + r_hi + 1 < s.end ? first_pos + r_hi + 1 : s.end);
  const int any_lo = a.window > 0 && first_pos + r_lo + 1 > a.window ? first_pos + r_lo + 1 - a.window : 0;

  kv_f4 o[CT][kE];
  // p = 2^(s - base); a base is kShift below a column's first scores' maximum, and moves when scores come to be more than
  // kShift + kSlack above it. limit: what is above it, or anything finite before the first.
  float base[CT], limit[CT], sum[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) {
#pragma unroll
    for (int e = 0; e < kE; ++e) o[t][e] = kv_f4{0.f, 0.f, 0.f, 0.f};
    base[t] = 0.f;
    limit[t] = -__builtin_inff();
    sum[t] = 0.f;
  }

  if (t0 < t1) {
    // blocks of 16 tokens of 16 tiles, one per lane: pages for the requests; scales; blocks without a page as bits
    int page = 0;
    uint64_t holes = 0;
    float kf = 0.f, lvs = 0.f, iv = 0.f;
    auto find = [&](int t) __attribute__((always_inline)) {
      const int tok = t * kTile + 16 * lane;
      return tok < end ? kv_page(a.c, b, tok) : -1;
    };
    auto look = [&](int t) __attribute__((always_inline)) {
      const int p = find(t);
      const int64_t at = int64_t(p < 0 ? 0 : p) * a.c.Hkv + head;
      const float ks = a.c.ks[at], vs = a.c.vs[at], v = vs > kLeast ? vs : kLeast;
      holes = __ballot(p < 0);
      kf = p < 0 ? 0.f : ks * a.scale2;
      lvs = __builtin_amdgcn_logf(v);
      iv = __builtin_amdgcn_rcpf(v);
    };
    auto number = [&](float v, int l) __attribute__((always_inline)) {
      return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
    };
    kv_u4 raw[2][kU];   // keys, values
    auto request = [&](int t) __attribute__((always_inline)) {   // this wavefront's block of tile t
      const int tok = t * kTile + 16 * wave;
      const int p = __builtin_amdgcn_readlane(page, ((t - t0) & 15) * 4 + wave);
      const int64_t off = kv_page_offset<D>(a.c, p, head) + int64_t((tok & ((1 << a.c.pshift) - 1)) >> 4) * 16 * D;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* base = h == 1 ? a.c.v : a.c.k;
#pragma unroll
        for (int k = 0; k < kU; ++k) raw[h][k] = *reinterpret_cast<const kv_u4*>(base + off + k * 1024 + uint32_t(lane * 16));
      }
    };
    auto decode = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        lk[buf][(wave * kF + 2 * k) * 64 + lane] = codes8(raw[0][k].x, raw[0][k].y);
        lk[buf][(wave * kF + 2 * k + 1) * 64 + lane] = codes8(raw[0][k].z, raw[0][k].w);
      }
#pragma unroll
      for (int k = 0; k < kU; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          reinterpret_cast<kv_h4*>(&lv[buf][((wave >> 1) * kE + 4 * k + e) * 64 + lane])[wave & 1] = codes4(raw[1][k][e]);
    };
    auto pages = [&](int t) __attribute__((always_inline)) {
      const int p = find(t);
      page = p < 0 ? 0 : p;
    };
    pages(t0);
    look(t0);
    request(t0);
    decode(0);
    request(t0 + 1 < t1 ? t0 + 1 : t0);
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1;
      // this tile is decoded, and everyone is done with the other buffer: a barrier for LDS only, requests stay on their way
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
      decode(buf ^ 1);
      const int tn = t + 2 < t1 ? t + 2 : t1 - 1;
      if (t + 2 < t1 && ((tn - t0) & 15) == 0) pages(tn);
      request(tn);
      if (t > t0 && ((t - t0) & 15) == 0) look(t);
      const int tok = t * kTile;
      if (tok >= any_hi || tok + kTile <= any_lo) continue;
      float kj[4], lj[4], rj[4];
      const uint32_t gone = uint32_t(holes >> (((t - t0) & 15) * 4)) & 15u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int l = ((t - t0) & 15) * 4 + j;
        kj[j] = number(kf, l);
        lj[j] = number(lvs, l);
        rj[j] = number(iv, l);
      }
      kv_f4 sc[CT][4];
#pragma unroll
      for (int f = 0; f < kF; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const kv_h8 k = lk[buf][(j * kF + f) * 64 + lane];
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            if (f == 0) sc[c][j] = kv_f4{0.f, 0.f, 0.f, 0.f};
            sc[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qf[c][f], sc[c][j], 0, 0, 0);
          }
        }
      kv_h8 ph[CT][2], pl[CT][2];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float add = lj[j] - base[c];
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[c][j][i] = __builtin_fmaf(sc[c][j][i], kj[j], add);
        }
        if (tok < all_lo || tok + kTile > all_hi || gone != 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int at = tok + 16 * j + 4 * q4 + i;
              sc[c][j][i] = at < hi[c] && at >= lo[c] && !(gone >> j & 1) ? sc[c][j][i] : -__builtin_inff();
            }
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[c][j][i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > limit[c])) {   // scores that are too large for the columns' bases, or their first
          // columns with none keep theirs; `by` is finite where there is a score
          const float by = top > limit[c] ? top - kShift : 0.f, r = limit[c] < 0.f ? 0.f : __builtin_amdgcn_exp2f(-by);
          sum[c] *= r;
#pragma unroll
          for (int e = 0; e < kE; ++e) o[c][e] *= r;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[c][j][i] -= by;
          base[c] += by;
          limit[c] = top > limit[c] ? kShift + kSlack : limit[c];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const float p0 = __builtin_amdgcn_exp2f(sc[c][j][i]), p1 = __builtin_amdgcn_exp2f(sc[c][j][i + 1]);
            // p before it is rounded: a weight on values of a tiny scale may be lost in p, but not in the sum
            sum[c] = __builtin_fmaf(p0, rj[j], sum[c]);
            sum[c] = __builtin_fmaf(p1, rj[j], sum[c]);
            // the first number cut off (a pair an instruction), the second the rest of it, rounded: 21 bits
            const kv_h2 up = __builtin_bit_cast(kv_h2, __builtin_amdgcn_cvt_pkrtz(p0, p1));
            const int at = 4 * (j & 1) + i;
            ph[c][j >> 1][at] = up.x;
            ph[c][j >> 1][at + 1] = up.y;
            pl[c][j >> 1][at] = _Float16(__builtin_fmaf(float(up.x), -1.f, p0));
            pl[c][j >> 1][at + 1] = _Float16(__builtin_fmaf(float(up.y), -1.f, p1));
          }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const kv_h8 v = lv[buf][(j * kE + e) * 64 + lane];
#pragma unroll
          for (int c = 0; c < CT; ++c) o[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[c][j], o[c][e], 0, 0, 0);
#pragma unroll
          for (int c = 0; c < CT; ++c) o[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl[c][j], o[c][e], 0, 0, 0);
        }
    }
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    sum[c] += __shfl_xor(sum[c], 16);
    sum[c] += __shfl_xor(sum[c], 32);
    const float r = sum[c] == 0.f ? 0.f : 1.f / sum[c];
#pragma unroll
    for (int e = 0; e < kE; ++e)
      store_out(a, s, head, cb * kCols + (wave * CT + c) * 16 + m16, 16 * e + 4 * q4, o[c][e] * r);
  }
}

int attention_wgs(int cus) { return 2 * cus; }

// Prompt chunks where their workgroups (four wavefronts of 32 columns each, 16 for D = 256) are one per CU at least: fresh
// causal prompts of 64 heads over 8, 128 / 256 / 512 rows 10.6 / 14.7 / 24 us, by the other kernel 8.6 / 15.8 / 40; of 32 heads
// over 32, 512 / 1000 / 1024 rows 22 / 37 / 45 and 21 / 81 / 62; of 8 over 1, 2048 / 4096 rows 66 / 127 and 54 / 185; 256 / 512
// rows of 64 over 8 on 8192 tokens 250 / 350 and 163 / 320 (few workgroups and long contexts: the other kernel splits them).
// And where sequences have on average as many columns as a workgroup: 64 of 12 rows, 64 heads over 8, 37 us and 34; of 16 rows
// 20 and 44. Sequences with fewer columns than one workgroup's among them go to the other kernel, which splits their
// tokens: one workgroup would take 2 us for every 64 tokens of a long context.
template <int D>
void attention_launch(Kv8AttnArgs a, int cus, hipStream_t stream) {
  constexpr int CT = D == 256 ? 1 : 2, cols = 16 * CT * kWaves;
  const int64_t blocks = int64_t(a.c.T) * a.G / cols;
  a.chunk_from = INT32_MAX;
  if (blocks * a.c.Hkv >= cus && blocks >= a.c.B) {
    a.chunk_from = a.c.B > 1 ? cols : 0;
    hipLaunchKernelGGL((k_kv8_chunk<D, CT>), dim3(unsigned(blocks + a.c.B), unsigned(a.c.Hkv)), dim3(64 * kWaves), 0, stream, a);
    if (a.c.B == 1) return;
  }
  // Short tables: items are not split, which saves the second kernel. Single tokens of up to 900 / 1800 tokens, whole and split:
  // one sequence of 32 heads 10.8 / 16 and 13.6 / 14 us, 8 of 64 heads over 8 11 / 16.5 and 14.7 / 17.
  a.whole = (int64_t(a.c.max_blocks) << a.c.pshift) <= 15 * kTile;
  // Single tokens of groups of up to 16 heads: 32 sequences of 256 to 8192 tokens 42.5 us with streaming requests, 45 without,
  // 4 of 16384 with 40 heads 109 and 121; eight tokens of 8 sequences of 8192 (four column tiles) 56.7 and 55.3.
  if (a.c.T <= a.c.B && a.G <= 16)
    hipLaunchKernelGGL((k_kv8_attention<D, true, false>), dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv8_attention<D, false, false>), dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  if (!a.whole) hipLaunchKernelGGL(k_kv8_join<D>, dim3(unsigned(a.wgs - 1), 4), dim3(512), 0, stream, a);
}

}  // namespace

// Trees of few columns (fluxbin_kv8_tree.hip has the others' kernel).
template <int D>
static void few_launch(Kv8AttnArgs a, hipStream_t stream) {
  // nearly all have one column tile: one node on 64 sequences of 4000 tokens, 64 heads over 8, 98 us, 106 without streaming requests
  if (int64_t(a.c.T) * a.G <= int64_t(a.c.B) * 16)
    hipLaunchKernelGGL((k_kv8_attention<D, true, true>), dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv8_attention<D, false, true>), dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  if (!a.whole) hipLaunchKernelGGL(k_kv8_join<D>, dim3(unsigned(a.wgs - 1), 4), dim3(512), 0, stream, a);
}

void launch_kv8_tree_few(Kv8AttnArgs a, int D, int cus, hipStream_t stream) {
  a.wgs = attention_wgs(cus);
  if (D == 64)
    few_launch<64>(a, stream);
  else if (D == 128)
    few_launch<128>(a, stream);
  else
    few_launch<256>(a, stream);
}

uint64_t kv8_workspace(int32_t D, int cus) {
  return round_up256(uint64_t(attention_wgs(cus)) * (2u * uint64_t(16 * D + 32) * 4u + sizeof(Joint)));
}

fluxbin_status launch_kv8_attention(Kv8AttnArgs a, int D, int cus, hipStream_t stream) {
  a.wgs = attention_wgs(cus);
  if (D == 64)
    attention_launch<64>(a, cus, stream);
  else if (D == 128)
    attention_launch<128>(a, cus, stream);
  else
    attention_launch<256>(a, cus, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the attention");
}

}  // namespace fluxbin

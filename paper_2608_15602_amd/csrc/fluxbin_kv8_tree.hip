// Attention of trees of drafted tokens over the paged 8-bit cache on the matrix cores, for trees of many columns (rows times
// query heads of a cached head). The mathematics are those of fluxbin_kv8_attention.hip: S^T = K Q^T and O^T += V^T P^T of codes
// that are exact in fp16, the scales apart, p as the sum of two fp16 numbers.
//
// A tree's rows all attend the whole history, which is long, and there are more columns than one wavefront takes: a workgroup
// decodes a tile of 64 tokens once, into LDS in operand order, for its four wavefronts of 16 CT columns each, and the tiles are
// shared out over all workgroups, of a long history over many of them, whose partial results a second kernel joins.
#include "fluxbin_kv8_walk.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

// A partial result in the order in which a workgroup holds it: [wavefront][column tile][16 elements][lane] four elements, then
// the columns' bases and sums. Two for each workgroup (its first and its last item), then a record for each.
template <int D, int CT>
constexpr int tree_part() { return 64 * CT * (D + 2); }

template <int D, int CT>
__global__ void __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) k_kv8_tree(Kv8AttnArgs a) {
  constexpr int kCols = 16 * CT * kWaves, kF = D / 32, kE = D / 16, kU = D / 64;
  __shared__ __attribute__((aligned(16))) kv_h8 lk[2][4 * kF * 64], lv[2][2 * kE * 64];   // [block][f][lane], [pair][e][lane]
  const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int m16 = lane & 15, q4 = lane >> 4;
  Walk<true> walk(a);
  const int64_t total = walk.total(), quota = quota_of(a, total);
  const int64_t u0 = quota * blockIdx.x;
  const int64_t u1 = u0 + quota < total ? u0 + quota : total;
  Joint joint = {};
  for (int64_t u = u0; u < u1;) {
    int64_t first;
    const Seq s = walk.find(u, first);
    if (s.n == 0) break;
    const int64_t rel = u - first;
    const int item = a.whole ? int(rel) : int(quotient(rel, s.nt));   // column block, head
    const int ta = a.whole ? 0 : int(rel - int64_t(item) * s.nt);
    const int64_t room = a.whole ? s.nt : u1 - u;
    const int tb = room < s.nt - ta ? ta + int(room) : s.nt;
    const int cb = item / a.c.Hkv, head = item - cb * a.c.Hkv;
    const int t0 = s.t0 + ta, t1 = s.t0 + tb, fresh = s.ctx - s.n;

    int lo[CT];
    const uint64_t* mask[CT];
    bool has[CT];
    kv_h8 qf[CT][kF];
    int all_lo = 0;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int col = cb * kCols + (wave * CT + t) * 16 + m16, ci = col / a.G, cg = col - ci * a.G;
      has[t] = ci < s.n;
      const int64_t row = s.start + (has[t] ? ci : 0);   // no such column: never stored
      mask[t] = a.masks + row * a.words;
      lo[t] = tree_low(a, mask[t], fresh, s.n);
      all_lo = lo[t] > all_lo ? lo[t] : all_lo;
      const uint16_t* p = a.q + row * a.qts + int64_t(head * a.G + (has[t] ? cg : 0)) * a.qhs;
#pragma unroll
      for (int f = 0; f < kF; ++f) __builtin_memcpy(&qf[t][f], p + 32 * f + 8 * q4, 16);
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const int other = __shfl_xor(all_lo, o);
      all_lo = other > all_lo ? other : all_lo;
    }
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    const int all_hi = fresh < s.end ? fresh : s.end;
    const bool work = cb * kCols + wave * CT * 16 < s.n * a.G;   // this wavefront has columns

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

    // blocks of 16 tokens of 16 tiles, one per lane: pages for the requests; scales; blocks without a page as bits
    int page = 0;
    uint64_t holes = 0;
    float kf = 0.f, lvs = 0.f, iv = 0.f;
    auto find = [&](int t) __attribute__((always_inline)) {
      const int tok = t * kTile + 16 * lane;
      return tok < s.end ? kv_page(a.c, s.b, tok) : -1;
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
        const uint8_t* from = h == 1 ? a.c.v : a.c.k;
#pragma unroll
        for (int k = 0; k < kU; ++k) raw[h][k] = *reinterpret_cast<const kv_u4*>(from + off + k * 1024 + uint32_t(lane * 16));
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
      if (!work) continue;
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
          const uint64_t seen = has[c] ? tree_bits(mask[c], a.words, tok - fresh, s.n) : 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int at = tok + 16 * j + 4 * q4 + i;
              const bool in = at < s.end && at >= lo[c] && !(gone >> j & 1) && (seen >> (16 * j + 4 * q4 + i) & 1);
              sc[c][j][i] = in ? sc[c][j][i] : -__builtin_inff();
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
    const bool whole = ta == 0 && tb == s.nt;
    float* part = a.part + (int64_t(blockIdx.x) * 2 + (u == u0 ? 0 : 1)) * tree_part<D, CT>();
    if (work) {
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        sum[c] += __shfl_xor(sum[c], 16);
        sum[c] += __shfl_xor(sum[c], 32);
        if (whole) {
          const float r = sum[c] == 0.f ? 0.f : 1.f / sum[c];
#pragma unroll
          for (int e = 0; e < kE; ++e)
            store_out(a, s, head, cb * kCols + (wave * CT + c) * 16 + m16, 16 * e + 4 * q4, o[c][e] * r);
        } else {
          kv_f4* to = reinterpret_cast<kv_f4*>(part) + (wave * CT + c) * kE * 64 + lane;
#pragma unroll
          for (int e = 0; e < kE; ++e) to[e * 64] = o[c][e];
          if (q4 == 0) {
            float* at = part + kCols * D + (wave * CT + c) * 16 + m16;
            at[0] = limit[c] < 0.f ? -__builtin_inff() : base[c];
            at[kCols] = sum[c];
          }
        }
      }
    }
    if (ta == 0 && tb < s.nt) joint = Joint{int(quotient(u + s.nt - 1, int(quota))), u == u0 ? 0 : 1, s.start, s.n, cb, head, {0, 0}};
    u += a.whole ? 1 : tb - ta;
    __syncthreads();   // lds of the next item
  }
  if (threadIdx.x == 0) reinterpret_cast<Joint*>(a.part + int64_t(a.wgs) * 2 * tree_part<D, CT>())[blockIdx.x] = joint;
}

// Adds the partial results of the items that several workgroups have worked on, in their order. The items are listed first;
// then a workgroup takes 16 columns and 64 elements of one at a time: 256 threads four elements each, in four slices of the
// contributions, whose sums are added in LDS.
constexpr int kJoinWgs = 1024;

template <int D, int CT>
__global__ void __launch_bounds__(1024) k_kv8_tree_join(Kv8AttnArgs a) {
  constexpr int kCols = 16 * CT * kWaves, kE = D / 16, kPieces = CT * kWaves * (kE / 4);
  __shared__ kv_f4 sums[1024];
  __shared__ float tops[1024], ls[1024];
  __shared__ int list[kJoinWgs], found[16];
  const Joint* joints = reinterpret_cast<const Joint*>(a.part + int64_t(a.wgs) * 2 * tree_part<D, CT>());
  const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = tid < a.wgs ? joints[tid].last : 0;
  const uint64_t mine = __ballot(last > tid && last < a.wgs);
  if (lane == 0) found[wave] = __popcll((unsigned long long)mine);
  __syncthreads();
  int at = 0, count = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) at += found[w];
    count += found[w];
  }
  if (mine >> lane & 1) list[at + __popcll((unsigned long long)(mine & ((uint64_t(1) << lane) - 1)))] = tid;
  __syncthreads();
  const int slice = tid >> 8, e4 = (tid >> 6) & 3;
  for (int64_t p = blockIdx.x; p < int64_t(count) * kPieces; p += gridDim.x) {
    const int w0 = list[p / kPieces], piece = int(p % kPieces), tile = piece / (kE / 4), e = (piece % (kE / 4)) * 4 + e4;
    const Joint it = joints[w0];
    const int n = it.last - w0 + 1, col = tile * 16 + (lane & 15);
    if (it.ct * kCols + tile * 16 >= it.n * a.G) continue;   // no such columns; the same for the whole workgroup
    const float* parts = a.part + int64_t(w0) * 2 * tree_part<D, CT>();
    float top = -__builtin_inff(), l = 0.f;
    kv_f4 v = {0.f, 0.f, 0.f, 0.f};
    for (int w = slice; w < n; w += 16) {
      float m[4], s[4];
      kv_f4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // contributions past the last repeat it, with no weight
        const int wi = w + 4 * i < n ? w + 4 * i : n - 1;
        const float* from = parts + int64_t(2 * wi + (wi == 0 ? it.slot : 0)) * tree_part<D, CT>();
        m[i] = from[kCols * D + col];
        s[i] = from[kCols * D + kCols + col];
        x[i] = reinterpret_cast<const kv_f4*>(from)[(tile * kE + e) * 64 + lane];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (w + 4 * i >= n) break;
        const float now = fmaxf(top, m[i]);
        const float r = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now), k = m[i] == now ? 1.f : __builtin_amdgcn_exp2f(m[i] - now);
        l = l * r + s[i] * k;
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d] = v[d] * r + x[i][d] * k;
        top = now;
      }
    }
    __syncthreads();   // the piece before
    tops[tid] = top;
    ls[tid] = l;
    sums[tid] = v;
    __syncthreads();
    if (slice > 0) continue;
    float most = top;
#pragma unroll
    for (int i = 1; i < 4; ++i) most = fmaxf(most, tops[tid + 256 * i]);
    v = kv_f4{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float mi = tops[tid + 256 * i], r = mi == most ? 1.f : __builtin_amdgcn_exp2f(mi - most);
      const kv_f4 x = sums[tid + 256 * i];
      l = __builtin_fmaf(ls[tid + 256 * i], r, l);
#pragma unroll
      for (int d = 0; d < 4; ++d) v[d] = __builtin_fmaf(x[d], r, v[d]);
    }
    Seq q;
    q.start = it.start;
    q.n = it.n;
    store_out(a, q, it.head, it.ct * kCols + col, 16 * e + 4 * (lane >> 4), v * (l == 0.f ? 0.f : 1.f / l));
  }
}

int tree_wgs(int cus) { return 2 * cus < kJoinWgs ? 2 * cus : kJoinWgs; }

template <int D>
constexpr int most_tiles() { return D == 256 ? 1 : 2; }   // column tiles of a wavefront

template <int D, int CT>
void many_launch(Kv8AttnArgs a, hipStream_t stream) {
  a.col_shift = CT == 1 ? 6 : 7;
  hipLaunchKernelGGL((k_kv8_tree<D, CT>), dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  if (!a.whole) hipLaunchKernelGGL((k_kv8_tree_join<D, CT>), dim3(unsigned(a.wgs)), dim3(1024), 0, stream, a);
}

template <int D>
void tree_launch(Kv8AttnArgs a, int cus, hipStream_t stream) {
  const int64_t mean = ceil_div(int64_t(a.c.T) * a.G, a.c.B);   // columns of a sequence and cached head
  if (mean <= 16) {
    a.col_shift = 4;
    launch_kv8_tree_few(a, D, cus, stream);
    return;
  }
  a.wgs = tree_wgs(cus);
  a.chunk_from = INT32_MAX;
  a.whole = (int64_t(a.c.max_blocks) << a.c.pshift) <= 15 * kTile;
  if (mean <= 64)
    many_launch<D, 1>(a, stream);
  else
    many_launch<D, most_tiles<D>()>(a, stream);
}

}  // namespace

uint64_t kv8_tree_workspace(int32_t D, int cus) {
  const uint64_t columns = D == 256 ? 64 : 128;
  const uint64_t many = round_up256(uint64_t(tree_wgs(cus)) * (2u * columns * (uint64_t(D) + 2) * 4u + sizeof(Joint)));
  const uint64_t few = kv8_workspace(D, cus);
  return many > few ? many : few;
}

fluxbin_status launch_kv8_tree_attention(Kv8AttnArgs a, int D, int cus, hipStream_t stream) {
  if (D == 64)
    tree_launch<64>(a, cus, stream);
  else if (D == 128)
    tree_launch<128>(a, cus, stream);
  else
    tree_launch<256>(a, cus, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the attention of trees");
}

}  // namespace fluxbin

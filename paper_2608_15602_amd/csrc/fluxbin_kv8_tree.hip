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
// the columns' bases and sums. Two for each workgroup (its first and its last item), then a record for each, then the records'
// `last` alone.
template <int D, int CT>
constexpr int tree_part() { return 64 * CT * (D + 2); }

// p less one half of `up`, exactly.
template <int HI>
__device__ __forceinline__ float rest(kv_h2 up, float p) {
  float r;
  if (HI)
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(up), "v"(p));
  else
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(up), "v"(p));
  return r;
}

// A step's matrix instructions, each followed by vector instructions that run beside it (2 to 6 of them: equal; in any order: 2%
// slower).
template <int MATRIX, int VECTOR>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < MATRIX; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Workgroup: a share of the units, as k_kv8_attention's; an item is 64 CT columns of a sequence and cached head. A tile's decoding,
// scores, weights and output are one barrier apart: the next tile is decoded, from requests sent a tile before, beside the last
// products, and the weights of the tile's second half beside those of its first; the row sums' 16 CT fused steps, two chains, come
// behind the last product, where the compiler puts them and no product runs beside them. CT = 2 halves the traffic from LDS for a column;
// its 256 registers allow two workgroups per CU, as do 64 KB of LDS (D = 256: 128 KB, one).
// Heads of 128, 64 over 8: trees of 48 to 64 rows on 8 sequences of 256 to 8192 tokens 94 us a call, 80 of them here and 13 the join
// (52 MB of partial results), 428 TFLOP/s by the formula's products, 640 by those done; 13 to 16 rows on 50000 and 65536 tokens
// 105 us, the join 10, 790 by those done. A wavefront takes 4770 cycles a tile beside another one's, of which its 96 matrix
// instructions fill 1536 and its 340 others 1900 at their issue; the clock is then at 1.95 GHz. Without the requests the second
// call takes 20 us less, with requests that hit the cache 3, without the second number of p 14, without exponentials 3.
// Tried, no faster: products of 32 x 32 with their operands (94, 113), wavefront priorities, uneven shares for a CU's two
// workgroups, one workgroup per CU, requests two tiles ahead (registers spill: 99 -> 111, 113 -> 123), pages and scales of the
// next 16 tiles looked up a tile before they are needed (99, 115 against 99, 113 on the same day).
template <int D, int CT>
__global__ void __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) k_kv8_tree(Kv8AttnArgs a) {
  constexpr int kCols = 16 * CT * kWaves, kF = D / 32, kE = D / 16, kU = D / 64, kSteps = 2 * kF;
  __shared__ __attribute__((aligned(16))) kv_h8 lk[2][4 * kF * 64];       // [block of 16 tokens][f][lane]
  __shared__ __attribute__((aligned(16))) kv_h4 lv[2][2 * kE * 2 * 64];   // [pair of blocks][e][block][lane]
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
    int rows[CT];   // the columns' rows, -1: there is no such column
    kv_h8 qf[CT][kF];
    int all_lo = 0;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int col = cb * kCols + (wave * CT + t) * 16 + m16, ci = col / a.G, cg = col - ci * a.G;
      const bool has = ci < s.n;
      const int64_t row = s.start + (has ? ci : 0);   // no such column: never stored
      rows[t] = has ? s.start + ci : -1;
      lo[t] = tree_low(a, a.masks + row * a.words, fresh, s.n);
      all_lo = lo[t] > all_lo ? lo[t] : all_lo;
      const uint16_t* p = a.q + row * a.qts + int64_t(head * a.G + (has ? cg : 0)) * a.qhs;
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

    // blocks of 16 tokens of 16 tiles, one per lane: their places in the codes, for the requests; scales; blocks without a page
    // as bits
    int64_t place = 0;
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
    auto places = [&](int t) __attribute__((always_inline)) {
      const int p = find(t), tok = t * kTile + 16 * lane;
      place = kv_page_offset<D>(a.c, p < 0 ? 0 : p, head) + ((tok & ((1 << a.c.pshift) - 1)) >> 4) * 16 * D;
    };
    auto number = [&](float v, int l) __attribute__((always_inline)) {
      return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
    };
    kv_u4 raw[2][kU];   // keys, values
    auto request = [&](int t) __attribute__((always_inline)) {   // this wavefront's block of tile t
      const int l = ((t - t0) & 15) * 4 + wave;
      const uint32_t lo32 = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(uint64_t(place))), l));
      const uint32_t hi32 = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(uint64_t(place) >> 32)), l));
      const int64_t off = int64_t((uint64_t(hi32) << 32) | lo32);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < kU; ++k)
          raw[h][k] = *reinterpret_cast<const kv_u4*>((h == 1 ? a.c.v : a.c.k) + off + k * 1024 + uint32_t(lane * 16));
    };
    // One of kSteps parts of a tile's decoding: 8 elements of the keys' units, or 4 of two of the values'.
    auto decode = [&](int buf, int i) __attribute__((always_inline)) {
      if (i < 2 * kU) {
        const kv_u4 w = raw[0][i >> 1];
        lk[buf][(wave * kF + i) * 64 + lane] = i & 1 ? codes8(w.z, w.w) : codes8(w.x, w.y);
      } else {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int e = 2 * (i - 2 * kU) + n;
          lv[buf][(((wave >> 1) * kE + e) * 2 + (wave & 1)) * 64 + lane] = codes4(raw[1][e >> 2][e & 3]);
        }
      }
    };
    places(t0);
    look(t0);
    request(t0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) decode(0, i);
    request(t0 + 1 < t1 ? t0 + 1 : t0);
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1, tok = t * kTile;
      // this tile is decoded, and everyone is done with the other buffer: a barrier for LDS only, requests stay on their way
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
      if (t > t0 && ((t - t0) & 15) == 0) look(t);
      // the next tile's decoding is beside the last products, and its request, for the tile after it, behind them: it has a
      // tile's time to come
      auto ahead = [&]() __attribute__((always_inline)) {
        if (t + 2 < t1 && ((t + 2 - t0) & 15) == 0) places(t + 2);
        request(t + 2 < t1 ? t + 2 : t1 - 1);
      };
      if (!work) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) decode(buf ^ 1, i);
        ahead();
        continue;
      }
      // S: kSteps steps of 2 CT products (half of the tile, 32 elements), operands two steps ahead.
      kv_h8 kx[3][2];
      auto keys = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) kx[i % 3][j] = lk[buf][((2 * (i / kF) + j) * kF + i % kF) * 64 + lane];
      };
      kv_f4 sc[CT][4];
      keys(0);
      keys(1);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (i + 2 < kSteps) keys(i + 2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            kv_f4& d = sc[c][2 * (i / kF) + j];
            if (i % kF == 0) d = kv_f4{0.f, 0.f, 0.f, 0.f};
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kx[i % 3][j], qf[c][i % kF], d, 0, 0, 0);
          }
      }

      kv_h8 vx[4];
      auto values = [&](int g) __attribute__((always_inline)) {   // half g / kE of the tile, 16 elements
        const kv_h4* at = &lv[buf][g * 128 + lane];
        const kv_h4 x = at[0], y = at[64];
        vx[g & 3] = kv_h8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      };
      const uint32_t gone = uint32_t(holes >> (((t - t0) & 15) * 4)) & 15u;
      float rj[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int l = ((t - t0) & 15) * 4 + j;
        const float kj = number(kf, l), lj = number(lvs, l);
        rj[j] = number(iv, l);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          const float add = lj - base[c];
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[c][j][i] = __builtin_fmaf(sc[c][j][i], kj, add);
        }
      }
      if (tok < all_lo || tok + kTile > all_hi || gone != 0) {
        uint64_t in = s.end - tok < 64 ? (uint64_t(1) << (s.end > tok ? s.end - tok : 0)) - 1 : ~uint64_t(0);
#pragma unroll
        for (int j = 0; j < 4; ++j) in &= gone >> j & 1 ? ~(uint64_t(0xFFFF) << (16 * j)) : ~uint64_t(0);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          uint64_t v = rows[c] < 0 ? 0 : in & tree_bits(a.masks + int64_t(rows[c]) * a.words, a.words, tok - fresh, s.n);
          if (lo[c] > tok) v = lo[c] - tok < 64 ? v & (~uint64_t(0) << (lo[c] - tok)) : 0;
          v >>= 4 * q4;   // from this lane's first token on
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[c][j][i] = v >> (16 * j + i) & 1 ? sc[c][j][i] : -__builtin_inff();
        }
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[c][j][i]);
        if (__any(top > limit[c])) {   // scores that are too large for the columns' bases, or their first
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
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
      }
      // P and O: the weights of one half of the tile are made beside the products of the other.
      kv_h8 ph[2][CT], pl[2][CT];
      auto weights = [&](int h, int n) __attribute__((always_inline)) {   // two of a half's 8 CT of a lane
        const int c = n >> 2, j = (n >> 1) & 1, i = 2 * (n & 1);
        const float p0 = __builtin_amdgcn_exp2f(sc[c][2 * h + j][i]), p1 = __builtin_amdgcn_exp2f(sc[c][2 * h + j][i + 1]);
        // p before it is rounded: a weight on values of a tiny scale may be lost in p, but not in the sum (built behind the products)
        sum[c] = __builtin_fmaf(p0, rj[2 * h + j], sum[c]);
        sum[c] = __builtin_fmaf(p1, rj[2 * h + j], sum[c]);
        // the first number cut off (a pair an instruction), the second the rest of it, rounded: 21 bits
        const kv_h2 up = __builtin_bit_cast(kv_h2, __builtin_amdgcn_cvt_pkrtz(p0, p1));
        ph[h][c][4 * j + i] = up.x;
        ph[h][c][4 * j + i + 1] = up.y;
        pl[h][c][4 * j + i] = _Float16(rest<0>(up, p0));
        pl[h][c][4 * j + i + 1] = _Float16(rest<1>(up, p1));
      };
#pragma unroll
      for (int g = 0; g < 3; ++g) values(g);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 4 * CT; ++n) weights(0, n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < 2 * kE; ++g) {
        const int h = g / kE, e = g % kE;
        if (g + 3 < 2 * kE) values(g + 3);
        if (h == 0) {
#pragma unroll
          for (int n = e * 4 * CT / kE; n < (e + 1) * 4 * CT / kE; ++n) weights(1, n);
        } else {
#pragma unroll
          for (int n = e * kSteps / kE; n < (e + 1) * kSteps / kE; ++n) decode(buf ^ 1, n);
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vx[g & 3], ph[h][c], o[c][e], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vx[g & 3], pl[h][c], o[c][e], 0, 0, 0);
        interleave<2 * CT, 4>();
      }
      ahead();
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
  if (threadIdx.x == 0) {
    Joint* joints = reinterpret_cast<Joint*>(a.part + int64_t(a.wgs) * 2 * tree_part<D, CT>());
    joints[blockIdx.x] = joint;
    reinterpret_cast<int*>(joints + a.wgs)[blockIdx.x] = joint.last;
  }
}

// Adds the partial results of the items that several workgroups have worked on, in their order. The items are listed first;
// then a workgroup takes 16 columns and 64 elements of one at a time, its wavefronts each a share of the contributions, 4 KB
// of one at a time; their sums are added in LDS. 512 workgroups' results, 52 MB, take 13 us: 4 TB/s.
constexpr int kJoinWgs = 1024;   // at most as many records

template <int D, int CT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_kv8_tree_join(Kv8AttnArgs a) {
  constexpr int kCols = 16 * CT * kWaves, kE = D / 16, kPieces = CT * kWaves * (kE / 4);
  __shared__ kv_f4 sums[WAVES][4][64];
  __shared__ float tops[WAVES][16], ls[WAVES][16];
  __shared__ int list[kJoinWgs], found[kJoinWgs / 64];
  const Joint* joints = reinterpret_cast<const Joint*>(a.part + int64_t(a.wgs) * 2 * tree_part<D, CT>());
  const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m16 = lane & 15;
  uint64_t mine[kJoinWgs / (64 * WAVES)];   // of 64 records each
#pragma unroll
  for (int i = 0; i < kJoinWgs / (64 * WAVES); ++i) {
    const int r = i * 64 * WAVES + tid, last = r < a.wgs ? reinterpret_cast<const int*>(joints + a.wgs)[r] : 0;
    mine[i] = __ballot(last > r && last < a.wgs);
    if (lane == 0) found[i * WAVES + wave] = __popcll((unsigned long long)mine[i]);
  }
  __syncthreads();
  int count = 0;
#pragma unroll
  for (int i = 0; i < kJoinWgs / 64; ++i) {
    if (i % WAVES == wave && (mine[i / WAVES] >> lane & 1))
      list[count + __popcll((unsigned long long)(mine[i / WAVES] & ((uint64_t(1) << lane) - 1)))] = i * 64 + lane;
    count += found[i];
  }
  __syncthreads();
  for (int64_t p = blockIdx.x; p < int64_t(count) * kPieces; p += gridDim.x) {
    const int w0 = list[p / kPieces], piece = int(p % kPieces), tile = piece / (kE / 4), e0 = (piece % (kE / 4)) * 4;
    const Joint it = joints[w0];
    const int n = it.last - w0 + 1, col = tile * 16 + m16;
    if (it.ct * kCols + tile * 16 >= it.n * a.G) continue;   // no such columns; the same for the whole workgroup
    const float* parts = a.part + int64_t(w0) * 2 * tree_part<D, CT>();
    float top = -__builtin_inff(), l = 0.f;
    kv_f4 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = kv_f4{0.f, 0.f, 0.f, 0.f};
    for (int w = wave; w < n; w += 2 * WAVES) {
      float m[2], s[2];
      kv_f4 x[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {   // contributions past the last repeat it, with no weight
        const int wi = w + WAVES * i < n ? w + WAVES * i : n - 1;
        const float* from = parts + int64_t(2 * wi + (wi == 0 ? it.slot : 0)) * tree_part<D, CT>();
        m[i] = from[kCols * D + col];
        s[i] = from[kCols * D + kCols + col];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = reinterpret_cast<const kv_f4*>(from)[(tile * kE + e0 + e) * 64 + lane];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (w + WAVES * i >= n) break;
        const float now = fmaxf(top, m[i]);
        const float r = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now), k = m[i] == now ? 1.f : __builtin_amdgcn_exp2f(m[i] - now);
        l = l * r + s[i] * k;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < 4; ++d) v[e][d] = v[e][d] * r + x[i][e][d] * k;
        top = now;
      }
    }
    __syncthreads();   // the piece before
    if (lane < 16) {
      tops[wave][lane] = top;
      ls[wave][lane] = l;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][e][lane] = v[e];
    __syncthreads();
    if (wave >= 4) continue;   // the others have a quarter of the elements each
    float most = tops[0][m16];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) most = fmaxf(most, tops[i][m16]);
    kv_f4 y = {0.f, 0.f, 0.f, 0.f};
    l = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float mi = tops[i][m16], r = mi == most ? 1.f : __builtin_amdgcn_exp2f(mi - most);
      const kv_f4 x = sums[i][wave][lane];
      l = __builtin_fmaf(ls[i][m16], r, l);
#pragma unroll
      for (int d = 0; d < 4; ++d) y[d] = __builtin_fmaf(x[d], r, y[d]);
    }
    Seq q;
    q.start = it.start;
    q.n = it.n;
    store_out(a, q, it.head, it.ct * kCols + col, 16 * (e0 + wave) + 4 * (lane >> 4), y * (l == 0.f ? 0.f : 1.f / l));
  }
}

int tree_wgs(int cus) { return 2 * cus < kJoinWgs ? 2 * cus : kJoinWgs; }

template <int D>
constexpr int most_tiles() { return D == 256 ? 1 : 2; }   // column tiles of a wavefront

template <int D, int CT>
void many_launch(Kv8AttnArgs a, int64_t items, int64_t tiles, hipStream_t stream) {
  a.col_shift = CT == 1 ? 6 : 7;
  hipLaunchKernelGGL((k_kv8_tree<D, CT>), dim3(unsigned(a.wgs)), dim3(64 * kWaves), 0, stream, a);
  if (a.whole) return;
  // Contributions to an item, as far as the host can tell. Many: 16 wavefronts to a piece. One sequence of 100000 tokens and 16 heads
  // over one, 64, 128 and 256 columns, 38, 44 and 45 us, 62, 68 and 59 with 4; 16 of 2000, 256 columns, 8 contributions, 29 and 26; 32: equal.
  const int64_t each = a.wgs / items;
  if ((each < tiles / kWaves ? each : tiles / kWaves) >= 64)
    hipLaunchKernelGGL((k_kv8_tree_join<D, CT, 16>), dim3(unsigned(a.wgs)), dim3(1024), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv8_tree_join<D, CT, 4>), dim3(unsigned(4 * a.wgs)), dim3(256), 0, stream, a);
}

// Which kernel, by columns of a sequence and cached head (their mean: only the device knows each) and by the table's length,
// which bounds the contexts. Where it is far longer than they are, short items are split and joined all the same (table four times
// as long and more, heads of 128: one sequence of 200 tokens, 8 columns 7.4 -> 9.7, 64 columns 8 -> 15; 8 of 900, 64 columns 12.5 -> 21;
// 64 of 300, 32 columns 15 -> 28, 128 columns 28 -> 41; 8 of 8192 and 64 of 2000 as long as before), and the steps below are more than
// there are (heads of 256, 32 of 400 to 2048, 16 columns 27 -> 36). Graph-timed, us:
//   Long tables, 16 columns at a time / 64 a workgroup. Up to 16 columns, the first: every code is decoded once in either, for one
//   wavefront; one node of 64 heads over 8 on 64 sequences of 4000 tokens 98 / 112, heads of 64 42 / 56 (800 to 4000 tokens). Heads of
//   256 on middle sizes, whose join has more to add, the second. 426 cases of one sequence to 64, even and ragged, mean of the first's
//   time over the second's by steps (below): 9 to 16 columns, steps 0, 1, 2, 4, 8, 10, 11, 12, 16, 20 and more: 0.92, 0.97, 1.11, 1.31,
//   1.25, 1.07, 0.93, 1.02, 0.98, 0.78 (4 sequences of 1600 to 8192 tokens, 8 heads 43 / 36; 32 of 400 to 2048, 2 heads 36 / 27; 64 of
//   800 to 4000, 8 heads 145 / 182; one of 2000 16 / 18; steps of 1 are about even, but one of 16384, 2 heads, 27 / 22); up to 8
//   columns, steps 1, 2, 3, 4, 7, 8, 10, 16: 0.86, 0.92, 1.06, 1.07, 0.99, 1.02 (even ones 0.9), 0.95, 0.85.
//   17 to 32 columns are two tiles, whose codes the first decodes twice: 32 on 64 of 240 to 1200 tokens, 8 heads of 128 50 / 43, of 64
//   41 / 33; 64 of 800 to 4000, 32 heads 460 / 329, 271 / 219; 8 of 800 to 4096, 8 heads 25 / 26, 20 / 21, 4 of 8192 even 35 / 31.
//   64 / 128 columns a workgroup, heads of 128 over 8: 4 sequences of 8192 tokens, 64, 96, 128 columns 30, 41, 44 / 37, 40, 43; 2 of
//   32768 49, 75, 78 / 56, 60, 65.
//   Tables of up to 15 tiles, whose items are not split (a.whole): 16 at a time where those are at most two a CU: 8 sequences of 900
//   tokens, 64, 128, 256, 512 columns 13, 18, 33, 60 / 24, 25, 26, 37 (64 a workgroup) / 31, 33, 34, 36 (128); 64 of 300, 32, 64, 128
//   columns 22, 41, 75 / 17, 20, 33 / 20, 25, 30; 256 of 500, 4 columns of heads of 256 135 / 173, 16 columns 161 / 174.
template <int D>
void tree_launch(Kv8AttnArgs a, int cus, hipStream_t stream) {
  const int64_t mean = ceil_div(int64_t(a.c.T) * a.G, a.c.B), tiles = ceil_div(int64_t(a.c.max_blocks) << a.c.pshift, kTile);
  const auto items = [&](int columns) { return int64_t(a.c.B) * ceil_div(mean, columns) * a.c.Hkv; };
  a.chunk_from = INT32_MAX;
  a.whole = tiles <= 15;
  const int64_t steps = items(16) * tiles / (2 * cus);   // of 16 columns and a workgroup, if contexts are as long as the table
  bool few;
  if (mean <= 16)
    few = a.whole || D != 256 || steps < (mean > 8 ? 1 : 3) || steps >= (mean > 8 ? 11 : 8);
  else if (a.whole)
    few = items(16) <= 2 * cus;
  else
    few = D != 256 && mean <= 32 && steps < 24;
  if (few) {
    a.col_shift = 4;
    launch_kv8_tree_few(a, D, cus, stream);
    return;
  }
  a.wgs = D == 256 ? tree_wgs(cus) / 2 : tree_wgs(cus);   // as many as run at a time
  if (mean <= 64 || (a.whole && items(64) <= 2 * cus))
    many_launch<D, 1>(a, items(64), tiles, stream);
  else
    many_launch<D, most_tiles<D>()>(a, items(64 * most_tiles<D>()), tiles, stream);
}

}  // namespace

uint64_t kv8_tree_workspace(int32_t D, int cus) {
  const uint64_t columns = D == 256 ? 64 : 128;
  const uint64_t many = round_up256(uint64_t(tree_wgs(cus)) * (2u * columns * (uint64_t(D) + 2) * 4u + sizeof(Joint) + 4u));
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

// What the attention kernels over the paged 8-bit cache share: codes as operands, the sequences of a call as a wavefront goes
// over them, masks of drafted trees, and results.
#pragma once

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

__device__ __forceinline__ kv_h4 codes4(uint32_t a) {
  const kv_h2 off = {_Float16(-1152.f), _Float16(-1152.f)};
  const uint32_t k = 0x64646464u;
  const kv_h2 x = __builtin_bit_cast(kv_h2, __builtin_amdgcn_perm(k, a, 0x04010400u)) + off;
  const kv_h2 y = __builtin_bit_cast(kv_h2, __builtin_amdgcn_perm(k, a, 0x04030402u)) + off;
  return kv_h4{x.x, x.y, y.x, y.y};
}

// Work of a sequence: column tiles (of 16 columns, for trees of what a wavefront or a workgroup takes; row i of the sequence and
// head g of the group are column i G + g), and token tiles that some row of it attends.
struct Seq {
  int b, start, n, ctx, end;   // first row, rows, tokens, attendable tokens
  int qt, t0, nt;              // column tiles, first token tile, token tiles
};

template <bool TREE>
__device__ __forceinline__ Seq seq_of(const Kv8AttnArgs& a, int b) {
  Seq s;
  const int o0 = a.c.offsets[b], o1 = a.c.offsets[b + 1];
  s.start = o0;
  s.n = o0 >= 0 && o1 <= a.c.T && o1 > o0 ? o1 - o0 : 0;
  if (TREE && s.n > 64 * a.words) s.n = 0;
  s.ctx = kv_context(a.c, b);
  const int cap = a.c.max_blocks << a.c.pshift;
  s.end = s.ctx < cap ? s.ctx : cap;
  int begin = 0;
  // of a tree, a row may attend only cached tokens
  if (a.window > 0 && s.ctx - s.n + (TREE ? 0 : 1) > a.window) begin = s.ctx - s.n + (TREE ? 0 : 1) - a.window;
  if (begin > s.end) begin = s.end;
  const int shift = TREE ? a.col_shift : 4;   // columns of a tile
  s.qt = s.n * a.G >= a.chunk_from ? 0 : (s.n * a.G + (1 << shift) - 1) >> shift;   // the others are the prompt chunks' kernel's
  s.t0 = begin / kTile;
  s.nt = (s.end + kTile - 1) / kTile - s.t0;
  if (s.nt < 1) s.nt = 1;   // nothing to attend: one tile, all of it masked
  return s;
}

__device__ __forceinline__ int64_t units_of(const Kv8AttnArgs& a, const Seq& s) {
  return int64_t(s.qt) * a.c.Hkv * (a.whole ? 1 : s.nt);
}

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uint64_t(v)))));
  const uint32_t hi = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uint64_t(v) >> 32))));
  return int64_t((uint64_t(hi) << 32) | lo);
}

__device__ __forceinline__ int64_t quotient(int64_t v, int by) {   // v >= 0, by > 0
  return (v >> 32) == 0 ? int64_t(uint32_t(v) / uint32_t(by)) : v / by;
}

// The sequences of a call as a wavefront sees them: 64 at a time, one per lane.
template <bool TREE>
struct Walk {
  const Kv8AttnArgs& a;
  int lane, base;     // the lanes hold sequences base ..
  Seq mine;
  int64_t before;     // units of the sequences before base
  int64_t upto;       // and of base .. this lane's

  __device__ __forceinline__ Walk(const Kv8AttnArgs& args) : a(args), lane(int(threadIdx.x) & 63), base(0), before(0) { load(); }

  __device__ __forceinline__ void load() {
    const int b = base + lane;
    mine = seq_of<TREE>(a, b < a.c.B ? b : a.c.B - 1);
    if (b >= a.c.B) mine.qt = 0;
    int64_t v = units_of(a, mine);
    for (int o = 1; o < 64 && o < a.c.B; o <<= 1) {   // lanes past the last sequence: not whole sums
      const int64_t u = __shfl_up(v, o);
      if (lane >= o) v += u;
    }
    upto = before + v;
  }
  __device__ __forceinline__ void next() {
    before = uniform64(__shfl(upto, 63));
    base += 64;
    load();
  }
  __device__ __forceinline__ int64_t total() {
    int64_t sum = uniform64(__shfl(upto, a.c.B < 64 ? a.c.B - 1 : 63));
    for (int b = 64 + lane; b - lane < a.c.B; b += 64) {
      int64_t v = b < a.c.B ? units_of(a, seq_of<TREE>(a, b)) : 0;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
      sum += uniform64(v);
    }
    return sum;
  }
  // The sequence that holds unit u (before the total, not before an earlier call's), and its first unit. n = 0: there is
  // none (lengths that change while a call reads them), so that the walk ends whatever it reads.
  __device__ __forceinline__ Seq find(int64_t u, int64_t& first) {
    uint64_t hit;
    while ((hit = __ballot(upto > u)) == 0) {
      if (base + 64 >= a.c.B) {
        Seq none = {};
        return none;
      }
      next();
    }
    const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
    Seq s;
    s.start = __builtin_amdgcn_readlane(mine.start, l);
    s.n = __builtin_amdgcn_readlane(mine.n, l);
    s.ctx = __builtin_amdgcn_readlane(mine.ctx, l);
    s.end = __builtin_amdgcn_readlane(mine.end, l);
    s.qt = __builtin_amdgcn_readlane(mine.qt, l);
    s.t0 = __builtin_amdgcn_readlane(mine.t0, l);
    s.nt = __builtin_amdgcn_readlane(mine.nt, l);
    s.b = base + l;
    first = uniform64(__shfl(upto, l)) - units_of(a, s);
    return s;
  }
};

// Of a row's mask: bits `from` .. from + 63 of a tree of n rows, with the positions before the tree (negative) set.
__device__ __forceinline__ uint64_t tree_bits(const uint64_t* mask, int words, int from, int n) {
  if (from <= -64) return ~uint64_t(0);
  if (from >= n) return 0;
  const int w = from >> 6, sh = from & 63;   // w = -1: the word before the tree's
  const uint64_t lo = w < 0 ? ~uint64_t(0) : mask[w], hi = w + 1 < words ? mask[w + 1] : 0;
  uint64_t v = sh ? (lo >> sh) | (hi << (64 - sh)) : lo;
  if (n - from < 64) v &= (uint64_t(1) << (n - from)) - 1;
  return v;
}

// The first position that a row attends: with a window, its last attended ones from there on are `window`, those of the tree
// counted by its mask.
__device__ __forceinline__ int tree_low(const Kv8AttnArgs& a, const uint64_t* mask, int fresh, int n) {
  if (a.window <= 0) return 0;
  int left = a.window;
  for (int w = (n - 1) >> 6; w >= 0; --w) {
    uint64_t v = tree_bits(mask, a.words, 64 * w, n);
    if (fresh < 0) {   // positions below 0 are nobody's
      const int below = -fresh - 64 * w;
      v = below >= 64 ? 0 : below > 0 ? v & (~uint64_t(0) << below) : v;
    }
    const int bits = __popcll((unsigned long long)v);
    if (bits >= left) {
      for (int i = bits; i > left; --i) v &= v - 1;
      return fresh + 64 * w + __ffsll((unsigned long long)v) - 1;
    }
    left -= bits;
  }
  return fresh > left ? fresh - left : 0;
}

// Units per workgroup: an even share, at least one step for each wavefront.
__device__ __forceinline__ int64_t quota_of(const Kv8AttnArgs& a, int64_t total) {
  const int64_t q = quotient(total + a.wgs - 1, a.wgs);
  return q < kWaves && !a.whole ? kWaves : q;
}

// The item that a workgroup begins and does not end, for the kernel that joins it.
struct Joint {
  int last;             // workgroup that ends it; 0: none
  int slot;             // its place among this workgroup's two, the others' is their first
  int start, n;         // of the sequence
  int ct, head;         // column tile, head
  int unused[2];
};

// Four elements of a column, if there is such a column.
__device__ __forceinline__ void store_out(const Kv8AttnArgs& a, const Seq& s, int head, int col, int d, kv_f4 v) {
  const int i = col / a.G, g = col - i * a.G;
  if (i >= s.n) return;
  const kv_h4 h = {_Float16(v[0]), _Float16(v[1]), _Float16(v[2]), _Float16(v[3])};
  __builtin_memcpy(a.out + int64_t(s.start + i) * a.ots + int64_t(head * a.G + g) * a.ohs + d, &h, 8);
}

}  // namespace

}  // namespace fluxbin

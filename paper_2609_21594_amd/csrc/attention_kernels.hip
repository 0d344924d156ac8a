// gfx950 kernels of the attention block: rotary positions, attention forward
// and backward, the clip of query and key weights by their heads' logits.
//
// Attention works on 32-row MFMA blocks whose accumulator layout makes the
// next product's operand: with S^T = K Q^T (A = K rows from LDS, B = Q rows in
// registers) a lane holds, for the one query lane % 32, the 4 consecutive keys
// 8g + 4 (lane / 32) + i of every group g of 8.  The contraction over keys of
// the next product may take the keys in any order as long as both operands
// agree, so these registers, rounded and packed, are its B operand as they
// lie, and the A operand (V^T, K^T) takes the same keys through transposing
// LDS reads.  Row statistics of a softmax are then per lane (plus one exchange
// between the halves of the wave).  The key/value gradient swaps the roles:
// S = Q K^T with keys in the lanes, and dV^T = dO^T P, dK^T = Q^T dS.
//
// LDS tiles keep rows of DP elements; the 16-byte chunk c of row r lies at
// chunk c ^ key(r), so that both the 16-byte reads of 32 rows at one chunk and
// the transposing reads of 4 rows at 4 chunks spread over the banks.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attention_internal.h"
#include "gfx950_util.h"

namespace muon {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();
constexpr float kSlack = 6.f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// x of the lane in the other half of the wave, combined.
__device__ __forceinline__ uint2 swap32(uint32_t a, uint32_t b) {
  const auto v = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return make_uint2(v[0], v[1]);
}
__device__ __forceinline__ float max32(float x) {
  const uint2 v = swap32(__float_as_uint(x), __float_as_uint(x));
  return fmaxf(__uint_as_float(v.x), __uint_as_float(v.y));
}
__device__ __forceinline__ float sum32(float x) {
  const uint2 v = swap32(__float_as_uint(x), __float_as_uint(x));
  return __uint_as_float(v.x) + __uint_as_float(v.y);
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
  return max32(x);
}
// The order of finite floats and infinities is that of their bits as signed
// integers where positive, reversed as unsigned ones where negative; x is no
// NaN.  Maxima do not depend on the order of the updates.
__device__ __forceinline__ void atomic_max_f32(float* p, float x) {
  x += 0.f;  // no negative zero
  // (most updates change nothing, and thousands of atomics on one cache line
  // take longer than a pass over short sequences: look first)
  if (!(x > __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))) return;
  if (x >= 0.f) atomicMax(reinterpret_cast<int*>(p), __float_as_int(x));
  else atomicMin(reinterpret_cast<unsigned*>(p), __float_as_uint(x));
}

// Every load of the wave has landed, the direct ones to LDS too.  The builtin
// and not inline assembly: the compiler then knows that the operands loaded
// before the loop have arrived, and puts no wait of its own at their use in it,
// which would wait for the next tile's loads as well.
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0), the other counters at their largest
}

// Raises the wave's claim on the SIMD around a row of MFMAs, so that of two
// waves on a SIMD one runs its products while the other has its softmax,
// instead of both wanting the same unit.
template <int P>
__device__ __forceinline__ void wave_priority() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_setprio(P);
  __builtin_amdgcn_sched_barrier(0);
}

// Orders the instructions of a row of M products and R LDS reads that feed
// them: AHEAD reads first, then the products one by one, each followed by its
// share of the remaining reads, so that a read is issued about AHEAD reads
// before the product that takes it.  (Left alone, the compiler saves registers
// and waits for each read right after issuing it.)
template <int M, int R, int AHEAD, int I = 0>
__device__ __forceinline__ void interleave() {
  constexpr auto upto = [](int i) { return AHEAD + (R * i + M - 1) / M < R ? AHEAD + (R * i + M - 1) / M : R; };
  if constexpr (I == 0) __builtin_amdgcn_sched_group_barrier(0x100, upto(0), 0);
  if constexpr (I < M) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (upto(I + 1) > upto(I)) __builtin_amdgcn_sched_group_barrier(0x100, upto(I + 1) - upto(I), 0);
    interleave<M, R, AHEAD, I + 1>();
  }
}

// Tiles of heads of up to DU elements, in rows of DP bf16 (a power of two).
template <int DU>
struct Lay {
  static constexpr int DP = DU <= 64 ? 64 : 128;
  static constexpr int CH = DP / 8, RB = DP * 2;  // 16-byte chunks and bytes of a row
  static constexpr int STEPS = DU / 16;           // MFMA steps over the head: 2 chunks each, one per half of the wave
  static constexpr int DB = DU / 32;              // 32-row blocks of the head
  __device__ __forceinline__ static constexpr int key(int r) {
    if constexpr (CH == 8) return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3);
    else return ((r & 3) << 2) | ((r >> 2) & 3);
  }
  __device__ __forceinline__ static int at(int r, int c) { return r * RB + ((c ^ key(r)) << 4); }
};

// The products' operands: bf16 (PL = 1), or fp32 values as the exact sum of
// PL = 3 bf16 planes, x = h + m + l (each the rounding of what the ones before
// it leave; 8 bits each, so 24 in all unless l falls below bf16's range, from
// |x| < 2^-109 on).  A product of two such values is hh + hm + mh + mm + hl +
// lh, six bf16 MFMAs in fp32 accumulation; what is left out is 2^-23 of it at most.
// (fp32 MFMAs have a sixteenth of the bf16 rate, so this is 2.7 times theirs.)
template <int PL> struct Io { using T = uint16_t; };
template <> struct Io<3> { using T = float; };
template <int PL> struct Frag { u32x4_t v[PL]; };
// SWAP: the operands are the other way round than in the pass that this one
// has to agree with bit for bit; the products then come in its order.
template <int PL, bool SWAP = false>
__device__ __forceinline__ void mma(const Frag<PL>& a, const Frag<PL>& b, f32x16_t& c) {
  if constexpr (PL == 3) {
    Mma<uint16_t>::run(a.v[1], b.v[1], c);
    Mma<uint16_t>::run(a.v[SWAP ? 2 : 0], b.v[SWAP ? 0 : 2], c);
    Mma<uint16_t>::run(a.v[SWAP ? 0 : 2], b.v[SWAP ? 2 : 0], c);
    Mma<uint16_t>::run(a.v[SWAP ? 1 : 0], b.v[SWAP ? 0 : 1], c);
    Mma<uint16_t>::run(a.v[SWAP ? 0 : 1], b.v[SWAP ? 1 : 0], c);
  }
  Mma<uint16_t>::run(a.v[0], b.v[0], c);
}
// The same where b is an accumulator's operand: PA planes of it against one
// bf16 operand (PL = 1), or as above.
template <int PL, int PA>
__device__ __forceinline__ void mma_acc(const Frag<PL>& a, const Frag<PA>& b, f32x16_t& c) {
  if constexpr (PL == 3) {
    mma<3>(a, b, c);
  } else {
#pragma unroll
    for (int p = PA - 1; p >= 0; --p) Mma<uint16_t>::run(a.v[0], b.v[p], c);
  }
}
// Planes that probabilities and their gradients are taken in as operands: one
// rounding to bf16 (up to 2^-8 of each, as much as the result's own rounding costs),
// three for fp32.  FINE: two, so that what is left is 2^-16; for requests of
// few rows (fine_of), where single roundings do not average out and the
// products cost little.
template <int PL, bool FINE> constexpr int kAccPlanes = PL == 3 ? 3 : FINE ? 2 : 1;
// A pair of values as words of the planes.
template <int PL>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t* w) {
  w[0] = pack_bf16x2(x, y);
  if constexpr (PL >= 2) {
    x -= __uint_as_float(w[0] << 16);
    y -= __uint_as_float(w[0] & 0xffff0000u);
    w[1] = pack_bf16x2(x, y);
  }
  if constexpr (PL == 3) {
    x -= __uint_as_float(w[1] << 16);
    y -= __uint_as_float(w[1] & 0xffff0000u);
    w[2] = pack_bf16x2(x, y);
  }
}

// LDS by byte address.
typedef const __attribute__((address_space(3))) u32x4_t* lds_u32x4_p;
__device__ __forceinline__ u32x4_t lds16(uint32_t at) { return *reinterpret_cast<lds_u32x4_p>(at); }
__device__ __forceinline__ uint2 lds_tr8(uint32_t at) {
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) v4i16*>(at)));
}

// Stages ROWS rows of `dch` chunks, plane by plane, into LDS by direct loads of
// the whole workgroup of NW waves.  Rows beyond the sequence repeat its last one and
// chunks from dch on the last one: what they hold is finite where the operand
// is, and meets zeros or is never read.  Load i of a thread has the row of load
// 0 plus i * STEP; 16 divides STEP, so its chunk is that of load 0, and its
// 32-bit offset that of load 0 plus a scalar.
template <int PL, int DU, int ROWS, int NW = 4>
struct Stager {
  using L = Lay<DU>;
  static constexpr int NT = 64 * NW, STEP = NT / L::CH, N = ROWS * L::CH / NT;
  static_assert(ROWS * L::CH % NT == 0 && STEP % 16 == 0, "whole loads");
  uint32_t off, stride;
  __device__ __forceinline__ void init(uint32_t stride_, int dch) {
    stride = stride_;
    off = threadIdx.x / L::CH * stride + chunk(dch) * 16;
  }
  __device__ __forceinline__ static int chunk(int dch) {
    return min((static_cast<int>(threadIdx.x) % L::CH) ^ L::key(threadIdx.x / L::CH), dch - 1);
  }
  // base: row 0 of the tile; plane: bytes from one plane of a row to the next;
  // left: rows from there to the sequence's end.
  __device__ __forceinline__ void issue(const char* base, int plane, int left, int dch, uint32_t lds, int wave) const {
    if (left >= ROWS) {
#pragma unroll
      for (int p = 0; p < PL; ++p)
#pragma unroll
        for (int i = 0; i < N; ++i)
          load_lds16(base + p * plane + static_cast<int64_t>(i * STEP) * stride, off,
                     lds + p * ROWS * L::RB + (i * NT + wave * 64) * 16);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t at = static_cast<uint32_t>(min(static_cast<int>(threadIdx.x) / L::CH + i * STEP, left - 1)) * stride +
                            chunk(dch) * 16;
#pragma unroll
        for (int p = 0; p < PL; ++p)
          load_lds16(base + p * plane, at, lds + p * ROWS * L::RB + (i * NT + wave * 64) * 16);
      }
    }
  }
};

// 4 elements, aligned to their size.
template <typename T>
__device__ __forceinline__ float4 load4(const char* p) {
  if constexpr (sizeof(T) == 4) return *reinterpret_cast<const float4*>(p);
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xffff0000u));
}

// 8 elements from c * 8 on of a row (zeros from `dim` on), as operand planes.
template <int PL>
__device__ __forceinline__ Frag<PL> load_chunk(const char* row, int c, int dim) {
  Frag<PL> f;
  if constexpr (PL == 1) {
    f.v[0] = 8 * c < dim ? *reinterpret_cast<const u32x4_t*>(row + c * 16) : u32x4_t{0, 0, 0, 0};
  } else {
    float x[8] = {};
    if (8 * c < dim) *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(row + c * 32);
    if (8 * c + 4 < dim) *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(row + c * 32 + 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t w[3];
      split_pair<PL>(x[2 * k], x[2 * k + 1], w);
#pragma unroll
      for (int p = 0; p < PL; ++p) f.v[p][k] = w[p];
    }
  }
  return f;
}
// The lane's row of an operand kept in registers: chunks 2 s + half.
template <int PL, int DU>
__device__ __forceinline__ void load_operand(const char* row, int dim, int half, Frag<PL>* f) {
#pragma unroll
  for (int s = 0; s < Lay<DU>::STEPS; ++s) f[s] = load_chunk<PL>(row, 2 * s + half, dim);
}
// A operand of the contraction over the head: rows r0 + lane % 32 of a tile,
// chunks 2 st + half.  As 2 st has no bit in common with half, the swizzled
// address is a lane's base with bits flipped by a constant, plus a constant:
// `base` is rows_base + the tile's address (a multiple of 1024, so that the
// flipped bits are the lane's own), `off` the rest; PLANE: bytes of a plane.
template <int DU>
__device__ __forceinline__ uint32_t rows_base(int lane) {
  return Lay<DU>::at(lane & 31, lane >> 5);
}
template <int PL, int PLANE>
__device__ __forceinline__ Frag<PL> frag_rows(uint32_t base, int off, int st) {
  Frag<PL> f;
#pragma unroll
  for (int p = 0; p < PL; ++p) f.v[p] = lds16((base ^ (st << 5)) + (off + p * PLANE));
  return f;
}
// A operand of the contraction over tile rows: elements 32 db + lane % 32 of
// the 16 rows that step `st` (of 2) of accumulator block rows r0 .. r0 + 31
// holds (r0 a multiple of 32, in `off`).  Rows further by 8 flip key bits in
// the same way.
template <int DU>
__device__ __forceinline__ uint32_t cols_base(int lane) {
  const int G = lane >> 4, q = lane & 15;
  return Lay<DU>::at(4 * (G >> 1) + (q >> 2), 2 * (G & 1) + ((q & 3) >> 1)) + (q & 1) * 8;
}
template <int PL, int DU, int PLANE>
__device__ __forceinline__ Frag<PL> frag_cols(uint32_t base, int off, int st, int db) {
  using L = Lay<DU>;
  constexpr int flip = L::key(8) << 4;
  const uint32_t b = base ^ (db << 6);
  Frag<PL> f;
#pragma unroll
  for (int p = 0; p < PL; ++p) {
    const int o = off + p * PLANE + 16 * st * L::RB;
    const uint2 lo = lds_tr8(b + o), hi = lds_tr8((b ^ flip) + (o + 8 * L::RB));
    f.v[p] = u32x4_t{lo.x, lo.y, hi.x, hi.y};
  }
  return f;
}
// The B operand of that step: accumulator registers, rounded or split.
template <int PL>
__device__ __forceinline__ Frag<PL> frag_acc(const f32x16_t& s, int st) {
  Frag<PL> f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w[3];
    split_pair<PL>(s[8 * st + 2 * i], s[8 * st + 2 * i + 1], w);
#pragma unroll
    for (int p = 0; p < PL; ++p) f.v[p][i] = w[p];
  }
  return f;
}

__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// Writes the lane's row (a transposed accumulator: element 32 db + 8 g +
// 4 half + i in register 4 g + i of block db), times `f`.  To `res` goes what the
// rounding took, or nothing where the result is `exact`.  All lanes of the wave
// call it; `on`: this lane writes.
template <typename T, int DB>
__device__ __forceinline__ void store_row(const f32x16_t* o, float f, char* row, char* res, int dim, int half, bool on,
                                          bool exact = false) {
  const uint32_t keep = exact ? 0u : ~0u;
  const int dch = dim / (16 / static_cast<int>(sizeof(T)));
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t w[4], e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // k / 2: group 2 p + k / 2, pairs of elements
          const float x = o[db][8 * p + 2 * k] * f, y = o[db][8 * p + 2 * k + 1] * f;
          w[k] = pack_bf16x2(x, y);
          e[k] = res ? pack_bf16x2(x - __uint_as_float(w[k] << 16), y - __uint_as_float(w[k] & 0xffff0000u)) & keep : 0u;
        }
        // halves exchange so that each lane holds 8 consecutive elements
        const uint2 a = swap32(w[0], w[2]), b = swap32(w[1], w[3]);
        const int c = 4 * db + 2 * p + half;
        if (on && c < dch) *reinterpret_cast<u32x4_t*>(row + c * 16) = u32x4_t{a.x, b.x, a.y, b.y};
        if (res) {
          const uint2 u = swap32(e[0], e[2]), v = swap32(e[1], e[3]);
          if (on && c < dch) *reinterpret_cast<u32x4_t*>(res + c * 16) = u32x4_t{u.x, v.x, u.y, v.y};
        }
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = 8 * db + 2 * g + half;
        if (on && c < dch)
          *reinterpret_cast<float4*>(row + c * 16) =
              make_float4(o[db][4 * g] * f, o[db][4 * g + 1] * f, o[db][4 * g + 2] * f, o[db][4 * g + 3] * f);
      }
    }
  }
}

// A row that sees one key has that key's value, exactly.  p / sum p is 1 but for
// the exponent's rounding, which the sum holds to 24 bits and an operand of p may
// not.  bf16: what the quotient rounds to is the value, and the rounding took
// nothing.  fp32: a tenth of such rows would be a step off, and its gradients not
// 0, so they take the value itself: here as an accumulator's row, where `on`.
template <int DB>
__device__ __forceinline__ void take_row(f32x16_t* o, const char* row, int dim, int half, bool on) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * db + 8 * g + 4 * half;
      if (!on || d >= dim) continue;
      const float4 x = *reinterpret_cast<const float4*>(row + d * 4);
      o[db][4 * g] = x.x; o[db][4 * g + 1] = x.y; o[db][4 * g + 2] = x.z; o[db][4 * g + 3] = x.w;
    }
}

// fp32 arrays that tiles are staged from, as planes: rows [batch][heads]
// [tokens][3][head, padded to 8].  A thread has 8 elements.  (4 us for a small
// call; without it every workgroup would split the tiles that it shares with others.)
struct SplitArgs {
  Heads from[4];
  char* to[4];
  int32_t tokens[4], heads[4];
  int64_t first[5];   // first thread of each array
  int32_t n, dim;
};
__global__ __launch_bounds__(256) void k_split(SplitArgs a) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (at >= a.first[a.n]) return;
  int k = 0;
  while (k + 1 < a.n && a.first[k + 1] <= at) ++k;
  const int chunks = (a.dim + 7) / 8;
  const int64_t i = at - a.first[k];
  const int c = static_cast<int>(i % chunks);
  const int64_t bth = i / chunks;  // heads vary fastest: reads are consecutive in the usual layout
  const int head = static_cast<int>(bth % a.heads[k]);
  const int64_t bt = bth / a.heads[k];
  const int64_t b = bt / a.tokens[k], t = bt % a.tokens[k];
  const Heads& h = a.from[k];
  const Frag<3> f = load_chunk<3>(h.p + b * h.batch + t * h.token + head * h.head, c, a.dim);
  char* to = a.to[k] + (((b * a.heads[k] + head) * a.tokens[k] + t) * 3 * chunks + c) * 16;
#pragma unroll
  for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4_t*>(to + p * chunks * 16) = f.v[p];
}

// ---------------------------------------------------------------------------
// Which work a workgroup has.
// ---------------------------------------------------------------------------
// Workgroup -> (batch, key head, head or part of the group, tile).  Workgroup b
// runs on XCD b % 8: where the (batch, key head) units divide evenly, each XCD
// has units of its own, so that it reads their keys and values once.  Tiles
// change slowest, `reverse` puts the last ones first: a causal pass starts with
// its longest tiles, over all heads, and ends with the shortest (heads changing
// slowest instead: 4 x 2048 tokens x 16 heads of 64 causal take 74 instead of
// 52 us forward, 215 instead of 160 backward; windows and long sequences 2% less).
struct Item { int b, kvh, g, tile; };
__device__ __forceinline__ Item item_of(int bid, const AttnArgs& a, int parts, int tiles, bool reverse) {
  const int units = static_cast<int>(a.seqs.batch) * a.kv_heads;
  int unit, rest;
  if (units % 8 == 0) {
    const int n = units >> 3, j = bid >> 3;
    unit = (bid & 7) * n + j / parts % n;
    rest = j / (parts * n) * parts + j % parts;
  } else {
    unit = bid % units;
    rest = bid / units;
  }
  Item it;
  it.b = unit / a.kv_heads;
  it.kvh = unit % a.kv_heads;
  it.g = rest % parts;
  it.tile = rest / parts;
  if (reverse) it.tile = tiles - 1 - it.tile;
  return it;
}

// A sequence: tokens q0 .. q0 + nq - 1 and k0 .. k0 + nk - 1 of batch b's
// axes; the rows of it that are written are q_rows / k_rows (dense: the whole
// axis, rows behind the length being zeros).  tile: of this sequence.
struct Seq { int q0, nq, k0, nk, q_rows, k_rows, tile; bool ok; };

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Sum over the wave's lanes of non-negative numbers below 2^bits, by bit planes.
__device__ __forceinline__ int wave_count(int x, int bits) {
  int sum = 0;
  for (int b = 0; b < bits; ++b) sum += __popcll(__ballot((x >> b) & 1)) << b;
  return sum;
}

// The sequence that holds tile `tile` (of `tiles`) of `bt` queries, or keys
// where by_key.  Packed, each wave finds it from the offsets, the tiles being
// numbered in one of three ways:
//   - more than 64 sequences: sequence s has the numbers from offset / bt + s on,
//     its tiles and at most one number without work, so that a search finds it,
//     64 probes at a time (4000 sequences of 32 tokens x 8 heads of 64: 225 us
//     forward; 924 where each wave added up the tiles of all sequences before
//     its own).  Numbers are taken in another order inside each 64: those without
//     work often alternate with the others, and a launch deals its workgroups out
//     to the parts of an XCD in turn (256 sequences of 128: 32 us, 43 in the
//     numbers' order);
//   - up to 64, a lane for each, causal without a window: by the number of keys
//     that a tile passes over, largest first.  By sequence, the launch would end
//     with the long tiles of one (8 sequences of 4096 x 8 heads of 64: 194 us
//     forward, 221 by sequence);
//   - otherwise one sequence's after the other's, which keeps the tiles that read
//     the same keys together (11 sequences of 745 x 16 heads of 64, a window of 1024:
//     45 us forward, 52 ranked, 51 in the order of many).
__device__ __forceinline__ bool ranks_tiles(const AttnArgs& a) { return a.seqs.q_off && a.causal && !a.window && a.seqs.n_seq <= 64; }
__device__ __forceinline__ Seq find_seq(const AttnArgs& a, int b, int tile, int tiles, int bt, bool by_key) {
  const Seqs& s = a.seqs;
  Seq r;
  r.ok = true;
  r.tile = tile;
  if (!s.q_off) {
    r.q0 = r.k0 = 0;
    r.nq = s.q_len ? clampi(s.q_len[b], 0, s.q_tokens) : s.q_tokens;
    r.nk = s.k_len ? clampi(s.k_len[b], 0, s.k_tokens) : s.k_tokens;
    r.q_rows = s.q_tokens;
    r.k_rows = s.k_tokens;
    return r;
  }
  const int lane = threadIdx.x & 63;
  const bool many = s.n_seq > 64;
  if (many && tile < (tiles & ~63)) tile = (tile & ~63) | (tile & 7) << 3 | (tile >> 3 & 7);
  // the search, down to 64 sequences from `lo` on, one a lane
  int lo = 0, n = s.n_seq;
  while (n > 64) {
    const int32_t* off = by_key ? s.k_off : s.q_off;
    const int step = (n + 63) >> 6, i = lo + lane * step;
    const bool start = lane * step < n && clampi(off[i], 0, by_key ? s.k_tokens : s.q_tokens) / bt + i <= tile;
    const int skip = max(__popcll(__ballot(start)) - 1, 0) * step;
    lo += skip;
    n = min(n - skip, step);
  }
  int q0 = 0, nq = 0, k0 = 0, nk = 0;
  if (lane < n) {
    const int32_t *qo = s.q_off + lo + lane, *ko = s.k_off + lo + lane;
    const int qa = qo[0], qb = qo[1], ka = ko[0], kb = ko[1];
    q0 = clampi(qa, 0, s.q_tokens);
    nq = clampi(qb, q0, s.q_tokens) - q0;
    k0 = clampi(ka, 0, s.k_tokens);
    nk = clampi(kb, k0, s.k_tokens) - k0;
  }
  unsigned long long hit;
  const int mine = ((by_key ? nk : nq) + bt - 1) / bt;
  if (many) {
    r.tile = tile - (by_key ? k0 : q0) / bt - lo - lane;
    const int starts = __popcll(__ballot(lane < n && r.tile >= 0));
    hit = starts ? 1ull << (starts - 1) : 0;
  } else if (ranks_tiles(a)) {
    // level i: the i-th tiles of all sequences that have it; above(i): the tiles
    // of higher levels.  The number's level is the lowest with above(i) <= tile.
    const int top = (by_key ? s.k_tokens : s.q_tokens) / bt + 1, bits = 32 - __clz(top);
    int level = 0, end = top;
    while (level < end) {
      const int mid = (level + end) >> 1;
      if (wave_count(max(mine - mid - 1, 0), bits) <= tile) end = mid;
      else level = mid + 1;
    }
    const unsigned long long have = __ballot(mine > level);
    const int nth = tile - wave_count(max(mine - level - 1, 0), bits);
    const int below = __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(have >> 32),
                                                __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(have), 0));
    hit = __ballot(mine > level && below == nth);
    r.tile = by_key ? mine - 1 - level : level;
  } else {
    int upto = mine;  // tiles of this lane's sequence and those before it
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    hit = __ballot(upto > tile);
    r.tile = tile - (upto - mine);
  }
  const int at = hit ? __ffsll(hit) - 1 : 0;
  r.tile = __builtin_amdgcn_readlane(r.tile, at);
  r.q0 = __builtin_amdgcn_readlane(q0, at);
  r.nq = r.q_rows = __builtin_amdgcn_readlane(nq, at);
  r.k0 = __builtin_amdgcn_readlane(k0, at);
  r.nk = r.k_rows = __builtin_amdgcn_readlane(nk, at);
  r.ok = hit && r.tile * bt < (by_key ? r.nk : r.nq);
  return r;
}

// Packed: fills the rows of a head that no sequence holds, [0, first offset)
// and [last offset, tokens), with zeros; the whole workgroup.
__device__ __forceinline__ void outside_of(const Seqs& s, bool keys, int& lo, int& hi) {
  const int32_t* off = keys ? s.k_off : s.q_off;
  const int n = keys ? s.k_tokens : s.q_tokens;
  lo = s.n_seq > 0 ? clampi(off[0], 0, n) : 0;
  hi = s.n_seq > 0 ? clampi(off[s.n_seq], lo, n) : 0;
}
__device__ __forceinline__ void zero_outside(const Seqs& s, bool keys, const Heads& h, int head, int bytes) {
  int lo, hi;
  outside_of(s, keys, lo, hi);
  const int n = keys ? s.k_tokens : s.q_tokens, chunks = bytes / 16;
  const int64_t total = static_cast<int64_t>(lo + n - hi) * chunks;
  for (int64_t i = threadIdx.x; i < total; i += blockDim.x) {
    const int r = static_cast<int>(i / chunks), c = static_cast<int>(i % chunks);
    const int64_t row = r < lo ? r : hi + r - lo;
    *reinterpret_cast<u32x4_t*>(h.p + row * h.token + head * h.head + c * 16) = u32x4_t{0, 0, 0, 0};
  }
}

__device__ __forceinline__ const char* at_row(const Heads& h, int b, int token, int head) {
  return h.p + b * h.batch + token * h.token + head * h.head;
}
__device__ __forceinline__ char* at_row_w(const Heads& h, int b, int token, int head) {
  return h.p + b * h.batch + token * h.token + head * h.head;
}
// Index of a row's log-sum-exp.
__device__ __forceinline__ int64_t row_index(const AttnArgs& a, int b, int head, int token) {
  return (static_cast<int64_t>(b) * a.q_heads + head) * a.seqs.q_tokens + token;
}

// Keys that queries lo .. hi (of one sequence) see: any of them [beg, end),
// all of them [all_beg, all_end).
struct KeyRange { int beg, end, all_beg, all_end; };
__device__ __forceinline__ KeyRange keys_of(const AttnArgs& a, const Seq& s, int lo, int hi) {
  KeyRange r{0, s.nk, 0, s.nk};
  if (hi < lo) return KeyRange{0, 0, 0, 0};
  const int shift = s.nk - s.nq;
  if (a.causal) {
    r.end = clampi(hi + shift + 1, 0, s.nk);
    r.all_end = clampi(lo + shift + 1, 0, s.nk);
    if (a.window) {
      r.beg = max(0, lo + shift - a.window + 1);
      r.all_beg = max(0, hi + shift - a.window + 1);
    }
  }
  return r;
}

// ---------------------------------------------------------------------------
// Forward.  A wave holds 32 queries and passes over the keys in tiles of BN,
// staged in LDS (NST stages), keeping the running maximum and sum.  WS = 1: the
// workgroup's NW waves hold 32 queries each and share each tile (8 waves: SUB
// tiles a stage, so that the two waves of a SIMD drift apart between barriers
// and one has its products while the other has its softmax).  WS > 1: WS waves
// share their queries and take every WS-th tile, and are joined at the end; for
// requests with too few rows to fill the device.
//
// Bound by MFMA and vector issue together: per 64 keys and 32 queries of 128
// elements 32 MFMAs (1024 cycles) and 32 x 4.2 vector instructions, of which 32
// are exponentials (about 1000), overlapped across the waves of a SIMD in part
// (MFMAs busy 54%, vector issue 53% of a busy CU's cycles, LDS 27%, no bank
// conflicts).  4096 tokens, 32 heads on 8 of 128, causal: 132 us, 1040 TFLOP/s; 2
// x 8192 without a mask: 1170; 4 x 4096, 16 heads of 64: 970; fp32, 2 x 2048, 16
// heads of 128: 162.  Few rows: by memory, 268 MB of keys and values in 45 us.
// ---------------------------------------------------------------------------
template <int PL, int DU, int BN, int WS, int NST, bool FINE, bool SPLIT, int NW>
__global__ __launch_bounds__(64 * NW, WS == 1 && (PL == 1 || DU <= 64) ? 2 : 1) void k_attn_fwd(AttnArgs a, int tiles, int pack) {
  constexpr int PA = kAccPlanes<PL, FINE>;
  constexpr int PR = PL == 3 ? 6 : 1, PP = PL == 3 ? 6 : PA;  // MFMAs of a product, and of one with an accumulator
  using L = Lay<DU>;
  using T = typename Io<PL>::T;
  constexpr int SUB = NW == 8 ? 2 : 1;  // tiles of a stage, for each wave
  constexpr int BM = 32 * NW / WS, KB = BN / 32, SR = BN * WS * SUB, PLANE = SR * L::RB, TILE = PL * PLANE, STAGE = 2 * TILE;
  constexpr int JOIN = (WS - 1) * (NW / WS) * (L::DB * 16 + 3) * 256;
  __shared__ __attribute__((aligned(1024))) char smem[NST * STAGE > JOIN ? NST * STAGE : JOIN];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ws = wave % WS, dch = (a.dim + 7) / 8;
  int bid = blockIdx.x, split = 0;
  if constexpr (SPLIT) {
    const int items = gridDim.x / a.splits;
    split = bid / items;
    bid -= split * items;
  }
  const Item it = item_of(bid, a, pack ? 1 : a.group, tiles, a.causal && !ranks_tiles(a));
  if (a.fill && it.tile == tiles - 1) {  // one tile more than sequences can have
    const int h = it.kvh * a.group + it.g;
    zero_outside(a.seqs, false, a.out, h, a.dim * sizeof(T));
    if (a.res.p) zero_outside(a.seqs, false, a.res, h, a.dim * sizeof(T));
    int lo, hi;
    outside_of(a.seqs, false, lo, hi);
    for (int i = threadIdx.x; i < lo + a.seqs.q_tokens - hi; i += 64 * NW)
      a.lse[row_index(a, 0, h, i < lo ? i : hi + i - lo)] = -kInf;
    return;
  }
  const Seq s = find_seq(a, it.b, it.tile, tiles, BM, false);
  if (!s.ok) return;
  const int shift = s.nk - s.nq;

  // the lane's rows.  pack: the rows are all heads of the group, each with all queries
  const int rows = pack ? s.q_rows * a.group : s.q_rows;
  const int r0 = s.tile * BM + wave / WS * 32;
  const int r = r0 + (lane & 31);
  const bool in = r < rows;
  int iq = min(r, rows - 1), g = it.g;
  if (pack) {
    g = iq / s.q_rows;
    iq -= g * s.q_rows;
  }
  const int head = it.kvh * a.group + g;
  const int jmax = a.causal ? min(s.nk - 1, iq + shift) : s.nk - 1;
  const int jmin = a.causal && a.window ? max(0, iq + shift - a.window + 1) : 0;

  // the keys of the workgroup and of the wave
  const int last = min(s.q_rows, s.nq) - 1;
  const KeyRange wg = pack ? keys_of(a, s, 0, last) : keys_of(a, s, s.tile * BM, min(s.tile * BM + BM - 1, last));
  const KeyRange wv = r0 >= rows ? KeyRange{0, 0, 0, 0} : pack ? wg : keys_of(a, s, r0, min(r0 + 31, last));
  int t0 = wg.beg / SR, t1 = (wg.end + SR - 1) / SR;
  if constexpr (SPLIT) {
    const int per = (max(t1 - t0, 0) + a.splits - 1) / a.splits;
    t0 += split * per;
    t1 = min(t1, t0 + per);
  }

  const uint32_t lds0 = lds_offset(smem);
  const uint32_t own = lds0 + ws * BN * L::RB, rbase = own + rows_base<DU>(lane), cbase = own + cols_base<DU>(lane);
  Stager<PL, DU, SR, NW> ks, vs;
  ks.init(static_cast<uint32_t>(a.sk.token), dch);
  vs.init(static_cast<uint32_t>(a.sv.token), dch);
  const char* const krow = at_row(a.sk, it.b, s.k0, it.kvh);
  const char* const vrow = at_row(a.sv, it.b, s.k0, it.kvh);
  auto issue = [&](int t) __attribute__((always_inline)) {
    const uint32_t at = lds0 + t % NST * STAGE;
    const int64_t j = t * SR;
    ks.issue(krow + j * a.sk.token, a.plane, s.nk - t * SR, dch, at, wave);
    vs.issue(vrow + j * a.sv.token, a.plane, s.nk - t * SR, dch, at + TILE, wave);
  };

  f32x16_t o[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) o[db] = zero16();
  float m = -kInf, l = 0.f, top = -kInf;
  if (NST > 1 && t0 < t1) issue(t0);
  Frag<PL> qf[L::STEPS];
  load_operand<PL, DU>(at_row(a.q, it.b, s.q0 + iq, head), a.dim, half, qf);
  for (int t = t0; t < t1; ++t) {
    if constexpr (NST == 1) {
      __syncthreads();
      issue(t);
    }
    wait_loads();
    __syncthreads();  // tile t has landed, and every wave is done with tile t - 1
    if (NST > 1 && t + 1 < t1) issue(t + 1);
#pragma unroll 1
    for (int sub = 0; sub < SUB; ++sub) {
      const int j0 = t * SR + (ws + sub) * BN;
      if (j0 >= wv.end || j0 + BN <= wv.beg) continue;
      const uint32_t at = t % NST * STAGE + sub * BN * L::RB, rb = rbase + at, cb = cbase + at;
      f32x16_t p[KB];
      wave_priority<NW == 8>();
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) p[kb] = zero16();
#pragma unroll
      for (int st = 0; st < L::STEPS; ++st)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) mma<PL>(frag_rows<PL, PLANE>(rb, 32 * kb * L::RB, st), qf[st], p[kb]);
      interleave<PR * KB * L::STEPS, PL * KB * L::STEPS, 4>();
      wave_priority<0>();
      if (j0 + BN > wv.all_end || j0 < wv.all_beg) {
        asm volatile("; a tile that the mask cuts");  // (a branch: else every tile pays for the comparisons)
        const int lo = jmin - j0 - 4 * half, hi = jmax - j0 - 4 * half;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = 32 * kb + 8 * (r >> 2) + (r & 3);
            if (j < lo || j > hi) p[kb][r] = -kInf;
          }
      }
      float mx = -kInf;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, p[kb][r]);
      mx = max32(mx);
      top = fmaxf(top, mx);
      // Probabilities are taken relative to m, which follows the maximum only
      // when that has grown by 2^kSlack: binary32 sums have room for the factor,
      // bf16 rounds relatively, and most tiles leave o as it is.  (The parts of a
      // split key axis report m as their maximum.)
      const float mn = mx * a.scale2;
      if (__any(mn > m + (SPLIT ? 0.f : kSlack))) {
        const float up = fmaxf(m, mn), alpha = m == up ? 1.f : exp2_(m - up);
        m = up;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < L::DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
      }
      const float mu = m == -kInf ? 0.f : m;
      float sum = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[kb][r] = exp2_(fmaf(p[kb][r], a.scale2, -mu));
          sum += p[kb][r];
        }
      l += sum;
      wave_priority<NW == 8>();
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const Frag<PA> pf = frag_acc<PA>(p[kb], st);
#pragma unroll
          for (int db = 0; db < L::DB; ++db)
            mma_acc<PL, PA>(frag_cols<PL, DU, PLANE>(cb, TILE + 32 * kb * L::RB, st, db), pf, o[db]);
        }
      interleave<PP * KB * 2 * L::DB, PL * KB * 4 * L::DB, 8>();
      wave_priority<0>();
    }
  }

  l = sum32(l);
  if constexpr (WS > 1) {  // the waves that shared the queries, in order
    float* const at = reinterpret_cast<float*>(smem) + wave / WS * (WS - 1) * (L::DB * 16 + 3) * 64 + lane;
    __syncthreads();
    if (ws > 0) {
      float* const x = at + (ws - 1) * (L::DB * 16 + 3) * 64;
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[(db * 16 + e) * 64] = o[db][e];
      x[L::DB * 16 * 64] = m;
      x[(L::DB * 16 + 1) * 64] = l;
      x[(L::DB * 16 + 2) * 64] = top;
    }
    __syncthreads();
    if (ws > 0) return;
    float all = m;
#pragma unroll
    for (int w = 0; w < WS - 1; ++w) all = fmaxf(all, at[(w * (L::DB * 16 + 3) + L::DB * 16) * 64]);
    const float f = m == -kInf ? 0.f : exp2_(m - all);
    m = all;
    l *= f;
#pragma unroll
    for (int db = 0; db < L::DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] *= f;
#pragma unroll
    for (int w = 0; w < WS - 1; ++w) {
      const float* const x = at + w * (L::DB * 16 + 3) * 64;
      const float mw = x[L::DB * 16 * 64], fw = mw == -kInf ? 0.f : exp2_(mw - all);
      l = fmaf(x[(L::DB * 16 + 1) * 64], fw, l);
      top = fmaxf(top, x[(L::DB * 16 + 2) * 64]);
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] = fmaf(x[(db * 16 + e) * 64], fw, o[db][e]);
    }
  }
  const int64_t row = row_index(a, it.b, head, s.q0 + iq);
  if constexpr (SPLIT) {
    const int64_t all = static_cast<int64_t>(a.seqs.batch) * a.q_heads * a.seqs.q_tokens;
    float* po = a.part_o + (split * all + row) * a.dim;
    store_row<float, L::DB>(o, 1.f, reinterpret_cast<char*>(po), nullptr, a.dim, half, in);
    if (in && half == 0) a.part_ml[split * all + row] = make_float2(m, l);
    return;
  }
  const bool live = in && iq < s.nq;
  const bool one = live && jmin == jmax && l > 0.f && l < kInf;  // (NaN stays)
  float inv = !live || l == 0.f ? 0.f : 1.f / l;
  if constexpr (PL == 3) {
    if (__any(one)) take_row<L::DB>(o, at_row(a.v, it.b, s.k0 + jmin, it.kvh), a.dim, half, one);
    if (one) inv = 1.f;
  } else if (PA == 1 && one) {
    inv = 1.f / to_f32<uint16_t>(f32_to_bf16(l));  // l is the row's p, and o has its one plane
  }
  if (!live) {
#pragma unroll
    for (int db = 0; db < L::DB; ++db) o[db] = zero16();
  }
  char* orow = at_row_w(a.out, it.b, s.q0 + iq, head);
  char* rrow = a.res.p ? at_row_w(a.res, it.b, s.q0 + iq, head) : nullptr;
  store_row<T, L::DB>(o, inv, orow, rrow, a.dim, half, in, one);
  if (in && half == 0) a.lse[row] = live && l != 0.f ? (m + __log2f(l)) * kLn2 : -kInf;
  if (a.max_logits) {
    float x = live ? top * a.scale : -kInf;
    if (pack) {
      if (half == 0 && x > -kInf) atomic_max_f32(a.max_logits + head, x);
    } else {
      x = wave_max(x);
      if (lane == 0 && x > -kInf) atomic_max_f32(a.max_logits + head, x);
    }
  }
}

// Joins the splits (4 to 5 us for 128 rows of 16 parts): a workgroup a row, 32 lanes along the head (4 elements
// each) times 8 parts of the splits, summed through LDS in a fixed order.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  __shared__ float4 sums[8][32];
  __shared__ float mx[8], ls[8];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int64_t all = static_cast<int64_t>(a.seqs.batch) * a.q_heads * a.seqs.q_tokens, row = blockIdx.x;
  const int i = static_cast<int>(row % a.seqs.q_tokens);
  const int64_t bh = row / a.seqs.q_tokens;
  const int head = static_cast<int>(bh % a.q_heads), b = static_cast<int>(bh / a.q_heads);
  const bool live = !a.seqs.q_len || i < a.seqs.q_len[b];
  const int d = 4 * lane;
  // the part's own maximum and sums
  float m = -kInf;
  for (int s = part; s < a.splits; s += 8) m = fmaxf(m, a.part_ml[s * all + row].x);
  float l = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = part; s < a.splits; s += 8) {
    const float2 v = a.part_ml[s * all + row];
    if (v.x == -kInf && v.y == 0.f) continue;  // a part that sees nothing (one of NaN alone has no maximum either)
    const float w = exp2_(v.x - m);
    l = fmaf(w, v.y, l);
    if (d < a.dim) {
      const float4 y = *reinterpret_cast<const float4*>(a.part_o + (s * all + row) * a.dim + d);
      x.x = fmaf(w, y.x, x.x); x.y = fmaf(w, y.y, x.y); x.z = fmaf(w, y.z, x.z); x.w = fmaf(w, y.w, x.w);
    }
  }
  sums[part][lane] = x;
  if (lane == 0) { mx[part] = m; ls[part] = l; }
  __syncthreads();
  if (part != 0) return;
  m = mx[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) m = fmaxf(m, mx[k]);
  l = 0.f;
  x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float w = mx[k] == -kInf ? 0.f : exp2_(mx[k] - m);
    const float4 y = sums[k][lane];
    l = fmaf(w, ls[k], l);
    x.x = fmaf(w, y.x, x.x); x.y = fmaf(w, y.y, x.y); x.z = fmaf(w, y.z, x.z); x.w = fmaf(w, y.w, x.w);
  }
  const bool some = live && l != 0.f;
  if (lane == 0) {
    a.lse[row] = some ? (m + __log2f(l)) * kLn2 : -kInf;
    if (a.max_logits && some && m > -kInf) atomic_max_f32(a.max_logits + head, m * kLn2);
  }
  if (d >= a.dim) return;
  const float inv = some ? 1.f / l : 0.f;
  float o[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
  if (!some) o[0] = o[1] = o[2] = o[3] = 0.f;
  // the keys that the row sees: 0 .. last, as split passes have no window
  const int nq = a.seqs.q_len ? clampi(a.seqs.q_len[b], 0, a.seqs.q_tokens) : a.seqs.q_tokens;
  const int nk = a.seqs.k_len ? clampi(a.seqs.k_len[b], 0, a.seqs.k_tokens) : a.seqs.k_tokens;
  if (some && l > 0.f && l < kInf && (a.causal ? i + nk - nq : nk - 1) == 0) {  // one: its value (take_row)
    const float4 y = load4<T>(at_row(a.v, b, 0, head / a.group) + d * sizeof(T));
    o[0] = y.x; o[1] = y.y; o[2] = y.z; o[3] = y.w;
  }
  char* orow = at_row_w(a.out, b, i, head);
  if constexpr (sizeof(T) == 2) {
    const uint2 w = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
    *reinterpret_cast<uint2*>(orow + 2 * d) = w;
    if (a.res.p)
      *reinterpret_cast<uint2*>(at_row_w(a.res, b, i, head) + 2 * d) =
          make_uint2(pack_bf16x2(o[0] - __uint_as_float(w.x << 16), o[1] - __uint_as_float(w.x & 0xffff0000u)),
                     pack_bf16x2(o[2] - __uint_as_float(w.y << 16), o[3] - __uint_as_float(w.y & 0xffff0000u)));
  } else {
    *reinterpret_cast<float4*>(orow + 4 * d) = make_float4(o[0], o[1], o[2], o[3]);
  }
}

// ---------------------------------------------------------------------------
// Backward.
// ---------------------------------------------------------------------------
// Sums the accumulators of the WS waves that share their rows, in order, into
// the first of them, through LDS that nothing else is read from any more; true
// in that wave.
template <int WS, int DB>
__device__ __forceinline__ bool join_waves(f32x16_t* acc, char* smem, int wave, int lane) {
  const int ws = wave % WS;
  float* const at = reinterpret_cast<float*>(smem) + wave / WS * (WS - 1) * DB * 1024 + lane;
  __syncthreads();
  if (ws > 0) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) at[((ws - 1) * DB * 16 + db * 16 + e) * 64] = acc[db][e];
  }
  __syncthreads();
  if (ws > 0) return false;
#pragma unroll
  for (int w = 0; w < WS - 1; ++w)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[db][e] += at[(w * DB * 16 + db * 16 + e) * 64];
  return true;
}

// Sums over a row, which have to be more exact than the factor that they tell:
// the 16 values of a step by pairs, the steps' sums with what each addition
// rounded off carried into the next.  That is 6 roundings for a row of any
// length.  (One value after the other, near equal ones all round the same way:
// rows of 200 to 1598 equal probabilities came out up to 4.1e-6 off.)
struct LongSum {
  float sum = 0.f, over = 0.f;
  __device__ __forceinline__ void add(float x) {
    x -= over;
    const float to = sum + x;
    over = (to - sum) - x;
    sum = to;
  }
};
__device__ __forceinline__ float sum16(const f32x16_t& x) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x[2 * e] + x[2 * e + 1];
#pragma unroll
  for (int n = 4; n > 0; n /= 2)
#pragma unroll
    for (int e = 0; e < n; ++e) y[e] = y[2 * e] + y[2 * e + 1];
  return y[0];
}

// fp32: what a row's probabilities are multiplied with, 0: they stay.  lse2 holds
// the log-sum-exp to half a step of its own size, 2^-24 |lse2|, twice (as lse, and
// times log2 e), which all probabilities of the row have as a common factor: at
// |lse2| = 72 up to 5e-6 of the gradients, ten times their other errors.  Their
// own sum tells the factor.  A sum further from 1 than such roundings is what lse
// says (it may be that of more keys).  Rows so normalised also know what their
// dS should sum to, which takes the rounding of out from delta.  Measured, errors
// of dq and dk of 200 to 4000 tokens, heads of 64: 0.2 to 0.9e-6 instead of 0.3 to
// 1.2e-6 with logits up to 24, heads of 128 up to 45: 1.9 to 2.2e-6 instead of 2.2
// to 2.4e-6, for 5% more time.
__device__ __forceinline__ float row_norm(float total, float lse2) {
  return total > 0.5f && fabsf(total - 1.f) <= 0x1p-22f * (fabsf(lse2) + 8.f) ? 1.f / total : 0.f;
}

// dout . (out + res) of the lane's row, as the diagonal of the products of 32
// rows of out with those of dout: the same operation, in the same order, as
// that of dout with a value row.  A row that sees one key has out equal to it
// bit for bit, so its dP - delta, and with it its gradient, is exactly 0.
template <int PL, int DU>
__device__ __forceinline__ float row_dots(const Frag<PL>* df, const char* out, const char* res, int dim, int lane) {
  const int half = lane >> 5, c = lane & 31;
  f32x16_t p = zero16();
#pragma unroll
  for (int st = 0; st < Lay<DU>::STEPS; ++st) mma<PL>(load_chunk<PL>(out, 2 * st + half, dim), df[st], p);
  if (res) {
#pragma unroll
    for (int st = 0; st < Lay<DU>::STEPS; ++st) mma<PL>(load_chunk<PL>(res, 2 * st + half, dim), df[st], p);
  }
  // column c's row c is in the half (c / 4) % 2, register 4 (c / 8) + c % 4
  float x = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (e == 4 * (c >> 3) + (c & 3) && ((c >> 2) & 1) == half) x = p[e];
  return sum32(x);
}

// dQ: a wave holds 32 queries (Q and dO rows in registers), the workgroup
// passes over the keys: S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.
// First it forms each row's dout . out in fp32, with what the rounding took
// from out where the caller kept it, and writes it and log2 of the sum of
// exponentials for k_attn_dkv: +inf where no key is visible, so that every
// probability recomputed from it is 0.  Bound as the forward pass is, with half
// more products: 4096 tokens, 32 heads on 8 of 128, causal: 223 us (206 GFLOP,
// MFMAs busy 55%).
template <int PL, int DU, int BN, int WS, int NST, bool FINE>
__global__ __launch_bounds__(256, WS == 1 && (PL == 1 || DU <= 64) ? 2 : 1) void k_attn_dq(AttnArgs a, int tiles) {
  constexpr int PA = kAccPlanes<PL, FINE>;
  constexpr int PR = PL == 3 ? 6 : 1, PP = PL == 3 ? 6 : PA;  // MFMAs of a product, and of one with an accumulator
  using L = Lay<DU>;
  using T = typename Io<PL>::T;
  constexpr int BM = 128 / WS, SR = BN * WS, PLANE = SR * L::RB, TILE = PL * PLANE, STAGE = 2 * TILE;
  constexpr int JOIN = (WS - 1) * (4 / WS) * L::DB * 4096, USED = JOIN + (PL == 3 && WS > 1 ? 2048 : 0);
  __shared__ __attribute__((aligned(1024))) char smem[NST * STAGE > USED ? NST * STAGE : USED];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ws = wave % WS, dch = (a.dim + 7) / 8;
  const Item it = item_of(blockIdx.x, a, a.group, tiles, a.causal && !ranks_tiles(a));
  if (a.fill && it.tile == tiles - 1) {
    zero_outside(a.seqs, false, a.dq, it.kvh * a.group + it.g, a.dim * sizeof(T));
    return;
  }
  const Seq s = find_seq(a, it.b, it.tile, tiles, BM, false);
  if (!s.ok) return;
  const int shift = s.nk - s.nq, head = it.kvh * a.group + it.g;
  const int r0 = s.tile * BM + wave / WS * 32;
  const int t0q = s.tile * BM;
  const KeyRange wg = keys_of(a, s, t0q, min(t0q + BM, s.nq) - 1);
  const KeyRange wv = keys_of(a, s, r0, min(r0 + 32, s.nq) - 1);
  const int t0 = wg.beg / SR, t1 = (wg.end + SR - 1) / SR;

  const uint32_t lds0 = lds_offset(smem);
  const uint32_t own = lds0 + ws * BN * L::RB, rbase = own + rows_base<DU>(lane), cbase = own + cols_base<DU>(lane);
  Stager<PL, DU, SR> ks, vs;
  ks.init(static_cast<uint32_t>(a.sk.token), dch);
  vs.init(static_cast<uint32_t>(a.sv.token), dch);
  const char* const krow = at_row(a.sk, it.b, s.k0, it.kvh);
  const char* const vrow = at_row(a.sv, it.b, s.k0, it.kvh);
  auto issue = [&](int t) __attribute__((always_inline)) {
    const uint32_t at = lds0 + t % NST * STAGE;
    const int64_t j = t * SR;
    ks.issue(krow + j * a.sk.token, a.plane, s.nk - t * SR, dch, at, wave);
    vs.issue(vrow + j * a.sv.token, a.plane, s.nk - t * SR, dch, at + TILE, wave);
  };
  if (NST > 1 && t0 < t1) issue(t0);

  Frag<PL> qf[L::STEPS], df[L::STEPS];
  const int r = r0 + (lane & 31), iq = min(r, s.q_rows - 1);
  const char* const dorow = at_row(a.dout, it.b, s.q0 + iq, head);
  load_operand<PL, DU>(at_row(a.q, it.b, s.q0 + iq, head), a.dim, half, qf);
  load_operand<PL, DU>(dorow, a.dim, half, df);
  const float delta = row_dots<PL, DU>(df, at_row(a.out, it.b, s.q0 + iq, head),
                                       PL == 1 && a.res.p ? at_row(a.res, it.b, s.q0 + iq, head) : nullptr, a.dim, lane);
  const int64_t row = row_index(a, it.b, head, s.q0 + iq);
  const float lse = r < s.nq ? a.lse[row] : -kInf;
  const float lse2 = lse == -kInf ? kInf : lse * kLog2e;
  if (ws == 0 && half == 0 && r < s.nq) {
    a.lse2[row] = lse2;
    a.delta[row] = delta;
  }
  const int jmax = a.causal ? min(s.nk - 1, iq + shift) : s.nk - 1;
  const int jmin = a.causal && a.window ? max(0, iq + shift - a.window + 1) : 0;
  f32x16_t acc[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) acc[db] = zero16();
  // fp32: the sums of the row's probabilities and of dS, and sum_j p_j k_j to bf16's accuracy
  LongSum total_j, rest_j;
  f32x16_t pk[PL == 3 ? L::DB : 1];
  if constexpr (PL == 3) {
#pragma unroll
    for (int db = 0; db < L::DB; ++db) pk[db] = zero16();
  }
  for (int t = t0; t < t1; ++t) {
    if constexpr (NST == 1) {
      __syncthreads();
      issue(t);
    }
    wait_loads();
    __syncthreads();
    if (NST > 1 && t + 1 < t1) issue(t + 1);
    const uint32_t rb = rbase + t % NST * STAGE, cb = cbase + t % NST * STAGE;
#pragma unroll
    for (int kb = 0; kb < BN / 32; ++kb) {
      const int j0 = t * SR + ws * BN + 32 * kb;
      if (j0 >= wv.end || j0 + 32 <= wv.beg) continue;
      f32x16_t p = zero16(), d = zero16();
      wave_priority<PL == 1>();
#pragma unroll
      for (int st = 0; st < L::STEPS; ++st) mma<PL>(frag_rows<PL, PLANE>(rb, 32 * kb * L::RB, st), qf[st], p);
#pragma unroll
      for (int st = 0; st < L::STEPS; ++st) mma<PL>(frag_rows<PL, PLANE>(rb, TILE + 32 * kb * L::RB, st), df[st], d);
      interleave<PR * 2 * L::STEPS, PL * 2 * L::STEPS, 4>();
      wave_priority<0>();
      if (j0 + 32 > wv.all_end || j0 < wv.all_beg) {
        asm volatile("; a tile that the mask cuts");
        const int lo = jmin - j0 - 4 * half, hi = jmax - j0 - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = 8 * (e >> 2) + (e & 3);
          if (j < lo || j > hi) p[e] = -kInf;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = exp2_(fmaf(p[e], a.scale2, -lse2));
        d[e] = x * (d[e] - delta);
        if constexpr (PL == 3) p[e] = x;
      }
      if constexpr (PL == 3) {
        total_j.add(sum16(p));
        rest_j.add(sum16(d));
      }
      wave_priority<PL == 1>();
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const Frag<PA> f = frag_acc<PA>(d, st);
#pragma unroll
        for (int db = 0; db < L::DB; ++db)
          if constexpr (PL == 3) {
            const Frag<3> c = frag_cols<3, DU, PLANE>(cb, 32 * kb * L::RB, st, db);
            mma<3>(c, f, acc[db]);
            Mma<uint16_t>::run(c.v[0], frag_acc<1>(p, st).v[0], pk[db]);
          } else {
            mma_acc<PL, PA>(frag_cols<PL, DU, PLANE>(cb, 32 * kb * L::RB, st, db), f, acc[db]);
          }
      }
      interleave<(PL == 3 ? 7 : PP) * 2 * L::DB, PL * 4 * L::DB, 6>();
      wave_priority<0>();
    }
  }
  float total = 0.f, rest = 0.f;
  if constexpr (PL == 3) {
    total = sum32(total_j.sum);
    rest = sum32(rest_j.sum);
  }
  if constexpr (WS > 1) {
    float2* const sums = reinterpret_cast<float2*>(smem + JOIN) + wave * 64 + lane;
    if constexpr (PL == 3) {
      join_waves<WS, L::DB>(pk, smem, wave, lane);
      *sums = make_float2(total, rest);
    }
    if (!join_waves<WS, L::DB>(acc, smem, wave, lane)) return;
    if constexpr (PL == 3) {
#pragma unroll
      for (int w = 1; w < WS; ++w) {
        total += sums[w * 64].x;
        rest += sums[w * 64].y;
      }
    }
  }
  float f = a.scale;
  if constexpr (PL == 3) {
    const float norm = row_norm(total, lse2);
    if (norm != 0.f) {
      // rows of dS sum to 0; what delta leaves, out being rounded, goes into it
      f *= norm;
      rest *= norm;
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] = fmaf(-rest, pk[db][e], acc[db][e]);
    }
    if (half == 0 && r < s.nq) {
      a.norm[row] = norm != 0.f ? norm : 1.f;
      if (norm != 0.f) a.delta[row] = delta + rest;
    }
  }
  if (r >= s.nq) {
#pragma unroll
    for (int db = 0; db < L::DB; ++db) acc[db] = zero16();
  }
  store_row<T, L::DB>(acc, f, at_row_w(a.dq, it.b, s.q0 + iq, head), nullptr, a.dim, half, r < s.q_rows);
}

// dK, dV: a wave holds 32 keys (K rows in registers, V rows there or, VL, in LDS;
// of three planes the smallest, where the registers do not hold all), the workgroup passes over the queries of one head, or of several heads
// of the group: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.  Its two
// accumulators and K leave no registers for a second row of queries, so that a
// step has 32 of them; V's place in LDS frees what two waves a SIMD need.  The
// case above: 279 us (275 GFLOP, MFMAs busy 55%, LDS 41%).
template <int PL, int DU, int BM, int WS, int NST, bool VL, bool FINE>
__global__ __launch_bounds__(256, WS == 1 && PL == 1 ? 2 : 1) void k_attn_dkv(AttnArgs a, int tiles) {
  constexpr int PA = kAccPlanes<PL, FINE>;
  constexpr int PR = PL == 3 ? 6 : 1, PP = PL == 3 ? 6 : PA;  // MFMAs of a product, and of one with an accumulator
  using L = Lay<DU>;
  using T = typename Io<PL>::T;
  constexpr int BK = 128 / WS, SR = BM * WS, PLANE = SR * L::RB, TILE = PL * PLANE, STAGE = 2 * TILE;
  constexpr int VPLANE = BK * L::RB, VT = VL ? VPLANE : 0;
  constexpr int JOIN = (WS - 1) * (4 / WS) * L::DB * 4096;
  static_assert(SR <= 128, "the rows' statistics");
  // V, the stages of Q and dO, those of the rows' statistics (128 floats of each kind)
  constexpr int STATS = PL == 3 ? 1536 : 1024, USED = VT + NST * (STAGE + STATS);
  __shared__ __attribute__((aligned(1024))) char smem[USED > JOIN ? USED : JOIN];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ws = wave % WS, dch = (a.dim + 7) / 8;
  const int heads = a.group / a.kv_parts;
  const Item it = item_of(blockIdx.x, a, a.kv_parts, tiles, false);
  if (a.fill && it.tile == tiles - 1) {
    if (a.kv_parts == 1) {  // (else the sum of the parts does)
      zero_outside(a.seqs, true, a.dk, it.kvh, a.dim * sizeof(T));
      zero_outside(a.seqs, true, a.dv, it.kvh, a.dim * sizeof(T));
    }
    return;
  }
  const Seq s = find_seq(a, it.b, it.tile, tiles, BK, true);
  if (!s.ok) return;
  const int shift = s.nk - s.nq;
  const int k0 = s.tile * BK, w0 = k0 + wave / WS * 32;
  // queries that see a key of the workgroup
  int qb = 0, qe = s.nq;
  if (a.causal) {
    qb = max(0, k0 - shift);
    if (a.window) qe = min(qe, min(k0 + BK, s.nk) - 1 - shift + a.window);
  }
  if (k0 >= s.nk) qe = 0;
  const int t0 = qb / SR, per = max(0, (qe + SR - 1) / SR - t0);
  const int steps = per * heads, h0 = it.kvh * a.group + it.g * heads;

  const uint32_t lds0 = lds_offset(smem), stats = lds0 + VT + NST * STAGE;
  const uint32_t own = lds0 + VT + ws * BM * L::RB, rbase = own + rows_base<DU>(lane), cbase = own + cols_base<DU>(lane);
  const uint32_t vbase = lds0 + wave / WS * 32 * L::RB + rows_base<DU>(lane);
  Stager<PL, DU, SR> qs, ds;
  qs.init(static_cast<uint32_t>(a.sq.token), dch);
  ds.init(static_cast<uint32_t>(a.sdo.token), dch);
  const char* const qrow = at_row(a.sq, it.b, s.q0, h0);
  const char* const drow = at_row(a.sdo, it.b, s.q0, h0);
  const int64_t srow = row_index(a, it.b, h0, s.q0);
  // the next tile to load: tile nt of head h0 + nh
  int nt = t0, nh = 0;
  auto issue = [&](int i) __attribute__((always_inline)) {
    const uint32_t at = lds0 + VT + i % NST * STAGE;
    const int64_t q = nt * SR;
    const int left = s.nq - nt * SR;
    qs.issue(qrow + nh * a.sq.head + q * a.sq.token, a.plane, left, dch, at, wave);
    ds.issue(drow + nh * a.sdo.head + q * a.sdo.token, a.plane, left, dch, at + TILE, wave);
    // the rows' statistics, 64 a wave (queries behind the last repeat it, and are masked)
    if (wave < 2 || SR > 64) {
      const float* p = (wave & 1 ? a.delta : a.lse2) + srow + nh * static_cast<int64_t>(a.seqs.q_tokens) + q;
      load_lds4(reinterpret_cast<const char*>(p), min(min((wave >> 1) * 64 + lane, SR - 1), left - 1) * 4,
                stats + i % NST * STATS + (wave & 1) * 512 + (wave >> 1) * 256);
    }
    if (PL == 3 && (SR > 64 ? wave < 2 : wave == 2)) {
      const int at64 = SR > 64 ? wave * 64 : 0;
      load_lds4(reinterpret_cast<const char*>(a.norm + srow + nh * static_cast<int64_t>(a.seqs.q_tokens) + q),
                min(min(at64 + lane, SR - 1), left - 1) * 4, stats + i % NST * STATS + 1024 + at64 * 4);
    }
    if (++nt == t0 + per) { nt = t0; ++nh; }
  };
  if (NST > 1 && steps > 0) issue(0);

  constexpr int VR = PL - VL;  // V's planes in registers
  Frag<PL> kf[L::STEPS];
  Frag<VR ? VR : 1> vf[VR ? L::STEPS : 1];
  const int r = w0 + (lane & 31), j = min(r, s.k_rows - 1);
  load_operand<PL, DU>(at_row(a.k, it.b, s.k0 + j, it.kvh), a.dim, half, kf);
  if constexpr (VR > 0) {
#pragma unroll
    for (int st = 0; st < L::STEPS; ++st) {
      const Frag<PL> f = load_chunk<PL>(at_row(a.v, it.b, s.k0 + j, it.kvh), 2 * st + half, a.dim);
#pragma unroll
      for (int p = 0; p < VR; ++p) vf[st].v[p] = f.v[p];
    }
  }
  const int qmin = a.causal ? j - shift : 0;
  const int qmax = a.causal && a.window ? min(s.nq - 1, j - shift + a.window - 1) : s.nq - 1;
  if constexpr (VL) {
    if (steps > 0)  // zeros beyond the head: dO's tiles repeat a chunk there
      for (int p = threadIdx.x; p < BK * L::CH; p += 256) {
        const int vr = p / L::CH, c = p % L::CH;
        const Frag<PL> f = load_chunk<PL>(at_row(a.v, it.b, s.k0 + min(k0 + vr, s.nk - 1), it.kvh), c, a.dim);
        *reinterpret_cast<u32x4_t*>(smem + L::at(vr, c)) = f.v[PL - 1];
      }
  }
  f32x16_t dk[L::DB], dv[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) dk[db] = dv[db] = zero16();
  const int w_hi = min(w0 + 32, s.nk) - 1;  // the wave's last key
  int ct = t0;
  for (int i = 0; i < steps; ++i) {
    if constexpr (NST == 1) {
      __syncthreads();
      issue(i);
    }
    wait_loads();
    __syncthreads();
    if (NST > 1 && i + 1 < steps) issue(i + 1);
    const uint32_t rb = rbase + i % NST * STAGE, cb = cbase + i % NST * STAGE;
    const uint32_t sb = stats + i % NST * STATS + ws * BM * 4 + 16 * half;
    const int q0 = ct * SR + ws * BM;
    if (++ct == t0 + per) ct = t0;
#pragma unroll
    for (int qk = 0; qk < BM / 32; ++qk) {
      const int q = q0 + 32 * qk;
      if (q >= s.nq || w_hi < w0) continue;
      if (a.causal && q + 31 + shift < w0) continue;
      if (a.causal && a.window && q + shift - w_hi >= a.window) continue;
      f32x16_t p = zero16(), d = zero16();
      wave_priority<PL == 1>();
#pragma unroll
      for (int st = 0; st < L::STEPS; ++st) mma<PL, true>(frag_rows<PL, PLANE>(rb, 32 * qk * L::RB, st), kf[st], p);
#pragma unroll
      for (int st = 0; st < L::STEPS; ++st) {
        const Frag<PL> f = frag_rows<PL, PLANE>(rb, TILE + 32 * qk * L::RB, st);
        Frag<PL> v;
        if constexpr (VL) v.v[PL - 1] = frag_rows<1, VPLANE>(vbase, 0, st).v[0];
#pragma unroll
        for (int p = 0; p < VR; ++p) v.v[p] = vf[st].v[p];
        mma<PL, true>(f, v, d);
      }
      interleave<PR * 2 * L::STEPS, (2 * PL + VL) * L::STEPS, 6>();
      wave_priority<0>();
      if (q + 32 > s.nq || (a.causal && q + shift < w0 + 31) ||
          (a.causal && a.window && q + 31 + shift - w0 >= a.window)) {
        asm volatile("; a tile that the mask cuts");
        const int lo = qmin - q - 4 * half, hi = qmax - q - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int x = 8 * (e >> 2) + (e & 3);
          if (x < lo || x > hi) p[e] = -kInf;
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const u32x4_t ls = lds16(sb + (32 * qk + 8 * g) * 4), de = lds16(sb + 512 + (32 * qk + 8 * g) * 4);
        u32x4_t norm;
        if constexpr (PL == 3) norm = lds16(sb + 1024 + (32 * qk + 8 * g) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = exp2_(fmaf(p[4 * g + e], a.scale2, -__uint_as_float(ls[e])));
          if constexpr (PL == 3) x *= __uint_as_float(norm[e]);
          p[4 * g + e] = x;
          d[4 * g + e] = x * (d[4 * g + e] - __uint_as_float(de[e]));
        }
      }
      wave_priority<PL == 1>();
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const Frag<PA> f = frag_acc<PA>(p, st);
#pragma unroll
        for (int db = 0; db < L::DB; ++db)
          mma_acc<PL, PA>(frag_cols<PL, DU, PLANE>(cb, TILE + 32 * qk * L::RB, st, db), f, dv[db]);
      }
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const Frag<PA> f = frag_acc<PA>(d, st);
#pragma unroll
        for (int db = 0; db < L::DB; ++db) mma_acc<PL, PA>(frag_cols<PL, DU, PLANE>(cb, 32 * qk * L::RB, st, db), f, dk[db]);
      }
      interleave<PP * 4 * L::DB, PL * 8 * L::DB, 6>();
      wave_priority<0>();
    }
  }
  if constexpr (WS > 1) {
    join_waves<WS, L::DB>(dk, smem, wave, lane);
    if (!join_waves<WS, L::DB>(dv, smem, wave, lane)) return;
  }
  if (r >= s.nk) {
#pragma unroll
    for (int db = 0; db < L::DB; ++db) dk[db] = dv[db] = zero16();
  }
  const bool on = r < s.k_rows;
  if (a.kv_parts > 1) {
    const int64_t row = ((static_cast<int64_t>(it.b) * a.seqs.k_tokens + s.k0 + j) * a.kv_heads + it.kvh) * a.kv_parts + it.g;
    store_row<float, L::DB>(dk, a.scale, reinterpret_cast<char*>(a.part_dk + row * a.dim), nullptr, a.dim, half, on);
    store_row<float, L::DB>(dv, 1.f, reinterpret_cast<char*>(a.part_dv + row * a.dim), nullptr, a.dim, half, on);
  } else {
    store_row<T, L::DB>(dk, a.scale, at_row_w(a.dk, it.b, s.k0 + j, it.kvh), nullptr, a.dim, half, on);
    store_row<T, L::DB>(dv, 1.f, at_row_w(a.dv, it.b, s.k0 + j, it.kvh), nullptr, a.dim, half, on);
  }
}

// Sums the parts of each group, in order: a thread has 4 elements of dk or dv.
// At memory's rate: 134 MB in 23 us.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sum_heads(AttnArgs a) {
  const int quads = a.dim / 4;
  const int64_t n = static_cast<int64_t>(a.seqs.batch) * a.seqs.k_tokens * a.kv_heads * quads;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (at >= 2 * n) return;
  const bool second = at >= n;
  const int64_t i = second ? at - n : at;
  const int quad = static_cast<int>(i % quads);
  const int64_t kh = i / quads, tok = kh / a.kv_heads;
  const int head = static_cast<int>(kh % a.kv_heads);
  const int b = static_cast<int>(tok / a.seqs.k_tokens), j = static_cast<int>(tok % a.seqs.k_tokens);
  bool held = true;  // by a sequence
  if (a.seqs.q_off) {
    int lo, hi;
    outside_of(a.seqs, true, lo, hi);
    held = j >= lo && j < hi;
    if (!held && !a.fill) return;
  }
  const float* p = (second ? a.part_dv : a.part_dk) + (tok * a.kv_heads + head) * a.kv_parts * a.dim + 4 * quad;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int g = 0; g < a.kv_parts && held; ++g, p += a.dim) {
    const float4 y = *reinterpret_cast<const float4*>(p);
    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
  }
  char* row = at_row_w(second ? a.dv : a.dk, b, j, head);
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(row + quad * 8) = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
  else
    *reinterpret_cast<float4*>(row + quad * 16) = x;
}

// ---------------------------------------------------------------------------
// Rotary positions.  A workgroup takes a few tokens: their angles once (fp64
// product and reduction to a fraction of a turn, then fp32 sine and cosine),
// through LDS to every head.  HBM-bound: each element is read and written once
// (8192 tokens of 40 heads of 128 bf16, 168 MB, in 28 us).
// ---------------------------------------------------------------------------
// Unit u of a head: a piece that turns (u < turning), else one that is copied.
template <typename T>
__device__ __forceinline__ void rotary_unit(const RotaryArgs& a, const T* x, T* y, const float2* w, int u, int turning,
                                            bool vec) {
  constexpr int EPC = 16 / sizeof(T);
  const int half = a.rot / 2, width = vec ? EPC : 1;
  if (u >= turning) {
    const int d = a.rot + (u - turning) * width;
    if (vec) *reinterpret_cast<u32x4_t*>(y + d) = *reinterpret_cast<const u32x4_t*>(x + d);
    else y[d] = x[d];
  } else if (!vec) {
    const int p = a.interleaved ? 2 * u : u, q = a.interleaved ? p + 1 : u + half;
    const float c = w[u].x, sn = w[u].y, e = to_f32<T>(x[p]), f = to_f32<T>(x[q]);
    y[p] = from_f32<T>(e * c - f * sn);
    y[q] = from_f32<T>(e * sn + f * c);
  } else {
    // a piece of EPC elements: pairs of it (interleaved), or it and the piece
    // half a rotation further
    float e[8], f[8];
    if constexpr (sizeof(T) == 2) load8(x, u * EPC, e);
    else *reinterpret_cast<float4*>(e) = *reinterpret_cast<const float4*>(x + u * EPC);
    if (a.interleaved) {
#pragma unroll
      for (int q = 0; q < EPC / 2; ++q) {
        const float2 cw = w[u * (EPC / 2) + q];
        const float g = e[2 * q], h = e[2 * q + 1];
        e[2 * q] = g * cw.x - h * cw.y;
        e[2 * q + 1] = g * cw.y + h * cw.x;
      }
    } else {
      if constexpr (sizeof(T) == 2) load8(x, u * EPC + half, f);
      else *reinterpret_cast<float4*>(f) = *reinterpret_cast<const float4*>(x + u * EPC + half);
#pragma unroll
      for (int q = 0; q < EPC; ++q) {
        const float2 cw = w[u * EPC + q];
        const float g = e[q], h = f[q];
        e[q] = g * cw.x - h * cw.y;
        f[q] = g * cw.y + h * cw.x;
      }
      if constexpr (sizeof(T) == 2) store8(y, u * EPC + half, f);
      else *reinterpret_cast<float4*>(y + u * EPC + half) = *reinterpret_cast<const float4*>(f);
    }
    if constexpr (sizeof(T) == 2) store8(y, u * EPC, e);
    else *reinterpret_cast<float4*>(y + u * EPC) = *reinterpret_cast<const float4*>(e);
  }
}

constexpr int kRotPairs = 512;  // angles of a workgroup
template <typename T>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a, int per_block) {
  constexpr int EPC = 16 / sizeof(T);
  __shared__ float2 turn[kRotPairs];
  const int half = a.rot / 2;
  const int64_t all = a.batch * a.tokens, first = static_cast<int64_t>(blockIdx.x) * per_block;
  const int n = static_cast<int>(min(static_cast<int64_t>(per_block), all - first));
  for (int i = threadIdx.x; i < n * half; i += 256) {
    const int64_t tok = first + i / half, b = tok / a.tokens, t = tok % a.tokens;
    int64_t pos = t;
    if (a.positions) {
      const int64_t at = b * a.pos_batch + t * a.pos_token;
      pos = a.positions64 ? static_cast<const int64_t*>(a.positions)[at] : static_cast<const int32_t*>(a.positions)[at];
    }
    const double rev = static_cast<double>(pos + a.first) * (a.freqs[i % half] * 0.15915494309189533577);
    float sn, cs;
    sincospif(static_cast<float>(2.0 * (rev - rint(rev))), &sn, &cs);
    turn[i] = make_float2(cs * a.scale, sn * a.scale * a.sign);
  }
  __syncthreads();
  for (int k = 0; k < a.n; ++k) {
    const RotaryTensor& t = a.t[k];
    const bool vec = t.vec != 0, same = t.x.p == t.y.p;
    // units of a head: pieces that turn, then pieces that are copied
    const int width = vec ? EPC : 1;
    const int turning = (a.interleaved ? a.rot / (vec ? EPC : 2) : half / width);
    const int units = turning + (same ? 0 : (a.dim - a.rot) / width);
    if (units == 0 || t.heads == 0) continue;
    // unit u of head `head` of token tk, by steps of 256 units
    int u = threadIdx.x % units, head = threadIdx.x / units, tk = head / t.heads;
    head -= tk * t.heads;
    const int du = 256 % units, dh = 256 / units % t.heads, dt = 256 / units / t.heads;
    while (tk < n) {
      const int64_t tok = first + tk, b = tok / a.tokens, at = tok - b * a.tokens;
      const T* x = reinterpret_cast<const T*>(t.x.p + b * t.x.batch + at * t.x.token + head * t.x.head);
      T* y = reinterpret_cast<T*>(t.y.p + b * t.y.batch + at * t.y.token + head * t.y.head);
      rotary_unit<T>(a, x, y, turn + tk * half, u, turning, vec);
      u += du;
      head += dh;
      tk += dt;
      if (u >= units) { u -= units; ++head; }
      if (head >= t.heads) { head -= t.heads; ++tk; }
    }
  }
}

// ---------------------------------------------------------------------------
// The clip.  A workgroup has a few rows of one entry; rows whose factor is 1
// are not touched.  HBM-bound on the rows that change: 671 MB in 120 us.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float clip_gamma(float m, float threshold) {
  return m > threshold && m < kInf ? fmaxf(threshold / m, 0x1p-126f) : 1.f;  // (0 would have no root to divide by)
}
template <typename T>
__global__ __launch_bounds__(256) void k_qk_clip(ClipArgs a) {
  constexpr int EPC = 16 / sizeof(T);
  __shared__ float factor[kClipRows];
  int k = 0;
  for (int step = kClipMax / 2; step > 0; step /= 2)  // the last entry that starts at or before this workgroup
    if (k + step < a.n && a.first[k + step] <= static_cast<int>(blockIdx.x)) k += step;
  const ClipEntry& e = a.e[k];
  const int lane = threadIdx.x & 63, group = e.q_heads / e.kv_heads;
  const int rows_q = e.q_heads * e.dim, rows = rows_q + e.kv_heads * e.dim;
  const int base = (blockIdx.x - a.first[k]) * a.rows;
  bool any = false;
  if (static_cast<int>(threadIdx.x) < a.rows) {
    const int row = base + threadIdx.x;
    float f = 1.f;
    if (row < rows) {
      const bool is_q = row < rows_q;
      const int head = (is_q ? row : row - rows_q) / e.dim, kvh = is_q ? head / group : head;
      float least = 1.f;
      for (int g = 0; g < group; ++g) least = fminf(least, clip_gamma(e.logits[kvh * group + g], e.threshold));
      const float key = sqrtf(least);
      f = is_q ? clip_gamma(e.logits[head], e.threshold) / key : key;
    }
    factor[threadIdx.x] = f;
    any = f != 1.f;
  }
  if (!__syncthreads_or(any)) return;
  for (int i = threadIdx.x >> 6; i < a.rows; i += 4) {
    const int row = base + i;
    const float f = factor[i];
    if (f == 1.f) continue;
    const bool is_q = row < rows_q;
    const int at = is_q ? row : row - rows_q;
    T* w = reinterpret_cast<T*>(is_q ? e.wq + at * e.ldq : e.wk + at * e.ldk);
    int done = 0;
    if (e.vec) {
      const int chunks = e.cols / EPC;
      done = chunks * EPC;
      u32x4_t* const w16 = reinterpret_cast<u32x4_t*>(w);
      for (int c = lane; c < chunks; c += 8 * 64) {
        u32x4_t v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c + q * 64 < chunks) v[q] = w16[c + q * 64];
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c + q * 64 < chunks) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if constexpr (sizeof(T) == 2)
                v[q][x] = pack_bf16x2(__uint_as_float(v[q][x] << 16) * f, __uint_as_float(v[q][x] & 0xffff0000u) * f);
              else
                v[q][x] = __float_as_uint(__uint_as_float(v[q][x]) * f);
            }
            w16[c + q * 64] = v[q];
          }
      }
    }
    for (int c = done + lane; c < e.cols; c += 64) w[c] = from_f32<T>(to_f32<T>(w[c]) * f);
  }
}
__global__ __launch_bounds__(256) void k_reset_logits(ClipArgs a) {
  const ClipEntry& e = a.e[blockIdx.x];
  for (int i = threadIdx.x; i < e.q_heads; i += 256) e.logits[i] = -kInf;
}

// Tiles of `bt` tokens: exactly per sequence (dense), or as many as packed
// sequences can have.
int64_t tiles_of(const Seqs& s, int64_t tokens, int bt) {
  return (tokens + bt - 1) / bt + (s.q_off ? s.n_seq : 0);
}
// The tiles of a launch: one more for the rows that no sequence holds.
int64_t launch_tiles(const AttnArgs& a, int64_t tokens, int bt) { return tiles_of(a.seqs, tokens, bt) + (a.fill ? 1 : 0); }
// Visible pairs of a dense request: of keys 1 .. nk that the last query sees, each
// query before sees one less (causal), and none more than the window.  Where
// lengths or offsets on the device cut it, no less than what they leave.
double pairs_of(const AttnArgs& a) {
  const double nq = a.seqs.q_tokens, nk = a.seqs.k_tokens, all = double(a.seqs.batch) * a.q_heads;
  if (!a.causal) return all * nq * nk;
  const double first = std::max(0.0, nk - nq), most = a.window ? std::min(double(a.window), nk) : nk;
  const auto upto = [](double n) { return n * (n + 1) / 2; };
  return all * (upto(most) - upto(std::min(first, most)) + most * (nk - std::max(first, most)));
}

// One tile of rows holds every query of every head of a group.
bool packs_heads(const Seqs& s, int group) {
  return !s.q_off && group > 1 && int64_t(s.q_tokens) * group <= 128;
}

// The arrays that the tiles of a pass come from: the caller's, or (fp32) the
// planes, which this launches the making of.
hipError_t stage_sources(AttnArgs& a, int dtype, bool backward, hipStream_t st) {
  a.sq = a.q; a.sk = a.k; a.sv = a.v; a.sdo = a.dout;
  a.plane = 0;
  if (dtype == DT_BF16) return hipSuccess;
  const int chunks = (a.dim + 7) / 8;
  a.plane = chunks * 16;
  SplitArgs x{};
  x.dim = a.dim;
  const auto add = [&](const Heads& from, char* to, int tokens, int heads, Heads& staged) {
    x.from[x.n] = from;
    x.to[x.n] = to;
    x.tokens[x.n] = tokens;
    x.heads[x.n] = heads;
    x.first[x.n + 1] = x.first[x.n] + a.seqs.batch * tokens * heads * chunks;
    ++x.n;
    staged = Heads{to, int64_t(heads) * tokens * 3 * a.plane, int64_t(3) * a.plane, int64_t(tokens) * 3 * a.plane};
  };
  add(a.k, a.split_k, a.seqs.k_tokens, a.kv_heads, a.sk);
  add(a.v, a.split_v, a.seqs.k_tokens, a.kv_heads, a.sv);
  if (backward) {
    add(a.q, a.split_q, a.seqs.q_tokens, a.q_heads, a.sq);
    add(a.dout, a.split_do, a.seqs.q_tokens, a.q_heads, a.sdo);
  }
  if (x.first[x.n] == 0) return hipSuccess;
  hipLaunchKernelGGL(k_split, dim3(static_cast<unsigned>((x.first[x.n] + 255) / 256)), dim3(256), 0, st, x);
  return hipGetLastError();
}

template <int PL, int DU, int BN, int WS, int NST, bool FINE = false, int NW = 4>
hipError_t forward_of(const AttnArgs& a, hipStream_t st) {
  const bool pack = packs_heads(a.seqs, a.group);
  const int64_t tiles = launch_tiles(a, int64_t(a.seqs.q_tokens) * (pack ? a.group : 1), 32 * NW / WS);
  const int64_t grid = a.seqs.batch * a.kv_heads * (pack ? 1 : a.group) * tiles * a.splits;
  const dim3 g(static_cast<unsigned>(grid)), b(64 * NW);
  if (a.splits == 1) {
    hipLaunchKernelGGL((k_attn_fwd<PL, DU, BN, WS, NST, FINE, false, NW>), g, b, 0, st, a, int(tiles), int(pack));
    return hipGetLastError();
  }
  // split passes are of few queries: no 8 waves, and rows beyond fine_of's are so
  // many heads that their parts are many workgroups too
  if constexpr (NW == 8 || (PL == 1 && WS == 4 && !FINE)) return hipErrorInvalidValue;
  else hipLaunchKernelGGL((k_attn_fwd<PL, DU, BN, WS, NST, FINE, true, NW>), g, b, 0, st, a, int(tiles), int(pack));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = a.seqs.batch * a.q_heads * int64_t(a.seqs.q_tokens);
  hipLaunchKernelGGL((k_attn_join<typename Io<PL>::T>), dim3(static_cast<unsigned>(rows)), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int PL, int DU, int BN, int WS, int NST, bool FINE = false>
hipError_t dq_of(const AttnArgs& a, hipStream_t st) {
  const int64_t tiles = launch_tiles(a, a.seqs.q_tokens, 128 / WS);
  hipLaunchKernelGGL((k_attn_dq<PL, DU, BN, WS, NST, FINE>), dim3(static_cast<unsigned>(a.seqs.batch * a.q_heads * tiles)),
                     dim3(256), 0, st, a, int(tiles));
  return hipGetLastError();
}
template <int PL, int DU, int BM, int WS, int NST, bool VL, bool FINE = false>
hipError_t dkv_of(const AttnArgs& a, hipStream_t st) {
  const int64_t tiles = launch_tiles(a, a.seqs.k_tokens, 128 / WS);
  const int64_t grid = a.seqs.batch * a.kv_heads * a.kv_parts * tiles;
  hipLaunchKernelGGL((k_attn_dkv<PL, DU, BM, WS, NST, VL, FINE>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, st, a,
                     int(tiles));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.kv_parts == 1) return e;
  const int64_t n = 2 * a.seqs.batch * int64_t(a.seqs.k_tokens) * a.kv_heads * (a.dim / 4);
  hipLaunchKernelGGL((k_attn_sum_heads<typename Io<PL>::T>), dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0,
                     st, a);
  return hipGetLastError();
}

// How many waves share their rows (WS in the kernels): more than one where
// workgroups of 128 rows would leave compute units idle and a row has enough to
// pass over, as long as the device holds all of them at once (256 workgroups of
// heads of more than 64 elements, 512 of narrower ones; a causal pass ends half
// or a third of them early).  Measured on an MI355X, WS = 1 / 2 / 4, us forward
// (gradients), 4096 tokens unless said otherwise:
//   heads of 128, no mask:  64 workgroups 76 / 63 / 42 (266 / 199 / 134), 128:
//     76 / 64 / 83 (273 / 204 / 258), 160: 78 / 84 / 131 (275 / 393 / 391)
//   causal: 128: 77 / 63 / 50 (270 / 201 / 157), 256: 78 / 69 / 97 (274 / 226 /
//     297), 384: 83 / 79 / 153 (288 / 357 / 454)
//   heads of 64, no mask: 128: 56 / 50 / 36 (173 / 131 / 106), 160: 57 / 58 / 59
//     (177 / 151 / 172), 256: 56 / 60 / 68 (177 / 165 / 198), 288: 81 / 77 / 89
//     (221 / 245 / 266)
//   causal: 192: 56 / 49 / 34 (174 / 135 / 98), 256: 57 / 49 / 41 (176 / 137 /
//     121), 384: 59 / 51 / 58 (184 / 149 / 173), 512: 61 / 58 / 75 (192 / 174 /
//     221), 512 of 1024 tokens: 20 / 23 / 34 (60 / 65 / 96)
//   windows of 1024, heads of 128, 384: 44 / 66 / 106 (125 / 196 / 296)
//   fp32, 1024 tokens, WS = 1 / 2 (more than 64 elements) or 4 (one stage in LDS;
//   gradients before their rows were normalised, which takes 4% more):
//     128, no mask, 128: 93 / 70 (313 / 196), 192: 95 / 127 (322 / 360); causal,
//     256: 96 / 84 (329 / 231), 320: 100 / 112 (344 / 323)
//     64, no mask, 128: 55 / 55 (159 / 140), 192: 57 / 77 (164 / 205); causal,
//     192: 57 / 56 (162 / 141), 256: 57 / 69 (166 / 180); 144 of 128 tokens:
//     21 / 32 (48 / 75)
int waves_a_row(const AttnArgs& a, int dtype, int64_t workgroups, int64_t stream) {
  const bool window = a.causal && a.window, narrow = a.dim <= 64;
  if (window) stream = std::min<int64_t>(stream, int64_t(a.window) + 128);
  const int64_t whole = workgroups, slots = narrow ? 512 : 256;
  if (a.causal && !window && stream >= 512) workgroups = narrow ? workgroups * 2 / 3 : workgroups / 2;
  if (dtype != DT_BF16) {
    const int ws = narrow ? 4 : 2;
    return stream >= 512 ? (workgroups * ws <= slots ? ws : 1) : stream >= 96 && whole * ws <= 256 ? ws : 1;
  }
  if (stream >= 512 && workgroups * 4 <= slots) return 4;
  return stream >= 256 && workgroups * 2 <= slots ? 2 : 1;
}

// Whether a forward workgroup has 8 waves, which halves the loads of tiles into
// LDS and leaves one barrier to 128 keys, but makes waves wait for those that the
// mask leaves more keys, and a tile of 256 rows out of a short sequence.
// Measured on an MI355X, 8 waves' time to 4's (workgroups of 8):
//   no mask, heads of 64 / 128: 0.94 / 0.99 for 8 x 512 tokens (256), 0.90 /
//     0.94 for 4 x 1024 (256), 0.89 / 0.92 for 4096 (256), - / 0.85 (160), but
//     1.05 for 64 x 130 (1024), and 11 sequences in 8192: 1.07
//   causal, heads of 128: 1.07 (256), 0.98 (384) and 0.89 (512) for 4096 tokens,
//     0.92 for 4 x 2048 (512), 1.0 for 8 x 1024 (512), 1.03 for 32 x 256 (512);
//     of 64: 1.05 (512), 0.95 (1024), 0.91 for 16 x 2048 (2048), 0.97 for 32 x
//     1024 (2048); 6 sequences in 16384: 0.97 / 0.97, 40 in 8192: 1.14
//   causal in a window, heads of 64: 0.89 to 0.95 for windows of 128 to 1024 in
//     4096 and 8192 tokens (256 and 512), of 96: 0.96, of 128: 0.98 to 1.09; 20
//     sequences in 16384: 1.04
bool eight_waves(const AttnArgs& a, int64_t workgroups, int64_t rows) {
  if (a.seqs.q_off) rows = a.seqs.n_seq ? rows / a.seqs.n_seq : 0;
  if (rows < (a.seqs.q_off || a.causal ? 2048 : 512)) return false;
  if (!a.causal) return workgroups >= 160;
  if (a.window) return workgroups >= 256 && a.dim <= 96;
  return workgroups >= (a.dim <= 64 ? 1024 : 512);
}

// Whether probabilities and their gradients are taken in two planes: where the
// rows are few.  With one, an output's error is 1.4 times that of the exact one
// rounded (up to 2^-8 of each probability beside 2^-8 of the result), on average; of
// 300 random requests 7 with up to 4096 rows came to 1.5 to 2.  Query gradients
// of heads of up to 32 elements too: the few keys that a query selects resemble
// each other there, their terms cancel, and one plane leaves 1.6 times.
bool fine_of(const AttnArgs& a) { return a.seqs.batch * a.q_heads * int64_t(a.seqs.q_tokens) <= 4096; }

// Kernels for heads of up to 64, 96 and 128 elements: those of up to 96 skip a
// quarter of the products and LDS reads of 128.
template <typename F>
hipError_t by_width(int dim, F&& f) {
  if (dim <= 64) return f(std::integral_constant<int, 64>{});
  if (dim <= 96) return f(std::integral_constant<int, 96>{});
  return f(std::integral_constant<int, 128>{});
}

}  // namespace

// A single pass where its workgroups fill the device or its keys are few; else
// parts of at least four tiles each, for two workgroups a CU.  Measured on an
// MI355X, one part / these, us:
//   one token, 32 heads on 8 of 128: 32 x 4096 keys 119 / 115 (2 parts); 16 heads
//     of 64, 16 x 4096: 78 / 48 (2); 32 x 1024: 29 / 30 (2)
//   more than 128 queries, heads of 128 (waves sharing rows / these): 512 on 8192
//     keys, 32 heads 159 / 97 (4 parts), on 4096 80 / 62, on 2048 45 / 46; 256 on
//     3000 34 / 37; 1024 on 4096, 16 heads 75 / 63; 4096 on 4096, 4 heads 54 / 60;
//     200 on 2 x 8192 167 / 92; of 64: 512 on 8192, 16 heads 51 / 42, on 4096, 8
//     heads 32 / 26; 1024 on 4096, 8 heads 28 / 34; 4 x 256 on 4096, 16 heads 41 / 50
int forward_splits(const Seqs& s, int q_heads, int kv_heads, int dim, bool causal, int window) {
  if (s.q_off || (causal && window)) return 1;
  const bool many = s.q_tokens > 128, pack = packs_heads(s, q_heads / kv_heads);
  if (many && (s.k_tokens < 4096 || s.k_tokens / s.q_tokens < (dim <= 64 ? 8 : 4))) return 1;
  const int64_t items = s.batch * (pack ? int64_t(kv_heads) : q_heads * tiles_of(s, s.q_tokens, 128));
  if (items == 0 || items > (!many ? 256 : dim <= 64 ? 64 : 255)) return 1;
  const int64_t parts = std::min<int64_t>(512 / items, s.k_tokens / 256);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(parts, 64)));
}

// The smallest number of parts that gives the device enough workgroups: parts
// cost fp32 gradients written and added up, too few workgroups leave compute
// units idle, most in a long causal pass, whose first keys take longest.
// Measured on an MI355X, groups of 4, 1 / 2 / 4 parts, us (workgroups of 1 part):
//   causal, 4096 tokens x 8 heads of 128: 657 / 567 / 481 (256); 2 of them: 1065
//     / 915 / 957 (512); 4: 1722 / 1794 / 1905 (1024); 4 x 2048: 562 / 512 / 577
//     (512); 8 x 1024: 321 / 333 / 400 (512); 4 x 1024: 197 / 185 / 188 (256);
//     8 x 512: 127 / 124 / 145 (256); 4 x 512: 88 / 87 / 77 (128); 32 x 128: 77 /
//     85 / 114 (256); 16 x 128, heads of 64: 27 / 34 / 38 (128)
//   a window of 1024 in 8192: 474 / 519 / 575 (512); of 512 in 4096: 181 / 170 /
//     195 (256); no mask, 4096: 987 / 845 / 866 (256), 4 x 2048: 833 / 885 / 955
//     (512), 2048: 311 / 273 / 242 (128)
int backward_parts(const Seqs& s, int q_heads, int kv_heads, bool causal, int window) {
  const int group = q_heads / kv_heads;
  const int64_t items = s.batch * kv_heads * tiles_of(s, s.k_tokens, 128);
  const int64_t length = s.q_off ? s.k_tokens / std::max(1, s.n_seq) : s.k_tokens;
  const int64_t enough = length <= 128 ? 128 : length >= 2048 && causal && !window ? 1024 : 512;
  for (int p = 1; p < group; ++p)
    if (group % p == 0 && items * p >= enough) return p;
  return group;
}

hipError_t run_attention_forward(AttnArgs a, int dtype, hipStream_t st, LaunchTimer* timer) {
  if (a.seqs.batch * a.seqs.q_tokens == 0) return hipSuccess;
  Timed tm(timer, KK_ATTENTION_FWD, st);
  hipError_t e = stage_sources(a, dtype, false, st);
  if (e != hipSuccess) return e;
  const bool pack = packs_heads(a.seqs, a.group);
  const int64_t rows = pack ? int64_t(a.seqs.q_tokens) * a.group : a.seqs.q_tokens;
  const int64_t items = a.seqs.batch * a.kv_heads * (pack ? 1 : a.group);
  const int ws = waves_a_row(a, dtype, items * tiles_of(a.seqs, rows, 128) * a.splits, a.seqs.k_tokens / a.splits);
  const bool wide = ws == 1 && a.splits == 1 && eight_waves(a, items * tiles_of(a.seqs, rows, 256), rows);
  e = by_width(a.dim, [&](auto w) {
    constexpr int DU = decltype(w)::value;
    if (dtype != DT_BF16) return ws > 1 ? forward_of<3, DU, 32, DU <= 64 ? 4 : 2, 1>(a, st) : forward_of<3, DU, 32, 1, 2>(a, st);
    if (fine_of(a)) return ws == 4 ? forward_of<1, DU, 32, 4, 2, true>(a, st) : forward_of<1, DU, 64, 1, 2, true>(a, st);
    if (ws == 4) return forward_of<1, DU, 32, 4, 2>(a, st);
    if (ws == 2) return forward_of<1, DU, 32, 2, 2>(a, st);
    return wide ? forward_of<1, DU, 64, 1, 2, false, 8>(a, st) : forward_of<1, DU, 64, 1, 2>(a, st);
  });
  const double es = dtype == DT_BF16 ? 2 : 4, b = double(a.seqs.batch);
  if (e == hipSuccess)
    tm.done(4.0 * pairs_of(a) * a.dim, 0,
            b * a.dim * es * 2.0 * (double(a.seqs.q_tokens) * a.q_heads + double(a.seqs.k_tokens) * a.kv_heads));
  return e;
}

hipError_t run_attention_backward(AttnArgs a, int dtype, hipStream_t st, LaunchTimer* timer) {
  if (a.seqs.batch == 0) return hipSuccess;
  Timed tm(timer, KK_ATTENTION_BWD, st);
  hipError_t e = stage_sources(a, dtype, true, st);
  if (e != hipSuccess) return e;
  const int ws_q = waves_a_row(a, dtype, a.seqs.batch * a.q_heads * tiles_of(a.seqs, a.seqs.q_tokens, 128), a.seqs.k_tokens);
  const int ws_k = waves_a_row(a, dtype, a.seqs.batch * a.kv_heads * a.kv_parts * tiles_of(a.seqs, a.seqs.k_tokens, 128),
                               int64_t(a.seqs.q_tokens) * (a.group / a.kv_parts));
  e = by_width(a.dim, [&](auto w) {
    constexpr int DU = decltype(w)::value, WS3 = DU <= 64 ? 4 : 2;
    constexpr bool VL = DU > 64;
    hipError_t r = hipSuccess;
    if (a.seqs.q_tokens > 0) {
      if (dtype != DT_BF16) r = ws_q > 1 ? dq_of<3, DU, 32, WS3, 1>(a, st) : dq_of<3, DU, 32, 1, 2>(a, st);
      else if (fine_of(a) || a.dim <= 32) r = ws_q == 4 ? dq_of<1, DU, 32, 4, 2, true>(a, st) : dq_of<1, DU, 64, 1, 2, true>(a, st);
      else if (ws_q == 4) r = dq_of<1, DU, 32, 4, 2>(a, st);
      else r = ws_q == 2 ? dq_of<1, DU, 32, 2, 2>(a, st) : dq_of<1, DU, 64, 1, 2>(a, st);
    }
    if (r != hipSuccess || a.seqs.k_tokens == 0) return r;
    if (dtype != DT_BF16) return ws_k > 1 ? dkv_of<3, DU, 32, WS3, 1, false>(a, st) : dkv_of<3, DU, 32, 1, 2, DU == 128>(a, st);
    if (fine_of(a)) return ws_k == 4 ? dkv_of<1, DU, 32, 4, 2, VL, true>(a, st) : dkv_of<1, DU, 32, 1, 2, VL, true>(a, st);
    if (ws_k == 4) return dkv_of<1, DU, 32, 4, 2, VL>(a, st);
    return ws_k == 2 ? dkv_of<1, DU, 32, 2, 2, VL>(a, st) : dkv_of<1, DU, 32, 1, 2, VL>(a, st);
  });
  const double es = dtype == DT_BF16 ? 2 : 4, b = double(a.seqs.batch);
  if (e == hipSuccess)
    tm.done(10.0 * pairs_of(a) * a.dim, 0,
            b * a.dim * es * 4.0 * (double(a.seqs.q_tokens) * a.q_heads + double(a.seqs.k_tokens) * a.kv_heads));
  return e;
}

hipError_t run_rotary(const RotaryArgs& a, int dtype, hipStream_t st, LaunchTimer* timer) {
  const int64_t all = a.batch * a.tokens;
  if (all == 0) return hipSuccess;
  Timed tm(timer, KK_ROTARY, st);
  // tokens a workgroup, 1 / 2 / 4 / 8, us on an MI355X: 2048 of 16 heads of 64 fp32
  // 5.7 / 5.1 / 5.2 / 6.3; 4094 of 24 of 96 fp32 15.6 / 15.4 / 15.5 / 20.3; 8192 of
  // 40 of 128 bf16 27.4 / 27.9 / 28.1 / 28.4, 1024: 6.1 / 6.1 / 7.1 / 10.5, 256: 4.3 /
  // 4.9 / 6.2 / 9.6
  int per = std::max(1, std::min(2, kRotPairs / std::max(1, a.rot / 2)));
  if ((all + per - 1) / per < 512) per = 1;
  const dim3 g(static_cast<unsigned>((all + per - 1) / per)), b(256);
  if (dtype == DT_BF16) hipLaunchKernelGGL((k_rotary<uint16_t>), g, b, 0, st, a, per);
  else hipLaunchKernelGGL((k_rotary<float>), g, b, 0, st, a, per);
  const hipError_t e = hipGetLastError();
  double heads = 0;
  for (int i = 0; i < a.n; ++i) heads += a.t[i].heads;
  if (e == hipSuccess) tm.done(0, 0, 2.0 * double(all) * heads * a.dim * (dtype == DT_BF16 ? 2 : 4));
  return e;
}

hipError_t run_qk_clip(const ClipArgs& a, int dtype, hipStream_t st, LaunchTimer* timer) {
  if (a.n == 0 || a.first[a.n] == 0) return hipSuccess;
  Timed tm(timer, KK_QK_CLIP, st);
  const dim3 g(static_cast<unsigned>(a.first[a.n])), b(256);
  if (dtype == DT_BF16) hipLaunchKernelGGL((k_qk_clip<uint16_t>), g, b, 0, st, a);
  else hipLaunchKernelGGL((k_qk_clip<float>), g, b, 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) tm.done(0, 0, 0);
  return e;
}

hipError_t run_reset_logits(const ClipArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(k_reset_logits, dim3(a.n), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace muon

// Attention of few new rows over a paged cache: up to 16 query rows per sequence and kv head (a token of 16 grouped heads, four drafted
// tokens of four).  Bound: HBM; each cached byte is read once, whatever the number of rows.
//
// Both products run on mma.sync with the cached side as the A operand, so that a query row is one of 8 columns and nothing is computed for
// 16: S^T = K q^T (16 tokens x 8 rows per step), O^T += V^T P^T.  The sum over channels of the first and the rows of the second may come
// in any order, so a lane takes 16-byte pieces of rows as they lie: no transposes.  Codes become values in registers, two at a time (a fused
// multiply-add of 16 bits: the rounding that the cache's definition has).  A warp walks through 16-token steps, which come into a ring of
// its own in shared memory by bulk copies (a lane each for keys, values and their parameters), several steps ahead; the warps of a CTA
// take turns.  (With the next step's loads held in registers instead, 16-bit rows waited for memory, 64 ragged contexts up to 8192 168 us,
// now 134, 86 % of the copy bandwidth; and codes spent 616 instructions per 16 tokens, half of them on addresses, 12 contexts of 32768 in 4
// bits 161 us, now 428 and 129, bound by the issue of instructions and by their latency at 16 warps per SM.)
//
// Work: where there are few (sequence, kv head) units for the CTAs, each is cut evenly into parts of its own, a CTA each; else the steps of
// all units, one after the other, are cut into equal ranges, one per CTA.  (Ranges that begin in one unit and end in the next cost a
// call of little work a second latency: 8 heads x 1000 tokens 13.9 us.)  A unit that several CTAs share is joined by the one that finishes last,
// part by part in their order.
#pragma once
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "gear_paged.cuh"
#include "gear_pi.cuh"
#include "gear_quant.cuh"

namespace gear {

// (sequence, kv head) units have parts of their own where CTAs are at least kOwnShare times as many (and the sequences kOwnSeqs at most)
constexpr int kOwnShare = 4, kOwnSeqs = 96;
constexpr int kFineTokens = 1024;            // tokens that a sequence's rows see, up to which codes get probabilities in two parts
constexpr int kStep = 16;                    // tokens of a product: every page holds whole ones
// products of a step: with codes two, which share what a step costs apart from its tokens (12 contexts of 32768 in 4 bits: 612 instructions
// per 16 tokens and 171 us with one); rows as they are wait for memory either way and would fill shared memory
template <int BITS> constexpr int kStepParts = BITS == 16 ? 1 : 2;

template <class T> __device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// x * step + low in the type, both halves, one rounding
template <class T> __device__ __forceinline__ uint32_t code_value(uint32_t biased, uint32_t bias, uint32_t step, uint32_t low) {
  using T2 = typename Two<T>::type;
  const T2 c = __hsub2(*reinterpret_cast<T2*>(&biased), *reinterpret_cast<T2*>(&bias));
  const T2 v = __hfma2(c, *reinterpret_cast<T2*>(&step), *reinterpret_cast<T2*>(&low));
  return *reinterpret_cast<const uint32_t*>(&v);
}
// A constant that stays in a register: with two of them as immediates an instruction of three inputs became two
__device__ __forceinline__ uint32_t held(uint32_t x) {
  uint32_t y;
  asm("mov.b32 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// (w & mask) | high
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t high) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(w), "r"(mask), "r"(high));
  return y;
}
template <class T> struct IsHalf { static constexpr bool value = false; };
template <> struct IsHalf<__half> { static constexpr bool value = true; };

// Probabilities and their sums are kept beside a base: 2^-kSpare of the largest of them when it was last moved, and moved again once one
// passes 2^(kSpare + 8).  An operand of fp16 is subnormal below 2^-14, zero below 2^-25, and has room up to 2^16: with the seven powers that the
// lag leaves spare, the tail behind a token that takes nearly all of the sum keeps its bits down to 2^-21 of it, and what it has at all down to
// 2^-32.  (With none, tails 2^-20 to 2^-26 below such tokens were off by 1.5 to 7 times what their roundings allow: the sum takes them unrounded.)
template <class T> constexpr float kSpare = IsHalf<T>::value ? 7.f : 0.f;
template <class T> constexpr float kRise = kSpare<T> + 8.f;

// Four packed pairs of codes 4 bits wide from a word, x = (nibble 0, nibble 4), (1, 5), (2, 6), (3, 7): the code is put below a constant whose
// last place is one, which is then subtracted
template <class T> struct Biases {
  // of fp16: 1024 + code below it, 64 + code one digit higher up; of bf16: 128 + code
  uint32_t first = held(IsHalf<T>::value ? 0x64006400u : 0x43004300u), second = held(0x54005400u);
  // the high byte of 1024 + code (fp16), 128 + code (bf16); of 2^23 + code in 32 bits
  uint32_t byte = held(IsHalf<T>::value ? 0x64646464u : 0x43434343u), wide = held(0x4B000000u);
};
template <class T> __device__ __forceinline__ void nibbles(uint32_t w, uint32_t step, uint32_t low, const Biases<T>& b, uint32_t (&x)[4]) {
  if (IsHalf<T>::value) {
    const uint32_t u = w >> 8;
    x[0] = code_value<T>(and_or(w, 0x000f000fu, b.first), 0x64006400u, step, low);
    x[1] = code_value<T>(and_or(w, 0x00f000f0u, b.second), 0x54005400u, step, low);
    x[2] = code_value<T>(and_or(u, 0x000f000fu, b.first), 0x64006400u, step, low);
    x[3] = code_value<T>(and_or(u, 0x00f000f0u, b.second), 0x54005400u, step, low);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = code_value<T>(and_or(w >> (4 * i), 0x000f000fu, b.first), 0x43004300u, step, low);
  }
}
// byte i of word x and byte j of word y as a pair of values of T, through pairs of 32-bit operations
template <class T>
__device__ __forceinline__ uint32_t bytes_value(uint32_t x, uint32_t y, int i, int j, const Biases<T>& b, F32x2 step, F32x2 low) {
  const F32x2 biased = pack2(__uint_as_float(prmt(x, b.wide, 0x7440u + i)), __uint_as_float(prmt(y, b.wide, 0x7440u + j)));
  const float2 v = unpack2(fma2(add2(biased, pack2(-8388608.f, -8388608.f)), step, low));
  return Two<T>::pack(v.x, v.y);
}

template <int BYTES> __device__ __forceinline__ void shared_piece(uint32_t* w, const unsigned char* p) {
  if (BYTES == 16) { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
  if (BYTES == 8) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
  if (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
}

// What sequence s asks for: its rows, the tokens that they see, the steps (of SPAN tokens) of each of its kv heads (one at least where it
// has rows, which may see nothing)
struct RowsUnit { int row0, rows, pos0, len, lo, hi, first, steps; bool bad; };
template <int SPAN> __device__ __forceinline__ RowsUnit rows_unit(const PagedAttnArgs& a, int s) {
  const RowRange r = rows_of(a.c.row_start, s, a.c.n_rows);
  const Length n = length_of(a.c.lengths, s, a.c.table_stride, a.c.page_size);
  RowsUnit u;
  u.bad = r.bad || n.bad || r.hi - r.lo > a.max_rows;
  u.row0 = r.lo;
  u.rows = min(r.hi - r.lo, a.max_rows);
  u.pos0 = n.n - (r.hi - r.lo);
  u.len = n.n;
  const Span v = seen_by(u.pos0, u.pos0 + u.rows - 1, n.n, a.causal, a.window);
  u.lo = v.lo; u.hi = v.hi;
  u.first = v.lo & ~(SPAN - 1);
  u.steps = u.rows == 0 ? 0 : max(1, (v.hi - u.first + SPAN - 1) / SPAN);
  return u;
}

// Shared memory of a CTA: the warps' rings, in whose place their results are joined, and the query rows
template <int BITS, int D, int NQ, int W> struct RowsRing {
  static constexpr int kRowBytes = D * BITS / 8, kCodes = kStep * kRowBytes, kParams = BITS == 16 ? 0 : kStep * D / 32 * 4;    // of a side
  static constexpr int kPart = 2 * (kCodes + kParams), kStage = kStepParts<BITS> * kPart;
  // Room for two CTAs per SM (one with D = 128 and W = 8).  D = 64 with eight warps: 64 ragged contexts up to 8192, 8 heads, 154 us with four stages,
  // whose second CTA had no room, now 135 (four warps with four stages 137)
  static constexpr int kStages = BITS == 16 ? (D == 128 || W == 8 ? 3 : 4) : 2;
  static constexpr int kQPitch = D * 2 + 16, kOPitch = D + 2;
  static constexpr int kRings = W * kStages * kStage, kJoin = W * NQ * 8 * kOPitch * 4;
  static constexpr int kQuery = kRings > kJoin ? kRings : (kJoin + 127) / 128 * 128;         // byte where the query rows begin
  static constexpr int kBytes = kQuery + NQ * 8 * kQPitch;
};

// W warps, NQ blocks of 8 query rows.  Fine: probabilities as a rounded part and the rest rounded (16 bits and more between them).  Rounded
// once, few tokens that share most of the sum leave outputs half as far off again as their own rounding does.  Rows as they are have the
// time for it (131 -> 133 us); with codes it costs 8 % (12 contexts of 32768 in 4 bits 134 -> 147 us), and only sequences whose rows see
// at most kFineTokens tokens get it.
template <class T, int BITS, int D, int NQ, int W, int MINB>
__global__ void __launch_bounds__(W * 32, MINB) paged_rows_kernel(PagedAttnArgs a, int group_shift, int least, int own_units) {
  using S = RowsRing<BITS, D, NQ, W>;
  const PagedArgs& c = a.c;
  constexpr int kRows = NQ * 8, NS = S::kStages, SUB = kStepParts<BITS>, kSpan = kStep * SUB;
  constexpr int kKeyBytes = D * BITS / 32;                   // of a token's key, a lane's share
  constexpr int kKeyPiece = kKeyBytes < 16 ? kKeyBytes : 16, kKeyPieces = kKeyBytes / kKeyPiece, kKeyChannels = kKeyPiece * 8 / BITS;
  constexpr int kValBytes = D * BITS / 64;                   // of a token's value
  constexpr int kValPiece = kValBytes < 16 ? kValBytes : 16, kValPieces = kValBytes / kValPiece, kValChannels = kValPiece * 8 / BITS;
  constexpr int MT = D / 16;                                 // blocks of 16 channels of the output
  constexpr int kQPitch = S::kQPitch, kOPitch = S::kOPitch;
  extern __shared__ __align__(128) unsigned char smem[];
  unsigned char* qs = smem + S::kQuery;
  float* os = reinterpret_cast<float*>(smem);
  __shared__ float ms[W][kRows], ls[W][kRows];
  __shared__ uint64_t full[W][NS], dead;
  __shared__ long long scan[W + 1];
  __shared__ long long start_at[1];
  __shared__ int start_seq, last_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, i4 = lane & 3;
  unsigned char* ring = smem + warp * NS * S::kStage;
  if (lane < NS) bar_init(&full[warp][lane]);
  if (tid == 0) bar_init(&dead);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  // Bit s: phase of stage s; bit 8 + stage * SUB + part: there is data, or on its way; bit 31: a wait gave up, go on without data (every loop
  // still ends).  From then on the others stay those of the copies in flight.  (In a register each: 12 contexts of 32768 in 4 bits 132 us, now 129.)
  uint32_t ring_state = 0;
  constexpr uint32_t kGaveUp = 1u << 31;
  auto data_of = [&](int stage) { return ring_state >> (8 + stage * SUB) & ((1u << SUB) - 1); };
  const Biases<T> biases;
  after_previous();

  // ---- where this CTA's range begins.  f counts steps of all units, or, where units have parts of their own, those.
  int s = -1;
  long long seq_at = 0, total = 0, per, f0, f1;
  auto parts_of = [&](int steps) { return own_units > 0 ? (int)((steps + per - 1) / per) : steps; };
  if (own_units > 0) {
    // few sequences: every warp for itself, a lane per sequence.  With this `per` there are no more parts than CTAs.
    int steps[kOwnSeqs / 32];
#pragma unroll
    for (int x = 0; x < kOwnSeqs / 32; ++x) {
      steps[x] = 0;
      if (x * 32 + lane < c.n_seqs) {
        const RowsUnit u = rows_unit<kSpan>(a, x * 32 + lane);
        if (u.bad) paged_bad(c);
        steps[x] = u.steps;
        total += u.steps;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    per = max((long long)least, (total * c.heads + gridDim.x - own_units - 1) / (gridDim.x - own_units));
    f0 = blockIdx.x;
    long long at = 0;
#pragma unroll
    for (int x = 0; x < kOwnSeqs / 32; ++x) {
      const int mine = parts_of(steps[x]) * c.heads;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += up;
      }
      const uint32_t here = __ballot_sync(0xffffffffu, f0 >= at + upto - mine && f0 < at + upto);
      if (here) {
        s = x * 32 + __ffs(here) - 1;
        seq_at = at + __shfl_sync(0xffffffffu, upto - mine, __ffs(here) - 1);
      }
      at += __shfl_sync(0xffffffffu, upto, 31);
      if (x * 32 + 32 >= c.n_seqs) break;
    }
    total = at;
    f1 = min(total, f0 + 1);
  } else {
    // sums of the sequences' steps over the threads, then within one thread's sequences
    const int per_thread = (c.n_seqs + W * 32 - 1) / (W * 32);
    const int s_begin = min(c.n_seqs, tid * per_thread), s_end = min(c.n_seqs, s_begin + per_thread);
    long long mine = 0;
    for (int q = s_begin; q < s_end; ++q) {
      const RowsUnit u = rows_unit<kSpan>(a, q);
      if (u.bad) paged_bad(c);
      mine += u.steps;
    }
    mine *= c.heads;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    long long before = incl - mine;
#pragma unroll
    for (int w = 0; w < W; ++w) { if (w < warp) before += scan[w]; total += scan[w]; }
    per = max((long long)least, (total + gridDim.x - 1) / gridDim.x);
    f0 = blockIdx.x * per;
    f1 = min(total, f0 + per);
    if (f0 < f1 && before <= f0 && f0 < before + mine) {
      long long at = before;
      for (int q = s_begin; q < s_end; ++q) {
        const long long n = (long long)rows_unit<kSpan>(a, q).steps * c.heads;
        if (f0 < at + n) { start_seq = q; start_at[0] = at; break; }
        at += n;
      }
    }
    __syncthreads();
    if (f0 < f1) { s = start_seq; seq_at = start_at[0]; }
  }
  if (tid == 0 && __ldcg(c.row_start) != 0) paged_bad(c);
  if (f0 >= f1) return;
  const bool own_parts = own_units > 0;

  for (long long f = f0; f < f1;) {
    RowsUnit u = rows_unit<kSpan>(a, s);
    int parts = parts_of(u.steps);
    while (f >= seq_at + (long long)parts * c.heads) {       // next sequence with rows
      seq_at += (long long)parts * c.heads;
      if (++s >= c.n_seqs) return;                           // tables that changed meanwhile
      u = rows_unit<kSpan>(a, s);
      parts = parts_of(u.steps);
    }
    const int head = (int)((f - seq_at) / parts);
    const long long unit_at = seq_at + (long long)head * parts;
    const int p0 = (int)(f - unit_at);
    const int st0 = own_parts ? (int)((long long)u.steps * p0 / parts) : p0;
    const int st1 = own_parts ? (int)((long long)u.steps * (p0 + 1) / parts) : (int)min((long long)u.steps, f1 - unit_at);
    const int R = u.rows * a.share;

    // what the two rows of each block that this lane keeps see; steps that every row sees whole lie in lo_max .. hi_min
    int see_lo[NQ][2], see_hi[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int pos = u.pos0 + min(n * 8 + i4 * 2 + e, R - 1) / a.share;
        const Span v = seen_by(pos, pos, u.len, a.causal, a.window);
        see_lo[n][e] = v.lo; see_hi[n][e] = v.hi;
      }
    const int last = u.pos0 + u.rows - 1;
    const int lo_max = seen_by(last, last, u.len, a.causal, a.window).lo, hi_min = seen_by(u.pos0, u.pos0, u.len, a.causal, a.window).hi;
    float o[NQ][MT][4], m[NQ][2], l[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][t][e] = 0.f;
      m[n][0] = m[n][1] = -FLT_MAX;
      l[n][0] = l[n][1] = 0.f;
    }

    // ---- steps into the ring.  Of four lanes per part of a step the first copies keys, the second values, the others their parameters; all
    // lanes look up the pages of the warp's next steps at once
    constexpr int kLook = 32 / SUB;                          // steps per look-up
    const int32_t* table = c.table + (size_t)s * c.table_stride;
    const int side = lane & 1, sub_mine = lane >> 2, steps_mine = st1 - st0 > warp ? (st1 - st0 - warp + W - 1) / W : 0;
    const bool params = lane & 2, copies = sub_mine < SUB && !(BITS == 16 && params);
    const uint32_t row_bytes = params ? c.param_row_bytes : S::kRowBytes, copy_bytes = kStep * row_bytes;
    const long long page_bytes = params ? c.param_bytes : c.page_bytes;
    const unsigned char* pool = (params ? params_of(c, side) : pages_of(c, side)) + (size_t)head * c.page_size * row_bytes;
    unsigned char* place = ring + sub_mine * S::kPart + (params ? 2 * S::kCodes + side * S::kParams : side * S::kCodes);
    const uint32_t part_bytes = 2 * kStep * (S::kRowBytes + (BITS == 16 ? 0 : c.param_row_bytes));
    int pages = 0;
    ring_state &= kGaveUp | 0xffu;
    // step k of this warp
    auto request = [&](int k, int stage) {
      if (k >= steps_mine || (ring_state & kGaveUp)) return;
      if (k % kLook == 0) {
        const int mine = k + lane / SUB, t = u.first + (st0 + warp + mine * W) * kSpan + lane % SUB * kStep;
        pages = -1;
        if (mine < steps_mine && t < u.hi && t + kStep > u.lo) {
          pages = __ldcg(table + (t >> c.page_shift));
          if ((unsigned)pages >= (unsigned)c.n_pages) { paged_bad(c); pages = -1; }
        }
      }
      const int page = __shfl_sync(0xffffffffu, pages, k % kLook * SUB + (sub_mine & (SUB - 1)));
      const uint32_t good = __ballot_sync(0xffffffffu, page >= 0 && lane < 4 * SUB);    // bits 0 and 4
      const uint32_t bits = (good & 1u) | (SUB == 2 ? good >> 3 & 2u : 0u);
      ring_state = (ring_state & ~(((1u << SUB) - 1) << (8 + stage * SUB))) | bits << (8 + stage * SUB);
      if (bits == 0) return;
      if (lane == 0) bar_expect(&full[warp][stage], part_bytes * __popc(bits));
      __syncwarp();
      const int slot = (u.first + (st0 + warp + k * W) * kSpan + sub_mine * kStep) & (c.page_size - 1);
      if (copies && page >= 0) bulk_copy(place + stage * S::kStage, pool + page * page_bytes + slot * row_bytes, copy_bytes, &full[warp][stage]);
    };
#pragma unroll
    for (int x = 0; x < NS; ++x) request(x, x);

    // ---- query rows into shared memory: [row][channels], a row past the last one zero; for 4-bit codes the eight channels of a piece in
    // the order in which their word gives them up
    for (int x = tid; x < kRows * (D / 8); x += W * 32) {
      const int n = x / (D / 8), p = x % (D / 8);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (n < R)
        v = *reinterpret_cast<const uint4*>(a.q + (u.row0 + n / a.share) * a.q_stride + (((size_t)head * a.share + n % a.share) * D + p * 8) * 2);
      if (BITS == 4) v = make_uint4(prmt(v.x, v.z, 0x5410), prmt(v.x, v.z, 0x7632), prmt(v.y, v.w, 0x5410), prmt(v.y, v.w, 0x7632));
      *reinterpret_cast<uint4*>(qs + n * kQPitch + p * 16) = v;
    }
    __syncthreads();
    // The same as B operands: rows as they are hold them for every step.  With codes they, and where parameters lie, are looked up again each time:
    // 128 registers are too few beside the conversion (12 contexts of 32768 in 4 bits 135 -> 127 us, drafted tokens in 8 bits 75 -> 71).
    auto query = [&](int n, int p, int w) {
      return *reinterpret_cast<const uint4*>(qs + (n * 8 + r) * kQPitch + ((p * 4 + i4) * kKeyChannels + w * 8) * 2);
    };
    uint4 qf[NQ][BITS == 16 ? D / 32 : 1];
    if (BITS == 16) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) qf[n][BITS == 16 ? x : 0] = query(n, x / (kKeyChannels / 8), x % (kKeyChannels / 8));
    }

    if (a.test_dead_wait == 1 && warp == 0 && !bar_wait(&dead, 0, kTestSpinLimit)) ring_state |= kGaveUp;
    int stage = 0;
    for (int k = 0; k < steps_mine; ++k) {
      const int t0 = u.first + (st0 + warp + k * W) * kSpan;
      uint32_t there = data_of(stage);
      if (there) {
        if (__all_sync(0xffffffffu, !(ring_state & kGaveUp) && bar_wait(&full[warp][stage], ring_state >> stage & 1u))) {
          ring_state ^= 1u << stage;
        } else {
          ring_state |= kGaveUp;
          there = 0;
        }
      }
      // The arithmetic of a step, made with and without masks, as most steps have nothing to mask (selected by a condition in one piece of
      // code, masks were computed in every step), and fine or not
      auto step = [&](auto kind) {
        constexpr bool kWhole = decltype(kind)::value & 1, kFine = decltype(kind)::value & 2;
        // ---- scores: z[..][n][0..1] token r, z[..][n][2..3] token r + 8, rows 2 i4 and 2 i4 + 1 of block n
        float z[SUB][NQ][4];
#pragma unroll
        for (int h = 0; h < SUB; ++h) {
          const unsigned char* data = ring + stage * S::kStage + h * S::kPart;
          uint32_t kr[2][kKeyPieces * kKeyPiece / 4], kp[2][kKeyPieces];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int p = 0; p < kKeyPieces; ++p) {
              shared_piece<kKeyPiece>(&kr[e][p * kKeyPiece / 4], data + (r + 8 * e) * S::kRowBytes + (p * 4 + i4) * kKeyPiece);
              if (BITS != 16)
                shared_piece<4>(&kp[e][p], data + 2 * S::kCodes + (r + 8 * e) * c.param_row_bytes + ((p * 4 + i4) * kKeyChannels >> group_shift) * 4);
            }
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) z[h][n][e] = 0.f;
#pragma unroll
          for (int p = 0; p < kKeyPieces; ++p) {
            constexpr int kWords = kKeyChannels / 2;             // packed pairs of a piece
            uint32_t x[2][kWords];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if (BITS == 16) {
#pragma unroll
                for (int w = 0; w < kWords; ++w) x[e][w] = kr[e][p * kKeyPiece / 4 + (BITS == 16 ? w : 0)];
              } else {
                const uint32_t step = prmt(kp[e][p], 0, 0x1010), low = prmt(kp[e][p], 0, 0x3232);
                const float2 sl = Two<T>::wide(kp[e][p]);
#pragma unroll
                for (int w = 0; w < kKeyPiece / 4; ++w) {
                  const uint32_t word = kr[e][p * kKeyPiece / 4 + w];
                  if (BITS == 4) {
                    uint32_t y[4];
                    nibbles<T>(word, step, low, biases, y);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[e][(w * 4 + j) % kWords] = y[j];
                  } else if (IsHalf<T>::value) {
                    x[e][(w * 2) % kWords] = code_value<T>(prmt(word, biases.byte, 0x4140), 0x64006400u, step, low);
                    x[e][(w * 2 + 1) % kWords] = code_value<T>(prmt(word, biases.byte, 0x4342), 0x64006400u, step, low);
                  } else {
                    x[e][(w * 2) % kWords] = bytes_value<T>(word, word, 0, 1, biases, pack2(sl.x, sl.x), pack2(sl.y, sl.y));
                    x[e][(w * 2 + 1) % kWords] = bytes_value<T>(word, word, 2, 3, biases, pack2(sl.x, sl.x), pack2(sl.y, sl.y));
                  }
                }
              }
            }
#pragma unroll
            for (int w = 0; w < kWords; w += 4) {
#pragma unroll
              for (int n = 0; n < NQ; ++n) {
                const uint4 qv = BITS == 16 ? qf[n][BITS == 16 ? p * (kKeyChannels / 8) + w / 4 : 0] : query(n, p, w / 4);
                const uint32_t a0[4] = {x[0][w], x[1][w], x[0][w + 1], x[1][w + 1]};
                const uint32_t a1[4] = {x[0][w + 2], x[1][w + 2], x[0][w + 3], x[1][w + 3]};
                mma16<T>(z[h][n], a0, qv.x, qv.y);
                mma16<T>(z[h][n], a1, qv.z, qv.w);
              }
            }
          }
        }
        // ---- probabilities beside a base that lags by up to 2^8
        bool rises = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < SUB; ++h)
#pragma unroll
              for (int x = e; x < 4; x += 2) {
                if (!kWhole) {
                  const int tok = t0 + h * kStep + r + 8 * (x >> 1);
                  if (!(there >> h & 1u) || tok < see_lo[n][e] || tok >= see_hi[n][e]) z[h][n][x] = -INFINITY;
                }
                top = fmaxf(top, z[h][n][x]);
              }
            rises = rises || top * a.scale_log2 > m[n][e] + kRise<T>;
          }
        if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float top = -INFINITY;
#pragma unroll
              for (int h = 0; h < SUB; ++h) top = fmaxf(top, fmaxf(z[h][n][e], z[h][n][e + 2]));
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
              top = fmaxf(m[n][e], fmaf(top, a.scale_log2, -kSpare<T>));
              const float keep = exp2_fast(m[n][e] - top);
              m[n][e] = top;
              l[n][e] *= keep;
#pragma unroll
              for (int k = 0; k < MT; ++k) { o[n][k][e] *= keep; o[n][k][e + 2] *= keep; }
            }
        }
        uint32_t pbs[SUB][NQ][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int h = 0; h < SUB; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float p0 = exp2_fast(fmaf(z[h][n][2 * x], a.scale_log2, -m[n][0])), p1 = exp2_fast(fmaf(z[h][n][2 * x + 1], a.scale_log2, -m[n][1]));
              l[n][0] += p0; l[n][1] += p1;                    // the log of the sum is an output: not from the rounded ones
              const uint32_t head = Two<T>::pack(p0, p1);
              const float2 w = Two<T>::wide(head);
              pbs[h][n][x] = transpose8(head);
              if (kFine) pbs[h][n][x + 2] = transpose8(Two<T>::pack(p0 - w.x, p1 - w.y));
            }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
          const unsigned char* data = ring + stage * S::kStage + sub * S::kPart;
          [[maybe_unused]] const int t = t0 + sub * kStep;
          uint32_t (&pb)[NQ][4] = pbs[sub];
          uint32_t vr[4][kValPieces * kValPiece / 4], vp[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = 2 * i4 + (e & 1) + 8 * (e >> 1);
#pragma unroll
            for (int p = 0; p < kValPieces; ++p)
              shared_piece<kValPiece>(&vr[e][p * kValPiece / 4], data + S::kCodes + tok * S::kRowBytes + (p * 8 + r) * kValPiece);
            if (BITS != 16)
              shared_piece<4>(&vp[e], data + 2 * S::kCodes + S::kParams + tok * c.param_row_bytes + (r * kValChannels >> group_shift) * 4);
            // values that no row sees may be no numbers, which a probability of zero does not hide
            if (!kWhole) {
              const bool in = (there >> sub & 1u) && t + tok >= u.lo && t + tok < u.hi;
              if (BITS != 16) vp[e] = in ? vp[e] : 0;
              else
#pragma unroll
                for (int w = 0; w < kValPieces * kValPiece / 4; ++w) vr[e][w] = in ? vr[e][w] : 0;
            }
          }
          // ---- values
          if (BITS == 16) {
#pragma unroll
            for (int k = 0; k < MT; ++k) {
              const int w = k % (kValBytes / 4);
              const uint32_t x[4] = {prmt(vr[0][w], vr[1][w], 0x5410), prmt(vr[0][w], vr[1][w], 0x7632),
                                     prmt(vr[2][w], vr[3][w], 0x5410), prmt(vr[2][w], vr[3][w], 0x7632)};
#pragma unroll
              for (int n = 0; n < NQ; ++n) {
                mma16<T>(o[n][k], x, pb[n][0], pb[n][1]);
                if (kFine) mma16<T>(o[n][k], x, pb[n][2], pb[n][3]);
              }
            }
          } else {
            uint32_t step[2], low[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              step[h] = prmt(vp[2 * h], vp[2 * h + 1], 0x5410);
              low[h] = prmt(vp[2 * h], vp[2 * h + 1], 0x7632);
            }
#pragma unroll
            for (int w = 0; w < kValBytes / 4; ++w) {
              constexpr int kPer = 32 / BITS;                    // codes of a word
              uint32_t x[2][kPer];                               // [token pair][channel]
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t wa = vr[2 * h][w], wb = vr[2 * h + 1][w];
                if (BITS == 4) {
                  uint32_t y[4];
                  nibbles<T>(prmt(wa, wb, 0x5410), step[h], low[h], biases, y);
#pragma unroll
                  for (int j = 0; j < 4; ++j) x[h][j] = y[j];
                  nibbles<T>(prmt(wa, wb, 0x7632), step[h], low[h], biases, y);
#pragma unroll
                  for (int j = 0; j < 4; ++j) x[h][(4 + j) % kPer] = y[j];
                } else if (IsHalf<T>::value) {
                  const uint32_t t0 = prmt(wa, wb, 0x5140), t1 = prmt(wa, wb, 0x7362);
                  x[h][0] = code_value<T>(prmt(t0, biases.byte, 0x4140), 0x64006400u, step[h], low[h]);
                  x[h][1] = code_value<T>(prmt(t0, biases.byte, 0x4342), 0x64006400u, step[h], low[h]);
                  x[h][2] = code_value<T>(prmt(t1, biases.byte, 0x4140), 0x64006400u, step[h], low[h]);
                  x[h][3] = code_value<T>(prmt(t1, biases.byte, 0x4342), 0x64006400u, step[h], low[h]);
                } else {
                  const float2 pa = Two<T>::wide(vp[2 * h]), pb2 = Two<T>::wide(vp[2 * h + 1]);
#pragma unroll
                  for (int j = 0; j < kPer; ++j) x[h][j] = bytes_value<T>(wa, wb, j, j, biases, pack2(pa.x, pb2.x), pack2(pa.y, pb2.y));
                }
              }
#pragma unroll
              for (int j = 0; j < kPer; j += 2) {
                const uint32_t y[4] = {x[0][j], x[0][j + 1], x[1][j], x[1][j + 1]};
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                mma16<T>(o[n][(w * kPer + j) / 2], y, pb[n][0], pb[n][1]);
                if (kFine) mma16<T>(o[n][(w * kPer + j) / 2], y, pb[n][2], pb[n][3]);
              }
              }
            }
          }
        }
      };
      const bool whole = there == (1u << SUB) - 1 && t0 >= lo_max && t0 + kSpan <= hi_min;
      if (BITS == 16 || u.hi - u.lo <= kFineTokens) {
        if (whole) step(std::integral_constant<int, 3>()); else step(std::integral_constant<int, 2>());
      } else if constexpr (BITS != 16) {
        if (whole) step(std::integral_constant<int, 1>()); else step(std::integral_constant<int, 0>());
      }
      // everything of the step has been used: the stage may be written again
      __syncwarp();
      request(k + NS, stage);
      if (++stage == NS) stage = 0;
    }
    if (ring_state & kGaveUp) {                              // let the copies in flight land (bounded)
      for (int x = 0; x < NS; ++x)
        if (data_of(x)) bar_wait(&full[warp][x], ring_state >> x & 1u, 100);
      if (lane == 0) atomicExch(c.status, GEAR_ERR_TIMEOUT);
    }
    __syncthreads();                                         // the rings are done with

    // ---- the warps' results joined in shared memory.  Output block k, element e of a lane: channel below, row n * 8 + 2 i4 + (e & 1)
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sum = l[n][e];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        if (r == 0) { ms[warp][n * 8 + 2 * i4 + e] = m[n][e]; ls[warp][n * 8 + 2 * i4 + e] = sum; }
#pragma unroll
        for (int k = 0; k < MT; ++k) {
          const int ch = BITS == 16 ? (k / 4) * 64 % D + r * 8 + (k % 4) * 2 : r * (D / 8) + k * 2;
          *reinterpret_cast<float2*>(os + (warp * kRows + n * 8 + 2 * i4 + e) * kOPitch + ch) = make_float2(o[n][k][e], o[n][k][e + 2]);
        }
      }
    __syncthreads();
    const bool alone = st0 == 0 && st1 == u.steps;
    const int heads_q = c.heads * a.share;
    // parts of the unit: those of CTAs first_cta .. last_cta; a CTA's part is its first one (slot 0) or its last (slot 1)
    const int first_cta = (int)(own_parts ? unit_at : unit_at / per);
    const int last_cta = (int)(own_parts ? unit_at + parts - 1 : (unit_at + u.steps - 1) / per);
    constexpr int kPart = kRows * (D + 2);
    auto part = [&](int cta) { return a.partial + ((size_t)cta * 2 + (own_parts || cta * per >= unit_at ? 0 : 1)) * kPart; };
    constexpr int kQuads = D / 4;
    for (int x = tid; x < R * kQuads; x += W * 32) {
      const int row = x / kQuads, ch = x % kQuads * 4;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, ms[w][row]);
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float k = exp2_fast(ms[w][row] - base);
        sum = fmaf(k, ls[w][row], sum);
        const float* src = os + (w * kRows + row) * kOPitch + ch;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(k, src[j], v[j]);
      }
      if (alone) {
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        const size_t at = (size_t)(u.row0 + row / a.share) * heads_q + head * a.share + row % a.share;
        *reinterpret_cast<uint2*>(a.out + (at * D + ch) * 2) = make_uint2(Two<T>::pack(v[0] * inv, v[1] * inv), Two<T>::pack(v[2] * inv, v[3] * inv));
        if (a.lse != nullptr && ch == 0) a.lse[at] = sum > 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
      } else {
        float* dst = part(blockIdx.x);
        *reinterpret_cast<float4*>(dst + row * D + ch) = make_float4(v[0], v[1], v[2], v[3]);
        if (ch == 0) { dst[kRows * D + row * 2] = top; dst[kRows * D + row * 2 + 1] = sum; }
      }
    }
    if (!alone) {
      __syncthreads();
      if (tid == 0) {
        int* ticket = a.tickets + first_cta;                 // a CTA's range ends inside one unit at most
        __threadfence();
        const bool last = atomicAdd(ticket, 1) == last_cta - first_cta;
        if (last) *ticket = 0;
        __threadfence();
        last_flag = last;
      }
      __syncthreads();
      if (last_flag) {
        for (int x = tid; x < R * kQuads; x += W * 32) {
          const int row = x / kQuads, ch = x % kQuads * 4;
          float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
          constexpr int kBatch = 8;                          // parts on their way at once
          for (int p0 = first_cta; p0 <= last_cta; p0 += kBatch) {
            float2 ml[kBatch];
            float4 y[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              const float* src = part(min(p0 + b, last_cta));
              ml[b] = __ldcg(reinterpret_cast<const float2*>(src + kRows * D + row * 2));
              y[b] = __ldcg(reinterpret_cast<const float4*>(src + row * D + ch));
              if (p0 + b > last_cta) ml[b] = make_float2(-INFINITY, 0.f);
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              const float next = fmaxf(top, ml[b].x), base = next == -INFINITY ? 0.f : next;
              const float ka = exp2_fast(top - base), kb = exp2_fast(ml[b].x - base);
              top = next;
              sum = sum * ka + ml[b].y * kb;
              v[0] = v[0] * ka + y[b].x * kb; v[1] = v[1] * ka + y[b].y * kb;
              v[2] = v[2] * ka + y[b].z * kb; v[3] = v[3] * ka + y[b].w * kb;
            }
          }
          const float inv = sum > 0.f ? 1.f / sum : 0.f;
          const size_t at = (size_t)(u.row0 + row / a.share) * heads_q + head * a.share + row % a.share;
          *reinterpret_cast<uint2*>(a.out + (at * D + ch) * 2) =
              make_uint2(Two<T>::pack(v[0] * inv, v[1] * inv), Two<T>::pack(v[2] * inv, v[3] * inv));
          if (a.lse != nullptr && ch == 0) a.lse[at] = sum > 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
        }
      }
    }
    f = own_parts ? f1 : unit_at + st1;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the rings are written by copies again
    __syncthreads();
  }
}

// CTAs of a launch: the scratch holds two partial results of each
constexpr int kRowsMaxCtas = 148 * 4;
// Tokens of a CTA at least; half as many where several units have parts of their own (8 heads x 1000 tokens 9.6 -> 8.5 us, in 8 bits 10.0 -> 8.3,
// 64 heads x 500 12.0 -> 10.0; one head x 256 6.7 -> 7.6, x 8000 11.4 -> 12.8)
constexpr int kRowsLeastTokens = 256, kRowsSeveral = 8;

template <class T, int BITS, int D, int NQ, int W, int MINB>
cudaError_t launch_rows_t(const PagedAttnArgs& a, int group, cudaStream_t st) {
  constexpr int kBytes = RowsRing<BITS, D, NQ, W>::kBytes;
  // 228 KB per SM, of which each CTA takes 1 KB and less than one for its barriers beside what it asks for
  static_assert(MINB * (kBytes + 2048) <= 228 * 1024, "MINB CTAs have no room on an SM");
  int shift = 0, sms = 0;
  while ((1 << shift) < group) ++shift;
  static KernelReady ready;
  const cudaError_t e = ready.on_this_device(paged_rows_kernel<T, BITS, D, NQ, W, MINB>, kBytes, &sms);
  if (e != cudaSuccess) return e;
  // no more CTAs than the longest contexts that the table has room for could use
  constexpr int kSpan = kStep * kStepParts<BITS>;
  const long long units = (long long)a.c.n_seqs * a.c.heads, room = std::min(sms * MINB, kRowsMaxCtas);
  const int own_units = units * kOwnShare <= room && a.c.n_seqs <= kOwnSeqs ? (int)units : 0;
  const int least = kRowsLeastTokens / kSpan / (own_units >= kRowsSeveral ? 2 : 1);
  const long long most = units * ((long long)a.c.table_stride * a.c.page_size / kSpan + 2);
  const long long ctas = (most + least - 1) / least + own_units;
  count_launches(1);
  return launch_dependent(paged_rows_kernel<T, BITS, D, NQ, W, MINB>, dim3((unsigned)std::min(ctas, room)), W * 32, kBytes, st, a, shift, least,
                          own_units);
}
template <class T, int BITS, int D>
cudaError_t launch_rows_d(const PagedAttnArgs& a, int group, cudaStream_t st) {
  constexpr int W = BITS == 16 && D == 128 ? 4 : BITS == 8 && D == 128 ? 6 : 8;    // what two CTAs have room for
  // Few units of 16-bit rows: eight warps in one CTA per SM, whose parts are half as many (one head x 256 tokens 7.4 -> 6.7 us,
  // 8 heads x 32000 31.6 -> 30.0; 32 heads x 4000 16.6 -> 17.2)
  if constexpr (BITS == 16 && D == 128)
    if (a.max_rows * a.share <= 8 && (long long)a.c.n_seqs * a.c.heads * kOwnShare <= 148 && a.c.n_seqs <= kOwnSeqs)
      return launch_rows_t<T, BITS, D, 1, 8, 1>(a, group, st);
  return a.max_rows * a.share <= 8 ? launch_rows_t<T, BITS, D, 1, W, 2>(a, group, st) : launch_rows_t<T, BITS, D, 2, 4, 2>(a, group, st);
}
template <int BITS>
cudaError_t launch_paged_rows_bits(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st) {
  if (dtype == GEAR_F16) return a.c.head_dim == 128 ? launch_rows_d<__half, BITS, 128>(a, group, st) : launch_rows_d<__half, BITS, 64>(a, group, st);
  return a.c.head_dim == 128 ? launch_rows_d<__nv_bfloat16, BITS, 128>(a, group, st) : launch_rows_d<__nv_bfloat16, BITS, 64>(a, group, st);
}

}  // namespace gear

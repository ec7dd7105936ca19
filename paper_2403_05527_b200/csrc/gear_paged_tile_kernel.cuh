// The kernel of gear_paged_tile.cuh: one instantiation per width of the cached rows.
#pragma once
#include <limits.h>

#include "gear_paged_rows.cuh"
#include "gear_paged_tile.cuh"
#include "gear_quant.cuh"
#include "gear_tma.cuh"

namespace gear {

// ------------------------------------------------------------------ tensor memory, without the wait of gear_umma.cuh
__device__ __forceinline__ void tmem_ld32_begin(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld_end() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// nothing that uses these registers moves ahead of here
__device__ __forceinline__ void tmem_settled(uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i])::"memory");
}
__device__ __forceinline__ void tmem_st16_begin(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
               "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st_end() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// d (+)= A b, the A operand in tensor memory
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// one lane of the warp, the same each time
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void load_page_box(void* dst, const CUtensorMap* map, int x, int slot, int head, int page, uint64_t* b) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(smem_addr(dst)), "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(smem_addr(b)) : "memory");
}

__device__ __forceinline__ void load_rows_box(void* dst, const CUtensorMap* map, int x, int head, int row, uint64_t* b) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(smem_addr(dst)), "l"(map), "r"(x), "r"(head), "r"(row), "r"(smem_addr(b)) : "memory");
}

// bar_wait with a limit that is not known when compiling, which only a wait that is not over at once looks at (508 instead of 512 us for 2048 rows
// over 16384 tokens)
__device__ __forceinline__ bool wait_for(uint64_t* b, uint32_t parity, int limit) {
  return bar_wait(b, parity, 1) || bar_wait(b, parity, limit);
}

// ------------------------------------------------------------------ shared memory
// Warps: eight of rows, then those that bring keys and values (one requests copies; eight turn codes into values), then one that issues
// products; the rest fill up its warpgroup (registers are handed out by whole ones).
template <int BITS> constexpr int kBringWarps = BITS == 16 ? 1 : 8;
template <int BITS> constexpr int kTileThreads = BITS == 16 ? 384 : 640;
// Q tiles and stages, which take K and V blocks in turn: [D / 64 halves][128 rows][128 bytes], 128-byte swizzle (16-byte piece c of row i
// at c ^ (i & 7)).  Codes on their way lie behind them: kAhead blocks of a side, rows of codes and then their parameters.
template <int BITS, int D> struct TileSmem {
  static constexpr int kOperand = kTileRows * D * 2, kHalf = kTileRows * 128;
  static constexpr int kStages = D == 128 ? (BITS == 16 ? 4 : 3) : 6;
  static constexpr int kRowBytes = D * BITS / 8, kPieces = kRowBytes / 16, kCodes = 128 / BITS;    // 16-byte pieces of a row of codes
  static constexpr int kTimes = BITS == 16 ? 0 : kTileTokens * kPieces / (kBringWarps<BITS> * 32); // pieces of a thread
  static constexpr int kRawCodes = BITS == 16 ? 0 : kTileTokens * kRowBytes, kRawParams = BITS == 16 ? 0 : kTileTokens * D / 32 * 4;
  static constexpr int kAheadBytes = kRawCodes + kRawParams, kAhead = BITS == 16 ? 0 : 3;
  static constexpr int kBytes = 1024 + (2 + kStages) * kOperand + kAhead * kAheadBytes;
};
struct TileMaps { CUtensorMap kv[2], q; };

template <class T, int BITS, int D>
__global__ void __launch_bounds__(kTileThreads<BITS>, 1) paged_tile_kernel(PagedAttnArgs a, int group_shift, const __grid_constant__ TileMaps maps) {
  using S = TileSmem<BITS, D>;
  constexpr int NS = S::kStages;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t kv_full[NS], kv_empty[NS], q_full[2], q_empty[2], s_full[2], p_part[2], p_full[2], pv_done[2], edge, ended, dead;
  __shared__ uint64_t raw_full[S::kAhead + 1], raw_empty[S::kAhead + 1];
  __shared__ int2 raw_rows[S::kAhead + 1];
  __shared__ uint32_t tmem_slot;
  const PagedArgs& c = a.c;
  unsigned char* smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  unsigned char* stages = smem + 2 * S::kOperand;
  unsigned char* ahead = stages + NS * S::kOperand;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kProducts = 8 + kBringWarps<BITS>;           // the warp that issues products
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) { bar_init(&kv_full[i], kBringWarps<BITS>); bar_init(&kv_empty[i]); }
    for (int t = 0; t < 2; ++t) {
      for (uint64_t* b : {&q_full[t], &q_empty[t], &s_full[t], &pv_done[t]}) bar_init(b);
      bar_init(&p_part[t], 4);
      bar_init(&p_full[t], 4);
    }
    for (int i = 0; i < S::kAhead; ++i) { bar_init(&raw_full[i]); bar_init(&raw_empty[i], kBringWarps<BITS>); }
    for (uint64_t* b : {&edge, &ended, &dead}) bar_init(b);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kProducts) tmem_alloc<512>(&tmem_slot);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = tmem_slot;
  after_previous();

  const long long total = __ldcg(a.unit_sums + a.unit_first[c.n_seqs]) * c.heads;
  const long long per = max((long long)kTileLeast, (total + gridDim.x - 1) / gridDim.x);
  TileIter it;
  it.f = blockIdx.x * per;
  it.f1 = min(total, it.f + per);
  const bool any = it.f < it.f1;
  if (any) it.find(a);
  bool ok = true;                                            // a wait gave up: go on without waiting, every loop still ends
  auto test_wait = [&](int who) { if (a.test_dead_wait == who) ok = ok && bar_wait(&dead, 0, kTestSpinLimit); };

  // Registers a thread.  A kernel of three or five warpgroups starts with 168 or 96 of them (65536 / 384, / 640, to a multiple of eight);
  // what some warpgroups take, the others have to have given up, else the takers wait for ever.
  constexpr int kRowRegs = BITS == 16 ? 208 : 136, kBringRegs = 72, kLastRegs = BITS == 16 ? 88 : 64;
  static_assert(BITS == 16 ? 2 * kRowRegs + kLastRegs <= 3 * 168 : 2 * kRowRegs + 2 * kBringRegs + kLastRegs <= 5 * 96, "more than at the start");
  // Three quarters of a block's probabilities are announced ahead of the rest, whose products follow (458 -> 449 us for 2048 rows over 16384
  // tokens; with codes the warps that convert are in the way of either, 755 -> 775).
  constexpr bool kSplit = BITS == 16;
  constexpr int kEarly = kSplit ? 3 : 4;
  if (warp < 8) {
    // ================================================================ rows: a thread per query row of tile `t`
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRowRegs));
    // scores of a block that are held at once: all of them, or half, and they are read again for the probabilities
    constexpr int kHeld = BITS == 16 ? 4 : 2;
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lane_base = tmem + ((uint32_t)(row & 96) << 16), tS = lane_base + t * 128, tO = lane_base + 256 + t * 128;
    const int heads_q = c.heads * a.share, i_tile = row / a.share, g = row - i_tile * a.share;
    int n_blocks = 0;                                        // of this tile so far
    TileShared shared = {};
    if (warp == 0) test_wait(2);
    while (any && it.f < it.f1) {
      const int b0 = it.block(), nb = it.blocks_here();
      const int i_unit = it.unit * 2 * a.tile_new, i_first = i_unit + t * a.tile_new, i = i_first + i_tile;
      if (i_first < it.q.rows) {
        // ---- what the row sees, and the blocks that every row of the warp sees whole
        const bool mine = i_tile < a.tile_new && i < it.q.rows;
        const int pos = it.q.pos0 + min(i, it.q.rows - 1);
        const Span see = seen_by(pos, pos, it.q.len, a.causal, a.window);
        // of the warp's rows the first one ends first, and the last one begins last
        const int p_first = it.q.pos0 + min(it.q.rows - 1, i_first + (row & 96) / a.share);
        const int p_last = it.q.pos0 + min(it.q.rows - 1, i_first + min(a.tile_new - 1, (row | 31) / a.share));
        const int lo_max = seen_by(p_last, p_last, it.q.len, a.causal, a.window).lo;
        const int hi_min = seen_by(p_first, p_first, it.q.len, a.causal, a.window).hi;
        float m = -INFINITY, l = 0.f;
        for (int j = 0; j < nb; ++j) {
          ok = ok && wait_for(&s_full[t], (uint32_t)n_blocks & 1u, a.wait_limit);
          tmem_fence_after();
          const int t0 = it.span.first + (b0 + j) * kTileTokens;
          // the arithmetic of a block, made three times: most blocks have nothing to mask (with masks under conditions in one piece of
          // code 2048 rows over 16384 took 448 us instead of 428, 512 rows over 32768 in 8 bits 756 instead of 580), others end early
          // for some rows, windows begin late for some
          auto block = [&](auto kind) {
            constexpr bool kEnds = decltype(kind)::value & 1, kBegins = decltype(kind)::value & 2;
            uint32_t s[kHeld][32];
            // tokens from `upto` on, and before `from`, are not seen
            const int upto = see.hi - t0, from = see.lo - t0;
            auto mask = [&](uint32_t (&v)[32], int x0) {
#pragma unroll
              for (int x = 0; x < 32; ++x) {
                if (kEnds) v[x] = x0 + x < upto ? v[x] : 0xff800000u;
                if (kBegins) v[x] = x0 + x < from ? 0xff800000u : v[x];
              }
            };
            float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int x0 = 0; x0 < 4; x0 += kHeld) {
#pragma unroll
              for (int x = 0; x < kHeld; ++x) tmem_ld32_begin(s[x], tS + (x0 + x) * 32);
              tmem_ld_end();
#pragma unroll
              for (int x = 0; x < kHeld; ++x) {
                tmem_settled(s[x]);
                mask(s[x], (x0 + x) * 32);
              }
#pragma unroll
              for (int k = 0; k < 32; k += 4)
#pragma unroll
                for (int x = 0; x < kHeld; ++x) {
                  top[x % 2] = fmaxf(fmaxf(top[x % 2], __uint_as_float(s[x][k])), __uint_as_float(s[x][k + 1]));
                  top[x % 2 + 2] = fmaxf(fmaxf(top[x % 2 + 2], __uint_as_float(s[x][k + 2])), __uint_as_float(s[x][k + 3]));
                }
            }
            if (kHeld < 4) tmem_ld32_begin(s[0], tS);
            const float z = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale_log2;
            // m: the base (kSpare).  Only rows of the unit have a say: the others hold the next sequences' rows, nobody's, or what shared
            // memory held before
            if (__any_sync(0xffffffffu, mine && z > m + kRise<T>)) {
              const float next = fmaxf(m, z - kSpare<T>), keep = next == -INFINITY ? 1.f : exp2_fast(m - next);
              m = next;
              l *= keep;
              if (j > 0) {                                     // O of the blocks so far; the first product writes over what is there
                ok = ok && wait_for(&pv_done[t], (uint32_t)(n_blocks - 1) & 1u, a.wait_limit);
                tmem_fence_after();
#pragma unroll 1
                for (int x = 0; x < D; x += 32) {
                  uint32_t o[32];
                  tmem_ld32(o, tO + x);
#pragma unroll
                  for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * keep);
                  tmem_st32(tO + x, o);
                }
              }
            }
            const float base = m == -INFINITY ? 0.f : m;
            const F32x2 scale2 = pack2(a.scale_log2, a.scale_log2), base2 = pack2(-base, -base);
            F32x2 sum2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              uint32_t p[16];
              uint32_t (&v)[32] = s[x % kHeld];
              if (kHeld < 4) {
                tmem_ld_end();
                tmem_settled(v);
                if (x < 3) tmem_ld32_begin(s[(x + 1) % kHeld], tS + (x + 1) * 32);
                mask(v, x * 32);
              }
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                const float2 e = unpack2(fma2(pack2(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), scale2, base2));
                const float e0 = exp2_fast(e.x), e1 = exp2_fast(e.y);
                sum2[(k >> 1) & 1] = add2(sum2[(k >> 1) & 1], pack2(e0, e1));
                p[k / 2] = Two<T>::pack(e0, e1);
              }
              tmem_st16_begin(tS + x * 16, p);
              if (kSplit && x == kEarly - 1) {
                tmem_st_end();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&p_part[t]);
              }
            }
            const float2 both = unpack2(add2(sum2[0], sum2[1]));
            l += both.x + both.y;
          };
          if (t0 < lo_max) block(std::integral_constant<int, 3>());
          else if (t0 + kTileTokens > hi_min) block(std::integral_constant<int, 1>());
          else block(std::integral_constant<int, 0>());
          tmem_st_end();
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(&p_full[t]);
          ++n_blocks;
        }
        // ---- the unit's result, or this CTA's part of it
        ok = ok && wait_for(&pv_done[t], (uint32_t)(n_blocks - 1) & 1u, a.wait_limit);
        tmem_fence_after();
        const bool alone = b0 == 0 && nb == it.span.blocks, wide_out = ((uintptr_t)a.out & 31) == 0;
        float* part = a.partial + ((size_t)blockIdx.x * 2 + (it.unit_at <= (long long)blockIdx.x * per ? 0 : 1)) * kTilePartFloats<D>;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const size_t at = (size_t)(it.q.row0 + i) * heads_q + it.head * a.share + g;
#pragma unroll 1
        for (int x = 0; x < D; x += 32) {
          uint32_t o[32];
          tmem_ld32(o, tO + x);
          if (!alone) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)
              *reinterpret_cast<uint4*>(part + ((size_t)(x + k) / 4 * kTileUnit + t * kTileRows + row) * 4) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          } else if (mine) {
#pragma unroll
            for (int k = 0; k < 32; k += 16) {               // whole 32-byte sectors
              float2 f[4];
#pragma unroll
              for (int y = 0; y < 8; ++y) {
                const float x0 = l > 0.f ? __uint_as_float(o[k + 2 * y]) * inv : 0.f, x1 = l > 0.f ? __uint_as_float(o[k + 2 * y + 1]) * inv : 0.f;
                (y & 1 ? f[y >> 1].y : f[y >> 1].x) = __uint_as_float(Two<T>::pack(x0, x1));
              }
              if (wide_out) {
                store8(reinterpret_cast<float*>(a.out + (at * D + x + k) * 2), f);
              } else {
                *reinterpret_cast<float4*>(a.out + (at * D + x + k) * 2) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
                *reinterpret_cast<float4*>(a.out + (at * D + x + k) * 2 + 16) = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
              }
            }
          }
        }
        if (!alone) {
          *reinterpret_cast<float2*>(part + kTileUnit * D + (t * kTileRows + row) * 2) = make_float2(m, l);
        } else if (mine && a.lse != nullptr) {
          a.lse[at] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
        }
        tmem_fence_before();                                 // O has been read before the next unit's first P is announced
      }
      if (b0 == 0 && nb < it.span.blocks) {
        shared.last = (int)((it.unit_at + it.span.blocks - 1) / per);
        shared.slot = it.unit_at <= (long long)blockIdx.x * per ? 0 : 1;
        shared.row0 = it.q.row0 + i_unit;
        shared.rows = min(2 * a.tile_new, it.q.rows - i_unit);
        shared.head = it.head;
      }
      it.f += nb;
      it.settle(a);
    }
    if (tid == 0) static_cast<TileShared*>(a.shared_units)[blockIdx.x] = shared;
  } else if (BITS != 16 && warp < kProducts) {
    // ================================================================ codes into the stages, as values
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBringRegs));
    if constexpr (BITS != 16) {
      // A thread takes one 16-byte piece of every kRowStep-th token.
      constexpr int kPieces = S::kPieces, kCodes = S::kCodes, kTimes = S::kTimes, kRowStep = kBringWarps<BITS> * 32 / kPieces;
      const int tp = tid - 256, piece = tp % kPieces, row_first = tp / kPieces, groups = c.param_row_bytes >> 2, group = piece * kCodes >> group_shift;
      const Biases<T> biases;
      auto convert = [&](unsigned char* dst, int k, uint4 codes, uint32_t par) {
        const uint32_t raw[4] = {codes.x, codes.y, codes.z, codes.w};
        const uint32_t step = prmt(par, 0, 0x1010), low = prmt(par, 0, 0x3232);
        const float2 sl = Two<T>::wide(par);
        const F32x2 step2 = pack2(sl.x, sl.x), low2 = pack2(sl.y, sl.y);
        const int row = row_first + k * kRowStep;
        uint32_t x[kCodes / 2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t word = raw[w];
          if (BITS == 4) {
            const uint32_t even = word & 0x0f0f0f0fu, odd = word >> 4 & 0x0f0f0f0fu;
            constexpr uint32_t kBias = IsHalf<T>::value ? 0x64006400u : 0x43004300u;
            const uint32_t u = prmt(even, odd, 0x5140), v = prmt(even, odd, 0x7362);
            x[w * 4 % (kCodes / 2)] = code_value<T>(prmt(u, biases.byte, 0x4140), kBias, step, low);
            x[(w * 4 + 1) % (kCodes / 2)] = code_value<T>(prmt(u, biases.byte, 0x4342), kBias, step, low);
            x[(w * 4 + 2) % (kCodes / 2)] = code_value<T>(prmt(v, biases.byte, 0x4140), kBias, step, low);
            x[(w * 4 + 3) % (kCodes / 2)] = code_value<T>(prmt(v, biases.byte, 0x4342), kBias, step, low);
          } else if (IsHalf<T>::value) {
            x[w * 2] = code_value<T>(prmt(word, biases.byte, 0x4140), 0x64006400u, step, low);
            x[w * 2 + 1] = code_value<T>(prmt(word, biases.byte, 0x4342), 0x64006400u, step, low);
          } else {
            x[w * 2] = bytes_value<T>(word, word, 0, 1, biases, step2, low2);
            x[w * 2 + 1] = bytes_value<T>(word, word, 2, 3, biases, step2, low2);
          }
        }
#pragma unroll
        for (int y = 0; y < kCodes / 8; ++y) {
          const int p = piece * (kCodes / 8) + y;            // 16-byte piece of the row of values
          *reinterpret_cast<uint4*>(dst + (p >> 3) * S::kHalf + row * 128 + (((p & 7) ^ (row & 7)) << 4)) =
              make_uint4(x[4 * y], x[4 * y + 1], x[4 * y + 2], x[4 * y + 3]);
        }
      };
      uint32_t st = 0, phase = 0, from = 0, from_phase = 0;
      if (tp < 32) test_wait(6);
      for (long long left = any ? 2 * (it.f1 - it.f) : 0; left > 0; --left) {
        ok = __all_sync(0xffffffffu, ok && wait_for(&raw_full[from], from_phase, a.wait_limit) && wait_for(&kv_empty[st], phase ^ 1u, a.wait_limit));
        if (!ok) break;                                      // raw_empty may not be told of copies that have not landed
        const unsigned char* src = ahead + from * S::kAheadBytes;
        unsigned char* dst = stages + st * S::kOperand;
        const int2 rows = raw_rows[from];
        uint4 codes[kTimes];
        uint32_t par[kTimes];
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
          const int row = row_first + k * kRowStep;
          codes[k] = *reinterpret_cast<const uint4*>(src + (row * kPieces + piece) * 16);
          par[k] = *reinterpret_cast<const uint32_t*>(src + S::kRawCodes + (row * groups + group) * 4);
          // tokens of other rows may have anything there: a step and a minimum of zero stand for zero
          if (row < rows.x || row >= rows.y) par[k] = 0;
        }
#pragma unroll
        for (int k = 0; k < kTimes; ++k) convert(dst, k, codes[k], par[k]);
        async_fence();
        __syncwarp();
        if (lane == 0) { bar_arrive(&kv_full[st]); bar_arrive(&raw_empty[from]); }
        if (++st == NS) { st = 0; phase ^= 1u; }
        if (++from == S::kAhead) { from = 0; from_phase ^= 1u; }
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLastRegs));
    if (BITS == 16 && warp == 8) {
      // ============================================================== pages into the stages: a box of 64 channels by a page per lane
      constexpr int kHalves = D / 64;
      const int pages = kTileTokens >> c.page_shift, slot_page = lane % pages, half = lane / pages;
      uint32_t st = 0, phase = 0, edges = 0;
      int copies = 0;
      for (; any && ok; ++it.f) {
        it.settle(a);
        if (it.f >= it.f1) break;
        const int t0 = it.span.first + it.block() * kTileTokens, tp = t0 + (slot_page << c.page_shift);
        bool on = half < kHalves && tp < it.span.hi && tp + c.page_size > it.span.lo;
        int page = 0;
        if (on) { page = page_of(c, it.s, tp); on = page >= 0; }
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, on)) * c.page_size * 128u;
        const bool ragged = t0 < it.span.lo || t0 + kTileTokens > it.span.hi;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          ok = __all_sync(0xffffffffu, ok && wait_for(&kv_empty[st], phase ^ 1u, a.wait_limit));
          if (!ok) break;
          unsigned char* dst = stages + st * S::kOperand;
          // values behind the last token or ahead of the first may be no numbers, which a probability of zero does not hide: they
          // are zeroed before the block is announced
          const bool fix = side == 1 && ragged;
          uint64_t* bar = fix ? &edge : &kv_full[st];
          if (lane == 0) bar_expect(bar, bytes);
          __syncwarp();
          if (on) load_page_box(dst + half * S::kHalf + (slot_page << c.page_shift) * 128, &maps.kv[side], half * 64, 0, it.head, page, bar);
          if (fix) {
            ok = __all_sync(0xffffffffu, wait_for(&edge, edges++ & 1u, a.wait_limit));
            const int lo = max(0, it.span.lo - t0), hi = max(lo, min(kTileTokens, it.span.hi - t0));
            for (int x = lane; x < kTileTokens * (D / 8); x += 32) {
              const int row = x / (D / 8), p = x % (D / 8);
              if (row < lo || row >= hi) *reinterpret_cast<uint4*>(dst + (p >> 3) * S::kHalf + row * 128 + (p & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            async_fence();
            __syncwarp();
            if (lane == 0) bar_arrive(&kv_full[st]);
          }
          ++copies;
          if (++st == NS) { st = 0; phase ^= 1u; }
        }
        test_wait(3);
      }
      // copies land before their memory goes (bounded), whoever gave up
      if (edges) bar_wait(&edge, (edges - 1) & 1u, 100);
      for (int x = max(0, copies - NS); x < copies; ++x) bar_wait(&kv_full[x % NS], (uint32_t)(x / NS) & 1u, 100);
    }
    if (BITS != 16 && warp == kProducts + 2) {
      // ============================================================== codes and parameters of a page, a lane each
      const int pages = kTileTokens >> c.page_shift;
      const uint32_t code_bytes = c.page_size * S::kRowBytes, param_bytes = c.page_size * c.param_row_bytes;
      uint32_t from = 0, phase = 0;
      int copies = 0;
      for (; any && ok; ++it.f) {
        it.settle(a);
        if (it.f >= it.f1) break;
        const int t0 = it.span.first + it.block() * kTileTokens, tp = t0 + (lane << c.page_shift);
        bool on = lane < pages && tp < it.span.hi && tp + c.page_size > it.span.lo;
        long long page = 0;
        if (on) { page = page_of(c, it.s, tp); on = page >= 0; }
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, on)) * (code_bytes + param_bytes);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          ok = __all_sync(0xffffffffu, ok && wait_for(&raw_empty[from], phase ^ 1u, a.wait_limit));
          if (!ok) break;
          unsigned char* dst = ahead + from * S::kAheadBytes;
          if (lane == 0) {
            raw_rows[from] = make_int2(it.span.lo - t0, it.span.hi - t0);
            bar_expect(&raw_full[from], bytes);
          }
          __syncwarp();
          if (on) {
            bulk_copy(dst + lane * code_bytes, c.pages[side] + page * c.page_bytes + (long long)it.head * code_bytes, code_bytes, &raw_full[from]);
            bulk_copy(dst + S::kRawCodes + lane * param_bytes, c.params[side] + page * c.param_bytes + (long long)it.head * param_bytes, param_bytes,
                      &raw_full[from]);
          }
          ++copies;
          if (++from == S::kAhead) { from = 0; phase ^= 1u; }
        }
        test_wait(3);
      }
      for (int x = max(0, copies - S::kAhead); x < copies; ++x) bar_wait(&raw_full[x % max(1, S::kAhead)], (uint32_t)(x / max(1, S::kAhead)) & 1u, 100);     // as above
    }
    if (warp == kProducts + 1 && lane == 0) {
      // ============================================================== query rows into their tiles: a box of 64 channels by whole new rows
      uint32_t units_of[2] = {0, 0};
      const uint32_t bytes = (uint32_t)a.tile_new * a.share * D * 2;
      while (any && ok && it.f < it.f1) {
        for (int t = 0; t < 2 && ok; ++t) {
          const int i_first = (it.unit * 2 + t) * a.tile_new;
          if (i_first >= it.q.rows) break;
          ok = wait_for(&q_empty[t], ~units_of[t] & 1u, a.wait_limit);
          if (!ok) break;
          ++units_of[t];
          bar_expect(&q_full[t], bytes);
          for (int h = 0; h < D / 64; ++h)
            load_rows_box(smem + t * S::kOperand + h * S::kHalf, &maps.q, h * 64, it.head * a.share, it.q.row0 + i_first, &q_full[t]);
        }
        it.f += it.blocks_here();
        it.settle(a);
        test_wait(4);
      }
      for (int t = 0; t < 2; ++t)                            // as above
        if (units_of[t]) bar_wait(&q_full[t], (units_of[t] - 1) & 1u, 100);
    }
    if (warp == kProducts) {
      // ============================================================== products
      // The whole warp walks through the blocks, so that descriptors and addresses stay in uniform registers; one lane issues.
      // Descriptors: 128-byte swizzle, 8-row groups 1 KB apart.  Q and K lie along the contracted channels (K-major: 16 channels are 32
      // bytes, 64-channel halves kHalf apart); V across them (its 64-channel halves kHalf apart, 16 tokens 2 KB).
      constexpr uint64_t kDescK = (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
      constexpr uint64_t kDescV = ((uint64_t)(S::kHalf >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
      constexpr uint32_t kType = IsHalf<T>::value ? 0u : 1u;
      constexpr uint32_t kIdesc = (1u << 4) | (kType << 7) | (kType << 10) | ((128u >> 4) << 24);
      constexpr uint32_t kIdescS = kIdesc | ((128u >> 3) << 17), kIdescO = kIdesc | (1u << 16) | (((uint32_t)D >> 3) << 17);
      const bool leader = elect_one();
      const uint64_t descQ = kDescK | (smem_addr(smem) >> 4), descK = kDescK | (smem_addr(stages) >> 4), descV = kDescV | (smem_addr(stages) >> 4);
      constexpr uint32_t kStageStep = S::kOperand >> 4;
      auto scores = [&](int t, uint32_t st) {
        if (!leader) return;
        const uint64_t q = descQ + t * kStageStep, k = descK + st * kStageStep;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
          const uint32_t off = (x >> 2) * (S::kHalf >> 4) + (x & 3) * 2;
          umma_f16(tmem + t * 128, q + off, k + off, kIdescS, x == 0 ? 0u : 1u);
        }
        umma_commit(&s_full[t]);
      };
      auto outputs = [&](int t, uint32_t st, bool first, int part) {       // tokens of the first kEarly quarters, or the others
        if (!leader) return;
        const uint64_t v = descV + st * kStageStep;
#pragma unroll
        for (int x = 0; x < kTileTokens / 16; ++x)
          if ((x < 2 * kEarly) == (part == 0))
            umma_f16_ts(tmem + 256 + t * 128, tmem + t * 128 + x * 8, v + x * (2048 >> 4), kIdescO, first && x == 0 ? 0u : 1u);
        if (part == 1) umma_commit(&pv_done[t]);
      };
      auto release = [&](uint64_t* b) { if (leader) umma_commit(b); };
      // a place in the ring of stages: K and V blocks in turn
      struct Place { uint32_t st, phase; };
      auto after = [&](Place x) { return x.st + 1 == NS ? Place{0u, x.phase ^ 1u} : Place{x.st + 1, x.phase}; };
      Place k = {0, 0};                                      // of the present block's keys
      uint32_t blocks_of[2] = {0, 0}, units_of[2] = {0, 0};
      while (any && ok && it.f < it.f1) {
        const int nb = __shfl_sync(0xffffffffu, it.blocks_here(), 0);
        const bool two = __shfl_sync(0xffffffffu, (it.unit * 2 + 1) * a.tile_new < it.q.rows, 0);
        auto wait = [&](uint64_t* b, uint32_t parity) { ok = ok && wait_for(b, parity & 1u, a.wait_limit); ok = __all_sync(0xffffffffu, ok); tmem_fence_after(); return ok; };
        if (!wait(&kv_full[k.st], k.phase) || !wait(&q_full[0], units_of[0]++)) break;
        scores(0, k.st);
        if (nb == 1) release(&q_empty[0]);                   // the tile's next rows may come
        if (two) {
          if (!wait(&q_full[1], units_of[1]++)) break;
          scores(1, k.st);
          if (nb == 1) release(&q_empty[1]);
        }
        release(&kv_empty[k.st]);
        test_wait(5);
        for (int j = 0; j < nb; ++j) {
          const Place v = after(k), next = after(v);
          if (!wait(&kv_full[v.st], v.phase) || !wait(kSplit ? &p_part[0] : &p_full[0], blocks_of[0])) break;
          outputs(0, v.st, j == 0, 0);
          if (kSplit && !wait(&p_full[0], blocks_of[0])) break;
          ++blocks_of[0];
          outputs(0, v.st, j == 0, 1);
          if (j + 1 < nb) {
            if (!wait(&kv_full[next.st], next.phase)) break;
            scores(0, next.st);
            if (j + 2 == nb) release(&q_empty[0]);
          }
          if (two) {
            if (!wait(kSplit ? &p_part[1] : &p_full[1], blocks_of[1])) break;
            outputs(1, v.st, j == 0, 0);
            if (kSplit && !wait(&p_full[1], blocks_of[1])) break;
            ++blocks_of[1];
            outputs(1, v.st, j == 0, 1);
          }
          release(&kv_empty[v.st]);
          if (j + 1 < nb) {
            if (two) scores(1, next.st);
            if (two && j + 2 == nb) release(&q_empty[1]);
            release(&kv_empty[next.st]);
          }
          k = next;
        }
        it.f += nb;
        it.settle(a);
      }
      // products end before their operands' memory and tensor memory go (bounded); whoever reads the last ones may have given up
      if (any) {
        release(&ended);
        bar_wait(&ended, 0, 100);
      }
    }
    __syncwarp();
  }
  if (!ok) atomicExch(c.status, GEAR_ERR_TIMEOUT);
  tmem_fence_before();
  __syncthreads();
  if (warp == kProducts) {
    tmem_fence_after();
    tmem_free<512>(tmem);
  }
}

template <class T, int BITS, int D>
cudaError_t launch_tile_t(const PagedAttnArgs& a, int group, cudaStream_t st) {
  int shift = 0, sms = 0;
  while ((1 << shift) < group) ++shift;
  static KernelReady ready;
  cudaError_t e = ready.on_this_device(paged_tile_kernel<T, BITS, D>, TileSmem<BITS, D>::kBytes, &sms);
  if (e != cudaSuccess) return e;
  TileMaps maps = {};
  if (BITS == 16)
    for (int side = 0; side < 2; ++side) {
      e = make_page_map(&maps.kv[side], a.c.pages[side], IsHalf<T>::value, D, a.c.page_size, a.c.heads, a.c.n_pages, a.c.page_bytes);
      if (e != cudaSuccess) return e;
    }
  e = make_rows_map(&maps.q, a.q, IsHalf<T>::value, D, a.c.heads * a.share, a.c.n_rows, a.q_stride, a.share, a.tile_new);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_dependent(paged_tile_kernel<T, BITS, D>, dim3((unsigned)a.tile_ctas), kTileThreads<BITS>, TileSmem<BITS, D>::kBytes, st, a, shift, maps);
}
template <int BITS>
cudaError_t launch_tile_bits(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st) {
  if (dtype == GEAR_F16) return a.c.head_dim == 128 ? launch_tile_t<__half, BITS, 128>(a, group, st) : launch_tile_t<__half, BITS, 64>(a, group, st);
  return a.c.head_dim == 128 ? launch_tile_t<__nv_bfloat16, BITS, 128>(a, group, st) : launch_tile_t<__nv_bfloat16, BITS, 64>(a, group, st);
}

}  // namespace gear

// Attention of many new rows over a paged cache, on tcgen05.  Bound: the tensor cores and, as close behind, the exponentials (each of them busy
// 59 % of the time; 2048 rows of 32 heads over 16384 tokens 428 us, 1.2 PFLOP/s, and 508, 1.0, at the 1635 MHz of the power limit), between them the
// latency of a tile's softmax, which one warp per scheduler works through.
//
// A unit of work is 2 x 128 query rows of a sequence and kv head (row i * share + g of a tile: new row i, query head g of the kv head, so
// that a short chunk of grouped heads fills them; a tile takes whole new rows) against blocks of 128 tokens.  Its two tiles take turns: while one tile's
// probabilities are computed the tensor cores work for the other.  Per tile and block S = Q K^T (operands in shared memory) lands in
// tensor memory, one thread per row turns it into probabilities, which go back over the scores as the A operand of O += P V.  O
// stays in tensor memory and is scaled only when a maximum rises by more than 2^8 (sums and outputs are kept beside a lagging
// base, kSpare in gear_paged_rows.cuh).  Tensor memory: S0 | S1 | O0 | O1, 128 columns each.
//
// Probabilities are rounded once to the type, as the tensor cores take them; their sum is of those in 32 bits.  In two parts, as with few rows,
// the products with V would be twice as many.  Errors against 64 bits, and with probabilities in 32 bits: 2048 rows over 16384 in fp16 2.4e-4
// and 2.1e-4, ragged prompts in bf16 1.7e-3 and 1.5e-3, 512 rows over 32768 in 8 bits of bf16 1.9e-3 and 1.7e-3.
//
// Blocks of all units, one after the other, are cut into equal ranges, one per SM; units that lie in several ranges leave partial
// results for paged_tile_join_kernel.  paged_tile_plan_kernel sums the units' blocks beforehand.
#pragma once
#include "gear_paged.cuh"
#include "gear_umma.cuh"

namespace gear {

constexpr int kTileRows = 128, kTileUnit = 2 * kTileRows, kTileTokens = 128;
constexpr int kTileMaxCtas = 148;
constexpr int kTileLeast = 2;                    // blocks per CTA at least

// Rows and tokens of a unit
struct TileSeq { int row0, rows, pos0, len, units; bool bad; };
__device__ __forceinline__ TileSeq tile_seq(const PagedAttnArgs& a, int s) {
  const RowRange r = rows_of(a.c.row_start, s, a.c.n_rows);
  const Length n = length_of(a.c.lengths, s, a.c.table_stride, a.c.page_size);
  TileSeq q;
  q.bad = r.bad || n.bad || r.hi - r.lo > a.max_rows;
  q.row0 = r.lo;
  q.rows = min(r.hi - r.lo, a.max_rows);
  q.pos0 = n.n - (r.hi - r.lo);
  q.len = n.n;
  q.units = (q.rows + 2 * a.tile_new - 1) / (2 * a.tile_new);
  return q;
}
struct TileSpan { int lo, hi, first, blocks; };
__device__ __forceinline__ TileSpan tile_span(const PagedAttnArgs& a, const TileSeq& q, int unit) {
  const int i0 = unit * 2 * a.tile_new, i1 = min(q.rows, i0 + 2 * a.tile_new) - 1;
  const Span v = seen_by(q.pos0 + i0, q.pos0 + i1, q.len, a.causal, a.window);
  TileSpan t;
  t.lo = v.lo; t.hi = v.hi;
  t.first = v.lo & ~(kTileTokens - 1);
  t.blocks = max(1, (v.hi - t.first + kTileTokens - 1) / kTileTokens);
  return t;
}

// Where a CTA is in its range: blocks f .. of the unit that begins at unit_at
struct TileIter {
  long long f, f1, unit_at;
  int s, head, unit;
  TileSeq q;
  TileSpan span;
  __device__ __forceinline__ int block() const { return (int)(f - unit_at); }
  __device__ __forceinline__ int blocks_here() const { return (int)min((long long)span.blocks - block(), f1 - f); }
  // finds f among the planned sums: sums[i] blocks per head lie before unit i of all sequences
  __device__ __forceinline__ void find(const PagedAttnArgs& a) {
    const int* tf = a.unit_first;
    int lo = 0, hi = a.c.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.unit_sums[tf[mid + 1]] * a.c.heads > f) hi = mid; else lo = mid + 1;
    }
    s = lo;
    const int u0 = tf[s], u1 = tf[s + 1];
    const long long base = a.unit_sums[u0], per_head = a.unit_sums[u1] - base;
    head = (int)((f - base * a.c.heads) / per_head);
    const long long rest = f - base * a.c.heads - head * per_head;
    lo = u0; hi = u1 - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.unit_sums[mid + 1] - base > rest) hi = mid; else lo = mid + 1;
    }
    unit = lo - u0;
    unit_at = f - (rest - (a.unit_sums[lo] - base));
    q = tile_seq(a, s);
    span = tile_span(a, q, unit);
  }
  // on to the next unit once f has passed the present one
  __device__ __forceinline__ void settle(const PagedAttnArgs& a) {
    if (f >= f1 || f < unit_at + span.blocks) return;
    unit_at += span.blocks;
    if (++unit >= q.units) {
      unit = 0;
      if (++head >= a.c.heads) {
        head = 0;
        do {
          if (++s >= a.c.n_seqs) { f = f1; return; }         // tables that changed meanwhile
          q = tile_seq(a, s);
        } while (q.units == 0 || a.unit_first[s + 1] == a.unit_first[s]);
      }
    }
    span = tile_span(a, q, unit);
  }
};

// What a CTA whose range ends inside a unit that it began leaves for the kernel that joins the parts: the last CTA of the unit (0: there is no
// such unit), which of its own two parts is meant, the unit's first new row, how many it has, its kv head
struct TileShared { int last, slot, row0, rows, head, pad[3]; };

// floats of a part of a unit: O as [D / 4][256 rows][4], then (maximum, sum) of each row
template <int D> constexpr int kTilePartFloats = kTileUnit * (D + 2);

cudaError_t launch_tile_b16(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st);
cudaError_t launch_tile_b8(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st);
cudaError_t launch_tile_b4(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st);

}  // namespace gear

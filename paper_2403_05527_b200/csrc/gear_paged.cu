// Paged cache: argument checks, rows into pages (as they are or as codes of Eq. 2) and pages back into rows.
#include <cuda_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gear_paged.cuh"
#include "gear_quant.cuh"

namespace gear {

// 32 entries of 16 bits, 16-byte aligned; whole sectors at once where they are 32-byte aligned
__device__ __forceinline__ void load_32_entries(uint32_t (&x)[16], const unsigned char* src, bool on) {
#pragma unroll
  for (int k = 0; k < 16; ++k) x[k] = 0;
  if (!on) return;
  if (((uintptr_t)src & 31) == 0) {
#pragma unroll
    for (int k = 0; k < 16; k += 8)
      asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(x[k]), "=r"(x[k + 1]), "=r"(x[k + 2]), "=r"(x[k + 3]), "=r"(x[k + 4]), "=r"(x[k + 5]), "=r"(x[k + 6]), "=r"(x[k + 7])
                   : "l"(src + k * 4));
  } else {
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
      const uint4 v = __ldcg(reinterpret_cast<const uint4*>(src + k * 4));
      x[k] = v.x; x[k + 1] = v.y; x[k + 2] = v.z; x[k + 3] = v.w;
    }
  }
}
__device__ __forceinline__ void store_32_entries(unsigned char* dst, const uint32_t (&x)[16]) {
  if (((uintptr_t)dst & 31) == 0) {
#pragma unroll
    for (int k = 0; k < 16; k += 8)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst + k * 4), "r"(x[k]), "r"(x[k + 1]), "r"(x[k + 2]), "r"(x[k + 3]),
                   "r"(x[k + 4]), "r"(x[k + 5]), "r"(x[k + 6]), "r"(x[k + 7]) : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < 16; k += 4) *reinterpret_cast<uint4*>(dst + k * 4) = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
  }
}

// ------------------------------------------------------------------ rows into pages
constexpr int kAppendThreads = 256;

// Piece `block * pieces` as a row of per_row (at most 2^14) pieces and one of its pieces, in 32 bits (a division of 64 is a call)
__device__ __forceinline__ void first_piece(int block, int pieces, int per_row, int& row, int& piece) {
  const int q = block / per_row, rest = (block - q * per_row) * pieces;
  row = q * pieces + rest / per_row;
  piece = rest % per_row;
}

// Page and slot of row `row`, (-1, 0) where it has none
__device__ __forceinline__ int2 place_of_row(const PagedArgs& c, int row) {
  const int s = sequence_of(c.row_start, c.n_seqs, row, row);
  if (s < 0) {
    if (row < __ldcg(c.row_start + c.n_seqs)) paged_bad(c);
    return make_int2(-1, 0);
  }
  const RowRange rr = rows_of(c.row_start, s, c.n_rows);
  const Length len = length_of(c.lengths, s, c.table_stride, c.page_size);
  const int t = len.n - (rr.hi - row);
  if (rr.bad || len.bad || t < 0) { paged_bad(c); return make_int2(-1, 0); }
  return make_int2(page_of(c, s, t), t & (c.page_size - 1));
}

// What is wrong with the tables is found by the first CTA, whatever rows look up: a row within the ranges of two sequences finds one of them, and
// sequences without rows are found by none
__device__ __forceinline__ void check_tables(const PagedArgs& c) {
  if (blockIdx.x != 0 || blockIdx.y != 0) return;
  bool bad = threadIdx.x == 0 && __ldcg(c.row_start) != 0;
  for (int s = threadIdx.x; s < c.n_seqs; s += kAppendThreads) {
    const RowRange r = rows_of(c.row_start, s, c.n_rows);
    const Length n = length_of(c.lengths, s, c.table_stride, c.page_size);
    bad = bad || r.bad || n.bad || r.hi - r.lo > n.n;
  }
  if (bad) paged_bad(c);
}

// Rows as they are.  Bound: HBM.  A thread takes 16 bytes of a row of K and of V, PER times; the loads of the rows do not wait for the
// look-up of their slots.
template <int PER>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(PagedArgs c, const unsigned char* k_new, const unsigned char* v_new,
                                                                      long long k_stride, long long v_stride) {
  constexpr int kPieces = kAppendThreads * PER;
  __shared__ int2 where[kPieces / 8 + 2];          // page and slot of the rows that this CTA touches
  const int tid = threadIdx.x, per_head = c.head_dim >> 3, per_row = c.heads * per_head;
  int row0, off0;
  first_piece(blockIdx.x, kPieces, per_row, row0, off0);
  const int rows = min((off0 + kPieces - 1) / per_row + 1, c.n_rows - row0);
  after_previous();
  uint4 x[PER][2];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = off0 + j * kAppendThreads + tid, r = i / per_row, rem = i - r * per_row;
    if (r < rows) {
      x[j][0] = __ldcg(reinterpret_cast<const uint4*>(k_new + (row0 + r) * k_stride) + rem);
      x[j][1] = __ldcg(reinterpret_cast<const uint4*>(v_new + (row0 + r) * v_stride) + rem);
    }
  }
  check_tables(c);
  for (int r = tid; r < rows; r += kAppendThreads) where[r] = place_of_row(c, row0 + r);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = off0 + j * kAppendThreads + tid, r = i / per_row, rem = i - r * per_row;
    if (r >= rows || where[r].x < 0) continue;
    const int2 w = where[r];
    const int head = rem / per_head, piece = rem - head * per_head;
    const size_t at = w.x * c.page_bytes + ((size_t)head * c.page_size + w.y) * c.row_bytes + piece * 16;
#pragma unroll
    for (int side = 0; side < 2; ++side) *reinterpret_cast<uint4*>(c.pages[side] + at) = x[j][side];
  }
}

// 1 / x, rounded to nearest, for x of at most 11 bits between 2^-126 and 2^126: one Newton step behind the approximate reciprocal
// (Markstein 1990)
__device__ __forceinline__ float reciprocal_of(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return __fmaf_rn(__fmaf_rn(-x, y, 1.f), y, y);
}

// Rows as codes.  Bound: HBM by its bytes (8 x 4096 rows of 32 heads to 4 bits: 104 us), the issue of instructions in fact.  A thread takes
// 32 channels of a row of K or V (blockIdx.y): a group is one thread's or that of two or four, so that the step and its reciprocal
// come once per 32 entries (with eight channels a thread 282 us, now 137).  The extremes are found on packed pairs, as (minimum,
// -maximum) where lanes exchange them.  Eq. 2 runs on pairs of binary32 operations; the code is what lies below 1.5 * 2^23 once that has
// been added, which rounds to nearest even as rint does.  Codes above the last one come from steps that are rounded down far, and only a
// warp that has such a group bounds them.
template <class T, int BITS>
__global__ void __launch_bounds__(kAppendThreads) paged_append_codes_kernel(PagedArgs c, const unsigned char* k_new, const unsigned char* v_new,
                                                                            long long k_stride, long long v_stride, int group) {
  __shared__ int2 where[kAppendThreads / 2 + 2];
  const int tid = threadIdx.x, side = blockIdx.y, per_head = c.head_dim >> 5, per_row = c.heads * per_head;
  int row0, off0;
  first_piece(blockIdx.x, kAppendThreads, per_row, row0, off0);
  const int rows = min((off0 + kAppendThreads - 1) / per_row + 1, c.n_rows - row0);
  // (i + 1/2) / per_row, both below 2^15, is never within rounding of a whole number
  const int i = off0 + tid, r = (int)(((float)i + 0.5f) * __frcp_rn((float)per_row)), rem = i - r * per_row;
  const unsigned char* src = (side == 0 ? k_new + (row0 + r) * k_stride : v_new + (row0 + r) * v_stride) + (size_t)rem * 64;
  after_previous();
  uint32_t x[16];
  load_32_entries(x, src, r < rows);
  check_tables(c);
  for (int q = tid; q < rows; q += kAppendThreads) where[q] = place_of_row(c, row0 + q);

  uint32_t lo2 = x[0], hi2 = x[0];
#pragma unroll
  for (int k = 1; k < 16; ++k) { lo2 = Two<T>::min(lo2, x[k]); hi2 = Two<T>::max(hi2, x[k]); }
  // (minimum, -maximum) of the thread, then of the group's lanes
  hi2 ^= 0x80008000u;
  uint32_t both = Two<T>::min(__byte_perm(lo2, hi2, 0x5410), __byte_perm(lo2, hi2, 0x7632));
  for (int o = 1; o < group >> 5; o <<= 1) both = Two<T>::min(both, __shfl_xor_sync(0xffffffffu, both, o));
  const float2 ends = Two<T>::wide(both);
  const float lo = ends.x, hi = -ends.y;
  constexpr float kTop = (float)((1 << BITS) - 1);
  const float range = __fsub_rn(hi, lo);
  float step = Two<T>::round(__fmul_rn(range, 1.0f / kTop));
  if (!(step >= 1.17549435e-38f)) step = 0.f;
  const float inverse = step > 0.f ? reciprocal_of(step) : 0.f;
  const bool over = __any_sync(0xffffffffu, __fmul_rn(range, inverse) >= kTop + 0.5f);
  const F32x2 low2 = pack2(-lo, -lo), inverse2 = pack2(inverse, inverse), magic2 = pack2(12582912.f, 12582912.f), one2 = pack2(1.f, 1.f);
  uint32_t words[8];                               // four codes each, a byte apart
  auto codes = [&](auto bounded) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t b[4];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const float2 w = Two<T>::wide(x[2 * k + p]);
        F32x2 t = mul2(add2(pack2(w.x, w.y), low2), inverse2);
        if (decltype(bounded)::value) {
          const float2 y = unpack2(t);
          t = pack2(fminf(y.x, kTop), fminf(y.y, kTop));
        }
        // (as a sum, the product before it was contracted into it, and lost its own rounding)
        const float2 u = unpack2(fma2(t, one2, magic2));
        b[2 * p] = __float_as_uint(u.x); b[2 * p + 1] = __float_as_uint(u.y);
      }
      words[k] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
  };
  if (over) codes(std::true_type()); else codes(std::false_type());
  __syncthreads();
  if (r >= rows || where[r].x < 0) return;
  const int2 w = where[r];
  const int head = rem / per_head, piece = rem - head * per_head;
  const size_t row = (size_t)head * c.page_size + w.y;
  unsigned char* dst = pages_of(c, side) + w.x * c.page_bytes + row * c.row_bytes + piece * (4 * BITS);
  if (BITS == 8) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(words[0], words[1], words[2], words[3]);
    *reinterpret_cast<uint4*>(dst + 16) = make_uint4(words[4], words[5], words[6], words[7]);
  } else {
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)                    // bytes 0 and 2 of w | w >> 4 hold two codes each
      o[k] = __byte_perm(words[2 * k] | words[2 * k] >> 4, words[2 * k + 1] | words[2 * k + 1] >> 4, 0x6420);
    *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  const int lanes = group >> 5;
  if ((piece & (lanes - 1)) == 0)
    *reinterpret_cast<uint32_t*>(params_of(c, side) + w.x * c.param_bytes + row * c.param_row_bytes + piece / lanes * 4) = Two<T>::pack(step, lo);
}

template <int PER>
cudaError_t append_rows(const PagedArgs& c, const void* k, const void* v, long long ks, long long vs, cudaStream_t st) {
  const long long pieces = (long long)c.n_rows * c.heads * (c.head_dim >> 3);
  const long long grid = (pieces + kAppendThreads * PER - 1) / (kAppendThreads * PER);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  count_launches(1);
  return launch_dependent(paged_append_kernel<PER>, dim3((unsigned)grid), kAppendThreads, 0, st, c, (const unsigned char*)k,
                          (const unsigned char*)v, ks, vs);
}
template <class T, int BITS>
cudaError_t append_codes(const PagedArgs& c, const void* k, const void* v, long long ks, long long vs, int group, cudaStream_t st) {
  const long long pieces = (long long)c.n_rows * c.heads * (c.head_dim >> 5);
  const long long grid = (pieces + kAppendThreads - 1) / kAppendThreads;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  count_launches(1);
  return launch_dependent(paged_append_codes_kernel<T, BITS>, dim3((unsigned)grid, 2), kAppendThreads, 0, st, c, (const unsigned char*)k,
                          (const unsigned char*)v, ks, vs, group);
}
template <class T>
cudaError_t append_bits(const PagedArgs& c, int bits, const void* k, const void* v, long long ks, long long vs, int group, cudaStream_t st) {
  if (bits == 8) return append_codes<T, 8>(c, k, v, ks, vs, group, st);
  if (bits == 4) return append_codes<T, 4>(c, k, v, ks, vs, group, st);
  // two pieces a thread where every SM has eight CTAs of them
  const long long pieces = (long long)c.n_rows * c.heads * (c.head_dim >> 3);
  return pieces >= 148LL * 8 * 2 * kAppendThreads ? append_rows<2>(c, k, v, ks, vs, st) : append_rows<1>(c, k, v, ks, vs, st);
}

// ------------------------------------------------------------------ pages into rows
// Bound: HBM (codes in once, rows out once).  A CTA takes 64 tokens of a head, K and V.  Rows as they are: a thread 16 bytes of a token,
// twice two.  Codes: a thread 32 channels of a token, which share a step, and whole sectors both ways (with eight channels a thread 4 bits ran at
// 71 % of the copy bandwidth, bound by instructions).
constexpr int kReadThreads = 256, kReadTokens = 64;

__device__ __forceinline__ bool read_range(const PagedArgs& c, const int32_t* first, long long n, int s, int& from, long long& base, int& end) {
  const Length len = length_of(c.lengths, s, c.table_stride, c.page_size);
  from = first != nullptr ? __ldcg(first + s) : 0;
  if ((len.bad || from < 0) && threadIdx.x == 0) paged_bad(c);
  base = (long long)blockIdx.x * kReadTokens;
  if (from < 0 || from + base >= len.n) return false;
  end = (int)min((long long)kReadTokens, min(n, (long long)len.n - from) - base);
  return true;
}

__global__ void __launch_bounds__(kReadThreads) paged_read_kernel(PagedArgs c, unsigned char* k_out, unsigned char* v_out, const int32_t* first,
                                                                  long long n) {
  const int head = blockIdx.y, s = blockIdx.z, per_head = c.head_dim >> 3;
  const int piece = threadIdx.x & (per_head - 1), lane_token = threadIdx.x / per_head, step_tokens = kReadThreads / per_head;
  after_previous();
  int from, end;
  long long base;
  if (!read_range(c, first, n, s, from, base, end)) return;
  unsigned char* outs[2] = {k_out, v_out};
  for (int i0 = lane_token; i0 < kReadTokens; i0 += step_tokens * 2) {
    uint4 raw[2][2];
    int page[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = i0 + u * step_tokens, t = from + (int)base + i;
      page[u] = -1;
      if (i < end) page[u] = page_of(c, s, t);
      if (page[u] < 0) continue;
#pragma unroll
      for (int side = 0; side < 2; ++side)
        if (outs[side] != nullptr)
          raw[u][side] = __ldcs(reinterpret_cast<const uint4*>(c.pages[side] + page[u] * c.page_bytes + token_row(c, head, t) * c.row_bytes) + piece);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (page[u] < 0) continue;
      const size_t at = (((size_t)s * c.heads + head) * n + base + i0 + u * step_tokens) * c.head_dim * 2 + piece * 16;
#pragma unroll
      for (int side = 0; side < 2; ++side)
        if (outs[side] != nullptr) __stcs(reinterpret_cast<uint4*>(outs[side] + at), raw[u][side]);
    }
  }
}

template <class T, int BITS>
__global__ void __launch_bounds__(kReadThreads) paged_read_codes_kernel(PagedArgs c, unsigned char* k_out, unsigned char* v_out,
                                                                        const int32_t* first, long long n, int group_shift) {
  const int head = blockIdx.y, s = blockIdx.z, per_head = c.head_dim >> 5;
  const int piece = threadIdx.x & (per_head - 1), step_tokens = kReadThreads / per_head;
  after_previous();
  int from, end;
  long long base;
  if (!read_range(c, first, n, s, from, base, end)) return;
  unsigned char* outs[2] = {k_out, v_out};
  for (int i = threadIdx.x / per_head; i < end; i += step_tokens) {
    const int t = from + (int)base + i, page = page_of(c, s, t);
    if (page < 0) continue;
    const size_t row = token_row(c, head, t);
    uint32_t raw[2][BITS], par[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      if (outs[side] == nullptr) continue;
      const uint4* src = reinterpret_cast<const uint4*>(c.pages[side] + page * c.page_bytes + row * c.row_bytes + piece * (4 * BITS));
#pragma unroll
      for (int k = 0; k < BITS / 4; ++k) {
        const uint4 v = __ldcg(src + k);
        raw[side][4 * k] = v.x; raw[side][4 * k + 1] = v.y; raw[side][4 * k + 2] = v.z; raw[side][4 * k + 3] = v.w;
      }
      par[side] = __ldcg(reinterpret_cast<const uint32_t*>(c.params[side] + page * c.param_bytes + row * c.param_row_bytes) +
                        (piece * 32 >> group_shift));
    }
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      if (outs[side] == nullptr) continue;
      const float2 p = Two<T>::wide(par[side]);
      const F32x2 step = pack2(p.x, p.x), low = pack2(p.y, p.y), bias = pack2(-8388608.f, -8388608.f);
      // bytes a and b of words u and v as 2^23 + code in 32 bits; the product of a code and a step is exact there, so the value is rounded
      // once there and once more to the type
      auto value = [&](uint32_t u, int a, uint32_t v, int b) {
        const F32x2 biased = pack2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440u + a)), __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7440u + b)));
        const float2 x = unpack2(fma2(add2(biased, bias), step, low));
        return Two<T>::pack(x.x, x.y);
      };
      uint32_t out[16];
#pragma unroll
      for (int k = 0; k < BITS; ++k) {
        const uint32_t w = raw[side][k];
        if (BITS == 8) {
          out[2 * k] = value(w, 0, w, 1);
          out[2 * k + 1] = value(w, 2, w, 3);
        } else {
          const uint32_t even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
#pragma unroll
          for (int b = 0; b < 4; ++b) out[(4 * k + b) % 16] = value(even, b, odd, b);
        }
      }
      store_32_entries(outs[side] + ((((size_t)s * c.heads + head) * n + base + i) * c.head_dim + piece * 32) * 2, out);
    }
  }
}

static dim3 read_grid(const PagedArgs& c, long long n) { return dim3((unsigned)((n + kReadTokens - 1) / kReadTokens), (unsigned)c.heads, (unsigned)c.n_seqs); }

template <class T, int BITS>
cudaError_t read_codes(const PagedArgs& c, void* k, void* v, const int32_t* first, long long n, int group, cudaStream_t st) {
  int shift = 0;
  while ((1 << shift) < group) ++shift;
  count_launches(1);
  return launch_dependent(paged_read_codes_kernel<T, BITS>, read_grid(c, n), kReadThreads, 0, st, c, (unsigned char*)k, (unsigned char*)v, first,
                          n, shift);
}
template <class T>
cudaError_t read_bits(const PagedArgs& c, int bits, void* k, void* v, const int32_t* first, long long n, int group, cudaStream_t st) {
  if (bits == 8) return read_codes<T, 8>(c, k, v, first, n, group, st);
  if (bits == 4) return read_codes<T, 4>(c, k, v, first, n, group, st);
  count_launches(1);
  return launch_dependent(paged_read_kernel, read_grid(c, n), kReadThreads, 0, st, c, (unsigned char*)k, (unsigned char*)v, first, n);
}

// ------------------------------------------------------------------ argument checks
static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Everything about the cache that the host can see
static gear_status check_cache(const gear_paged_cache* c, PagedArgs* a) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table || !c->lengths) return GEAR_ERR_ARG;
  if (c->dtype != GEAR_F16 && c->dtype != GEAR_BF16) return GEAR_ERR_ARG;
  if (c->bits != 16 && c->bits != 8 && c->bits != 4) return GEAR_ERR_ARG;
  if (c->n_pages < 1 || c->n_seqs < 1 || c->n_seqs > 65535 || c->table_stride < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024)
    return GEAR_ERR_ARG;
  if (c->page_bytes < 0 || c->param_bytes < 0) return GEAR_ERR_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return GEAR_ERR_SHAPE;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return GEAR_ERR_SHAPE;
  if ((long long)c->table_stride * c->page_size >= 1LL << 30) return GEAR_ERR_SHAPE;      // a block past the last token still has 32-bit numbers
  if (c->bits == 16 ? c->group != 0 : (c->group != 32 && c->group != 64 && c->group != 128) || c->group > c->head_dim)
    return GEAR_ERR_SHAPE;
  if (c->bits != 16 && (!c->k_params || !c->v_params)) return GEAR_ERR_ARG;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return GEAR_ERR_ALIGN;
  if (c->bits != 16 && (!aligned16(c->k_params) || !aligned16(c->v_params))) return GEAR_ERR_ALIGN;
  if (((uintptr_t)c->page_table | (uintptr_t)c->lengths) & 3) return GEAR_ERR_ALIGN;
  a->row_bytes = c->head_dim * c->bits / 8;
  a->param_row_bytes = c->bits == 16 ? 0 : c->head_dim / c->group * 4;
  const long long page = (long long)c->n_kv_heads * c->page_size * a->row_bytes;
  const long long param = (long long)c->n_kv_heads * c->page_size * a->param_row_bytes;
  a->page_bytes = c->page_bytes ? c->page_bytes : page;
  a->param_bytes = c->param_bytes ? c->param_bytes : param;
  if (a->page_bytes < page || a->param_bytes < param || a->page_bytes >= 1LL << 40) return GEAR_ERR_SHAPE;
  if (a->page_bytes % 16 || a->param_bytes % 16) return GEAR_ERR_ALIGN;
  a->pages[0] = (unsigned char*)c->k_pages; a->pages[1] = (unsigned char*)c->v_pages;
  a->params[0] = (unsigned char*)c->k_params; a->params[1] = (unsigned char*)c->v_params;
  a->table = c->page_table; a->lengths = c->lengths; a->row_start = nullptr;
  a->n_pages = c->n_pages; a->page_size = c->page_size; a->n_seqs = c->n_seqs; a->table_stride = c->table_stride;
  a->page_shift = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  a->heads = c->n_kv_heads; a->head_dim = c->head_dim; a->n_rows = 0;
  return GEAR_OK;
}

static gear_status check_scratch(PagedArgs* a, void* scratch, size_t bytes, size_t least) {
  if (!scratch) return GEAR_ERR_ARG;
  if (!aligned16(scratch)) return GEAR_ERR_ALIGN;
  if (bytes < least) return GEAR_ERR_CAPACITY;
  a->status = (int*)scratch;
  return GEAR_OK;
}

static gear_status check_rows(PagedArgs* a, const int32_t* row_start, int64_t n_rows) {
  if (!row_start || n_rows < 0 || n_rows > 0x3fffffffLL) return GEAR_ERR_ARG;
  if ((uintptr_t)row_start & 3) return GEAR_ERR_ALIGN;
  a->row_start = row_start;
  a->n_rows = (int)n_rows;
  return GEAR_OK;
}

// Elements from a row to the next -> bytes
static gear_status check_stride(int64_t stride, int64_t width, long long* bytes) {
  if (stride == 0) stride = width;
  if (stride < width || stride > (1LL << 38)) return GEAR_ERR_SHAPE;
  if (stride % 8) return GEAR_ERR_ALIGN;
  *bytes = stride * 2;
  return GEAR_OK;
}

static std::atomic<int> test_dead_wait{0};

static gear_status launched(cudaError_t e) {
  if (e == cudaSuccess) return GEAR_OK;
  cudaGetLastError();
  return GEAR_ERR_CUDA;
}

}  // namespace gear

using namespace gear;

extern "C" gear_status gear_paged_scratch_init(void* scratch, size_t scratch_bytes, void* stream) {
  if (!scratch) return GEAR_ERR_ARG;
  if ((uintptr_t)scratch & 15) return GEAR_ERR_ALIGN;
  if (scratch_bytes < GEAR_PAGED_SCRATCH_MIN) return GEAR_ERR_CAPACITY;
  return launched(cudaMemsetAsync(scratch, 0, scratch_bytes, (cudaStream_t)stream));
}

extern "C" gear_status gear_paged_status(void* scratch, int32_t* code) { return gear_fp16_attn_status(scratch, code); }

extern "C" gear_status gear_paged_append(const gear_paged_cache* cache, const void* k_new, const void* v_new, int64_t k_stride,
                                         int64_t v_stride, const int32_t* row_start, int64_t n_rows, void* scratch,
                                         size_t scratch_bytes, void* stream) {
  PagedArgs a = {};
  long long ks = 0, vs = 0;
  gear_status e = check_cache(cache, &a);
  if (e == GEAR_OK) e = check_rows(&a, row_start, n_rows);
  if (e == GEAR_OK) e = check_scratch(&a, scratch, scratch_bytes, GEAR_PAGED_SCRATCH_MIN);
  if (e == GEAR_OK) e = check_stride(k_stride, (int64_t)a.heads * a.head_dim, &ks);
  if (e == GEAR_OK) e = check_stride(v_stride, (int64_t)a.heads * a.head_dim, &vs);
  if (e != GEAR_OK) return e;
  if (n_rows == 0) return GEAR_OK;
  if (!k_new || !v_new) return GEAR_ERR_ARG;
  if (!aligned16(k_new) || !aligned16(v_new)) return GEAR_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  return launched(cache->dtype == GEAR_F16 ? append_bits<__half>(a, cache->bits, k_new, v_new, ks, vs, cache->group, st)
                                           : append_bits<__nv_bfloat16>(a, cache->bits, k_new, v_new, ks, vs, cache->group, st));
}

extern "C" gear_status gear_paged_read(const gear_paged_cache* cache, void* K, void* V, const int32_t* first, int64_t n, void* scratch,
                                       size_t scratch_bytes, void* stream) {
  PagedArgs a = {};
  gear_status e = check_cache(cache, &a);
  if (e == GEAR_OK) e = check_scratch(&a, scratch, scratch_bytes, GEAR_PAGED_SCRATCH_MIN);
  if (e != GEAR_OK) return e;
  if (n < 0 || n > 0x7fffffffLL || (!K && !V)) return GEAR_ERR_ARG;
  if (!aligned16(K) || !aligned16(V) || ((uintptr_t)first & 3)) return GEAR_ERR_ALIGN;
  if (n == 0) return GEAR_OK;
  cudaStream_t st = (cudaStream_t)stream;
  return launched(cache->dtype == GEAR_F16 ? read_bits<__half>(a, cache->bits, K, V, first, n, cache->group, st)
                                           : read_bits<__nv_bfloat16>(a, cache->bits, K, V, first, n, cache->group, st));
}

extern "C" gear_status gear_paged_test_dead_wait(int32_t which) {
  if (which < 0 || which > 6) return GEAR_ERR_ARG;
  test_dead_wait.store(which, std::memory_order_relaxed);
  return GEAR_OK;
}

extern "C" size_t gear_paged_scratch_bytes(const gear_paged_cache* cache, int64_t n_rows, int32_t n_q_heads) {
  if (!cache || cache->n_seqs < 1 || cache->n_kv_heads < 1 || n_rows < 0 || n_q_heads < 1) return GEAR_PAGED_SCRATCH_MIN;
  return paged_attn_scratch(n_rows, (n_q_heads + cache->n_kv_heads - 1) / cache->n_kv_heads, cache->n_seqs);
}

extern "C" gear_status gear_paged_attn(const gear_paged_cache* cache, const void* q, int64_t q_stride, void* out, float* lse,
                                       const int32_t* row_start, int64_t n_rows, int64_t max_rows, int32_t n_q_heads, int32_t causal,
                                       int32_t window, float softmax_scale, void* scratch, size_t scratch_bytes, void* stream) {
  PagedAttnArgs a = {};
  gear_status e = check_cache(cache, &a.c);
  if (e == GEAR_OK) e = check_rows(&a.c, row_start, n_rows);
  if (e != GEAR_OK) return e;
  if (n_q_heads < 1 || window < 0 || max_rows < 0 || !isfinite(softmax_scale)) return GEAR_ERR_ARG;
  if (n_q_heads % a.c.heads || n_q_heads / a.c.heads > 128) return GEAR_ERR_SHAPE;
  e = check_stride(q_stride, (int64_t)n_q_heads * a.c.head_dim, &a.q_stride);
  if (e == GEAR_OK) e = check_scratch(&a.c, scratch, scratch_bytes, gear_paged_scratch_bytes(cache, n_rows, n_q_heads));
  if (e != GEAR_OK) return e;
  if (n_rows == 0) return GEAR_OK;
  if (!q || !out || max_rows < 1) return GEAR_ERR_ARG;
  if (!aligned16(q) || !aligned16(out) || ((uintptr_t)lse & 3)) return GEAR_ERR_ALIGN;
  const float sc = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)a.c.head_dim);
  a.q = (const unsigned char*)q; a.out = (unsigned char*)out; a.lse = lse;
  a.share = n_q_heads / a.c.heads;
  a.max_rows = (int)std::min<int64_t>(max_rows, n_rows);
  a.causal = causal != 0; a.window = window;
  a.scale_log2 = sc * 1.4426950408889634f;
  a.test_dead_wait = test_dead_wait.load(std::memory_order_relaxed);
  a.wait_limit = a.test_dead_wait ? kTestSpinLimit : kDecodeSpinLimit;
  return launched(launch_paged_attn(a, cache->bits, cache->dtype, cache->group, scratch, (cudaStream_t)stream));
}

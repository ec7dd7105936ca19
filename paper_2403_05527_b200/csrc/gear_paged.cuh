// The paged cache on the device: arguments, where a token lies, types.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/gear.h"
#include "gear_internal.cuh"
#include "gear_paged_index.h"

namespace gear {

struct PagedArgs {
  unsigned char* pages[2];      // keys, values
  unsigned char* params[2];
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* row_start;
  long long page_bytes, param_bytes;
  int n_pages, page_size, page_shift, n_seqs, table_stride, heads, head_dim, row_bytes, param_row_bytes;
  int n_rows;
  int* status;
};

struct PagedAttnArgs {
  PagedArgs c;
  const unsigned char* q;
  unsigned char* out;
  float* lse;
  long long q_stride;           // bytes from a row to the next
  int share;                    // query heads per kv head
  int max_rows, causal, window;
  float scale_log2;             // softmax scale * log2(e)
  float* partial;
  int* tickets;                 // few rows: by the first CTA of a unit of work that several share, how many of them are done
  int* unit_first;              // many rows: [n_seqs + 1] number of the first unit of a sequence
  long long* unit_sums;         // [units + 1] blocks of all units before it, of one head
  int unit_cap, tile_ctas;
  int tile_new;                 // new rows of a tile: 128 / share
  void* shared_units;           // [tile_ctas] TileShared
  int wait_limit;               // polls before a wait of the kernel of many rows gives up
  int test_dead_wait;           // test only: who waits on a barrier that nothing completes (gear_paged_test_dead_wait)
};

// What a kernel needs to be told once per device before it is launched there: the shared memory it takes beyond the default.  Calls from
// several threads may tell it twice.
class KernelReady {
 public:
  template <class K> cudaError_t on_this_device(K* kernel, int smem, int* sms) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev < kDevices;
    if (known && (*sms = sms_[dev].load(std::memory_order_acquire)) > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess && smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && known) sms_[dev].store(*sms, std::memory_order_release);
    return e;
  }

 private:
  static constexpr int kDevices = 64;
  std::atomic<int> sms_[kDevices] = {};                      // multiprocessors; 0: not told yet
};

// Pools of a side that is not known when compiling (indexed by it, the whole argument would be copied to memory of the thread)
__device__ __forceinline__ unsigned char* pages_of(const PagedArgs& c, int side) { return side == 0 ? c.pages[0] : c.pages[1]; }
__device__ __forceinline__ unsigned char* params_of(const PagedArgs& c, int side) { return side == 0 ? c.params[0] : c.params[1]; }

constexpr int kTestSpinLimit = 64;             // polls, of 20 us at most, of a wait under gear_paged_test_dead_wait
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ void paged_bad(const PagedArgs& c) { atomicExch(c.status, GEAR_ERR_STATE); }

// What the kernel in front may have written while this one was already resident (tables, pages, parameters) is read by coherent loads or bulk copies.

// Page of token t of sequence s, or -1 (recorded) where the table names none.  t lies below the sequence's clamped length.
__device__ __forceinline__ int page_of(const PagedArgs& c, int s, int t) {
  const int page = c.table[(size_t)s * c.table_stride + (t >> c.page_shift)];
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  paged_bad(c);
  return -1;
}
__device__ __forceinline__ size_t token_row(const PagedArgs& c, int head, int t) {
  return (size_t)head * c.page_size + (t & (c.page_size - 1));
}

// ------------------------------------------------------------------ types
template <class T> struct Two;
template <> struct Two<__half> {
  using type = __half2;
  static __device__ __forceinline__ float2 wide(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float round(float a) { return __half2float(__float2half_rn(a)); }
  static __device__ __forceinline__ uint32_t min(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
};
template <> struct Two<__nv_bfloat16> {
  using type = __nv_bfloat162;
  static __device__ __forceinline__ float2 wide(uint32_t x) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float round(float a) { return __bfloat162float(__float2bfloat16_rn(a)); }
  static __device__ __forceinline__ uint32_t min(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
};

constexpr int kRowsMost = 16;                  // query rows per sequence and kv head that the kernel of few rows takes
size_t paged_attn_scratch(long long n_rows, int share, int n_seqs);
cudaError_t launch_paged_rows_b16(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st);
cudaError_t launch_paged_rows_b8(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st);
cudaError_t launch_paged_rows_b4(const PagedAttnArgs& a, int dtype, int group, cudaStream_t st);
cudaError_t launch_paged_attn(const PagedAttnArgs& a, int bits, int dtype, int group, void* scratch, cudaStream_t st);

}  // namespace gear

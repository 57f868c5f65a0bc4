// Declarations shared by the paged cache's host code (kvp_paged.cu) and its attention kernel (kvp_paged_attn.cu).
#pragma once

#include <string>
#include <vector>

#include "kvp_internal.h"

// Quotient of a number n below 2^31 by a fixed divisor d, as a product and a shift: with l = ceil(log2 d) and
// M = floor(2^(31+l) / d) + 1, M exceeds 2^(31+l) / d by at most 1, so n M / 2^(31+l) exceeds n / d by less than 2^-l <= 1 / d:
// too little to reach the next whole number.
struct kvp_divisor {
    uint32_t mul;
    int32_t shift;
};

// One layer of the store, or all of it (layer 0), as kernels see it; strides in bytes.
struct kvp_store {
    char *k, *v;
    int64_t page_stride, head_stride, row_stride;
    int32_t page_size, n_pages;
    kvp_divisor by_page;
};

// Key tiles of `rows` rows, 0 to 2^31 - 1 of them (rounded up in 32 bits: the sum may pass 2^31).
#ifdef __CUDACC__
__host__ __device__
#endif
constexpr int32_t kvp_tiles(int32_t rows, int32_t keys) { return (int32_t)(((uint32_t)rows + (uint32_t)keys - 1) / (uint32_t)keys); }

#ifdef __CUDACC__
__device__ __forceinline__ int32_t divide(int32_t n, kvp_divisor d) { return (int32_t)(((uint64_t)(uint32_t)n * d.mul) >> d.shift); }

// Two fp32 numbers in a register pair, and the packed arithmetic on them.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi)
{
    f32x2 x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(lo), "f"(hi));
    return x;
}
__device__ __forceinline__ void unpack2(f32x2 x, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 x;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
    return x;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 x;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(a), "l"(b), "l"(c));
    return x;
}
#endif

// Partial results of units whose rows several CTAs share, and a count of the parts that are in per unit.
struct kvp_paged_ws {
    float *part_o;             // [2 * CTAs][16][head_dim]
    float2 *part_ml;           // [2 * CTAs][16]
    int32_t *arrived;          // [units], zero between launches
    int32_t *arrived_group;    // [2 * CTAs], by a group's first part; likewise
};

struct kvp_paged_args {
    kvp_store st;              // the layer's
    uint32_t page_units, head_units, row_units;    // its strides in units of 2^unit_shift bytes, which divide all of them
    int32_t unit_shift;
    const char *q;
    char *out;
    int64_t q_stride[2], out_stride[2];    // {request, head}, bytes
    const int32_t *table, *lens, *first;
    int64_t table_stride;
    int32_t room;              // rows that a line of the table holds, INT32_MAX at most
    int32_t batch, n_kv, group;
    float *lse;
    float scale;
    kvp_paged_ws ws;
};

// Most and fewest query rows of a full unit (bf16, fp32); a group of more heads is several units.
#define KVP_PAGED_ROWS 16
#define KVP_PAGED_LEAST_ROWS 8
int32_t kvp_paged_ctas(int32_t sm_count);
// whether key tiles of a call (of 8 keys at least) can be counted in 31 bits, were all lists as long as `room`
bool kvp_paged_fits(int64_t batch, int64_t n_kv, int64_t group, int64_t room);
cudaError_t kvp_paged_attn_prepare(int32_t dtype, int32_t head_dim);
cudaError_t kvp_launch_paged_attn(const kvp_paged_args &a, int32_t dtype, int32_t head_dim, int32_t sm_count, cudaStream_t st);

struct kvp_cache {
    kvp_cache_config cfg;
    int32_t elem_bytes, sm_count = 148, unit_shift = 0;
    float scale;
    kvp_divisor by_page;
    kvp_paged_ws ws = {};
    std::vector<int32_t> holders;          // per page
    std::vector<int32_t> free_pages;       // a stack: the lowest page on top at the start
    std::vector<int32_t> scratch;          // per page, zero between calls
    std::string err;
};

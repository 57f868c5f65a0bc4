// A cache in pages: host entry points, the kernel that norms, rotates and appends new tokens, and the kernels that copy
// and compact pages.  The attention kernel is in kvp_paged_attn.cu.
#include <cuda_bf16.h>

#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <new>

#include "kvp_paged.h"

namespace {

// A 16-byte word of elements as pairs of fp32 numbers, and back (rounded to nearest).
template <typename T> struct elem;
template <> struct elem<float> {
    static constexpr int kPerVec = 4;
    __device__ static void get(uint4 u, f32x2 (&x)[2])
    {
        x[0] = (f32x2)u.y << 32 | u.x;
        x[1] = (f32x2)u.w << 32 | u.z;
    }
    __device__ static uint4 put(const f32x2 (&x)[2]) { return make_uint4((uint32_t)x[0], (uint32_t)(x[0] >> 32), (uint32_t)x[1], (uint32_t)(x[1] >> 32)); }
    __device__ static float one(float x) { return x; }
};
template <> struct elem<__nv_bfloat16> {
    static constexpr int kPerVec = 8;
    __device__ static f32x2 wide(uint32_t w) { return (f32x2)(w & 0xffff0000u) << 32 | (w << 16); }
    __device__ static uint32_t narrow(f32x2 x)
    {
        float lo, hi;
        unpack2(x, lo, hi);
        uint32_t w;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
        return w;
    }
    __device__ static void get(uint4 u, f32x2 (&x)[4])
    {
        x[0] = wide(u.x); x[1] = wide(u.y); x[2] = wide(u.z); x[3] = wide(u.w);
    }
    __device__ static uint4 put(const f32x2 (&x)[4]) { return make_uint4(narrow(x[0]), narrow(x[1]), narrow(x[2]), narrow(x[3])); }
    __device__ static float one(__nv_bfloat16 x) { return __bfloat162float(x); }
};

// ---- norms, rotation, append ----------------------------------------------------------------------------------

struct rows_at {
    const char *p;
    int64_t stride[2];             // {token, head}, bytes
};
struct append_args {
    rows_at q, k, v, q_out, k_out;
    const int32_t *positions, *slots;
    const char *q_weight, *k_weight;
    kvp_store st;                  // st.k null: no pages
    int32_t n_tokens, n_q, n_k, n_v;   // heads of each that there is something to do for
    int32_t rotary, pairing;
    int32_t half_q, half_kv;       // q heads of a half of a token, and its k and v heads
    float eps, magnitude;
    double turns[64];              // f_i / 2 pi
};

// A row is one head of one token.  A thread takes two 16-byte words of it that are each other's rotation partners (half layout),
// so that neither layout needs an exchange between threads and a sum of squares takes log2(words / 2) shuffles.  A warp takes
// a token, or a part of its heads: the token's angles are formed once, and the sines, cosines and weights that a thread needs
// stay in its registers for all heads (read from shared memory for each head they took twice the wavefronts of the rows
// themselves).  The angle is formed in double precision, as a part of a turn, and its sine and cosine from the rounded
// remainder: |remainder| <= 1/2 turn, so that rounding moves the angle by 2^-26 turns at most, wherever the position lies (rows of
// fp32 4.3e-8 off in the 2-norm, 3.9e-8 with sines and cosines rounded from 64 bits).  The product in front of it is exact to
// 2^-53 of itself: less than that up to positions of 2^28, 2^-24 turns at 2^31.
template <typename T, int D> struct row_math {
    static constexpr int EV = elem<T>::kPerVec, P = EV / 2, L = D / EV / 2, R = 32 / L;   // elements and pairs of a word, threads of a row, rows of a warp
    int w0, w1;                            // the words
    bool turns;
    f32x2 c[P], s[P];                      // of this thread's pairs: the half layout's P pairs, or P / 2 of each word
    f32x2 gx[P], gy[P];                    // weights

    __device__ row_math(int rotary)
    {
        const int j = threadIdx.x % L, half = rotary / EV / 2;             // half: words of one half of the rotated part
        turns = j < half;
        w0 = turns ? j : half + j;
        w1 = w0 + (turns ? half : L - half);
    }
    __device__ void weigh(const char *weight)
    {
        elem<T>::get(reinterpret_cast<const uint4 *>(weight)[w0], gx);
        elem<T>::get(reinterpret_cast<const uint4 *>(weight)[w1], gy);
    }
    // norms: whether any row of the warp is normed (the same for all its threads)
    __device__ void row(uint4 &x, uint4 &y, bool norms, bool norm, bool rotate, float eps, int pairing) const
    {
        f32x2 fx[P], fy[P];
        elem<T>::get(x, fx);
        elem<T>::get(y, fy);
        float inv = 1.0f;
        if (norms) {
            f32x2 sum = 0;
#pragma unroll
            for (int e = 0; e < P; ++e) sum = fma2(fy[e], fy[e], fma2(fx[e], fx[e], sum));
            float ss, hi;
            unpack2(sum, ss, hi);
            ss += hi;
#pragma unroll
            for (int o = L / 2; o > 0; o /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            inv = rsqrtf(ss * (1.0f / D) + eps);
        }
        if (norm) {
            const f32x2 inv2 = pack2(inv, inv);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                fx[e] = mul2(mul2(fx[e], gx[e]), inv2);
                fy[e] = mul2(mul2(fy[e], gy[e]), inv2);
            }
        }
        if (turns && rotate) {
            if (pairing == 0) {
                const f32x2 minus = pack2(-1.0f, -1.0f);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const f32x2 p = fx[e], q = fy[e];
                    fx[e] = fma2(p, c[e], mul2(mul2(q, s[e]), minus));
                    fy[e] = fma2(q, c[e], mul2(p, s[e]));
                }
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    float c0, c1, s0, s1, p, q;
                    unpack2(c[e], c0, c1);
                    unpack2(s[e], s0, s1);
                    unpack2(fx[e], p, q);
                    fx[e] = pack2(p * c0 - q * s0, p * s0 + q * c0);
                    unpack2(fy[e], p, q);
                    fy[e] = pack2(p * c1 - q * s1, p * s1 + q * c1);
                }
            }
        }
        x = elem<T>::put(fx);
        y = elem<T>::put(fy);
    }
};

__device__ __forceinline__ uint4 *words_at(const rows_at &r, int token, int head)
{
    return reinterpret_cast<uint4 *>(const_cast<char *>(r.p) + token * r.stride[0] + head * r.stride[1]);
}

// A token's row in the pages.
struct page_row {
    char *k, *v;                   // null: nowhere
    __device__ page_row(const append_args &a, int32_t slot) : k(nullptr), v(nullptr)
    {
        if (slot < 0 || slot >= a.st.n_pages * a.st.page_size) return;
        const int32_t page = divide(slot, a.st.by_page), row = slot - page * a.st.page_size;
        const int64_t at = page * a.st.page_stride + row * a.st.row_stride;
        k = a.st.k + at;
        v = a.st.v + at;
    }
};

// The pairs of a thread, from a table of (cosine, sine): half layout, elements 2e and 2e + 1 of both words; the other, pair e of
// the first and of the second word.
template <typename T, int D>
__device__ __forceinline__ void take_angles(row_math<T, D> &m, const float2 *table, int pairing)
{
    constexpr int P = row_math<T, D>::P;
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const int i0 = !m.turns ? 0 : pairing == 0 ? m.w0 * 2 * P + 2 * e : m.w0 * P + e, i1 = !m.turns ? 0 : pairing == 0 ? i0 + 1 : m.w1 * P + e;
        const float2 t0 = table[i0], t1 = table[i1];
        m.c[e] = pack2(t0.x, t1.x);
        m.s[e] = pack2(t0.y, t1.y);
    }
}

__device__ __forceinline__ float2 angle_of(int position, double turns, float magnitude)
{
    const double turn = (double)position * turns;
    float sine, cosine;
    sincospif(2.0f * (float)(turn - rint(turn)), &sine, &cosine);
    return make_float2(magnitude * cosine, magnitude * sine);
}

// Many tokens: bound by DRAM (33,280 tokens of 32/8 heads of 128 with norms: 130 us, 6.3 TB/s read and written; a copy reaches
// 6.5).  A thread has four rows under way; warps take tokens in turn, so that the frequencies are fetched once (a token per
// warp and launch: 141 us), and the next token's position and slot are fetched a token ahead (137 without).  HALVES: a warp
// has half of one token's heads - where warps are left over (1,000 tokens: 8.9 us whole, 6.1 in halves; 2,048: 10.9, 14.7).
template <typename T, int D, bool HALVES>
__global__ void __launch_bounds__(256, 2)
append_many_kernel(const __grid_constant__ append_args a)
{
    typedef row_math<T, D> math;
    constexpr int R = math::R, U = 4;
    __shared__ float2 turned_by[8][D / 2];                 // (cosine, sine)
    pdl_launch_dependents();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, mine = lane / math::L;
    math m(a.rotary);
    double f[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) f[i] = lane + 32 * i < a.rotary / 2 ? a.turns[lane + 32 * i] : 0.0;
    pdl_wait();
    const int first = blockIdx.x * 8 + warp, part = HALVES ? first & 1 : 0;
    int token = HALVES ? first / 2 : first;
    if (token >= a.n_tokens) return;
    int position = a.rotary ? a.positions[token] : 0, slot = a.st.k ? a.slots[token] : -1;
    while (true) {
        const int next = token + gridDim.x * 8, next_position = next < a.n_tokens && a.rotary ? a.positions[next] : 0;
        const int next_slot = next < a.n_tokens && a.st.k ? a.slots[next] : -1;
        uint4 x[U], y[U];
        auto fetch = [&](const rows_at &r, int u, int head, int end) {
            if (head >= end) return;
            const uint4 *p = words_at(r, token, head);
            x[u] = p[m.w0];
            y[u] = p[m.w1];
        };
        auto store = [&](uint4 *p, int u) {
            p[m.w0] = x[u];
            p[m.w1] = y[u];
        };
        const int q0 = HALVES ? part * a.half_q : 0, q1 = HALVES ? min(q0 + a.half_q, a.n_q) : a.n_q;
        const int kv0 = HALVES ? part * a.half_kv : 0, k1 = HALVES ? min(kv0 + a.half_kv, a.n_k) : a.n_k, v1 = HALVES ? min(kv0 + a.half_kv, a.n_v) : a.n_v;
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(a.q, u, q0 + u * R + mine, q1);
        if (a.rotary) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < D / 64; ++i) turned_by[warp][lane + 32 * i] = angle_of(position, f[i], a.magnitude);
            __syncwarp();
            take_angles<T, D>(m, turned_by[warp], a.pairing);
        }
        if (a.q_weight) m.weigh(a.q_weight);
        for (int h0 = q0; h0 < q1; h0 += U * R) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int head = h0 + u * R + mine;
                if (head - mine >= q1) break;
                m.row(x[u], y[u], a.q_weight, a.q_weight, true, a.eps, a.pairing);
                if (head < q1) store(words_at(a.q_out, token, head), u);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) fetch(a.q, u, h0 + (U + u) * R + mine, q1);
        }
        if (a.k_weight) m.weigh(a.k_weight);
        const page_row to(a, slot);
        for (int h0 = kv0; h0 < max(k1, v1); h0 += U / 2 * R) {
#pragma unroll
            for (int u = 0; u < U / 2; ++u) {
                fetch(a.k, u, h0 + u * R + mine, k1);
                fetch(a.v, U / 2 + u, h0 + u * R + mine, v1);
            }
#pragma unroll
            for (int u = 0; u < U / 2; ++u) {
                const int head = h0 + u * R + mine;
                if (head - mine < k1) m.row(x[u], y[u], a.k_weight, a.k_weight, true, a.eps, a.pairing);
                if (head < k1 && a.k_out.p) store(words_at(a.k_out, token, head), u);
                if (head < k1 && to.k) store(reinterpret_cast<uint4 *>(to.k + head * a.st.head_stride), u);
                if (head < v1 && to.v) store(reinterpret_cast<uint4 *>(to.v + head * a.st.head_stride), U / 2 + u);
            }
        }
        if (HALVES || next >= a.n_tokens) return;
        token = next;
        position = next_position;
        slot = next_slot;
    }
}

// Few tokens: latency.  A block has as many rows of one token (q heads, then k, then v) as it has threads for, and forms the
// angles while they are fetched.
template <typename T, int D>
__global__ void __launch_bounds__(256, 4)
append_few_kernel(const __grid_constant__ append_args a)
{
    typedef row_math<T, D> math;
    __shared__ float2 turned_by[D / 2];
    pdl_launch_dependents();
    math m(a.rotary);
    const int token = blockIdx.x, n_qk = a.n_q + a.n_k, r = blockIdx.y * (256 / math::L) + threadIdx.x / math::L;
    const int kind = r < a.n_q ? 0 : r < n_qk ? 1 : r < n_qk + a.n_v ? 2 : 3, head = kind == 0 ? r : kind == 1 ? r - a.n_q : r - n_qk;   // q, k, v, nothing
    const double f = (int)threadIdx.x < a.rotary / 2 ? a.turns[threadIdx.x] : 0.0;
    pdl_wait();
    uint4 x = make_uint4(0, 0, 0, 0), y = x;
    if (kind < 3) {
        const uint4 *p = words_at(kind == 0 ? a.q : kind == 1 ? a.k : a.v, token, head);
        x = p[m.w0];
        y = p[m.w1];
    }
    const bool norm = (kind == 0 && a.q_weight) || (kind == 1 && a.k_weight);
    if (norm) m.weigh(kind == 0 ? a.q_weight : a.k_weight);
    if ((int)threadIdx.x < a.rotary / 2) turned_by[threadIdx.x] = angle_of(a.positions[token], f, a.magnitude);
    __syncthreads();
    if (a.rotary) take_angles<T, D>(m, turned_by, a.pairing);
    if (__any_sync(0xffffffffu, kind < 2)) {
        uint4 x1 = x, y1 = y;
        m.row(x1, y1, a.q_weight || a.k_weight, norm, a.rotary > 0, a.eps, a.pairing);
        if (kind < 2) {
            x = x1;
            y = y1;
        }
    }
    auto store = [&](uint4 *p) {
        p[m.w0] = x;
        p[m.w1] = y;
    };
    if (kind == 0) store(words_at(a.q_out, token, head));
    if (kind == 1 && a.k_out.p) store(words_at(a.k_out, token, head));
    if (kind == 1 || kind == 2) {
        const page_row to(a, a.st.k ? a.slots[token] : -1);
        if (to.k) store(reinterpret_cast<uint4 *>((kind == 1 ? to.k : to.v) + head * a.st.head_stride));
    }
}

kvp_divisor divisor(int32_t d)
{
    int l = 0;
    while ((1ll << l) < d) ++l;
    return {(uint32_t)((1ull << (31 + l)) / (uint64_t)d + 1), 31 + l};
}

template <typename T, int D>
cudaError_t launch_append(append_args &a, int sm_count, cudaStream_t st)
{
    // 512 tokens of 32/8 heads: 7.1 us as many, 4.9 as few; 1,000 of 28/4: 6.1, 11.4 (fewer heads, whose tokens are less work,
    // were not measured at these borders).  Twice as many blocks as fit, so that the last
    // ones even out (one wave: 8,000 tokens of fp32 73 us instead of 65).
    if (a.n_tokens >= 4 * sm_count) {
        if (a.n_tokens <= 8 * sm_count) {
            const int at_once = row_math<T, D>::R, kv = std::max(a.n_k, a.n_v);
            a.half_q = (a.n_q + 2 * at_once - 1) / (2 * at_once) * at_once;
            a.half_kv = (kv + 2 * at_once - 1) / (2 * at_once) * at_once;
            return launch_pdl(append_many_kernel<T, D, true>, dim3((2 * a.n_tokens + 7) / 8), dim3(256), 0, st, a);
        }
        return launch_pdl(append_many_kernel<T, D, false>, dim3(std::min((a.n_tokens + 7) / 8, 4 * sm_count)), dim3(256), 0, st, a);
    }
    const int rows = a.n_q + a.n_k + a.n_v, at_once = 256 / row_math<T, D>::L;
    return launch_pdl(append_few_kernel<T, D>, dim3(a.n_tokens, (rows + at_once - 1) / at_once), dim3(256), 0, st, a);
}

cudaError_t launch_append(append_args &a, int32_t dtype, int32_t head_dim, int sm_count, cudaStream_t st)
{
    if (dtype == KVP_DTYPE_BF16)
        return head_dim == 128 ? launch_append<__nv_bfloat16, 128>(a, sm_count, st) : launch_append<__nv_bfloat16, 64>(a, sm_count, st);
    return head_dim == 128 ? launch_append<float, 128>(a, sm_count, st) : launch_append<float, 64>(a, sm_count, st);
}

// ---- copies of pages --------------------------------------------------------------------------------------------

struct page_pair { int32_t src, dst, rows; };
constexpr int kPairs = 1300;       // of one launch; they travel as parameters
struct copy_pairs { page_pair p[kPairs]; };
struct copy_pairs_small { page_pair p[300]; };

constexpr int kCopyVecs = 8;       // words in flight per thread

// Block (pair, layer and K or V, part of the page): words of the rows to be copied, in the order they lie in the store.  Bound by
// DRAM: 520 pages of 64 rows, 8 layers, 331 us = 6.6 TB/s read and written, 1,000 of 16 rows 157 us = 6.7.
template <typename P>
__global__ void __launch_bounds__(256)
copy_pages_kernel(const __grid_constant__ P pairs, kvp_store st, int64_t layer_stride, int n_kv, int words, int heads_inside)
{
    pdl_launch_dependents();
    const page_pair p = pairs.p[blockIdx.x];
    const int layer = blockIdx.y >> 1;
    char *base = ((blockIdx.y & 1) ? st.v : st.k) + layer * layer_stride;
    const char *src = base + p.src * st.page_stride;
    char *dst = base + p.dst * st.page_stride;
    const int inner = heads_inside ? n_kv : p.rows;
    const int64_t s_in = heads_inside ? st.head_stride : st.row_stride, s_out = heads_inside ? st.row_stride : st.head_stride;
    const int n = n_kv * p.rows * words;
    pdl_wait();
    for (int w0 = blockIdx.z * 256 * kCopyVecs + threadIdx.x; w0 < n; w0 += gridDim.z * 256 * kCopyVecs) {
        uint4 x[kCopyVecs];
        int64_t at[kCopyVecs];
#pragma unroll
        for (int u = 0; u < kCopyVecs; ++u) {
            const int w = w0 + 256 * u;
            if (w >= n) break;
            const int r = w / words, c = w % words;
            at[u] = (int64_t)(r / inner) * s_out + (int64_t)(r % inner) * s_in + c * 16;
            x[u] = *reinterpret_cast<const uint4 *>(src + at[u]);
        }
#pragma unroll
        for (int u = 0; u < kCopyVecs; ++u) {
            if (w0 + 256 * u >= n) break;
            *reinterpret_cast<uint4 *>(dst + at[u]) = x[u];
        }
    }
}

// ---- compaction -------------------------------------------------------------------------------------------------

struct compact_args {
    kvp_store st;
    int64_t layer_stride;
    const int32_t *table, *lens, *new_table, *kept, *n_kept;
    int64_t table_stride, new_stride, kept_stride[3];
    int32_t table_cols, new_cols, max_kept, n_kv;
};

constexpr int kCompactRows = 32, kCompactVecs = 4;         // rows of a block; words in flight per thread

// Block (kCompactRows new rows, layer and head, request): where each row comes from and goes to is looked up once, then the
// words of K and V are moved.  Bound by DRAM; the look-ups, three round trips, hide behind other blocks, so blocks are small and
// many: 4 x 8,000-10,560 rows to two fifths, 8 layers, 64 rows and 8 words a thread (4 blocks per SM) 168 us, 64 and 4 (8
// blocks) 163, 32 and 4 161 = 6.4 TB/s.
template <int WORDS>
__global__ void __launch_bounds__(256, 8)
compact_kernel(const __grid_constant__ compact_args a)
{
    __shared__ int64_t from[kCompactRows], to[kCompactRows];
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.z, layer = blockIdx.y / a.n_kv, h = blockIdx.y % a.n_kv, i0 = blockIdx.x * kCompactRows;
    const int end = min(a.n_kept[b], a.max_kept);
    if (end <= i0) return;                         // (before anything is subtracted: n_kept may be any number)
    const int n = min(end - i0, kCompactRows);
    if ((int)threadIdx.x < n) {
        const int i = i0 + threadIdx.x, new_page = divide(i, a.st.by_page);
        const int dst = new_page < a.new_cols ? a.new_table[b * a.new_stride + new_page] : -1;
        const int row = a.kept[b * a.kept_stride[0] + layer * a.kept_stride[1] + h * a.kept_stride[2] + i];
        const int64_t base = layer * a.layer_stride + h * a.st.head_stride;
        int64_t f = -1, t = -1;
        if (row >= 0 && row < a.lens[b]) {
            const int page = divide(row, a.st.by_page);
            const int src = page < a.table_cols ? a.table[b * a.table_stride + page] : -1;
            if (src >= 0 && src < a.st.n_pages && dst >= 0 && dst < a.st.n_pages) {
                f = base + src * a.st.page_stride + (row - page * a.st.page_size) * a.st.row_stride;
                t = base + dst * a.st.page_stride + (i - new_page * a.st.page_size) * a.st.row_stride;
            }
        }
        from[threadIdx.x] = f;
        to[threadIdx.x] = t;
    }
    __syncthreads();
    // K and V of a row in turn
    for (int w0 = threadIdx.x; w0 < 2 * WORDS * n; w0 += 256 * kCompactVecs) {
        uint4 x[kCompactVecs];
#pragma unroll
        for (int u = 0; u < kCompactVecs; ++u) {
            const int w = w0 + 256 * u, r = w / (2 * WORDS), c = w % (2 * WORDS);
            if (r < n && from[r] >= 0) x[u] = *reinterpret_cast<const uint4 *>((c < WORDS ? a.st.k : a.st.v) + from[r] + c % WORDS * 16);
        }
#pragma unroll
        for (int u = 0; u < kCompactVecs; ++u) {
            const int w = w0 + 256 * u, r = w / (2 * WORDS), c = w % (2 * WORDS);
            if (r < n && from[r] >= 0) *reinterpret_cast<uint4 *>((c < WORDS ? a.st.k : a.st.v) + to[r] + c % WORDS * 16) = x[u];
        }
    }
}

cudaError_t launch_compact(const compact_args &a, int words, int n_layers, int batch, cudaStream_t st)
{
    const dim3 grid((unsigned)(((int64_t)a.max_kept + kCompactRows - 1) / kCompactRows), (unsigned)(n_layers * a.n_kv), (unsigned)batch);
    return words == 8 ? launch_pdl(compact_kernel<8>, grid, dim3(256), 0, st, a)
         : words == 16 ? launch_pdl(compact_kernel<16>, grid, dim3(256), 0, st, a) : launch_pdl(compact_kernel<32>, grid, dim3(256), 0, st, a);
}

// ---- host side --------------------------------------------------------------------------------------------------

thread_local std::string g_error;

int32_t fail(kvp_cache *c, int32_t code, const char *fmt, ...) __attribute__((format(printf, 3, 4)));
int32_t fail(kvp_cache *c, int32_t code, const char *fmt, ...)
{
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        (c ? c->err : g_error) = buf;
    } catch (const std::bad_alloc &) {             // without a text then
    }
    return code;
}

int32_t cuda_failed(kvp_cache *c, const char *what, cudaError_t e)
{
    (void)cudaGetLastError();                      // reported here, not to whoever asks next
    return fail(c, KVP_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// The device of a call while it launches; the caller's current one afterwards.
struct on_device {
    int before = -1;
    cudaError_t rc;
    explicit on_device(int device)
    {
        rc = cudaGetDevice(&before);
        if (rc == cudaSuccess && before != device) rc = cudaSetDevice(device);
        else before = -1;
    }
    ~on_device() { if (before >= 0) (void)cudaSetDevice(before); }
};

bool odd16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// Whether rows of `width` elements, numbered by n indices of the given counts and strides, lie apart: from the smallest stride on, each
// step is as long as all that the ones before it reach.
struct index_of_rows { int64_t count, stride; };
bool rows_apart(index_of_rows *x, int n, int64_t width)
{
    std::sort(x, x + n, [](const index_of_rows &a, const index_of_rows &b) { return llabs(a.stride) < llabs(b.stride); });
    double span = (double)width;
    for (int i = 0; i < n; ++i) {
        if (x[i].count <= 1) continue;
        if ((double)llabs(x[i].stride) < span) return false;
        span += (double)llabs(x[i].stride) * (double)(x[i].count - 1);
    }
    return true;
}

int32_t unit_shift_of(const kvp_cache_config *c);
bool rows_fit(const kvp_cache_config *c);

bool valid_cache(const kvp_cache_config *c)
{
    if (!c || c->struct_bytes != (int32_t)sizeof(kvp_cache_config)) return false;
    if (c->n_layers <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_q_heads % c->n_kv_heads) return false;
    if (c->n_layers > 32767 || c->n_q_heads > 65535) return false;
    if ((int64_t)c->n_layers * c->n_kv_heads > 65535) return false;              // y dimension of the copy and compaction grids
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    if (c->dtype != KVP_DTYPE_F32 && c->dtype != KVP_DTYPE_BF16) return false;
    if (c->page_size <= 0 || c->n_pages <= 0 || (int64_t)c->page_size * c->n_pages > INT32_MAX) return false;
    if ((int64_t)c->page_size * c->n_kv_heads > (1 << 24)) return false;         // words of a page are counted in 32 bits
    if ((int64_t)c->max_batch * c->n_q_heads > INT32_MAX / 4) return false;
    if (c->max_batch <= 0 || c->max_batch > 65535 || !(c->softmax_scale >= 0.0) || !isfinite(c->softmax_scale)) return false;
    const int64_t unit = c->dtype == KVP_DTYPE_BF16 ? 8 : 4;
    const int64_t strides[4] = {c->layer_stride, c->page_stride, c->head_stride, c->row_stride};
    for (int64_t s : strides)
        if (s < 0 || s % unit || s > (1ll << 56)) return false;
    index_of_rows rows[4] = {{c->n_layers, c->layer_stride}, {c->n_pages, c->page_stride}, {c->n_kv_heads, c->head_stride}, {c->page_size, c->row_stride}};
    return rows_apart(rows, 4, c->head_dim) && rows_fit(c);
}

// The largest power of two that divides all strides within a layer, in bytes; with it every row of a layer has to have a
// number of 32 bits.
int32_t unit_shift_of(const kvp_cache_config *c)
{
    const int64_t e = c->dtype == KVP_DTYPE_BF16 ? 2 : 4;
    return __builtin_ctzll((uint64_t)((c->page_stride | c->head_stride | c->row_stride) * e) | (1ull << 40));
}
bool rows_fit(const kvp_cache_config *c)
{
    const double e = c->dtype == KVP_DTYPE_BF16 ? 2 : 4;
    const double bytes = e * ((double)c->page_stride * (c->n_pages - 1) + (double)c->head_stride * (c->n_kv_heads - 1) + (double)c->row_stride * (c->page_size - 1));
    return bytes / (double)(1ull << unit_shift_of(c)) < 4294967296.0;
}

struct cache_layout { uint64_t o, ml, arrived, arrived_group, counted, total; int32_t units; };
cache_layout layout_of(const kvp_cache_config *c, int32_t sm_count)
{
    cache_layout l;
    const int64_t group = c->n_q_heads / c->n_kv_heads, slots = 2ll * kvp_paged_ctas(sm_count);
    l.units = (int32_t)std::min<int64_t>(INT32_MAX, (int64_t)c->max_batch * c->n_kv_heads * ((group + KVP_PAGED_LEAST_ROWS - 1) / KVP_PAGED_LEAST_ROWS));
    l.arrived = 0;
    l.arrived_group = l.arrived + 4ull * l.units;
    l.counted = l.arrived_group + 4ull * slots;            // end of what is zero between launches
    l.ml = (l.counted + 255) / 256 * 256;
    l.o = l.ml + 8ull * slots * KVP_PAGED_ROWS;
    l.total = l.o + 4ull * slots * KVP_PAGED_ROWS * c->head_dim;
    return l;
}

constexpr int32_t kMostSms = 256;              // the workspace is sized for: its size is asked before the device is known

int32_t check_rope(kvp_cache *c, const kvp_rope *r, int32_t head_dim)
{
    if (!r) return KVP_OK;
    if (r->struct_bytes != (int32_t)sizeof(kvp_rope) || r->reserved != 0) return fail(c, KVP_ERR_INVALID, "rope: not a kvp_rope of this version");
    if (r->pairing != 0 && r->pairing != 1) return fail(c, KVP_ERR_INVALID, "rope: pairing %d", r->pairing);
    if (r->rotary_dim < 0 || r->rotary_dim > head_dim || r->rotary_dim % 16)
        return fail(c, KVP_ERR_INVALID, "rope: rotary_dim %d is not a multiple of 16 up to %d", r->rotary_dim, head_dim);
    if (!r->inv_freq && !(r->theta > 0.0 && isfinite(r->theta))) return fail(c, KVP_ERR_INVALID, "rope: theta");
    if (!(r->scale >= 1.0 && isfinite(r->scale)) || !(r->magnitude > 0.0 && isfinite(r->magnitude)))
        return fail(c, KVP_ERR_INVALID, "rope: scale has to be at least 1, magnitude above 0");
    if (!(r->original_positions >= 0.0 && isfinite(r->original_positions)) ||
        (r->original_positions > 0.0 && !(r->low_rotations >= 0.0 && r->high_rotations > r->low_rotations && isfinite(r->high_rotations))))
        return fail(c, KVP_ERR_INVALID, "rope: original_positions, low_rotations < high_rotations");
    for (int i = 0; r->inv_freq && i < r->rotary_dim / 2; ++i)
        if (!isfinite(r->inv_freq[i])) return fail(c, KVP_ERR_INVALID, "rope: inv_freq[%d] is not finite", i);
    return KVP_OK;
}

double frequency(const kvp_rope *r, int i)
{
    const double f = r->inv_freq ? r->inv_freq[i] : pow(r->theta, -2.0 * i / r->rotary_dim);
    if (r->original_positions <= 0.0) return f / r->scale;
    const double t = r->original_positions * fabs(f) / (2.0 * M_PI);
    const double w = std::min(1.0, std::max(0.0, (t - r->low_rotations) / (r->high_rotations - r->low_rotations)));
    return w * f + (1.0 - w) * f / r->scale;
}

// Checks `t` and fills in `a`; c null: kvp_norm_rope.
int32_t token_args(kvp_cache *c, const kvp_tokens *t, const kvp_rope *rope, int32_t dtype, int32_t head_dim, append_args &a)
{
    if (!t || t->struct_bytes != (int32_t)sizeof(kvp_tokens)) return fail(c, KVP_ERR_INVALID, "tokens: not a kvp_tokens of this version");
    if (t->n_tokens < 0 || t->n_tokens > (1 << 30)) return fail(c, KVP_ERR_INVALID, "tokens: n_tokens is negative or above 2^30");
    a.n_tokens = 0;
    if (t->n_tokens == 0) return KVP_OK;           // nothing to do, and arrays of nothing have no address
    if ((t->q != nullptr) != (t->q_out != nullptr)) return fail(c, KVP_ERR_INVALID, "tokens: q and q_out go together");
    if (t->n_q_heads < 0 || t->n_q_heads > 65535 || t->n_kv_heads < 0 || t->n_kv_heads > 65535 || (t->q && t->n_q_heads == 0) || (t->k && t->n_kv_heads == 0))
        return fail(c, KVP_ERR_INVALID, "tokens: number of heads");
    if (c) {
        if (!t->k || !t->v || !t->slots) return fail(c, KVP_ERR_INVALID, "append: k, v and slots are needed");
        if (t->n_kv_heads != c->cfg.n_kv_heads || (t->q && t->n_q_heads != c->cfg.n_q_heads))
            return fail(c, KVP_ERR_INVALID, "append: heads of the tokens are not those of the cache");
    } else {
        if (t->v || t->slots) return fail(c, KVP_ERR_INVALID, "norm_rope: v and slots are for kvp_cache_append");
        if ((t->k != nullptr) != (t->k_out != nullptr)) return fail(c, KVP_ERR_INVALID, "norm_rope: k and k_out go together");
    }
    if ((t->q_weight && !t->q) || (t->k_weight && !t->k)) return fail(c, KVP_ERR_INVALID, "tokens: a weight without its rows");
    if ((t->q_weight || t->k_weight) && !(t->eps >= 0.0 && isfinite(t->eps))) return fail(c, KVP_ERR_INVALID, "tokens: eps");
    const int32_t e = dtype == KVP_DTYPE_BF16 ? 2 : 4;
    const bool turned = rope && rope->rotary_dim > 0 && (t->q || t->k);
    if (turned && !t->positions) return fail(c, KVP_ERR_INVALID, "tokens: a rotation needs positions");
    if (((uintptr_t)t->positions | (uintptr_t)t->slots) & 3) return fail(c, KVP_ERR_INVALID, "tokens: positions and slots must be aligned");
    if (odd16(t->q_weight) || odd16(t->k_weight)) return fail(c, KVP_ERR_INVALID, "tokens: weights must be 16-byte aligned");
    const struct { const void *p; const int64_t *s; rows_at &to; int32_t heads; } x[5] = {
        {t->q, t->q_stride, a.q, t->n_q_heads}, {t->k, t->k_stride, a.k, t->n_kv_heads}, {t->v, t->v_stride, a.v, t->n_kv_heads},
        {t->q_out, t->q_out_stride, a.q_out, t->n_q_heads}, {t->k_out, t->k_out_stride, a.k_out, t->n_kv_heads}};
    for (int i = 0; i < 5; ++i) {
        x[i].to = {(const char *)x[i].p, {0, 0}};
        if (!x[i].p) continue;
        if (odd16(x[i].p)) return fail(c, KVP_ERR_INVALID, "tokens: pointers must be 16-byte aligned");
        for (int k = 0; k < 2; ++k) {
            if (x[i].s[k] < -(1ll << 56) || x[i].s[k] > (1ll << 56) || x[i].s[k] * e % 16)
                return fail(c, KVP_ERR_INVALID, "tokens: strides must be multiples of 16 bytes");
            x[i].to.stride[k] = x[i].s[k] * e;
        }
        // rows that are written must not lie over one another
        index_of_rows rows[2] = {{t->n_tokens, x[i].s[0]}, {x[i].heads, x[i].s[1]}};
        if (i >= 3 && !rows_apart(rows, 2, head_dim)) return fail(c, KVP_ERR_INVALID, "tokens: rows of an output overlap");
    }
    // in place only row for row
    if ((t->q && t->q_out == t->q && (t->q_stride[0] != t->q_out_stride[0] || t->q_stride[1] != t->q_out_stride[1])) ||
        (t->k && t->k_out == t->k && (t->k_stride[0] != t->k_out_stride[0] || t->k_stride[1] != t->k_out_stride[1])))
        return fail(c, KVP_ERR_INVALID, "tokens: in place with other strides");
    a.positions = t->positions;
    a.slots = t->slots;
    a.q_weight = (const char *)t->q_weight;
    a.k_weight = (const char *)t->k_weight;
    a.st = {};
    a.n_tokens = t->n_tokens;
    a.n_q = t->q ? t->n_q_heads : 0;
    a.n_k = t->k ? t->n_kv_heads : 0;
    a.n_v = t->v ? t->n_kv_heads : 0;
    a.rotary = turned ? rope->rotary_dim : 0;
    a.pairing = rope ? rope->pairing : 0;
    a.eps = (float)t->eps;
    a.magnitude = rope ? (float)rope->magnitude : 1.0f;
    for (int i = 0; i < a.rotary / 2; ++i) a.turns[i] = frequency(rope, i) / (2.0 * M_PI);
    return KVP_OK;
}

kvp_store store_of(const kvp_cache *c, int32_t layer)
{
    const int64_t e = c->elem_bytes;
    kvp_store s;
    s.k = (char *)c->cfg.k + layer * c->cfg.layer_stride * e;
    s.v = (char *)c->cfg.v + layer * c->cfg.layer_stride * e;
    s.page_stride = c->cfg.page_stride * e;
    s.head_stride = c->cfg.head_stride * e;
    s.row_stride = c->cfg.row_stride * e;
    s.page_size = c->cfg.page_size;
    s.n_pages = c->cfg.n_pages;
    s.by_page = c->by_page;
    return s;
}

int32_t check_runs(kvp_cache *c, int32_t layer)
{
    if (c->cfg.device < 0) return fail(c, KVP_ERR_STATE, "host-only cache");
    if (layer < 0 || layer >= c->cfg.n_layers) return fail(c, KVP_ERR_INVALID, "layer %d of %d", layer, c->cfg.n_layers);
    return KVP_OK;
}

cudaError_t sms_of(int device, int *n)
{
    return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, device);
}

// The launches of a copy whose arguments have been checked.
int32_t launch_copies(kvp_cache *c, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *rows, cudaStream_t st)
{
    on_device dev(c->cfg.device);
    if (dev.rc != cudaSuccess) return cuda_failed(c, "cudaSetDevice", dev.rc);
    const kvp_store s = store_of(c, 0);
    const int words = c->cfg.head_dim * c->elem_bytes / 16, heads_inside = s.head_stride < s.row_stride;
    auto fill = [&](page_pair *p, int32_t i0, int32_t m) {
        int32_t most = 0;
        for (int32_t i = 0; i < m; ++i) {
            p[i] = {src[i0 + i], dst[i0 + i], rows ? rows[i0 + i] : c->cfg.page_size};
            most = std::max(most, p[i].rows);
        }
        return most;
    };
    for (int32_t i0 = 0; i0 < n;) {
        const int32_t m = std::min(n - i0, n - i0 <= 300 ? 300 : kPairs);
        copy_pairs pairs;
        copy_pairs_small few;
        const int64_t most = m <= 300 ? fill(few.p, i0, m) : fill(pairs.p, i0, m);
        i0 += m;
        if (most == 0) continue;
        const int64_t per = 256 * kCopyVecs * 4, z = std::min<int64_t>(65535, (most * c->cfg.n_kv_heads * words + per - 1) / per);
        const dim3 grid(m, 2 * c->cfg.n_layers, (unsigned)z);
        const int64_t layer_bytes = c->cfg.layer_stride * c->elem_bytes;
        const cudaError_t e = m <= 300 ? launch_pdl(copy_pages_kernel<copy_pairs_small>, grid, dim3(256), 0, st, few, s, layer_bytes, c->cfg.n_kv_heads, words, heads_inside)
                                       : launch_pdl(copy_pages_kernel<copy_pairs>, grid, dim3(256), 0, st, pairs, s, layer_bytes, c->cfg.n_kv_heads, words, heads_inside);
        if (e != cudaSuccess) return cuda_failed(c, "copy", e);
    }
    return KVP_OK;
}

}  // namespace

extern "C" {

int32_t kvp_rope_frequencies(const kvp_rope *rope, double *inv_freq)
{
    if (!rope || !inv_freq) return fail(nullptr, KVP_ERR_INVALID, "rope_frequencies: null pointer");
    if (int32_t rc = check_rope(nullptr, rope, INT32_MAX - 15)) return rc;
    for (int i = 0; i < rope->rotary_dim / 2; ++i) inv_freq[i] = frequency(rope, i);
    return KVP_OK;
}

int32_t kvp_norm_rope(int32_t device, int32_t dtype, int32_t head_dim, const kvp_tokens *tokens, const kvp_rope *rope, void *stream)
{
    if ((head_dim != 64 && head_dim != 128) || (dtype != KVP_DTYPE_F32 && dtype != KVP_DTYPE_BF16) || device < 0)
        return fail(nullptr, KVP_ERR_INVALID, "norm_rope: bad device, dtype or head_dim");
    if (int32_t rc = check_rope(nullptr, rope, head_dim)) return rc;
    append_args a;
    if (int32_t rc = token_args(nullptr, tokens, rope, dtype, head_dim, a)) return rc;
    if (a.n_tokens == 0 || a.n_q + a.n_k == 0) return KVP_OK;
    on_device dev(device);
    int sms = 0;
    cudaError_t e = dev.rc;
    if (e == cudaSuccess) e = sms_of(device, &sms);
    if (e == cudaSuccess) e = launch_append(a, dtype, head_dim, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? (int32_t)KVP_OK : cuda_failed(nullptr, "norm_rope", e);
}

uint64_t kvp_cache_workspace_bytes(const kvp_cache_config *cfg)
{
    return valid_cache(cfg) ? layout_of(cfg, kMostSms).total : 0;
}

int32_t kvp_cache_create(const kvp_cache_config *cfg, kvp_cache **out)
{
    if (!out) return fail(nullptr, KVP_ERR_INVALID, "cache_create: null pointer");
    *out = nullptr;
    if (!valid_cache(cfg)) return fail(nullptr, KVP_ERR_INVALID, "cache_create: invalid configuration");
    kvp_cache *c = new (std::nothrow) kvp_cache();
    if (!c) return fail(nullptr, KVP_ERR_CAPACITY, "cache_create: no host memory");
    c->cfg = *cfg;
    c->elem_bytes = cfg->dtype == KVP_DTYPE_BF16 ? 2 : 4;
    c->scale = (float)(cfg->softmax_scale > 0.0 ? cfg->softmax_scale : 1.0 / sqrt((double)cfg->head_dim));
    c->by_page = divisor(cfg->page_size);
    c->unit_shift = unit_shift_of(cfg);
    auto bail = [&](int32_t code) {
        delete c;
        return code;
    };
    try {
        c->holders.assign(cfg->n_pages, 0);
        c->scratch.assign(cfg->n_pages, 0);
        c->free_pages.resize(cfg->n_pages);
    } catch (const std::bad_alloc &) {
        return bail(fail(nullptr, KVP_ERR_CAPACITY, "cache_create: no host memory"));
    }
    for (int32_t i = 0; i < cfg->n_pages; ++i) c->free_pages[i] = cfg->n_pages - 1 - i;
    if (cfg->device >= 0) {
        if (!cfg->k || !cfg->v || odd16(cfg->k) || odd16(cfg->v)) return bail(fail(nullptr, KVP_ERR_INVALID, "cache_create: k and v must be non-null and 16-byte aligned"));
        if (!cfg->workspace || (uintptr_t)cfg->workspace % 256) return bail(fail(nullptr, KVP_ERR_INVALID, "cache_create: workspace must be non-null and 256-byte aligned"));
        on_device dev(cfg->device);
        cudaError_t e = dev.rc;
        if (e == cudaSuccess) e = sms_of(cfg->device, &c->sm_count);
        c->sm_count = std::min(c->sm_count, kMostSms);
        if (cfg->workspace_bytes < layout_of(cfg, kMostSms).total) return bail(fail(nullptr, KVP_ERR_CAPACITY, "cache_create: workspace too small"));
        const cache_layout l = layout_of(cfg, kMostSms);
        char *ws = (char *)cfg->workspace;
        c->ws = {(float *)(ws + l.o), (float2 *)(ws + l.ml), (int32_t *)(ws + l.arrived), (int32_t *)(ws + l.arrived_group)};
        if (e == cudaSuccess) e = kvp_paged_attn_prepare(cfg->dtype, cfg->head_dim);
        // whatever is still under way on this memory, on any stream, before it becomes the cache's
        if (e == cudaSuccess) e = cudaDeviceSynchronize();
        if (e == cudaSuccess) e = cudaMemsetAsync(ws, 0, l.counted, 0);
        if (e == cudaSuccess) e = cudaStreamSynchronize(0);
        if (e != cudaSuccess) return bail(cuda_failed(nullptr, "cache_create", e));
    }
    *out = c;
    return KVP_OK;
}

int32_t kvp_cache_destroy(kvp_cache *c)
{
    if (!c) return KVP_ERR_INVALID;
    delete c;
    return KVP_OK;
}

int32_t kvp_cache_append(kvp_cache *c, int32_t layer, const kvp_tokens *tokens, const kvp_rope *rope, void *stream)
{
    if (!c) return KVP_ERR_INVALID;
    if (int32_t rc = check_rope(c, rope, c->cfg.head_dim)) return rc;
    append_args a;
    if (int32_t rc = token_args(c, tokens, rope, c->cfg.dtype, c->cfg.head_dim, a)) return rc;
    if (int32_t rc = check_runs(c, layer)) return rc;
    if (a.n_tokens == 0) return KVP_OK;
    a.st = store_of(c, layer);
    on_device dev(c->cfg.device);
    cudaError_t e = dev.rc;
    if (e == cudaSuccess) e = launch_append(a, c->cfg.dtype, c->cfg.head_dim, c->sm_count, (cudaStream_t)stream);
    return e == cudaSuccess ? (int32_t)KVP_OK : cuda_failed(c, "append", e);
}

int32_t kvp_cache_attend(kvp_cache *c, int32_t layer, int32_t batch, const void *q, const int64_t *q_stride, const int32_t *table,
                         int64_t table_stride, int32_t table_cols, const int32_t *lens, const int32_t *first, void *out,
                         const int64_t *out_stride, float *lse, void *stream)
{
    if (!c) return KVP_ERR_INVALID;
    if (batch < 0 || table_cols < 0) return fail(c, KVP_ERR_INVALID, "attend: batch or table_cols is negative");
    if (batch > c->cfg.max_batch) return fail(c, KVP_ERR_CAPACITY, "attend: %d requests of %d", batch, c->cfg.max_batch);
    if (batch > 0) {
        if (!q || !out || !q_stride || !out_stride || !lens || (!table && table_cols > 0)) return fail(c, KVP_ERR_INVALID, "attend: null pointer");
        if (odd16(q) || odd16(out)) return fail(c, KVP_ERR_INVALID, "attend: q and out must be 16-byte aligned");
        if (((uintptr_t)table | (uintptr_t)lens | (uintptr_t)first | (uintptr_t)lse) & 3) return fail(c, KVP_ERR_INVALID, "attend: table, lens, first and lse must be aligned");
        for (int k = 0; k < 2; ++k)
            if (llabs(q_stride[k]) > (1ll << 56) || llabs(out_stride[k]) > (1ll << 56) || q_stride[k] * c->elem_bytes % 16 || out_stride[k] * c->elem_bytes % 16)
                return fail(c, KVP_ERR_INVALID, "attend: strides must be multiples of 16 bytes");
        index_of_rows rows[2] = {{batch, out_stride[0]}, {c->cfg.n_q_heads, out_stride[1]}};
        if (!rows_apart(rows, 2, c->cfg.head_dim)) return fail(c, KVP_ERR_INVALID, "attend: rows of out overlap");
        if (llabs(table_stride) > (1ll << 56)) return fail(c, KVP_ERR_INVALID, "attend: table_stride");
    }
    if (!kvp_paged_fits(batch, c->cfg.n_kv_heads, c->cfg.n_q_heads / c->cfg.n_kv_heads, std::min<int64_t>(INT32_MAX, (int64_t)table_cols * c->cfg.page_size)))
        return fail(c, KVP_ERR_CAPACITY, "attend: tables of %d pages for %d requests", table_cols, batch);
    if (int32_t rc = check_runs(c, layer)) return rc;
    if (batch == 0) return KVP_OK;
    kvp_paged_args a;
    a.st = store_of(c, layer);
    a.unit_shift = c->unit_shift;
    a.page_units = (uint32_t)(a.st.page_stride >> a.unit_shift);
    a.head_units = (uint32_t)(a.st.head_stride >> a.unit_shift);
    a.row_units = (uint32_t)(a.st.row_stride >> a.unit_shift);
    a.q = (const char *)q;
    a.out = (char *)out;
    for (int k = 0; k < 2; ++k) {
        a.q_stride[k] = q_stride[k] * c->elem_bytes;
        a.out_stride[k] = out_stride[k] * c->elem_bytes;
    }
    a.table = table;
    a.lens = lens;
    a.first = first;
    a.table_stride = table_stride;
    a.room = (int32_t)std::min<int64_t>(INT32_MAX, (int64_t)table_cols * c->cfg.page_size);
    a.batch = batch;
    a.n_kv = c->cfg.n_kv_heads;
    a.group = c->cfg.n_q_heads / c->cfg.n_kv_heads;
    a.lse = lse;
    a.scale = c->scale;
    a.ws = c->ws;
    on_device dev(c->cfg.device);
    cudaError_t e = dev.rc;
    if (e == cudaSuccess) e = kvp_launch_paged_attn(a, c->cfg.dtype, c->cfg.head_dim, c->sm_count, (cudaStream_t)stream);
    return e == cudaSuccess ? (int32_t)KVP_OK : cuda_failed(c, "attend", e);
}

int32_t kvp_cache_copy(kvp_cache *c, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *rows, void *stream)
{
    if (!c) return KVP_ERR_INVALID;
    if (n < 0 || (n > 0 && (!src || !dst))) return fail(c, KVP_ERR_INVALID, "copy: null pointer or negative count");
    // every page that is written is marked, so that one written twice or read as well shows
    int32_t rc = KVP_OK, marked = 0;
    for (int32_t i = 0; i < n && rc == KVP_OK; ++i) {
        if (src[i] < 0 || src[i] >= c->cfg.n_pages || dst[i] < 0 || dst[i] >= c->cfg.n_pages)
            rc = fail(c, KVP_ERR_INVALID, "copy: page %d -> %d of %d", src[i], dst[i], c->cfg.n_pages);
        else if (rows && (rows[i] < 0 || rows[i] > c->cfg.page_size)) rc = fail(c, KVP_ERR_INVALID, "copy: %d rows of %d", rows[i], c->cfg.page_size);
        else if (c->scratch[dst[i]]) rc = fail(c, KVP_ERR_INVALID, "copy: page %d is written twice", dst[i]);
        else if (c->holders[dst[i]] > 1) rc = fail(c, KVP_ERR_STATE, "copy: page %d is shared", dst[i]);
        else { c->scratch[dst[i]] = 1; marked = i + 1; }
    }
    for (int32_t i = 0; i < n && rc == KVP_OK; ++i)
        if (c->scratch[src[i]]) rc = fail(c, KVP_ERR_INVALID, "copy: page %d is read and written", src[i]);
    for (int32_t i = 0; i < marked; ++i) c->scratch[dst[i]] = 0;
    if (rc == KVP_OK) rc = check_runs(c, 0);
    if (rc != KVP_OK || n == 0) return rc;
    return launch_copies(c, n, src, dst, rows, (cudaStream_t)stream);
}

int32_t kvp_cache_compact(kvp_cache *c, int32_t batch, const int32_t *table, int64_t table_stride, int32_t table_cols, const int32_t *lens,
                          const int32_t *new_table, int64_t new_stride, int32_t new_cols, const int32_t *kept, const int64_t *kept_stride,
                          int32_t max_kept, const int32_t *n_kept, void *stream)
{
    if (!c) return KVP_ERR_INVALID;
    if (batch < 0 || batch > 65535 || table_cols < 0 || new_cols < 0 || max_kept < 0) return fail(c, KVP_ERR_INVALID, "compact: bad count");
    const bool any = batch > 0 && max_kept > 0;
    if (any) {
        if ((!table && table_cols > 0) || (!new_table && new_cols > 0) || !lens || !kept || !kept_stride || !n_kept) return fail(c, KVP_ERR_INVALID, "compact: null pointer");
        if (((uintptr_t)table | (uintptr_t)lens | (uintptr_t)new_table | (uintptr_t)kept | (uintptr_t)n_kept) & 3)
            return fail(c, KVP_ERR_INVALID, "compact: arrays must be aligned");
        if (llabs(table_stride) > (1ll << 56) || llabs(new_stride) > (1ll << 56)) return fail(c, KVP_ERR_INVALID, "compact: strides");
        for (int k = 0; k < 3; ++k)
            if (llabs(kept_stride[k]) > (1ll << 56)) return fail(c, KVP_ERR_INVALID, "compact: strides");
    }
    if (int32_t rc = check_runs(c, 0)) return rc;
    if (!any) return KVP_OK;
    compact_args a;
    a.st = store_of(c, 0);
    a.layer_stride = c->cfg.layer_stride * c->elem_bytes;
    a.table = table;
    a.lens = lens;
    a.new_table = new_table;
    a.kept = kept;
    a.n_kept = n_kept;
    a.table_stride = table_stride;
    a.new_stride = new_stride;
    for (int k = 0; k < 3; ++k) a.kept_stride[k] = kept_stride[k];
    a.table_cols = table_cols;
    a.new_cols = new_cols;
    a.max_kept = max_kept;
    a.n_kv = c->cfg.n_kv_heads;
    on_device dev(c->cfg.device);
    cudaError_t e = dev.rc;
    if (e == cudaSuccess) e = launch_compact(a, c->cfg.head_dim * c->elem_bytes / 16, c->cfg.n_layers, batch, (cudaStream_t)stream);
    return e == cudaSuccess ? (int32_t)KVP_OK : cuda_failed(c, "compact", e);
}

int32_t kvp_cache_take(kvp_cache *c, int32_t n, int32_t *pages)
{
    if (!c) return KVP_ERR_INVALID;
    if (n < 0 || (n > 0 && !pages)) return fail(c, KVP_ERR_INVALID, "take: null pointer or negative count");
    if ((size_t)n > c->free_pages.size()) return fail(c, KVP_ERR_CAPACITY, "take: %d pages, %d are free", n, (int)c->free_pages.size());
    for (int32_t i = 0; i < n; ++i) {
        pages[i] = c->free_pages.back();
        c->free_pages.pop_back();
        c->holders[pages[i]] = 1;
    }
    return KVP_OK;
}

int32_t kvp_cache_share(kvp_cache *c, int32_t n, const int32_t *pages)
{
    if (!c) return KVP_ERR_INVALID;
    if (n < 0 || (n > 0 && !pages)) return fail(c, KVP_ERR_INVALID, "share: null pointer or negative count");
    for (int32_t i = 0; i < n; ++i) {
        if (pages[i] < 0 || pages[i] >= c->cfg.n_pages) return fail(c, KVP_ERR_INVALID, "share: page %d of %d", pages[i], c->cfg.n_pages);
        if (c->holders[pages[i]] == 0) return fail(c, KVP_ERR_STATE, "share: page %d has no holder", pages[i]);
        if (c->holders[pages[i]] > INT32_MAX - n) return fail(c, KVP_ERR_CAPACITY, "share: page %d has too many holders", pages[i]);
    }
    for (int32_t i = 0; i < n; ++i) ++c->holders[pages[i]];
    return KVP_OK;
}

int32_t kvp_cache_release(kvp_cache *c, int32_t n, const int32_t *pages)
{
    if (!c) return KVP_ERR_INVALID;
    if (n < 0 || (n > 0 && !pages)) return fail(c, KVP_ERR_INVALID, "release: null pointer or negative count");
    int32_t rc = KVP_OK, counted = 0;
    for (int32_t i = 0; i < n && rc == KVP_OK; ++i) {
        if (pages[i] < 0 || pages[i] >= c->cfg.n_pages) rc = fail(c, KVP_ERR_INVALID, "release: page %d of %d", pages[i], c->cfg.n_pages);
        else if (++c->scratch[pages[i]] > c->holders[pages[i]]) {
            --c->scratch[pages[i]];
            rc = fail(c, KVP_ERR_STATE, "release: page %d is not held that often", pages[i]);
        } else counted = i + 1;
    }
    for (int32_t i = 0; i < counted; ++i) c->scratch[pages[i]] = 0;
    if (rc != KVP_OK) return rc;
    for (int32_t i = 0; i < n; ++i)
        if (--c->holders[pages[i]] == 0) c->free_pages.push_back(pages[i]);       // there is room: it held every page at the start
    return KVP_OK;
}

int32_t kvp_cache_fork(kvp_cache *c, int32_t n_tokens, const int32_t *pages, int32_t n_forks, int32_t *forks, void *stream)
{
    if (!c) return KVP_ERR_INVALID;
    if (n_tokens < 0 || n_forks < 0) return fail(c, KVP_ERR_INVALID, "fork: negative count");
    const int32_t whole = n_tokens / c->cfg.page_size, rest = n_tokens % c->cfg.page_size, cols = whole + (rest ? 1 : 0);
    if (n_forks == 0 || cols == 0) return KVP_OK;
    if (!pages || !forks) return fail(c, KVP_ERR_INVALID, "fork: null pointer");
    for (int32_t i = 0; i < cols; ++i) {
        if (pages[i] < 0 || pages[i] >= c->cfg.n_pages) return fail(c, KVP_ERR_INVALID, "fork: page %d of %d", pages[i], c->cfg.n_pages);
        if (c->holders[pages[i]] == 0) return fail(c, KVP_ERR_STATE, "fork: page %d has no holder", pages[i]);
        if (c->holders[pages[i]] > INT32_MAX / 2 || n_forks > INT32_MAX / 2 / cols) return fail(c, KVP_ERR_CAPACITY, "fork: too many holders");
    }
    if (rest) {
        if (int32_t rc = check_runs(c, 0)) return rc;
        if ((size_t)n_forks > c->free_pages.size()) return fail(c, KVP_ERR_CAPACITY, "fork: %d pages, %d are free", n_forks, (int)c->free_pages.size());
        std::vector<int32_t> src, dst, rows;
        try {
            src.assign(n_forks, pages[whole]);
            rows.assign(n_forks, rest);
            dst.assign(c->free_pages.end() - n_forks, c->free_pages.end());
        } catch (const std::bad_alloc &) {
            return fail(c, KVP_ERR_CAPACITY, "fork: no host memory");
        }
        if (int32_t rc = launch_copies(c, n_forks, src.data(), dst.data(), rows.data(), (cudaStream_t)stream)) return rc;
    }
    for (int32_t f = 0; f < n_forks; ++f) {
        for (int32_t i = 0; i < whole; ++i) {
            forks[(int64_t)f * cols + i] = pages[i];
            ++c->holders[pages[i]];
        }
        if (rest) (void)kvp_cache_take(c, 1, forks + (int64_t)f * cols + whole);
    }
    return KVP_OK;
}

int32_t kvp_cache_free_pages(kvp_cache *c, int32_t *n)
{
    if (!c) return KVP_ERR_INVALID;
    if (!n) return fail(c, KVP_ERR_INVALID, "free_pages: null pointer");
    *n = (int32_t)c->free_pages.size();
    return KVP_OK;
}

const char *kvp_cache_last_error(kvp_cache *c) { return c ? c->err.c_str() : g_error.c_str(); }

}  // extern "C"

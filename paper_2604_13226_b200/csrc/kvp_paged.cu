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

template <typename T> struct elem;
template <> struct elem<float> {
    static constexpr int kPerVec = 4;
    __device__ static float get(float x) { return x; }
    __device__ static float put(float x) { return x; }
};
template <> struct elem<__nv_bfloat16> {
    static constexpr int kPerVec = 8;
    __device__ static float get(__nv_bfloat16 x) { return __bfloat162float(x); }
    __device__ static __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
};
template <typename T> union vec16 {
    uint4 u;
    T e[elem<T>::kPerVec];
};

// ---- norms, rotation, append ----------------------------------------------------------------------------------

constexpr int kTokens = 4;         // most tokens of a block

struct append_args {
    const char *q, *k, *v;
    char *q_out, *k_out;
    int64_t q_stride[2], k_stride[2], v_stride[2], q_out_stride[2], k_out_stride[2];   // {token, head}, bytes
    const int32_t *positions, *slots;
    const char *q_weight, *k_weight;
    kvp_store st;                  // st.k null: no pages
    int32_t n_tokens, n_q, n_k, n_v;   // heads of each that there is something to do for
    int32_t tokens, rows;          // per block: tokens, and rows of a token (all, or a part of them)
    int32_t rotary, pairing;
    float eps, magnitude;
    double turns[64];              // f_i / 2 pi
};

// A row is one head of one token.  A thread takes two 16-byte words of it that are each other's rotation partners (half
// layout; the words behind rotary_dim in pairs as they come), so that neither layout needs an exchange between threads and
// the sum of squares takes log2(words/2) shuffles.  The angle is formed in double precision, as a part of a turn, and its
// sine and cosine from the rounded remainder: |remainder| <= 1/2 turn, so the rounding moves the angle by 2^-25 turns at
// most, wherever the position lies.
template <typename T, int D>
__global__ void __launch_bounds__(256)
append_tokens_kernel(const __grid_constant__ append_args a)
{
    constexpr int EV = elem<T>::kPerVec, V = D / EV, L = V / 2, RP = 256 / L;     // words of a row, threads of a row, rows at once
    __shared__ __align__(16) float2 cs[kTokens][D / 2];
    pdl_launch_dependents();
    const int t0 = blockIdx.x * a.tokens, n_t = min(a.tokens, a.n_tokens - t0), half_rot = a.rotary / 2;
    const int tt = threadIdx.x / 64, ti = threadIdx.x % 64;
    pdl_wait();
    if (tt < n_t && ti < half_rot) {
        const double turn = (double)a.positions[t0 + tt] * a.turns[ti];
        float s, c;
        sincospif(2.0f * (float)(turn - rint(turn)), &s, &c);
        cs[tt][ti] = make_float2(a.magnitude * c, a.magnitude * s);
    }
    __syncthreads();
    const int j = threadIdx.x % L, lane_row = threadIdx.x / L;
    const int half = a.rotary / EV / 2;                                            // words of one half of the rotated part
    const bool turns = j < half;
    const int w0 = turns ? j : 2 * half + 2 * (j - half), w1 = turns ? j + half : w0 + 1;
    const int rows = a.n_q + a.n_k + a.n_v, r0 = blockIdx.y * a.rows, n_rows = min(a.rows, rows - r0);
    for (int w = lane_row; w - lane_row < n_t * n_rows; w += RP) {
        const bool in = w < n_t * n_rows;
        const int t = t0 + (in ? w / n_rows : 0), tl = t - t0, r = in ? r0 + w % n_rows : r0;
        const int kind = r < a.n_q ? 0 : r < a.n_q + a.n_k ? 1 : 2;
        const int head = kind == 0 ? r : kind == 1 ? r - a.n_q : r - a.n_q - a.n_k;
        const char *src = kind == 0 ? a.q + t * a.q_stride[0] + head * a.q_stride[1]
                        : kind == 1 ? a.k + t * a.k_stride[0] + head * a.k_stride[1]
                                    : a.v + t * a.v_stride[0] + head * a.v_stride[1];
        vec16<T> x, y;
        x.u = reinterpret_cast<const uint4 *>(src)[w0];
        y.u = reinterpret_cast<const uint4 *>(src)[w1];
        const char *weight = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
        float fx[EV], fy[EV];
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < EV; ++e) {
            fx[e] = elem<T>::get(x.e[e]);
            fy[e] = elem<T>::get(y.e[e]);
            ss += fx[e] * fx[e] + fy[e] * fy[e];
        }
        if (a.q_weight || a.k_weight) {
#pragma unroll
            for (int o = L / 2; o > 0; o /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        }
        if (weight) {
            const float inv = rsqrtf(ss * (1.0f / D) + a.eps);
            vec16<T> gx, gy;
            gx.u = reinterpret_cast<const uint4 *>(weight)[w0];
            gy.u = reinterpret_cast<const uint4 *>(weight)[w1];
#pragma unroll
            for (int e = 0; e < EV; ++e) {
                fx[e] *= inv * elem<T>::get(gx.e[e]);
                fy[e] *= inv * elem<T>::get(gy.e[e]);
            }
        }
        if (kind < 2 && turns) {
            if (a.pairing == 0) {
#pragma unroll
                for (int e = 0; e < EV; ++e) {
                    const float2 c = cs[tl][w0 * EV + e];
                    const float p = fx[e], q = fy[e];
                    fx[e] = p * c.x - q * c.y;
                    fy[e] = p * c.y + q * c.x;
                }
            } else {
#pragma unroll
                for (int e = 0; e < EV; e += 2) {
                    float2 c = cs[tl][(w0 * EV + e) / 2];
                    float p = fx[e], q = fx[e + 1];
                    fx[e] = p * c.x - q * c.y;
                    fx[e + 1] = p * c.y + q * c.x;
                    c = cs[tl][(w1 * EV + e) / 2];
                    p = fy[e];
                    q = fy[e + 1];
                    fy[e] = p * c.x - q * c.y;
                    fy[e + 1] = p * c.y + q * c.x;
                }
            }
        }
        if (kind < 2) {
#pragma unroll
            for (int e = 0; e < EV; ++e) {
                x.e[e] = elem<T>::put(fx[e]);
                y.e[e] = elem<T>::put(fy[e]);
            }
        }
        if (!in) continue;
        char *out = kind == 0 ? a.q_out + t * a.q_out_stride[0] + head * a.q_out_stride[1]
                  : kind == 1 && a.k_out ? a.k_out + t * a.k_out_stride[0] + head * a.k_out_stride[1] : nullptr;
        if (out) {
            reinterpret_cast<uint4 *>(out)[w0] = x.u;
            reinterpret_cast<uint4 *>(out)[w1] = y.u;
        }
        if (kind > 0 && a.st.k) {
            const int32_t slot = a.slots[t];
            if (slot >= 0 && slot < a.st.n_pages * a.st.page_size) {
                const int32_t page = divide(slot, a.st.by_page), row = slot - page * a.st.page_size;
                char *to = (kind == 1 ? a.st.k : a.st.v) + page * a.st.page_stride + head * a.st.head_stride + row * a.st.row_stride;
                reinterpret_cast<uint4 *>(to)[w0] = x.u;
                reinterpret_cast<uint4 *>(to)[w1] = y.u;
            }
        }
    }
}

template <typename T>
cudaError_t launch_append(append_args &a, int head_dim, int sm_count, cudaStream_t st)
{
    const int at_once = 256 / (head_dim / elem<T>::kPerVec / 2), rows = a.n_q + a.n_k + a.n_v;
    // Few tokens: one pass of a block each, rows of a token spread over blocks; many: four tokens a block, so that every thread
    // forms an angle.
    int64_t parts = 1;
    if (a.n_tokens >= 8 * sm_count) {
        a.tokens = kTokens;
        a.rows = rows;
    } else {
        a.tokens = 1;
        a.rows = std::min(rows, at_once);
        parts = (rows + a.rows - 1) / a.rows;
    }
    const dim3 grid((a.n_tokens + a.tokens - 1) / a.tokens, (unsigned)parts);
    return head_dim == 128 ? launch_pdl(append_tokens_kernel<T, 128>, grid, dim3(256), 0, st, a)
                           : launch_pdl(append_tokens_kernel<T, 64>, grid, dim3(256), 0, st, a);
}

// ---- copies of pages --------------------------------------------------------------------------------------------

struct page_pair { int32_t src, dst, rows; };
constexpr int kPairs = 1300;       // of one launch; they travel as parameters
struct copy_pairs { page_pair p[kPairs]; };
struct copy_pairs_small { page_pair p[300]; };

constexpr int kCopyVecs = 8;       // words in flight per thread

// Block (pair, layer and K or V, part of the page): words of the rows to be copied, in the order they lie in the store.
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
    int32_t table_cols, new_cols, max_kept, n_kv, words;
};

constexpr int kCompactRows = 64;

// Block (64 new rows, layer and head, request): where each row comes from and goes to is looked up once, then the words of K
// and V are moved.
__global__ void __launch_bounds__(256)
compact_kernel(const compact_args a)
{
    __shared__ int64_t from[kCompactRows], to[kCompactRows];
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.z, layer = blockIdx.y / a.n_kv, h = blockIdx.y % a.n_kv, i0 = blockIdx.x * kCompactRows;
    const int n = min(min(a.n_kept[b], a.max_kept) - i0, kCompactRows);
    if (n <= 0) return;
    if ((int)threadIdx.x < n) {
        const int i = i0 + threadIdx.x;
        const int row = a.kept[b * a.kept_stride[0] + layer * a.kept_stride[1] + h * a.kept_stride[2] + i];
        const int64_t base = layer * a.layer_stride + h * a.st.head_stride;
        int64_t f = -1, t = -1;
        const int new_page = divide(i, a.st.by_page);
        if (row >= 0 && row < a.lens[b] && new_page < a.new_cols) {
            const int page = divide(row, a.st.by_page);
            const int src = page < a.table_cols ? a.table[b * a.table_stride + page] : -1, dst = a.new_table[b * a.new_stride + new_page];
            if (src >= 0 && src < a.st.n_pages && dst >= 0 && dst < a.st.n_pages) {
                f = base + src * a.st.page_stride + (row - page * a.st.page_size) * a.st.row_stride;
                t = base + dst * a.st.page_stride + (i - new_page * a.st.page_size) * a.st.row_stride;
            }
        }
        from[threadIdx.x] = f;
        to[threadIdx.x] = t;
    }
    __syncthreads();
    const int n_words = 2 * n * a.words;                   // K and V of a row in turn
    for (int w0 = threadIdx.x; w0 < n_words; w0 += 256 * kCopyVecs) {
        uint4 x[kCopyVecs];
#pragma unroll
        for (int u = 0; u < kCopyVecs; ++u) {
            const int w = w0 + 256 * u;
            if (w >= n_words) break;
            const int r = w / (2 * a.words), c = w % (2 * a.words);
            if (from[r] >= 0) x[u] = *reinterpret_cast<const uint4 *>((c < a.words ? a.st.k : a.st.v) + from[r] + (c % a.words) * 16);
        }
#pragma unroll
        for (int u = 0; u < kCopyVecs; ++u) {
            const int w = w0 + 256 * u;
            if (w >= n_words) break;
            const int r = w / (2 * a.words), c = w % (2 * a.words);
            if (from[r] >= 0) *reinterpret_cast<uint4 *>((c < a.words ? a.st.k : a.st.v) + to[r] + (c % a.words) * 16) = x[u];
        }
    }
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

kvp_divisor divisor(int32_t d)
{
    int l = 0;
    while ((1ll << l) < d) ++l;
    return {(uint32_t)((1ull << (31 + l)) / (uint64_t)d + 1), 31 + l};
}

bool odd16(const void *p) { return ((uintptr_t)p & 15) != 0; }

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
    // each index of more than one value moves by a row at least
    if ((c->n_layers > 1 && c->layer_stride < c->head_dim) || (c->n_pages > 1 && c->page_stride < c->head_dim) ||
        (c->n_kv_heads > 1 && c->head_stride < c->head_dim) || (c->page_size > 1 && c->row_stride < c->head_dim))
        return false;
    return true;
}

struct cache_layout { uint64_t o, ml, arrived, total; int32_t units; };
cache_layout layout_of(const kvp_cache_config *c, int32_t sm_count)
{
    cache_layout l;
    const int64_t group = c->n_q_heads / c->n_kv_heads, slots = 2ll * kvp_paged_ctas(sm_count);
    l.units = (int32_t)std::min<int64_t>(INT32_MAX, (int64_t)c->max_batch * c->n_kv_heads * ((group + KVP_PAGED_LEAST_ROWS - 1) / KVP_PAGED_LEAST_ROWS));
    l.arrived = 0;
    l.ml = (4ull * l.units + 255) / 256 * 256;
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
    if (t->n_tokens < 0) return fail(c, KVP_ERR_INVALID, "tokens: n_tokens is negative");
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
    const struct { const void *p; const int64_t *s; int64_t *to; int32_t heads; } x[5] = {
        {t->q, t->q_stride, a.q_stride, t->n_q_heads}, {t->k, t->k_stride, a.k_stride, t->n_kv_heads}, {t->v, t->v_stride, a.v_stride, t->n_kv_heads},
        {t->q_out, t->q_out_stride, a.q_out_stride, t->n_q_heads}, {t->k_out, t->k_out_stride, a.k_out_stride, t->n_kv_heads}};
    for (int i = 0; i < 5; ++i) {
        x[i].to[0] = x[i].to[1] = 0;
        if (!x[i].p) continue;
        if (odd16(x[i].p)) return fail(c, KVP_ERR_INVALID, "tokens: pointers must be 16-byte aligned");
        for (int k = 0; k < 2; ++k) {
            if (x[i].s[k] < -(1ll << 56) || x[i].s[k] > (1ll << 56) || x[i].s[k] * e % 16)
                return fail(c, KVP_ERR_INVALID, "tokens: strides must be multiples of 16 bytes");
            x[i].to[k] = x[i].s[k] * e;
        }
        // rows that are written must not lie over one another
        if (i >= 3 && ((t->n_tokens > 1 && llabs(x[i].s[0]) < head_dim) || (x[i].heads > 1 && llabs(x[i].s[1]) < head_dim)))
            return fail(c, KVP_ERR_INVALID, "tokens: rows of an output overlap");
    }
    // in place only row for row
    if ((t->q && t->q_out == t->q && (t->q_stride[0] != t->q_out_stride[0] || t->q_stride[1] != t->q_out_stride[1])) ||
        (t->k && t->k_out == t->k && (t->k_stride[0] != t->k_out_stride[0] || t->k_stride[1] != t->k_out_stride[1])))
        return fail(c, KVP_ERR_INVALID, "tokens: in place with other strides");
    a.q = (const char *)t->q;
    a.k = (const char *)t->k;
    a.v = (const char *)t->v;
    a.q_out = (char *)t->q_out;
    a.k_out = (char *)t->k_out;
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
    if (e == cudaSuccess) e = dtype == KVP_DTYPE_BF16 ? launch_append<__nv_bfloat16>(a, head_dim, sms, (cudaStream_t)stream)
                                                      : launch_append<float>(a, head_dim, sms, (cudaStream_t)stream);
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
        c->ws = {(float *)(ws + l.o), (float2 *)(ws + l.ml), (int32_t *)(ws + l.arrived)};
        if (e == cudaSuccess) e = kvp_paged_attn_prepare(cfg->dtype, cfg->head_dim);
        // whatever is still under way on this memory, on any stream, before it becomes the cache's
        if (e == cudaSuccess) e = cudaDeviceSynchronize();
        if (e == cudaSuccess) e = cudaMemsetAsync(c->ws.arrived, 0, 4ull * l.units, 0);
        if (e == cudaSuccess) e = cudaStreamSynchronize(0);
        if (e != cudaSuccess) return bail(cuda_failed(nullptr, "cache_create", e));
    }
    *out = c;
    return KVP_OK;
}

int32_t kvp_cache_destroy(kvp_cache *c)
{
    if (!c) return KVP_ERR_INVALID;
    if (c->cfg.device >= 0) {
        on_device dev(c->cfg.device);
        if (dev.rc == cudaSuccess) (void)cudaDeviceSynchronize();
    }
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
    if (e == cudaSuccess) e = c->cfg.dtype == KVP_DTYPE_BF16 ? launch_append<__nv_bfloat16>(a, c->cfg.head_dim, c->sm_count, (cudaStream_t)stream)
                                                             : launch_append<float>(a, c->cfg.head_dim, c->sm_count, (cudaStream_t)stream);
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
        if ((batch > 1 && llabs(out_stride[0]) < c->cfg.head_dim) || (c->cfg.n_q_heads > 1 && llabs(out_stride[1]) < c->cfg.head_dim))
            return fail(c, KVP_ERR_INVALID, "attend: rows of out overlap");
        if (llabs(table_stride) > (1ll << 56)) return fail(c, KVP_ERR_INVALID, "attend: table_stride");
    }
    if (!kvp_paged_fits(batch, c->cfg.n_kv_heads, c->cfg.n_q_heads / c->cfg.n_kv_heads, std::min<int64_t>(INT32_MAX, (int64_t)table_cols * c->cfg.page_size)))
        return fail(c, KVP_ERR_CAPACITY, "attend: tables of %d pages for %d requests", table_cols, batch);
    if (int32_t rc = check_runs(c, layer)) return rc;
    if (batch == 0) return KVP_OK;
    kvp_paged_args a;
    a.st = store_of(c, layer);
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
        if (!table || !lens || !new_table || !kept || !kept_stride || !n_kept) return fail(c, KVP_ERR_INVALID, "compact: null pointer");
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
    a.words = c->cfg.head_dim * c->elem_bytes / 16;
    on_device dev(c->cfg.device);
    cudaError_t e = dev.rc;
    const dim3 grid((unsigned)(((int64_t)max_kept + kCompactRows - 1) / kCompactRows), (unsigned)(c->cfg.n_layers * c->cfg.n_kv_heads), (unsigned)batch);
    if (e == cudaSuccess) e = launch_pdl(compact_kernel, grid, dim3(256), 0, (cudaStream_t)stream, a);
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

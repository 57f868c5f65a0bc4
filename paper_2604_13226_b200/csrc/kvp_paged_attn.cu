// Attention of one new token per request over a cache in pages (kvp_cache_attend).
//
// out = sum_j softmax(scale q.k_j) v_j over the request's visible rows, the group's query heads together against their kv head.
// Every K and V byte is used for at most 16 query rows, so reading the cache bounds the call: 6.5 TB/s are 23 bytes per SM and
// clock, 350 clocks for the 8 KB of 16 keys of 128 in bf16, where mma.sync needs 64 of them.  What matters is bytes in flight
// and an even share for every SM.
//
// * A unit is (request, kv head, up to 16 of its query heads).  Units are laid end to end, a unit counting as long as its key
//   tiles plus a fixed cost, and the line is cut into equal shares, one per CTA.  Every CTA finds its share itself, from the
//   lengths as they lie in device memory, so that a captured launch follows them.
// * A unit inside one CTA is written out by it.  The parts of a unit that several CTAs share go to the workspace, and the CTA
//   whose part is the last to arrive joins them, always in the order of the parts: results do not depend on who came last.
// * Inside a CTA every warp streams key tiles of its own (warp w takes every 4th) through a ring of cp.async stages, without
//   any barrier; the warps' running maxima, sums and outputs are joined in shared memory at a unit's end.  The ring runs on
//   into the next unit meanwhile.
// * Rows are looked up one by one through the page table, by any page size; rows that are not there - behind the length, in
//   front of `first`, on a page outside the store - are filled with zeros and masked, never read.
#include <cuda_bf16.h>

#include <algorithm>

#include "kvp_paged.h"

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kCtasPerSm = 2;
constexpr int kStages = 3;
constexpr int kStageBytes = 8192;          // K and V rows of a tile
constexpr int kUnitCost = 8;               // start and end of a unit, in key tiles of one warp
constexpr int kMinShare = 8;               // tiles that a CTA is worth starting for

template <typename T, int D> struct shape {
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kWords = kRowBytes / 16;                      // 16-byte words of a row
    static constexpr int kKeys = kStageBytes / 2 / kRowBytes;          // keys of a tile
    static constexpr int kSmemJoin = kWarps * 8 * D * 4;               // outputs of 8 rows of every warp
    static constexpr int kSmem = kWarps * kStages * kStageBytes + kSmemJoin + kWarps * 8 * 8;
    static_assert(kKeys <= 32, "a lane looks up a row");
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 16 bytes to shared memory; without `there` zeros, and src is not read
__device__ __forceinline__ void copy16(uint32_t dst, const char *src, bool there)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(__nv_bfloat16 lo, __nv_bfloat16 hi)
{
    return (uint32_t)__bfloat16_as_ushort(lo) | (uint32_t)__bfloat16_as_ushort(hi) << 16;
}
// a probability pair in two bf16 numbers each, value and rounding remainder
__device__ __forceinline__ void split(float p0, float p1, uint32_t &value, uint32_t &rest)
{
    const __nv_bfloat16 h0 = __float2bfloat16_rn(p0), h1 = __float2bfloat16_rn(p1);
    value = pack(h0, h1);
    rest = pack(__float2bfloat16_rn(p0 - __bfloat162float(h0)), __float2bfloat16_rn(p1 - __bfloat162float(h1)));
}

__device__ __forceinline__ float quad_max(float x)
{
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x)
{
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

// Visible rows of request b: [first, first + n).
__device__ __forceinline__ int visible(const kvp_paged_args &a, int b, int &first)
{
    const int64_t room = (int64_t)a.table_cols * a.st.page_size;
    int len = max(a.lens[b], 0);
    first = a.first ? max(a.first[b], 0) : 0;
    if (len > room) len = (int)room;
    return max(len - first, 0);
}

// Where on the line of all units a CTA's share lies, and a walk over the units that reach into it.
struct line {
    int64_t total, begin, end;
    int ctas;
    __device__ int64_t start(int cta) const { return total * cta / ctas; }
    __device__ int owner(int64_t x) const { return (int)(((x + 1) * ctas - 1) / total); }
};

template <int KEYS> struct walk {
    int b, u, first, rows, tiles;          // the request, unit in it, its rows and tiles
    int64_t at;                            // where the unit begins on the line
    __device__ void request(const kvp_paged_args &a)
    {
        if (b >= a.batch) return;
        rows = visible(a, b, first);
        tiles = (rows + KEYS - 1) / KEYS;
    }
    // To the next unit with something to do for this CTA: tiles [lo, hi), none for a unit without rows.  False: there is none.
    __device__ bool next(const kvp_paged_args &a, const line &ln, int units, int &lo, int &hi, int &ub, int &uu, int &ufirst, int &urows, int64_t &uat)
    {
        while (b < a.batch && at < ln.end) {
            const int64_t t0 = at + kUnitCost;
            lo = (int)max((int64_t)0, ln.begin - t0);
            hi = (int)min((int64_t)tiles, ln.end - t0);
            const bool mine = tiles == 0 ? at >= ln.begin : lo < hi;       // one without rows is its beginning's
            if (tiles == 0) lo = hi = 0;
            ub = b; uu = u; ufirst = first; urows = rows; uat = at;
            at += kUnitCost + tiles;
            if (++u == units) {
                u = 0;
                ++b;
                request(a);
            }
            if (mine) return true;
        }
        return false;
    }
};

// Every warp for itself: 32 requests at a time.
template <int KEYS>
__device__ __forceinline__ void find_share(const kvp_paged_args &a, int units, line &ln, walk<KEYS> &w)
{
    const int lane = threadIdx.x % 32;
    int64_t total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        int f;
        if (b0 + lane < a.batch) total += (int64_t)units * (kUnitCost + (visible(a, b0 + lane, f) + KEYS - 1) / KEYS);
    }
    for (int o = 16; o > 0; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
    ln.total = total;
    ln.ctas = (int)max((int64_t)1, min((int64_t)gridDim.x, total / kMinShare));
    ln.begin = ln.end = 0;
    if ((int)blockIdx.x >= ln.ctas) return;
    ln.begin = ln.start(blockIdx.x);
    ln.end = ln.start(blockIdx.x + 1);
    int64_t before = 0;
    for (int b0 = 0;; b0 += 32) {
        int f, n = 0;
        if (b0 + lane < a.batch) n = (visible(a, b0 + lane, f) + KEYS - 1) / KEYS + kUnitCost;
        int64_t upto = (int64_t)n * units;                 // of this and the lanes in front
        for (int o = 1; o < 32; o *= 2) {
            const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + upto > ln.begin);
        if (past || b0 + 32 >= a.batch) {
            const int who = past ? __ffs(past) - 1 : 31;
            const int64_t base = before + __shfl_sync(0xffffffffu, upto - (int64_t)n * units, who);
            const int len = __shfl_sync(0xffffffffu, n, who);
            w.b = b0 + who;
            w.u = len ? (int)((ln.begin - base) / len) : 0;
            w.at = base + (int64_t)w.u * len;
            w.request(a);
            return;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
}

// The tiles of a warp, one after the other, through the pieces of its CTA's share: what is loaded.
template <typename T, int D> struct loader {
    using S = shape<T, D>;
    walk<S::kKeys> w;
    int lo, hi, b, u, first, rows;         // the piece
    int64_t at;
    int tile, turn;                        // this warp's next tile; tiles of the CTA so far, modulo the warps
    bool more;
    int page;                              // of this lane's row in that tile, -1: not there
    int row;                               // and the row within it

    __device__ void piece(const kvp_paged_args &a, const line &ln, int units)
    {
        const int warp = threadIdx.x / 32;
        while (more) {
            more = w.next(a, ln, units, lo, hi, b, u, first, rows, at);
            if (!more) return;
            const int n = max(hi - lo, 0), mine = lo + (warp + kWarps - turn) % kWarps;
            turn = (turn + n) % kWarps;
            if (mine < hi) {
                tile = mine;
                return;
            }
        }
    }
    __device__ void look_up(const kvp_paged_args &a)
    {
        page = -1;
        const int lane = threadIdx.x % 32, i = tile * S::kKeys + lane;
        if (!more || lane >= S::kKeys || i >= rows) return;
        const int r = first + i, p = divide(r, a.st.by_page);
        row = r - p * a.st.page_size;
        page = a.table[b * a.table_stride + p];
        if (page >= a.st.n_pages) page = -1;
    }
    __device__ void advance(const kvp_paged_args &a, const line &ln, int units)
    {
        tile += kWarps;
        if (tile >= hi) piece(a, ln, units);
        look_up(a);
    }
    // Copies the tile to `stage` (shared address) and leaves which rows are there in *mask; then on to the next tile.
    __device__ void issue(const kvp_paged_args &a, const line &ln, int units, int row_tiles, uint32_t stage, uint32_t *mask)
    {
        if (more) {
            const int lane = threadIdx.x % 32;
            const int64_t off = page < 0 ? 0 : page * a.st.page_stride + (u / row_tiles) * a.st.head_stride + row * a.st.row_stride;
            const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
            if (lane == 0) *mask = there;
            constexpr int N = S::kKeys * S::kWords / 32;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int x = i * 32 + lane, r = x / S::kWords, c = x % S::kWords;
                const int64_t o = __shfl_sync(0xffffffffu, off, r) + c * 16;
                const bool in = (there >> r) & 1;
                // bf16 rows are read by ldmatrix, eight rows at a time: the words of a row are permuted by its number
                const uint32_t to = stage + r * S::kRowBytes + (sizeof(T) == 2 ? c ^ (r & 7) : c) * 16;
                copy16(to, a.st.k + o, in);
                copy16(to + S::kKeys * S::kRowBytes, a.st.v + o, in);
            }
            advance(a, ln, units);
        }
        copies_commit();
    }
};

// ---- the arithmetic of a warp ---------------------------------------------------------------------------------------

// bf16: mma.sync m16n8k16, query rows as M.  With a group of at most 8 the lower half of M is free, and takes the rounding
// remainders of the probabilities: P V with 16 bits of P in one instruction.  Wider groups take two.
template <typename T, int D, bool WIDE> struct tile_math;

template <int D, bool WIDE> struct tile_math<__nv_bfloat16, D, WIDE> {
    using S = shape<__nv_bfloat16, D>;
    static constexpr int kHalves = WIDE ? 2 : 1;           // rows of 8 that a thread has one of each
    uint32_t q[D / 16][4];
    float o[D / 8][4];
    float m[2], l[2];

    __device__ void begin(const char *q0, int64_t head_stride, int n_rows)
    {
        const int g = threadIdx.x % 32 / 4, t = threadIdx.x % 4;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const char *p = q0 + (g + 8 * h) * head_stride + (k * 16 + t * 2) * 2;
                const bool in = g + 8 * h < n_rows;
                q[k][h] = in ? *reinterpret_cast<const uint32_t *>(p) : 0u;
                q[k][h + 2] = in ? *reinterpret_cast<const uint32_t *>(p + 16) : 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.0f;
    }

    __device__ void tile(uint32_t stage, uint32_t there, float scale)
    {
        const int lane = threadIdx.x % 32, t = lane % 4;
        constexpr int N = S::kKeys / 8;                    // 8-key columns of S
        float s[N][4];
#pragma unroll
        for (int i = 0; i < N; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
        const int mi = lane / 8, mr = lane % 8;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const int row = i * 16 + (mi / 2) * 8 + mr;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                uint32_t f[4];
                ldmatrix4(stage + row * S::kRowBytes + (((k * 2 + (mi & 1)) ^ mr) * 16), f);
                mma16816(s[2 * i], q[k], f[0], f[1]);
                mma16816(s[2 * i + 1], q[k], f[2], f[3]);
            }
        }
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool in = (there >> (i * 8 + t * 2 + e)) & 1;
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    s[i][2 * h + e] = in ? s[i][2 * h + e] * scale : -INFINITY;
                    top[h] = fmaxf(top[h], s[i][2 * h + e]);
                }
            }
        float fix[2] = {1.0f, 1.0f};
        bool moved = false;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            top[h] = fmaxf(quad_max(top[h]), m[h]);
            if (top[h] > m[h]) {
                fix[h] = exp2_fast(m[h] - top[h]);
                m[h] = top[h];
                l[h] *= fix[h];
                moved = true;
            }
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                o[i][0] *= fix[0];
                o[i][1] *= fix[0];
                o[i][2] *= fix[WIDE ? 1 : 0];
                o[i][3] *= fix[WIDE ? 1 : 0];
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const float ref = m[h] == -INFINITY ? 0.0f : m[h];     // no key so far: exp2(-inf - 0) = 0
                s[i][2 * h] = exp2_fast(s[i][2 * h] - ref);
                s[i][2 * h + 1] = exp2_fast(s[i][2 * h + 1] - ref);
                l[h] += s[i][2 * h] + s[i][2 * h + 1];
            }
        const uint32_t v = stage + S::kKeys * S::kRowBytes;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            uint32_t p[4], r[4];
            split(s[2 * i][0], s[2 * i][1], p[0], r[0]);
            split(s[2 * i + 1][0], s[2 * i + 1][1], p[2], r[2]);
            if (WIDE) {
                split(s[2 * i][2], s[2 * i][3], p[1], r[1]);
                split(s[2 * i + 1][2], s[2 * i + 1][3], p[3], r[3]);
            } else {
                p[1] = r[0];
                p[3] = r[2];
            }
            const int row = i * 16 + (mi & 1) * 8 + mr;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t f[4];
                ldmatrix4_trans(v + row * S::kRowBytes + (((c * 2 + mi / 2) ^ mr) * 16), f);
                mma16816(o[2 * c], p, f[0], f[1]);
                mma16816(o[2 * c + 1], p, f[2], f[3]);
                if (WIDE) {
                    mma16816(o[2 * c], r, f[0], f[1]);
                    mma16816(o[2 * c + 1], r, f[2], f[3]);
                }
            }
        }
    }

    __device__ void end()
    {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) l[h] = quad_sum(l[h]);
    }
    // rows [8 half, 8 half + 8) of this warp to shared memory: out [8][D], ml [8]
    __device__ void store(int half, float *out, float2 *ml)
    {
        const int g = threadIdx.x % 32 / 4, t = threadIdx.x % 4;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            float2 x;
            if (WIDE) x = half == 0 ? make_float2(o[i][0], o[i][1]) : make_float2(o[i][2], o[i][3]);
            else x = make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]);
            *reinterpret_cast<float2 *>(out + g * D + i * 8 + t * 2) = x;
        }
        if (t == 0) ml[g] = make_float2(m[WIDE ? half : 0], l[WIDE ? half : 0]);
    }
};

// fp32: FMA pipe.  Q K^T: 8 lanes share a key, each with a sixteenth or an eighth of its words, four keys at once; P V: a lane
// has D/32 columns of every row.  8 query rows.
template <int D> struct tile_math<float, D, false> {
    using S = shape<float, D>;
    static constexpr int R = 8, C = D / 32;
    float q[R][D / 8];
    float o[R][C];
    float m, l;                            // of row (lane % 8)

    __device__ void begin(const char *q0, int64_t head_stride, int n_rows)
    {
        const int part = threadIdx.x % 8;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (r < n_rows) x = *reinterpret_cast<const float4 *>(q0 + r * head_stride + (j * 8 + part) * 16);
                q[r][4 * j] = x.x; q[r][4 * j + 1] = x.y; q[r][4 * j + 2] = x.z; q[r][4 * j + 3] = x.w;
            }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) o[r][c] = 0.0f;
        m = -INFINITY;
        l = 0.0f;
    }

    __device__ void tile(uint32_t stage, uint32_t there, float scale)
    {
        const int lane = threadIdx.x % 32, part = lane % 8, key4 = lane / 8;
        constexpr int N = S::kKeys / 4;
        float s[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float x[R];
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                float4 k;
                asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(k.x), "=f"(k.y), "=f"(k.z), "=f"(k.w)
                             : "r"(stage + (i * 4 + key4) * S::kRowBytes + (j * 8 + part) * 16) : "memory");
#pragma unroll
                for (int r = 0; r < R; ++r) x[r] += q[r][4 * j] * k.x + q[r][4 * j + 1] * k.y + q[r][4 * j + 2] * k.z + q[r][4 * j + 3] * k.w;
            }
            // the 8 lanes of a key add up; lane `part` keeps row `part`
#pragma unroll
            for (int w = 4; w > 0; w /= 2)
#pragma unroll
                for (int r = 0; r < w; ++r) {
                    const bool upper = part & w;
                    const float give = upper ? x[r] : x[r + w], keep = upper ? x[r + w] : x[r];
                    x[r] = keep + __shfl_xor_sync(0xffffffffu, give, w);
                }
            s[i] = (there >> (i * 4 + key4)) & 1 ? x[0] * scale : -INFINITY;
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const bool moved = top > m;
        const float fix = moved ? exp2_fast(m - top) : 1.0f, ref = top == -INFINITY ? 0.0f : top;
        m = top;
        l *= fix;
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = __shfl_sync(0xffffffffu, fix, r);
#pragma unroll
                for (int c = 0; c < C; ++c) o[r][c] *= f;
            }
        }
        const uint32_t v = stage + S::kKeys * S::kRowBytes;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = exp2_fast(s[i] - ref);
            l += p;                                        // of the keys of this lane
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x[C];
                if (C == 4)
                    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[C - 2]), "=f"(x[C - 1])
                                 : "r"(v + (i * 4 + k) * S::kRowBytes + lane * 16) : "memory");
                else
                    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(x[0]), "=f"(x[1]) : "r"(v + (i * 4 + k) * S::kRowBytes + lane * 8) : "memory");
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float w = __shfl_sync(0xffffffffu, p, k * 8 + r);
#pragma unroll
                    for (int c = 0; c < C; ++c) o[r][c] += w * x[c];
                }
            }
        }
    }

    __device__ void end()
    {
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
    }
    __device__ void store(int, float *out, float2 *ml)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) out[r * D + lane * C + c] = o[r][c];
        if (lane < R) ml[lane] = make_float2(m, l);
    }
};

// ---- the kernel -------------------------------------------------------------------------------------------------------

template <typename T, int D>
__device__ __forceinline__ void write_row(const kvp_paged_args &a, int b, int head, int c4, float4 o, float m, float l)
{
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);      // no row: zeros; NaN stays
    o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
    char *to = a.out + b * a.out_stride[0] + head * a.out_stride[1] + c4 * 4 * sizeof(T);
    if (sizeof(T) == 2) {
        uint2 x;
        x.x = pack(__float2bfloat16_rn(o.x), __float2bfloat16_rn(o.y));
        x.y = pack(__float2bfloat16_rn(o.z), __float2bfloat16_rn(o.w));
        *reinterpret_cast<uint2 *>(to) = x;
    } else {
        *reinterpret_cast<float4 *>(to) = o;
    }
    if (a.lse && c4 == 0)
        a.lse[(int64_t)b * a.n_kv * a.group + head] = l > 0.0f ? (m + log2f(l)) * 0.693147180559945309f : (l == 0.0f ? -INFINITY : l);
}

template <typename T, int D, bool WIDE>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
paged_attn_kernel(const __grid_constant__ kvp_paged_args a)
{
    using S = shape<T, D>;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint32_t masks[kWarps][kStages];
    __shared__ int last;
    pdl_launch_dependents();
    const int warp = threadIdx.x / 32;
    constexpr int kUnitRows = sizeof(T) == 2 ? 16 : 8;
    const int row_tiles = (a.group + kUnitRows - 1) / kUnitRows, units = a.n_kv * row_tiles;
    const float scale = a.scale * 1.44269504088896341f;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * kStages * kStageBytes;
    float *join_o = reinterpret_cast<float *>(smem + kWarps * kStages * kStageBytes);
    float2 *join_ml = reinterpret_cast<float2 *>(smem + kWarps * kStages * kStageBytes + S::kSmemJoin);
    pdl_wait();

    line ln;
    walk<S::kKeys> w;
    find_share<S::kKeys>(a, units, ln, w);
    if ((int)blockIdx.x >= ln.ctas) return;
    loader<T, D> ld;
    ld.w = w;
    ld.turn = 0;
    ld.tile = ld.hi = 0;
    ld.more = true;
    ld.piece(a, ln, units);
    ld.look_up(a);
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) ld.issue(a, ln, units, row_tiles, ring + s * kStageBytes, &masks[warp][s]);

    int stage = 0, turn = 0;
    int lo, hi, b, u, first, rows;
    int64_t at;
    tile_math<T, D, WIDE> tm;
    while (w.next(a, ln, units, lo, hi, b, u, first, rows, at)) {
        const int h = u / row_tiles, head0 = h * a.group + u % row_tiles * kUnitRows;
        const int n_rows = min(kUnitRows, a.group - u % row_tiles * kUnitRows);
        tm.begin(a.q + b * a.q_stride[0] + head0 * a.q_stride[1], a.q_stride[1], n_rows);
        for (int t = lo + (warp + kWarps - turn) % kWarps; t < hi; t += kWarps) {
            copies_wait<kStages - 2>();
            __syncwarp();
            const int ahead = stage == 0 ? kStages - 1 : stage - 1;
            const uint32_t there = masks[warp][stage];
            ld.issue(a, ln, units, row_tiles, ring + ahead * kStageBytes, &masks[warp][ahead]);
            tm.tile(ring + stage * kStageBytes, there, scale);
            stage = stage == kStages - 1 ? 0 : stage + 1;
        }
        turn = (turn + max(hi - lo, 0)) % kWarps;
        tm.end();

        // the warps' parts, 8 rows at a time; a thread has 4 columns of a row
        const int tiles = (rows + S::kKeys - 1) / S::kKeys;
        const bool whole = lo <= 0 && hi >= tiles;
        const int slot = 2 * blockIdx.x + (lo > 0 ? 0 : 1);
        for (int half = 0; half * 8 < n_rows; ++half) {
            tm.store(half, join_o + warp * 8 * D, join_ml + warp * 8);
            __syncthreads();
            for (int x = threadIdx.x; x < 8 * D / 4; x += kThreads) {
                const int r = x / (D / 4), c4 = x % (D / 4);
                if (half * 8 + r >= n_rows) break;
                float m = -INFINITY;
#pragma unroll
                for (int k = 0; k < kWarps; ++k) m = fmaxf(m, join_ml[k * 8 + r].x);
                const float ref = m == -INFINITY ? 0.0f : m;
                float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                float l = 0.0f;
#pragma unroll
                for (int k = 0; k < kWarps; ++k) {
                    const float2 ml = join_ml[k * 8 + r];
                    const float f = exp2_fast(ml.x - ref);
                    const float4 y = reinterpret_cast<const float4 *>(join_o + (k * 8 + r) * D)[c4];
                    o.x += f * y.x; o.y += f * y.y; o.z += f * y.z; o.w += f * y.w;
                    l += f * ml.y;
                }
                if (whole) {
                    write_row<T, D>(a, b, head0 + half * 8 + r, c4, o, m, l);
                } else {
                    const int64_t p = (int64_t)slot * KVP_PAGED_ROWS + half * 8 + r;
                    reinterpret_cast<float4 *>(a.ws.part_o + p * D)[c4] = o;
                    if (c4 == 0) a.ws.part_ml[p] = make_float2(m, l);
                }
            }
            __syncthreads();
        }
        if (whole) continue;

        // whoever's part is the last joins them
        const int64_t t0 = at + kUnitCost;
        const int c0 = ln.owner(t0), n_parts = ln.owner(t0 + tiles - 1) - c0 + 1;
        int32_t *arrived = a.ws.arrived + (int64_t)b * units + u;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            last = atomicAdd(arrived, 1) == n_parts - 1;
            if (last) *arrived = 0;
        }
        __syncthreads();
        if (!last) continue;
        __threadfence();
        for (int x = threadIdx.x; x < n_rows * D / 4; x += kThreads) {
            const int r = x / (D / 4), c4 = x % (D / 4);
            float m = -INFINITY, l = 0.0f;
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int p0 = 0; p0 < n_parts; p0 += 4) {
                float2 ml[4];
                float4 y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int cta = c0 + p0 + k;
                    const int64_t p = (int64_t)(2 * cta + (p0 + k == 0 ? 1 : 0)) * KVP_PAGED_ROWS + r;
                    ml[k] = make_float2(-INFINITY, 0.0f);
                    y[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (p0 + k < n_parts) {
                        ml[k] = __ldcg(a.ws.part_ml + p);
                        y[k] = __ldcg(reinterpret_cast<const float4 *>(a.ws.part_o + p * D) + c4);
                    }
                }
                float top = m;
#pragma unroll
                for (int k = 0; k < 4; ++k) top = fmaxf(top, ml[k].x);
                const float ref = top == -INFINITY ? 0.0f : top, f0 = exp2_fast(m - ref);
                m = top;
                o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
                l *= f0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float f = exp2_fast(ml[k].x - ref);
                    o.x += f * y[k].x; o.y += f * y[k].y; o.z += f * y[k].z; o.w += f * y[k].w;
                    l += f * ml[k].y;
                }
            }
            write_row<T, D>(a, b, head0 + r, c4, o, m, l);
        }
    }
    copies_wait<0>();
}

template <typename T, int D, bool WIDE>
cudaError_t launch(const kvp_paged_args &a, int sm_count, cudaStream_t st)
{
    // no more CTAs than the longest lists that the tables can hold are worth
    constexpr int kUnitRows = sizeof(T) == 2 ? 16 : 8;
    const int64_t units = (int64_t)a.batch * a.n_kv * ((a.group + kUnitRows - 1) / kUnitRows);
    const int64_t tiles = ((int64_t)a.table_cols * a.st.page_size + shape<T, D>::kKeys - 1) / shape<T, D>::kKeys;
    const int64_t most = std::min<int64_t>(sm_count * kCtasPerSm, units * std::min<int64_t>(tiles + kUnitCost, 1 << 24) / kMinShare);
    return launch_pdl(paged_attn_kernel<T, D, WIDE>, dim3((unsigned)std::max<int64_t>(1, most)), dim3(kThreads), shape<T, D>::kSmem, st, a);
}

template <typename T, int D, bool WIDE>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(paged_attn_kernel<T, D, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, shape<T, D>::kSmem);
}

}  // namespace

int32_t kvp_paged_ctas(int32_t sm_count) { return sm_count * kCtasPerSm; }

cudaError_t kvp_paged_attn_prepare(int32_t dtype, int32_t head_dim)
{
    if (dtype == KVP_DTYPE_F32) return head_dim == 128 ? prepare<float, 128, false>() : prepare<float, 64, false>();
    const cudaError_t e = head_dim == 128 ? prepare<__nv_bfloat16, 128, false>() : prepare<__nv_bfloat16, 64, false>();
    if (e != cudaSuccess) return e;
    return head_dim == 128 ? prepare<__nv_bfloat16, 128, true>() : prepare<__nv_bfloat16, 64, true>();
}

cudaError_t kvp_launch_paged_attn(const kvp_paged_args &a, int32_t dtype, int32_t head_dim, int32_t sm_count, cudaStream_t st)
{
    if (dtype == KVP_DTYPE_F32) return head_dim == 128 ? launch<float, 128, false>(a, sm_count, st) : launch<float, 64, false>(a, sm_count, st);
    if (a.group <= 8) return head_dim == 128 ? launch<__nv_bfloat16, 128, false>(a, sm_count, st) : launch<__nv_bfloat16, 64, false>(a, sm_count, st);
    return head_dim == 128 ? launch<__nv_bfloat16, 128, true>(a, sm_count, st) : launch<__nv_bfloat16, 64, true>(a, sm_count, st);
}

// Attention of one new token per request over a cache in pages (kvp_cache_attend).
//
// out = sum_j softmax(scale q.k_j) v_j over the request's visible rows, the group's query heads together against their kv head.
// Every K and V byte is used for at most 16 query rows, so reading the cache bounds the call: 6.5 TB/s are 23 bytes per SM and
// clock, 350 clocks for the 8 KB of 16 keys of 128 in bf16, where mma.sync needs 64 of them (the tensor pipe is 21 % busy);
// tiles of 128 rows, as tcgen05 has them, would be empty but for a few.  16 requests of 33,280 rows, 32/8 heads, take 325 us =
// 6.7 TB/s, one of 133,120 rows 88 us = 6.2 TB/s (DRAM is read at 7.5 TB/s while tiles stream; 3 us go by before the first
// rows are asked for, CTAs end 3 us before and after their mean, arriving and joining takes 3), one of 2,785 rows 8.5 us.
//
// * A unit is (request, kv head, up to 16 of its query heads).  Units are laid end to end, a unit counting as long as its key
//   tiles plus a fixed cost, and the line is cut into equal shares, one per CTA.  Every CTA finds its share itself, from the
//   lengths as they lie in device memory, so that a captured launch follows them.
// * A unit inside one CTA is written out by it.  The parts of a unit that several CTAs share go to the workspace, and the CTA
//   whose part is the last to arrive joins them, always in the order of the parts: results do not depend on who came last.
//   Dozens of parts are joined in two steps, groups of neighbours first.
// * Inside a CTA every warp streams key tiles of its own (one in 4 or 8 of the CTA's) through a ring of cp.async stages, without
//   any barrier; the warps' running maxima, sums and outputs are joined in shared memory at a unit's end.  The ring runs on
//   into the next unit meanwhile.
// * Rows are looked up one by one through the page table, by any page size; rows that are not there - behind the length, in
//   front of `first`, on a page outside the store - are filled with zeros and masked, never read.
#include <cuda_bf16.h>

#include <algorithm>

#include "kvp_paged.h"

namespace {

constexpr int kWarpsPerSm = 8;             // in CTAs of 4 or of 8
constexpr int kStages = 3;
constexpr int kStageBytes = 8192;          // K and V rows of a tile
constexpr int kUnitCost = 16;              // start and end of a unit, in key tiles of one warp
constexpr int kMinShare = 8;               // tiles that a CTA is worth starting for
constexpr int kJoin = 8;                   // parts that are read at once when a unit is joined
// Units of more than kFlat parts are joined in groups of kGroup first, groups at the same time; eight parts take 0.4 us, the
// second step 1.7.  One request of 54,000 rows: 28/4 heads 35.7 -> 29.0 us, 16/1 23.5 -> 18.3, 133,120 of 8/2
// 38.8 -> 31.2.  (kFlat 12: 2,785 rows 8.7 -> 9.6; 22: 9.5; kGroup 12, 16/1 18.3 -> 19.5.)
constexpr int kGroup = 8, kFlat = 30;
// Rows of parts that one CTA joins in the time a CTA of 4 or 8 warps takes for a tile.  A unit of t tiles in shares of s is joined
// from t/s parts of `rows` rows, and s + t/s rows/k is least at s = sqrt(t rows/k): shares are not made shorter than that - or
// than half of it, where that leaves so many parts that they are joined in groups (16/1 heads over 54,000 rows: the whole 20.6
// us, 0.7 19.7, a half 18.5, a third 19.2).  28/4 heads over 8,000 rows: 16.3 us without, 13.9 with; many or long units, whose
// shares are longer anyway, as before.  (Half of the first: 2,785 rows 8.5 -> 8.8; half or three times the second: 16/1 over
// 3 x 3,000-12,796 rows 15.3 -> 16.4, 16.5.)
constexpr float kJoin4 = 11.0f, kJoin8 = 16.0f;

template <typename T, int D> struct shape {
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kWords = kRowBytes / 16;                      // 16-byte words of a row
    static constexpr int kKeys = kStageBytes / 2 / kRowBytes;          // keys of a tile
    static_assert(kKeys <= 32, "a lane looks up a row");
};

template <int D, int W> struct smem_layout {
    static constexpr int kOut = W * kStages * kStageBytes;             // outputs of 8 rows of every warp, behind the rings
    static constexpr int kMl = kOut + W * 8 * D * 4;                   // their maxima and sums
    static constexpr int kBytes = kMl + W * 8 * 8;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 16 bytes to shared memory; without `there` zeros, and src is not read.  L2 fetches 256 bytes at a time: that is two rows of bf16
// heads of 64, the other one the next row's (pages by head: 146 requests of 674-8,335 rows, 32/8 heads, 239 us of a floor of 221)
// or another head's, which is read much later (pages by token: 339 us).
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
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    uint32_t x;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(hi), "f"(lo));
    return x;
}
// a probability pair in two bf16 numbers each, value and rounding remainder
__device__ __forceinline__ void split(float p0, float p1, uint32_t &value, uint32_t &rest)
{
    value = pack(p0, p1);
    rest = pack(p0 - __uint_as_float(value << 16), p1 - __uint_as_float(value & 0xffff0000u));
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
    const int len = min(max(a.lens[b], 0), a.room);
    first = a.first ? max(a.first[b], 0) : 0;
    return max(len - first, 0);
}

// Where on the line of all units a CTA's share lies (the host has seen to it that the line is shorter than 2^31), and a walk
// over the units that reach into it.
struct line {
    uint32_t share;
    int begin, end;
    __device__ int owner(int x) const { return (int)((uint32_t)x / share); }
};

struct piece {
    int b, u, first, rows;                 // request, unit of the request, first visible row, visible rows
    int lo, hi;                            // tiles; none for a unit without rows
    int at;                                // where the unit begins on the line
};

template <int KEYS> struct walk {
    int b, u, first, rows, tiles;
    int at;
    __device__ void request(const kvp_paged_args &a)
    {
        if (b >= a.batch) return;
        rows = visible(a, b, first);
        tiles = kvp_tiles(rows, KEYS);
    }
    // To the next unit with something to do for this CTA.  False: there is none.
    __device__ bool next(const kvp_paged_args &a, const line &ln, int units, piece &p)
    {
        while (b < a.batch && at < ln.end) {
            const int t0 = at + kUnitCost;
            p.lo = max(0, ln.begin - t0);
            p.hi = min(tiles, ln.end - t0);
            const bool mine = tiles == 0 ? at >= ln.begin : p.lo < p.hi;   // one without rows is its beginning's
            if (tiles == 0) p.lo = p.hi = 0;
            p.b = b; p.u = u; p.first = first; p.rows = rows; p.at = at;
            at = t0 + tiles;
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

// The lengths of more than 32 requests are added up by the whole CTA, a few requests per thread.  False: the CTA has no share.
template <int KEYS, int W>
__device__ __forceinline__ bool find_share(const kvp_paged_args &a, int units, float rows_per_join, line &ln, walk<KEYS> &w)
{
    __shared__ int sums[W], tops[W], found, found_at, found_len;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    auto length = [&](int b) {                             // of one of a request's units
        int f;
        return kvp_tiles(visible(a, b, f), KEYS) + kUnitCost;
    };
    auto cut = [&](int total, int longest) {               // this CTA's share of the line, of units of that length at most
        const uint32_t ctas = max(1u, min(gridDim.x, (uint32_t)total / kMinShare));
        const uint32_t even = ((uint32_t)total + ctas - 1) / ctas;
        const float least = sqrtf((float)longest * rows_per_join);
        ln.share = max(even, (uint32_t)least);
        if ((uint32_t)longest / kFlat >= ln.share) ln.share = max(even, (uint32_t)(least * 0.5f));
        if ((uint64_t)ln.share * blockIdx.x >= (uint32_t)total) return false;
        ln.begin = (int)(ln.share * blockIdx.x);
        ln.end = (int)min((uint32_t)total, ln.begin + ln.share);
        return true;
    };
    auto scan = [&](int n) {                               // of the lanes up to this one
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int x = __shfl_up_sync(0xffffffffu, n, o);
            if (lane >= o) n += x;
        }
        return n;
    };
    if (a.batch <= 32) {                                   // every warp for itself: no barrier on the way to the first rows
        const int len = lane < a.batch ? length(lane) : 0, upto = scan(len * units);
        if (!cut(__shfl_sync(0xffffffffu, upto, 31), __reduce_max_sync(0xffffffffu, len))) return false;
        const int who = __ffs(__ballot_sync(0xffffffffu, ln.begin < upto)) - 1;
        const int at = __shfl_sync(0xffffffffu, upto - len * units, who), one = __shfl_sync(0xffffffffu, len, who);
        w.b = who;
        w.u = (int)((uint32_t)(ln.begin - at) / (uint32_t)one);
        w.at = at + w.u * one;
        w.request(a);
        return true;
    }
    const int per = a.batch <= 32 * W ? 1 : (a.batch + 32 * W - 1) / (32 * W), b0 = threadIdx.x * per, b1 = min(b0 + per, a.batch);
    int mine = 0, top = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) {
        const int len = length(b);
        mine += len * units;
        top = max(top, len);
    }
    int upto = scan(mine);
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 31) {
        sums[warp] = upto;
        tops[warp] = top;
    }
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (i < warp) upto += sums[i];
        total += sums[i];
        top = max(top, tops[i]);
    }
    if (!cut(total, top)) return false;
    if (upto - mine <= ln.begin && ln.begin < upto) {      // one thread has the request that the share begins in
        int at = upto - mine;
        for (int b = b0; b < b1; ++b) {
            const int len = length(b);
            if (ln.begin < at + len * units) {
                found = b;
                found_at = at;
                found_len = len;
                break;
            }
            at += len * units;
        }
    }
    __syncthreads();
    w.b = found;
    w.u = (int)((uint32_t)(ln.begin - found_at) / (uint32_t)found_len);
    w.at = found_at + w.u * found_len;
    w.request(a);
    return true;
}

// The tiles of a warp, one after the other, through the pieces of its CTA's share: what is loaded.  Pages are looked up two
// tiles ahead, so that the table's latency is not in the way of the rows'.
template <typename T, int D, int W> struct loader {
    using S = shape<T, D>;
    walk<S::kKeys> w;
    piece p;
    int tile, turn;                        // this warp's next tile; tiles of the CTA so far, modulo the warps
    bool more;
    struct place {
        int page, row, head;               // of this lane's row in a tile; page -1: it is not there, -2: there is no tile
    } next[2];

    __device__ void start(const walk<S::kKeys> &from)
    {
        w = from;
        turn = tile = p.hi = 0;
        more = true;
    }
    __device__ void next_piece(const kvp_paged_args &a, const line &ln, int units)
    {
        const int warp = threadIdx.x / 32;
        while (more) {
            more = w.next(a, ln, units, p);
            if (!more) return;
            const int mine = p.lo + (warp + W - turn) % W;
            turn = (turn + p.hi - p.lo) % W;
            if (mine < p.hi) {
                tile = mine;
                return;
            }
        }
    }
    __device__ void look_up(const kvp_paged_args &a, const line &ln, int units, int row_tiles)
    {
        next[0] = next[1];
        place &x = next[1];
        x.page = -2;
        if (tile >= p.hi) next_piece(a, ln, units);
        if (!more) return;
        const int lane = threadIdx.x % 32;
        const uint32_t i = (uint32_t)(tile * S::kKeys) + lane;     // (a last tile may reach beyond 2^31)
        x.page = -1;
        if (lane < S::kKeys && i < (uint32_t)p.rows) {
            const int r = p.first + (int)i, col = divide(r, a.st.by_page);
            x.row = r - col * a.st.page_size;
            x.head = p.u / row_tiles;
            x.page = a.table[p.b * a.table_stride + col];
            if (x.page < 0 || x.page >= a.st.n_pages) x.page = -1;
        }
        tile += W;
    }
    // Copies the next tile to `stage` (shared address) and leaves which rows are there in *mask.
    __device__ void issue(const kvp_paged_args &a, uint32_t stage, uint32_t *mask)
    {
        const place x = next[0];
        if (x.page != -2) {
            const int lane = threadIdx.x % 32;
            // (in units that every row's place is a multiple of: 32 bits say it, whatever the size of the store)
            const uint32_t off = x.page < 0 ? 0 : (uint32_t)x.page * a.page_units + (uint32_t)x.head * a.head_units + (uint32_t)x.row * a.row_units;
            const uint32_t there = __ballot_sync(0xffffffffu, x.page >= 0);
            if (lane == 0) *mask = there;
            constexpr int N = S::kKeys * S::kWords / 32;
            const int c = lane % S::kWords;                // the same word of every row that this lane copies
            const char *k = a.st.k + c * 16, *v = a.st.v + c * 16;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = (i * 32 + lane) / S::kWords;
                const int64_t o = (int64_t)__shfl_sync(0xffffffffu, off, r) << a.unit_shift;
                const bool in = (there >> r) & 1;
                // bf16 rows are read by ldmatrix, eight rows at a time: the words of a row are permuted by its number
                const uint32_t to = stage + r * S::kRowBytes + (sizeof(T) == 2 ? c ^ (r & 7) : c) * 16;
                copy16(to, k + o, in);
                copy16(to + S::kKeys * S::kRowBytes, v + o, in);
            }
        }
        copies_commit();
    }
};

// Where column c of row r of a warp's part lies: the eight rows that a warp writes at once are permuted against one another by
// 32 bytes, else they would all fall on the same banks.
template <int D> __device__ __forceinline__ int join_at(int r, int c) { return r * D + ((c / 8) ^ r) * 8 + c % 8; }

// ---- the arithmetic of a warp ---------------------------------------------------------------------------------------

// bf16: mma.sync m16n8k16, query rows as M.  With a group of at most 8 the lower half of M is free, and takes the rounding
// remainders of the probabilities: P V with 16 bits of P in one instruction.  Wider groups take two.
// fp32 units have 8 rows, those of a group of at most 4 the arithmetic of 4.
template <typename T, int D, bool WIDE> struct tile_math;
template <typename T> __host__ __device__ constexpr int unit_rows(bool wide) { return sizeof(T) == 2 ? (wide ? 16 : 8) : (wide ? 8 : 4); }

template <int D, bool WIDE> struct tile_math<__nv_bfloat16, D, WIDE> {
    using S = shape<__nv_bfloat16, D>;
    static constexpr int kHalves = WIDE ? 2 : 1;           // rows of 8 that a thread has one of each
    uint32_t q[D / 16][2 * kHalves];
    float o[D / 8][4];
    float m[2], l[2];

    __device__ void queries(const char *q0, int64_t head_stride, int n_rows)
    {
        const int g = threadIdx.x % 32 / 4, t = threadIdx.x % 4;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const char *p = q0 + (g + 8 * h) * head_stride + (k * 16 + t * 2) * 2;
                const bool in = g + 8 * h < n_rows;
                q[k][h] = in ? *reinterpret_cast<const uint32_t *>(p) : 0u;
                q[k][h + kHalves] = in ? *reinterpret_cast<const uint32_t *>(p + 16) : 0u;
            }
        }
    }
    __device__ void begin()
    {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.0f;
    }

    __device__ void tile(uint32_t stage, uint32_t there, float scale, bool fresh)
    {
        const int lane = threadIdx.x % 32, t = lane % 4;
        constexpr int N = S::kKeys / 8;                    // 8-key columns of S
        float s[N][4], s1[N][4];                           // even and odd steps of the dot products: two chains, half as long
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i][e] = s1[i][e] = 0.0f;
        const int mi = lane / 8, mr = lane % 8;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const int row = i * 16 + (mi / 2) * 8 + mr;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                uint32_t f[4];
                ldmatrix4(stage + row * S::kRowBytes + (((k * 2 + (mi & 1)) ^ mr) * 16), f);
                const uint32_t qa[4] = {q[k][0], WIDE ? q[k][1] : 0u, q[k][kHalves], WIDE ? q[k][2 * kHalves - 1] : 0u};
                mma16816(k % 2 ? s1[2 * i] : s[2 * i], qa, f[0], f[1]);
                mma16816(k % 2 ? s1[2 * i + 1] : s[2 * i + 1], qa, f[2], f[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 2 * kHalves; ++e) s[i][e] += s1[i][e];
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
        if (__any_sync(0xffffffffu, moved) && !fresh) {      // (a unit's first tile has nothing to scale)
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
    // rows [8 half, 8 half + n), n <= 8, of this warp to shared memory: out [n][D], ml [n]
    __device__ void store(int half, int n, float *out, float2 *ml)
    {
        const int g = threadIdx.x % 32 / 4, t = threadIdx.x % 4;
        if (g >= n) return;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            float2 x;
            if (WIDE) x = half == 0 ? make_float2(o[i][0], o[i][1]) : make_float2(o[i][2], o[i][3]);
            else x = make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]);
            *reinterpret_cast<float2 *>(out + join_at<D>(g, i * 8 + t * 2)) = x;
        }
        if (t == 0) ml[g] = make_float2(m[WIDE ? half : 0], l[WIDE ? half : 0]);
    }
};

// fp32: FMA pipe, two numbers an instruction.  Q K^T: 8 lanes share a key, each with an eighth of its words, four keys at once;
// P V: a lane has D/32 columns of every row.  4 query rows, or 8 (WIDE).  Twice as many instructions, and probabilities handed
// round by shuffles, took 8 x 8,000 rows of 28/4 heads from 50.8 us to 54.0, heads of 64 from 31.6 to 35.7 (4 rows: no difference,
// DRAM).
template <int D, bool WIDE> struct tile_math<float, D, WIDE> {
    using S = shape<float, D>;
    static constexpr int R = WIDE ? 8 : 4, C = D / 32;
    f32x2 q[R][D / 16];
    f32x2 o[R / 2][C];                     // rows 2i and 2i + 1
    float m, l;                            // of row (lane % R)

    __device__ void queries(const char *q0, int64_t head_stride, int n_rows)
    {
        const int part = threadIdx.x % 8;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (r < n_rows) x = *reinterpret_cast<const float4 *>(q0 + r * head_stride + (j * 8 + part) * 16);
                q[r][2 * j] = pack2(x.x, x.y);
                q[r][2 * j + 1] = pack2(x.z, x.w);
            }
    }
    __device__ void begin()
    {
#pragma unroll
        for (int r = 0; r < R / 2; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) o[r][c] = 0;
        m = -INFINITY;
        l = 0.0f;
    }

    __device__ void tile(uint32_t stage, uint32_t there, float scale, bool fresh)
    {
        const int lane = threadIdx.x % 32, part = lane % 8, key4 = lane / 8;
        constexpr int N = S::kKeys / 4;
        float s[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f32x2 x2[R];
#pragma unroll
            for (int r = 0; r < R; ++r) x2[r] = 0;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                f32x2 k0, k1;
                asm volatile("ld.shared.v2.b64 {%0,%1}, [%2];" : "=l"(k0), "=l"(k1) : "r"(stage + (i * 4 + key4) * S::kRowBytes + (j * 8 + part) * 16) : "memory");
#pragma unroll
                for (int r = 0; r < R; ++r) x2[r] = fma2(q[r][2 * j + 1], k1, fma2(q[r][2 * j], k0, x2[r]));
            }
            float x[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float lo, hi;
                unpack2(x2[r], lo, hi);
                x[r] = lo + hi;
            }
            // the 8 lanes of a key add up; lane `part` keeps row `part % R`
            if (R == 4) {
#pragma unroll
                for (int r = 0; r < R; ++r) x[r] += __shfl_xor_sync(0xffffffffu, x[r], 4);
            }
#pragma unroll
            for (int w = R / 2; w > 0; w /= 2)
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
        if (__any_sync(0xffffffffu, moved) && !fresh) {      // (a unit's first tile has nothing to scale)
#pragma unroll
            for (int r = 0; r < R; r += 2) {
                const f32x2 f = pack2(__shfl_sync(0xffffffffu, fix, r), __shfl_sync(0xffffffffu, fix, r + 1));
#pragma unroll
                for (int c = 0; c < C; ++c) o[r / 2][c] = mul2(o[r / 2][c], f);
            }
        }
        // the probabilities go round the warp through the keys' place, which has been read: [key][row]
        __syncwarp();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = exp2_fast(s[i] - ref);
            l += p;                                        // of the keys of this lane
            if (part < R) asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage + ((i * 4 + key4) * R + part) * 4), "f"(p) : "memory");
        }
        __syncwarp();
        const uint32_t v = stage + S::kKeys * S::kRowBytes;
#pragma unroll
        for (int i = 0; i < S::kKeys; ++i) {
            f32x2 w[R / 2];
#pragma unroll
            for (int r = 0; r < R / 2; r += 2) asm volatile("ld.shared.v2.b64 {%0,%1}, [%2];" : "=l"(w[r]), "=l"(w[r + 1]) : "r"(stage + (i * R + 2 * r) * 4) : "memory");
            float x[C];
            if (C == 4)
                asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[C - 2]), "=f"(x[C - 1]) : "r"(v + i * S::kRowBytes + lane * 16) : "memory");
            else
                asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(x[0]), "=f"(x[1]) : "r"(v + i * S::kRowBytes + lane * 8) : "memory");
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const f32x2 x2 = pack2(x[c], x[c]);
#pragma unroll
                for (int r = 0; r < R / 2; ++r) o[r][c] = fma2(w[r], x2, o[r][c]);
            }
        }
    }

    __device__ void end()
    {
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
    }
    __device__ void store(int, int n, float *out, float2 *ml)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= n) break;
            float x[C], other;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (r % 2) unpack2(o[r / 2][c], other, x[c]);
                else unpack2(o[r / 2][c], x[c], other);
            }
            float *to = out + join_at<D>(r, lane * C);
            if (C == 4) *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[C - 2], x[C - 1]);
            else *reinterpret_cast<float2 *>(to) = make_float2(x[0], x[1]);
        }
        if (lane < n) ml[lane] = make_float2(m, l);
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
        x.x = pack(o.x, o.y);
        x.y = pack(o.z, o.w);
        *reinterpret_cast<uint2 *>(to) = x;
    } else {
        *reinterpret_cast<float4 *>(to) = o;
    }
    if (a.lse && c4 == 0)
        a.lse[(int64_t)b * a.n_kv * a.group + head] = l > 0.0f ? (m + log2f(l)) * 0.693147180559945309f : (l == 0.0f ? -INFINITY : l);
}

template <typename T, int D, bool WIDE, int W>
__global__ void __launch_bounds__(32 * W, kWarpsPerSm / W)
paged_attn_kernel(const __grid_constant__ kvp_paged_args a)
{
    using S = shape<T, D>;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint32_t masks[W][kStages];
    __shared__ int last;
    pdl_launch_dependents();
    const int warp = threadIdx.x / 32;
    constexpr int kUnitRows = unit_rows<T>(WIDE);
    const int row_tiles = WIDE ? (a.group + kUnitRows - 1) / kUnitRows : 1, units = a.n_kv * row_tiles;
    const float scale = a.scale * 1.44269504088896341f;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * kStages * kStageBytes;
    float *join_o = reinterpret_cast<float *>(smem + smem_layout<D, W>::kOut);
    float2 *join_ml = reinterpret_cast<float2 *>(smem + smem_layout<D, W>::kMl);
    // parameters are fetched while the kernel in front ends
    asm volatile("" ::"l"(a.lens), "l"(a.first), "l"(a.table), "l"(a.st.k), "l"(a.st.v), "l"(a.q), "r"(a.batch), "r"(a.room), "r"(units), "f"(scale));
    pdl_wait();

    line ln;
    walk<S::kKeys> w;
    if (!find_share<S::kKeys, W>(a, units, (float)min(a.group, kUnitRows) / (W == 8 ? kJoin8 : kJoin4), ln, w)) return;
    // (Code is kept short here: a CTA of a short call runs most of it once, and instructions that are not in the cache take as
    // long as the work.)
    loader<T, D, W> ld;
    ld.start(w);
#pragma unroll 1
    for (int s = -2; s < kStages - 1; ++s) {
        if (s >= 0) ld.issue(a, ring + s * kStageBytes, &masks[warp][s]);
        ld.look_up(a, ln, units, row_tiles);
    }

    int stage = 0, turn = 0, flip = 0;
    piece p = {}, p1;
    tile_math<T, D, WIDE> tm;
#pragma unroll 1
    for (bool any = false;; any = true) {
        // the next unit's queries are fetched while this one is joined
        const bool more = w.next(a, ln, units, p1);
        if (more) {
            const int rt = p1.u % row_tiles * kUnitRows;
            tm.queries(a.q + p1.b * a.q_stride[0] + (p1.u / row_tiles * a.group + rt) * a.q_stride[1], a.q_stride[1], min(kUnitRows, a.group - rt));
        }
        if (any) {
            const int rt = p.u % row_tiles * kUnitRows, head0 = p.u / row_tiles * a.group + rt, n_rows = min(kUnitRows, a.group - rt);
            [&]() {
                // the warps' parts, 8 rows at a time; a thread has 4 columns of a row
                const int tiles = kvp_tiles(p.rows, S::kKeys);
                const bool whole = p.lo == 0 && p.hi == tiles;
                const int slot = 2 * blockIdx.x + (p.lo > 0 ? 0 : 1);
                // (groups of up to four, whose units are all alike, take the two halves of the space in turn, and need no barrier
                // behind them: the next unit's lies in front of the one after)
                const bool alternate = !WIDE && n_rows <= 4;
                const int base = alternate ? (flip ^= 4) : 0;
                for (int half = 0; half * 8 < n_rows; ++half) {
                    tm.store(half, min(8, n_rows - half * 8), join_o + (warp * 8 + base) * D, join_ml + warp * 8 + base);
                    __syncthreads();
                    for (int x = threadIdx.x; x < 8 * D / 4; x += 32 * W) {
                        const int r = x / (D / 4), c4 = x % (D / 4);
                        if (half * 8 + r >= n_rows) break;
                        float m = -INFINITY;
#pragma unroll
                        for (int k = 0; k < W; ++k) m = fmaxf(m, join_ml[k * 8 + base + r].x);
                        const float ref = m == -INFINITY ? 0.0f : m;
                        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        float l = 0.0f;
#pragma unroll
                        for (int k = 0; k < W; ++k) {
                            const float2 ml = join_ml[k * 8 + base + r];
                            const float f = exp2_fast(ml.x - ref);
                            const float4 y = *reinterpret_cast<const float4 *>(join_o + (k * 8 + base) * D + join_at<D>(r, c4 * 4));
                            o.x += f * y.x; o.y += f * y.y; o.z += f * y.z; o.w += f * y.w;
                            l += f * ml.y;
                        }
                        if (whole) {
                            write_row<T, D>(a, p.b, head0 + half * 8 + r, c4, o, m, l);
                        } else {
                            const int to = slot * KVP_PAGED_ROWS + half * 8 + r;
                            reinterpret_cast<float4 *>(a.ws.part_o + to * D)[c4] = o;
                            if (c4 == 0) a.ws.part_ml[to] = make_float2(m, l);
                        }
                    }
                    if (!alternate || !whole) __syncthreads();
                }
                if (whole) return;

                // whoever's part is the last joins them
                const int t0 = p.at + kUnitCost;
                const int c0 = ln.owner(t0), n_parts = ln.owner(t0 + tiles - 1) - c0 + 1;
                auto slot_of = [&](int i) { return 2 * (c0 + i) + (i == 0); };
#pragma unroll 1
                for (bool inner = n_parts > kFlat;; inner = false) {
                    int step = !inner && n_parts > kFlat ? kGroup : 1;
                    asm volatile("" : "+r"(step));         // one join for both: made twice, it cost fp32 of 14/2 heads 4 %
                    const int i0 = inner ? ((int)blockIdx.x - c0) / kGroup * kGroup : 0;
                    const int count = inner ? min(kGroup, n_parts - i0) : (n_parts + step - 1) / step;     // parts i0, i0 + step, ...
                    // (a barrier lies behind the parts' stores: thread 0's release covers all of them, and its acquire what others released)
                    if (threadIdx.x == 0) {
                        int32_t *arrived = inner ? a.ws.arrived_group + slot_of(i0) : a.ws.arrived + p.b * units + p.u;
                        int before;
                        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(arrived) : "memory");
                        last = before == count - 1;
                        if (last) *arrived = 0;
                    }
                    __syncthreads();
                    if (!last) return;
                    // D/4 threads take a row, four columns each; each of them first weighs one part, then all add up kJoin parts at a time
                    constexpr int L = D / 4;
                    for (int x = threadIdx.x; x - (int)threadIdx.x % 32 < n_rows * L; x += 32 * W) {
                        const int r = min(x / L, n_rows - 1), c4 = x % L;
                        const int row0 = 2 * (c0 + i0) * KVP_PAGED_ROWS + r, row1 = 2 * step * KVP_PAGED_ROWS;
                        auto part = [&](int i) { return row0 + (i > 0 ? i * row1 : i0 == 0 ? KVP_PAGED_ROWS : 0); };
                        float m = -INFINITY, l = 0.0f;
                        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        for (int p0 = 0; p0 < count; p0 += L) {
                            const int n = min(L, count - p0);
                            const float2 ml = c4 < n ? __ldcg(a.ws.part_ml + part(p0 + c4)) : make_float2(-INFINITY, 0.0f);
                            float weight = 0.0f;
                            for (int k0 = 0; k0 < n; k0 += kJoin) {
                                float4 y[kJoin];
#pragma unroll
                                for (int k = 0; k < kJoin; ++k) y[k] = __ldcg(reinterpret_cast<const float4 *>(a.ws.part_o + part(p0 + min(k0 + k, n - 1)) * D) + c4);
                                if (k0 == 0) {
                                    float top = ml.x;
#pragma unroll
                                    for (int w = L / 2; w > 0; w /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                                    top = fmaxf(top, m);
                                    const float ref = top == -INFINITY ? 0.0f : top, f0 = exp2_fast(m - ref);
                                    m = top;
                                    weight = exp2_fast(ml.x - ref);
                                    float sum = weight * ml.y;
#pragma unroll
                                    for (int w = L / 2; w > 0; w /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                                    o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
                                    l = l * f0 + sum;
                                }
#pragma unroll
                                for (int k = 0; k < kJoin; ++k) {
                                    const float f = __shfl_sync(0xffffffffu, weight, (k0 + k) % L, L);
                                    if (k0 + k < n) { o.x += f * y[k].x; o.y += f * y[k].y; o.z += f * y[k].z; o.w += f * y[k].w; }
                                }
                            }
                        }
                        if (x >= n_rows * L) continue;
                        if (inner) {                                   // in the place of the group's first part
                            reinterpret_cast<float4 *>(a.ws.part_o + part(0) * D)[c4] = o;
                            if (c4 == 0) a.ws.part_ml[part(0)] = make_float2(m, l);
                        } else {
                            write_row<T, D>(a, p.b, head0 + r, c4, o, m, l);
                        }
                    }
                    if (!inner) return;
                    __syncthreads();
                }
            }();
        }
        if (!more) break;
        p = p1;
        tm.begin();
        bool fresh = true;
#pragma unroll 1
        for (int t = p.lo + (warp + W - turn) % W; t < p.hi; t += W) {
            copies_wait<kStages - 2>();
            __syncwarp();
            const int ahead = stage == 0 ? kStages - 1 : stage - 1;
            const uint32_t there = masks[warp][stage];
            ld.issue(a, ring + ahead * kStageBytes, &masks[warp][ahead]);
            ld.look_up(a, ln, units, row_tiles);
            tm.tile(ring + stage * kStageBytes, there, scale, fresh);
            fresh = false;
            stage = stage == kStages - 1 ? 0 : stage + 1;
        }
        turn = (turn + p.hi - p.lo) % W;
        tm.end();
    }
    copies_wait<0>();
}

template <typename T, int D, bool WIDE, int W>
cudaError_t launch(const kvp_paged_args &a, int64_t units, int sm_count, cudaStream_t st)
{
    // no more CTAs than the longest lists that the tables can hold are worth
    const int64_t tiles = (a.room + (int64_t)shape<T, D>::kKeys - 1) / shape<T, D>::kKeys;
    const int64_t most = std::min<int64_t>(sm_count * (kWarpsPerSm / W), units * (tiles + kUnitCost) / kMinShare);
    return launch_pdl(paged_attn_kernel<T, D, WIDE, W>, dim3((unsigned)std::max<int64_t>(1, most)), dim3(32 * W), smem_layout<D, W>::kBytes, st, a);
}

template <typename T, int D, bool WIDE>
cudaError_t launch_any(const kvp_paged_args &a, int sm_count, cudaStream_t st)
{
    constexpr int kUnitRows = unit_rows<T>(WIDE);
    const int64_t units = (int64_t)a.batch * a.n_kv * ((a.group + kUnitRows - 1) / kUnitRows);
    const int64_t tiles = units * ((a.room + (int64_t)shape<T, D>::kKeys - 1) / shape<T, D>::kKeys);
    if (tiles + units * kUnitCost > INT32_MAX) return cudaErrorInvalidValue;       // kvp_paged_fits
    // CTAs of 8 warps, one per SM, halve the parts that a unit is joined from: 8 x 8,000 rows of one kv head with 16 query heads
    // 27 -> 20 us, 133,120 rows 92.5 -> 90.0.  CTAs of 4 join within themselves more cheaply and hide one another's ends: 256 x
    // 200 rows 64 -> 48 us, 2,785 rows 9.7 -> 9.1, 16 x 16,000 rows of fp32 heads of 64 92 -> 86.  The lengths are not known
    // here; tables for long lists mean long ones.  Where they do not, tables of 133,120 rows as a recorded step has them: 433 rows
    // 7.2 -> 6.7 us, 2,785 8.8 -> 8.3, 8 x 2,000 17.9 -> 18.2, 16 x 2,000 27.6 -> 28.6, 16 x 433 11.1 -> 11.9.
    const bool eight = units < 2 * sm_count && (WIDE || (sizeof(T) == 2 && tiles >= 200ll * sm_count));
    return eight ? launch<T, D, WIDE, 8>(a, units, sm_count, st) : launch<T, D, WIDE, 4>(a, units, sm_count, st);
}

template <typename T, int D, bool WIDE, int W> cudaError_t prepare_one()
{
    return cudaFuncSetAttribute(paged_attn_kernel<T, D, WIDE, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_layout<D, W>::kBytes);
}
template <typename T, int D, bool WIDE> cudaError_t prepare()
{
    const cudaError_t e = prepare_one<T, D, WIDE, 4>();
    return e != cudaSuccess ? e : prepare_one<T, D, WIDE, 8>();
}

}  // namespace

bool kvp_paged_fits(int64_t batch, int64_t n_kv, int64_t group, int64_t room)
{
    return (double)batch * n_kv * ((group + KVP_PAGED_LEAST_ROWS - 1) / KVP_PAGED_LEAST_ROWS) * ((room + 7) / 8 + kUnitCost) <= INT32_MAX;
}

int32_t kvp_paged_ctas(int32_t sm_count) { return sm_count * kWarpsPerSm / 4; }

cudaError_t kvp_paged_attn_prepare(int32_t dtype, int32_t head_dim)
{
    cudaError_t e;
    if (dtype == KVP_DTYPE_F32) {
        e = head_dim == 128 ? prepare<float, 128, false>() : prepare<float, 64, false>();
        return e != cudaSuccess ? e : head_dim == 128 ? prepare<float, 128, true>() : prepare<float, 64, true>();
    }
    e = head_dim == 128 ? prepare<__nv_bfloat16, 128, false>() : prepare<__nv_bfloat16, 64, false>();
    return e != cudaSuccess ? e : head_dim == 128 ? prepare<__nv_bfloat16, 128, true>() : prepare<__nv_bfloat16, 64, true>();
}

template <typename T>
static cudaError_t launch_paged(const kvp_paged_args &a, int32_t head_dim, int32_t sm_count, cudaStream_t st)
{
    if (a.group <= unit_rows<T>(false))
        return head_dim == 128 ? launch_any<T, 128, false>(a, sm_count, st) : launch_any<T, 64, false>(a, sm_count, st);
    return head_dim == 128 ? launch_any<T, 128, true>(a, sm_count, st) : launch_any<T, 64, true>(a, sm_count, st);
}

cudaError_t kvp_launch_paged_attn(const kvp_paged_args &a, int32_t dtype, int32_t head_dim, int32_t sm_count, cudaStream_t st)
{
    return dtype == KVP_DTYPE_F32 ? launch_paged<float>(a, head_dim, sm_count, st) : launch_paged<__nv_bfloat16>(a, head_dim, sm_count, st);
}

// Selection of KV pages by their block keys, and attention over the selected
// pages.
#include <algorithm>

#include "common.hpp"
#include "outlets.h"
#include "paged.hpp"

namespace outlets {

namespace {

__device__ __forceinline__ double to_f64(float x) { return x; }
__device__ __forceinline__ double to_f64(__bf16 x) { return static_cast<double>(static_cast<float>(x)); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return static_cast<float>(x); }

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------- scores
// Selection is made of comparisons of s_b = max over the group's heads of
// q_h . kbar_b, and its result is defined by the 64-bit scores.  They are not
// computed for every page: scores in 32 bits (matrix instructions for bf16)
// come with a bound on their error, and only pages closer to the border than
// that bound are scored again in 64 bits.  The first pass is then bound by
// reading the block keys; at the sizes of a 512-request step (263 candidate
// pages, 59 wanted) one row in eight scores two or three pages again.
//
// Error of a 32-bit score: sums of at most 128 products, each step off by at
// most 2^-23 of the partial sum's magnitude, hence by 2^-16 sum |q k|; 2^-14
// leaves a factor of four.  Underflow is covered by the absolute term.
constexpr float kScoreErr2 = 0x1p-13f;               // twice the bound
constexpr float kScoreErrAbs = 0x1p-100f;

// What a call selects, and where its scores go.
struct SelectArgs {
    KvPages c;
    const int32_t* row_slot;
    const int32_t* positions;
    const void* q;
    int64_t ldq;
    int n_rows, G, top_k, sink, local;
    int tile;              // rows scored together where they belong to one slot
    uint64_t* keys;        // [rows, n_kv, max_pages]: 64-bit scores of crowded borders
    float* scores;         // [rows, n_kv, max_pages] (split form)
    float* bounds;         // [rows, n_kv, chunks] (split form)
    int32_t* sel;
};

// Visible pages of row r (0: none).
__device__ __forceinline__ int visible_pages(const SelectArgs& a, int r) {
    const int pos = a.positions[r], slot = a.row_slot[r];
    if (pos < 0 || slot < 0 || slot >= a.c.max_slots) return 0;
    const int nb = pos / kPage + 1;
    return nb > a.c.max_pages ? 0 : nb;
}

// The rows that the block of row r works on: the whole aligned tile for its
// first row when the tile's rows share a slot (a prompt's rows: each block
// key is then read once for all of them), none for the tile's others, and
// the row alone when they do not.
__device__ __forceinline__ int block_rows(const SelectArgs& a, int r) {
    if (a.tile == 1) return 1;
    const int r0 = r / a.tile * a.tile, r1 = min(r0 + a.tile, a.n_rows);
    bool same = true;
    for (int i = r0 + 1; i < r1; ++i) same = same && a.row_slot[i] == a.row_slot[r0];
    if (!same) return 1;
    return r == r0 ? r1 - r0 : 0;
}

constexpr int pow2_at_least(int g) { return g <= 1 ? 1 : g <= 2 ? 2 : g <= 4 ? 4 : g <= 8 ? 8 : 16; }

// Scores of pages [p0, p1) for rows r .. r + nr - 1 of one slot and KV head
// g, by the waves of the block: sc[j * ld + b] of row j and page b (all lo <= b
// < its last candidate); *bound receives the block's largest sum |q k|.
//
// bf16: v_mfma_f32_16x16x32_bf16 with the queries as A (rows: row j's head h
// at j GP + h, GP the group rounded up to a power of two with the last head
// repeated) and 16 pages as B; a lane then holds four heads of one page and
// the group's maximum takes at most two lane exchanges.  The same product of
// absolute values gives the bound.  A wave takes 64 pages at a time: one
// coalesced read of their ids, then 16 loads in flight.
template <int HD, int GP>
__device__ __forceinline__ void score_pages_bf16(const SelectArgs& a, int r, int nr, int g, int p0, int p1, float* sc,
                                                 int64_t ld, int nw, uint32_t* bound) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const __bf16* q = static_cast<const __bf16*>(a.q);
    const __bf16* keys = static_cast<const __bf16*>(a.c.block_keys);
    const int32_t* row = a.c.page_table + static_cast<int64_t>(a.row_slot[r]) * a.c.max_pages;
    bf16x8 qf[HD / 32], qm[HD / 32];
    {
        const int j = min(col / GP, nr - 1), h = min(col % GP, a.G - 1);
        const __bf16* src = q + (r + j) * a.ldq + (static_cast<int64_t>(g) * a.G + h) * HD + 8 * grp;
        const bool vec = (reinterpret_cast<uintptr_t>(q) & 15) == 0 && a.ldq % 8 == 0;
#pragma unroll
        for (int b = 0; b < HD / 32; ++b) {
            uint4 x;
            if (vec) {
                x = *reinterpret_cast<const uint4*>(src + 32 * b);
            } else {
                __bf16 e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = src[32 * b + i];
                x = *reinterpret_cast<const uint4*>(e);
            }
            qf[b] = __builtin_bit_cast(bf16x8, x);
            x.x &= 0x7FFF7FFFu; x.y &= 0x7FFF7FFFu; x.z &= 0x7FFF7FFFu; x.w &= 0x7FFF7FFFu;
            qm[b] = __builtin_bit_cast(bf16x8, x);
        }
    }
    // last candidates of the rows this lane stores
    constexpr int RL = GP >= 4 ? 1 : 4 / GP;         // rows of a lane's four values
    int hi[RL];
    const int j0 = GP >= 4 ? grp / (GP / 4) : grp * RL;
#pragma unroll
    for (int i = 0; i < RL; ++i) {
        const int nb = j0 + i < nr ? visible_pages(a, r + j0 + i) : 0;
        hi[i] = nb > a.top_k ? nb - a.local : 0;
    }
    uint32_t big = 0;
    const int tiles = (p1 - p0 + 15) / 16;
    const int t0 = tiles * w / nw, t1 = tiles * (w + 1) / nw;
    for (int t = t0; t < t1; t += 4) {
        const int mine = p0 + 16 * t + lane;
        int id = mine < p1 && 16 * t + lane < 16 * t1 ? row[mine] : -1;
        if (id >= a.c.num_pages) id = -1;
        uint4 kf[4][HD / 32];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t page = max(__shfl(id, 16 * u + col, 64), 0);
            const __bf16* src = keys + (page * a.c.n_kv + g) * HD + 8 * grp;
            if (t + u < t1)
#pragma unroll
                for (int b = 0; b < HD / 32; ++b) kf[u][b] = *reinterpret_cast<const uint4*>(src + 32 * b);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (t + u >= t1) break;
            f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, m = s;
#pragma unroll
            for (int b = 0; b < HD / 32; ++b) {
                uint4 x = kf[u][b];
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[b], __builtin_bit_cast(bf16x8, x), s, 0, 0, 0);
                x.x &= 0x7FFF7FFFu; x.y &= 0x7FFF7FFFu; x.z &= 0x7FFF7FFFu; x.w &= 0x7FFF7FFFu;
                m = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qm[b], __builtin_bit_cast(bf16x8, x), m, 0, 0, 0);
            }
            const int b = p0 + 16 * (t + u) + col;
            const bool there = __shfl(id, 16 * u + col, 64) >= 0;
            float v[RL];
#pragma unroll
            for (int i = 0; i < RL; ++i) {
                v[i] = s[i * (4 / RL)];
#pragma unroll
                for (int e = 1; e < 4 / RL; ++e) v[i] = fmaxf(v[i], s[i * (4 / RL) + e]);
                if (GP >= 8) v[i] = fmaxf(v[i], __shfl_xor(v[i], 16, 64));
                if (GP >= 16) v[i] = fmaxf(v[i], __shfl_xor(v[i], 32, 64));
                if (b >= a.sink && b < hi[i]) {
                    sc[(j0 + i) * ld + b] = there ? v[i] : -INFINITY;
                    if (there)
#pragma unroll
                        for (int e = 0; e < 4 / RL; ++e)     // as integers: NaN above infinity
                            big = max(big, __float_as_uint(m[i * (4 / RL) + e]));
                }
            }
        }
    }
    if (big) atomicMax(bound, big);
}

// fp32: 16 lanes a page, on the vector units.
template <int HD>
__device__ __forceinline__ void score_pages_f32(const SelectArgs& a, int r, int nr, int g, int p0, int p1, float* sc,
                                                int64_t ld, int nw, uint32_t* bound) {
    constexpr int LP = 16, CH = HD / LP;
    const float* q = static_cast<const float*>(a.q);
    const float* keys = static_cast<const float*>(a.c.block_keys);
    const int32_t* row = a.c.page_table + static_cast<int64_t>(a.row_slot[r]) * a.c.max_pages;
    const int ln = threadIdx.x % LP;
    uint32_t big = 0;
    for (int j = 0; j < nr; ++j) {
        const int nb = visible_pages(a, r + j), hi = nb > a.top_k ? min(nb - a.local, p1) : 0;
        for (int b = max(p0, a.sink) + static_cast<int>(threadIdx.x) / LP; b < hi; b += nw * 64 / LP) {
            const int page = row[b];
            float s = -INFINITY;
            if (page >= 0 && page < a.c.num_pages) {
                const float* kb = keys + (static_cast<int64_t>(page) * a.c.n_kv + g) * HD + ln * CH;
                float kr[CH];
#pragma unroll
                for (int e = 0; e < CH; ++e) kr[e] = kb[e];
                for (int h = 0; h < a.G; ++h) {
                    const float* qr = q + (r + j) * a.ldq + (static_cast<int64_t>(g) * a.G + h) * HD + ln * CH;
                    float x = 0.f, m = 0.f;
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        x = fmaf(kr[e], qr[e], x);
                        m = fmaf(fabsf(kr[e]), fabsf(qr[e]), m);
                    }
#pragma unroll
                    for (int o = 1; o < LP; o <<= 1) {
                        x += __shfl_xor(x, o, 64);
                        m += __shfl_xor(m, o, 64);
                    }
                    s = fmaxf(s, x);
                    big = max(big, __float_as_uint(m));
                }
            }
            if (ln == 0) sc[j * ld + b] = s;
        }
    }
    if (big) atomicMax(bound, big);
}

template <typename T, int HD, int GP>
__device__ __forceinline__ void score_pages(const SelectArgs& a, int r, int nr, int g, int p0, int p1, float* sc,
                                            int64_t ld, int nw, uint32_t* bound) {
    if constexpr (sizeof(T) == 2) score_pages_bf16<HD, GP>(a, r, nr, g, p0, p1, sc, ld, nw, bound);
    else score_pages_f32<HD>(a, r, nr, g, p0, p1, sc, ld, nw, bound);
}

// ---------------------------------------------------------------- selection
__device__ __forceinline__ int wave_inclusive(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(v, o, 64);
        if (lane >= o) v += x;
    }
    return v;
}

// Order-preserving maps of scores to unsigned keys; -0 counts as +0 and, in
// 64 bits, NaN as -infinity.
__device__ __forceinline__ uint32_t order_key(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);
    return u ^ ((u >> 31) ? ~0u : (1u << 31));
}
__device__ __forceinline__ uint64_t order_key(double s) {
    if (s != s) s = -__builtin_inf();
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
    return u ^ ((u >> 63) ? ~0ull : (1ull << 63));
}

constexpr int kNear = 256;           // candidates that are compared one with another

template <int NT>
struct PickShared {
    int hist[256];
    int red[NT / 64][2];
    float fred[NT / 64][2];
    float value[kNear];
    int index[kNear];
    double exact[kNear];
    uint64_t prefix;
    int bin, want, count, n;
    float t;
};

// Sums of a and b over the block, in every thread.
template <int NT>
__device__ __forceinline__ int2 block_sum2(int a, int b, PickShared<NT>& sh) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { a += __shfl_xor(a, o, 64); b += __shfl_xor(b, o, 64); }
    if ((threadIdx.x & 63) == 0) { sh.red[threadIdx.x >> 6][0] = a; sh.red[threadIdx.x >> 6][1] = b; }
    __syncthreads();
    int2 t = make_int2(0, 0);
    for (int i = 0; i < NT / 64; ++i) { t.x += sh.red[i][0]; t.y += sh.red[i][1]; }
    __syncthreads();
    return t;
}

// The histogram's bin (largest first) that holds the want-th entry: sh.bin,
// the rank within it in sh.want and its size in sh.count.
template <int NT>
__device__ __forceinline__ void find_bin(int want, PickShared<NT>& sh) {
    if (threadIdx.x < 64) {
        int h[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += h[j] = sh.hist[255 - 4 * threadIdx.x - j];
        int before = wave_inclusive(sum) - sum;
        if (before < want && before + sum >= want) {
            for (int j = 0; j < 4; ++j) {
                if (before + h[j] >= want) {
                    sh.bin = 255 - 4 * threadIdx.x - j;
                    sh.want = want - before;
                    sh.count = h[j];
                    break;
                }
                before += h[j];
            }
        }
    }
    __syncthreads();
}

// The want-th largest key of those that key(i, k) names for i in [lo, hi), by
// eight bits at a time; *left receives how many keys equal to it are wanted.
template <int NT, typename K, typename F>
__device__ __forceinline__ K radix_select(int lo, int hi, int want, F key, int* left, PickShared<NT>& sh) {
    K prefix = 0;
    constexpr int top = 8 * sizeof(K) - 8;
    for (int shift = top; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += NT) sh.hist[i] = 0;
        __syncthreads();
        for (int i = lo + threadIdx.x; i < hi; i += NT) {
            K k;
            if (key(i, k) && (shift == top || (k >> (shift + 8)) == (prefix >> (shift + 8))))
                atomicAdd(&sh.hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        find_bin<NT>(want, sh);
        prefix |= static_cast<K>(sh.bin) << shift;
        want = sh.want;
        __syncthreads();
    }
    *left = want;
    return prefix;
}

// 64-bit score of one page, by a wave; every lane gets it.
template <typename T, int HD>
__device__ __forceinline__ double exact_score(const KvPages& c, const T* q, int G, int g, int page) {
    double s = -__builtin_inf();
    if (page < 0 || page >= c.num_pages) return s;
    const int lane = threadIdx.x & 63;
    const T* kb = static_cast<const T*>(c.block_keys) + (static_cast<int64_t>(page) * c.n_kv + g) * HD;
    for (int h = 0; h < G; ++h) {
        double a = 0.0;
#pragma unroll
        for (int e = 0; e < HD / 64; ++e) a = fma(to_f64(kb[lane + 64 * e]), to_f64(q[h * HD + lane + 64 * e]), a);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) a += __shfl_xor(a, o, 64);
        s = a > s ? a : s;                           // NaN: never larger
    }
    return s;
}

// The selection of one row and KV head from its scores: pages below `lo`, from
// `hi` on and the `want` best between them, ascending.  Overwrites scores of
// the pages that were compared in 64 bits.  All threads of the block.
template <typename T, int HD, int NT>
__device__ void pick_row(const SelectArgs& a, int r, int g, int nb, float* sc, float bound, uint64_t* keys,
                         PickShared<NT>& sh) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int lo = a.sink, hi = nb - a.local, want = a.top_k - a.sink - a.local;
    int32_t* sel = a.sel + (static_cast<int64_t>(r) * a.c.n_kv + g) * a.top_k;
    const float d2 = bound * kScoreErr2 + kScoreErrAbs;
    float thr = INFINITY;                            // pages of at least this score are taken
    if (want > 0) {
        const bool bounded = d2 < INFINITY;          // not where a product overflows or is NaN
        float upper = 0.f, lower = 0.f;
        int need = want, crowd = hi - lo;            // of `crowd` pages near the border, `need` are taken
        if (bounded) {
            // the want-th largest score: 256 bins between the extremes (a bin
            // of a linear scale holds few pages, a bin of the first bits
            // most), then by comparison within its bin
            float mn = INFINITY, mx = -INFINITY;
            for (int i = lo + tid; i < hi; i += NT) {
                const float s = sc[i];
                mx = fmaxf(mx, s);
                if (s > -INFINITY) mn = fminf(mn, s);
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                mx = fmaxf(mx, __shfl_xor(mx, o, 64));
                mn = fminf(mn, __shfl_xor(mn, o, 64));
            }
            if (lane == 0) { sh.fred[w][0] = mx; sh.fred[w][1] = mn; }
            for (int i = tid; i < 256; i += NT) sh.hist[i] = 0;
            if (tid == 0) sh.n = 0;
            __syncthreads();
            for (int i = 0; i < NT / 64; ++i) { mx = fmaxf(mx, sh.fred[i][0]); mn = fminf(mn, sh.fred[i][1]); }
            const float scale = mx > mn ? 255.f / (mx - mn) : 0.f;
            auto bin = [&](float s) {                // nondecreasing in s
                return s > mn ? min(static_cast<int>((s - mn) * scale), 255) : 0;
            };
            for (int i = lo + tid; i < hi; i += NT) atomicAdd(&sh.hist[bin(sc[i])], 1);
            __syncthreads();
            find_bin<NT>(want, sh);
            float t;
            if (sh.count <= kNear) {
                const int B = sh.bin, rank = sh.want - 1, n = sh.count;
                for (int i = lo + tid; i < hi; i += NT) {
                    const float s = sc[i];
                    if (bin(s) == B) sh.value[atomicAdd(&sh.n, 1)] = s;
                }
                __syncthreads();
                for (int i = tid; i < n; i += NT) {
                    const float v = sh.value[i];
                    int above = 0;
                    for (int j = 0; j < n; ++j) above += sh.value[j] > v || (sh.value[j] == v && j < i);
                    if (above == rank) sh.t = v;
                }
                __syncthreads();
                t = sh.t;
            } else {
                int left;
                const uint32_t k = radix_select<NT, uint32_t>(
                    lo, hi, want, [&](int i, uint32_t& k) { k = order_key(sc[i]); return true; }, &left, sh);
                t = __uint_as_float(k ^ ((k >> 31) ? (1u << 31) : ~0u));
            }
            upper = t + d2;
            lower = t - d2;
            int in = 0, near = 0;
            for (int i = lo + tid; i < hi; i += NT) {
                const float s = sc[i];
                in += s > upper;
                near += s >= lower && !(s > upper);
            }
            const int2 sum = block_sum2<NT>(in, near, sh);
            need = want - sum.x;
            crowd = sum.y;
        }
        if (bounded && need == crowd) {
            thr = lower;
        } else {
            // the 64-bit scores of the crowd decide, ties by the page index
            auto near = [&](int i) { return !bounded || (sc[i] >= lower && !(sc[i] > upper)); };
            const T* q = static_cast<const T*>(a.q) + r * a.ldq + static_cast<int64_t>(g) * a.G * HD;
            const int32_t* row = a.c.page_table + static_cast<int64_t>(a.row_slot[r]) * a.c.max_pages;
            thr = bounded ? fmaxf(upper, -__FLT_MAX__) : 0.f;
            if (crowd <= kNear) {
                if (tid == 0) sh.n = 0;
                __syncthreads();
                for (int i = lo + tid; i < hi; i += NT)
                    if (near(i)) sh.index[atomicAdd(&sh.n, 1)] = i;
                __syncthreads();
                for (int i = w; i < crowd; i += NT / 64) {
                    const double s = exact_score<T, HD>(a.c, q, a.G, g, row[sh.index[i]]);
                    if (lane == 0) sh.exact[i] = s;
                }
                __syncthreads();
                for (int i = tid; i < crowd; i += NT) {
                    const double s = sh.exact[i];
                    int above = 0;
                    for (int j = 0; j < crowd; ++j)
                        above += sh.exact[j] > s || (sh.exact[j] == s && sh.index[j] < sh.index[i]);
                    sc[sh.index[i]] = above < need ? INFINITY : -INFINITY;
                }
                __syncthreads();
            } else {
                for (int i = lo + w; i < hi; i += NT / 64) {
                    if (!near(i)) continue;
                    const double s = exact_score<T, HD>(a.c, q, a.G, g, row[i]);
                    if (lane == 0) keys[i] = order_key(s);
                }
                __syncthreads();
                int left;
                const uint64_t k = radix_select<NT, uint64_t>(
                    lo, hi, need, [&](int i, uint64_t& k) { if (!near(i)) return false; k = keys[i]; return true; },
                    &left, sh);
                int ties = 0;
                for (int i0 = lo; i0 < hi; i0 += NT) {
                    const int i = i0 + tid;
                    const bool mine = i < hi && near(i);
                    const uint64_t x = mine ? keys[i] : 0;
                    const bool tie = mine && x == k;
                    const uint64_t tb = __ballot(tie);
                    if (lane == 0) sh.red[w][0] = __popcll(tb);
                    __syncthreads();
                    int t0 = ties;
                    for (int j = 0; j < NT / 64; ++j) {
                        if (j < w) t0 += sh.red[j][0];
                        ties += sh.red[j][0];
                    }
                    if (mine) {
                        const bool take = x > k || (tie && t0 + __popcll(tb & ((1ull << lane) - 1)) < left);
                        sc[i] = take ? INFINITY : -INFINITY;
                    }
                    __syncthreads();
                }
            }
        }
    }
    int done = 0;
    for (int b0 = 0; b0 < nb; b0 += NT) {
        const int b = b0 + tid;
        const bool take = b < nb && (b < lo || b >= hi || (want > 0 && sc[b] >= thr));
        const uint64_t m = __ballot(take);
        if (lane == 0) sh.red[w][0] = __popcll(m);
        __syncthreads();
        int at = done;
        for (int j = 0; j < NT / 64; ++j) {
            if (j < w) at += sh.red[j][0];
            done += sh.red[j][0];
        }
        if (take) sel[at + __popcll(m & ((1ull << lane) - 1))] = b;
        __syncthreads();
    }
}

// A row that reads every page it sees.
__device__ __forceinline__ void pick_all(const SelectArgs& a, int r, int g, int nb) {
    int32_t* sel = a.sel + (static_cast<int64_t>(r) * a.c.n_kv + g) * a.top_k;
    for (int i = threadIdx.x; i < a.top_k; i += blockDim.x) sel[i] = i < nb ? i : -1;
}

constexpr int kSelectThreads = 256;
constexpr int kPickThreads = 1024;
constexpr int kScorePages = 256;     // pages of a block of the split form
constexpr int kPickLdsPages = 12288; // scores of a row that are copied to LDS there (48 KB)

// One block per KV head and row (or tile of rows): scores in LDS, then the
// selection.  KV heads are the fast axis of the grid, so the blocks of one
// head share an XCD's L2 where there are eight heads, and a prompt's rows
// find the block keys there.
template <typename T, int HD, int GP>
__global__ void __launch_bounds__(kSelectThreads)
block_select_fused(SelectArgs a) {
    extern __shared__ float sc[];                    // [tile][max_pages]
    __shared__ PickShared<kSelectThreads> sh;
    __shared__ uint32_t bound;
    const int g = blockIdx.x, r = blockIdx.y;
    const int nr = block_rows(a, r);
    if (nr == 0) return;
    int most = 0;
    for (int j = 0; j < nr; ++j) most = max(most, visible_pages(a, r + j));
    if (threadIdx.x == 0) bound = 0;
    __syncthreads();
    const int ld = a.c.max_pages;
    if (most > a.top_k) {
        score_pages<T, HD, GP>(a, r, nr, g, a.sink, most - a.local, sc, ld, kSelectThreads / 64, &bound);
        __syncthreads();
    }
    for (int j = 0; j < nr; ++j) {
        const int nb = visible_pages(a, r + j);
        if (nb <= a.top_k) pick_all(a, r + j, g, nb);
        else
            pick_row<T, HD>(a, r + j, g, nb, sc + j * ld, __uint_as_float(bound),
                            a.keys + (static_cast<int64_t>(r + j) * a.c.n_kv + g) * ld, sh);
    }
}

// The split form, for few rows over long caches: scores by chunks of pages,
// then one block per row and KV head.
template <typename T, int HD, int GP>
__global__ void __launch_bounds__(kSelectThreads)
block_scores(SelectArgs a) {
    __shared__ uint32_t bound;
    const int g = blockIdx.x, r = blockIdx.y, p0 = blockIdx.z * kScorePages;
    const int nr = block_rows(a, r);
    if (nr == 0) return;
    int most = 0;
    for (int j = 0; j < nr; ++j) most = max(most, visible_pages(a, r + j));
    const int p1 = min(p0 + kScorePages, most - a.local);
    if (threadIdx.x == 0) bound = 0;
    __syncthreads();
    if (most > a.top_k && p0 < p1) {
        score_pages<T, HD, GP>(a, r, nr, g, p0, p1, a.scores + (static_cast<int64_t>(r) * a.c.n_kv + g) * a.c.max_pages,
                               static_cast<int64_t>(a.c.n_kv) * a.c.max_pages, kSelectThreads / 64, &bound);
        __syncthreads();
    }
    if (threadIdx.x < nr)
        a.bounds[(static_cast<int64_t>(r + threadIdx.x) * a.c.n_kv + g) * gridDim.z + blockIdx.z] =
            __uint_as_float(bound);
}

template <typename T, int HD, bool LDS>
__global__ void __launch_bounds__(kPickThreads)
block_pick(SelectArgs a, int chunks) {
    extern __shared__ float lds[];                   // [max_pages]
    __shared__ PickShared<kPickThreads> sh;
    __shared__ uint32_t bound;
    const int g = blockIdx.x, r = blockIdx.y, nb = visible_pages(a, r);
    if (nb <= a.top_k) {
        pick_all(a, r, g, nb);
        return;
    }
    const int64_t item = static_cast<int64_t>(r) * a.c.n_kv + g;
    float* sc = a.scores + item * a.c.max_pages;
    if (threadIdx.x == 0) bound = 0;
    __syncthreads();
    if (LDS)
        for (int i = a.sink + threadIdx.x; i < nb - a.local; i += kPickThreads) lds[i] = sc[i];
    for (int i = threadIdx.x; i < chunks; i += kPickThreads) {
        const uint32_t b = __float_as_uint(a.bounds[item * chunks + i]);
        if (b) atomicMax(&bound, b);
    }
    __syncthreads();
    if constexpr (LDS) pick_row<T, HD>(a, r, g, nb, lds, __uint_as_float(bound), a.keys + item * a.c.max_pages, sh);
    else pick_row<T, HD>(a, r, g, nb, sc, __uint_as_float(bound), a.keys + item * a.c.max_pages, sh);
}

// ---------------------------------------------------------------- attention
// Largest query heads per KV head: the columns of a 16-wide MFMA.
constexpr int kMaxGroup = 16;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Joins the states (m, l, o) that NW waves left in LDS, in wave order, for
// the G heads of an item; every thread of the block calls it.  A row without
// keys gives zeros.
template <typename T, int HD, int NW>
__device__ __forceinline__ void join_waves(int G, const float* sm, const float* sl, const float* so, const T* gate,
                                           T* out) {
    for (int e = threadIdx.x; e < G * HD; e += 64 * NW) {
        const int h = e / HD;
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sm[w * kMaxGroup + h]);
        float L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (sl[w * kMaxGroup + h] == 0.f) continue;          // a wave without keys
            const float f = fast_exp2(sm[w * kMaxGroup + h] - M);
            L = fmaf(sl[w * kMaxGroup + h], f, L);
            O = fmaf(so[w * G * HD + e], f, O);
        }
        float y = L == 0.f ? 0.f : O / L;
        if (gate) y /= 1.f + fast_exp2(-1.4426950408889634f * to_f32(gate[e]));
        out[e] = static_cast<T>(y);
    }
}

// bf16: one workgroup of NW waves per row and KV head, wave w the entries
// w, w + NW, .. of the row's list.  Per 16-key page S = K Q^T by
// v_mfma_f32_16x16x32_bf16 (the G heads in columns of B, the others zero);
// its output (lane: head l % 16, keys 4 (l / 16) + i) is the B operand of
// O^T += V^T P^T by v_mfma_f32_16x16x16_bf16, whose A operand is the
// transposed value page as it is stored, so no element changes lanes.
// Softmax statistics in fp32; the probabilities enter the second product as
// bf16 and the row sum adds the same rounded values.
template <int HD>
struct PageFrag {
    uint4 k[HD / 32];
    uint2 v[HD / 16];
};

template <int HD>
__device__ __forceinline__ void load_page(const KvPages& c, int64_t page, int g, int col, int grp, PageFrag<HD>& f) {
    const __bf16* kb = static_cast<const __bf16*>(c.k_pool) + (page * c.n_kv + g) * kPage * HD + col * HD + 8 * grp;
    const __bf16* vb = static_cast<const __bf16*>(c.v_pool) + (page * c.n_kv + g) * HD * kPage + col * kPage + 4 * grp;
#pragma unroll
    for (int b = 0; b < HD / 32; ++b) f.k[b] = *reinterpret_cast<const uint4*>(kb + 32 * b);
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) f.v[b] = *reinterpret_cast<const uint2*>(vb + 16 * kPage * b);
}

template <int HD>
__device__ __forceinline__ void add_page(int nkeys, int grp, float qscale, const bf16x8* qb, const PageFrag<HD>& f,
                                         float& m, float& l, f32x4* o) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < HD / 32; ++b)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f.k[b]), qb[b], s, 0, 0, 0);
    const bool part = nkeys < kPage;                 // wave-uniform: the page of the newest token
    if (part) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * grp + i >= nkeys) s[i] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    mx *= qscale;
    // the reference moves only when a page exceeds it by more than 8 (the
    // probabilities then stay below 2^8): most pages rescale nothing
    const bool grow = mx > m + 8.f;
    if (__any(grow)) {
        const float mn = grow ? mx : m;
        const float corr = m == mn ? 1.f : fast_exp2(m - mn);
        m = mn;
        l *= corr;
#pragma unroll
        for (int b = 0; b < HD / 16; ++b) o[b] = o[b] * corr;
    }
    const float nm = m == -INFINITY ? 0.f : -m;
    float ps = 0.f;
    s16x4 pb;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __bf16 p = static_cast<__bf16>(fast_exp2(fmaf(s[i], qscale, nm)));
        pb[i] = __builtin_bit_cast(short, p);
        ps += static_cast<float>(p);
    }
    ps += __shfl_xor(ps, 16, 64);
    ps += __shfl_xor(ps, 32, 64);
    l += ps;
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) {
        uint2 vv = f.v[b];
        if (part) {                                  // what stands behind the newest token is not read
            if (4 * grp + 0 >= nkeys) vv.x &= 0xFFFF0000u;
            if (4 * grp + 1 >= nkeys) vv.x &= 0x0000FFFFu;
            if (4 * grp + 2 >= nkeys) vv.y &= 0xFFFF0000u;
            if (4 * grp + 3 >= nkeys) vv.y &= 0x0000FFFFu;
        }
        o[b] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, vv), pb, o[b], 0, 0, 0);
    }
}

template <int HD, int NW>
__global__ void __launch_bounds__(64 * NW)
block_attend_bf16(KvPages c, const int32_t* __restrict__ row_slot, const int32_t* __restrict__ positions,
                  const __bf16* __restrict__ q, int64_t ldq, int G, const int32_t* __restrict__ sel_in, int top_k,
                  float qscale, const __bf16* __restrict__ gate, int64_t ldg, __bf16* __restrict__ out, int64_t ldo) {
    extern __shared__ __attribute__((aligned(16))) float so[];        // [NW][G][HD]
    __shared__ float sm[NW * kMaxGroup], sl[NW * kMaxGroup];
    const int64_t r = blockIdx.x;
    const int g = blockIdx.y;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const int pos = positions[r], slot = row_slot[r];
    const bool live = pos >= 0 && slot >= 0 && slot < c.max_slots && pos / kPage < c.max_pages;
    const int32_t* sel = sel_in + (r * c.n_kv + g) * top_k;
    const int32_t* row = c.page_table + static_cast<int64_t>(live ? slot : 0) * c.max_pages;
    bf16x8 qb[HD / 32];
#pragma unroll
    for (int b = 0; b < HD / 32; ++b) {
        uint4 x = *reinterpret_cast<const uint4*>(q + r * ldq + (static_cast<int64_t>(g) * G + min(col, G - 1)) * HD +
                                                  32 * b + 8 * grp);
        if (col >= G) x = make_uint4(0u, 0u, 0u, 0u);
        qb[b] = __builtin_bit_cast(bf16x8, x);
    }
    float m = -INFINITY, l = 0.f;
    f32x4 o[HD / 16];
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (live) {
        for (int e0 = 0; e0 < top_k; e0 += 64 * NW) {
            // 64 entries of this wave, one a lane; entries that are no visible
            // page of the row are dropped here
            const int e = e0 + lane * NW + w;
            const int idx = e < top_k ? sel[e] : -1;
            int page = -1;
            if (idx >= 0 && idx <= pos / kPage) page = row[idx];
            if (page >= c.num_pages) page = -1;
            uint64_t todo = __ballot(page >= 0);
            if (!todo) continue;
            PageFrag<HD> cur, nxt;
            int at = __builtin_ctzll(todo);
            todo &= todo - 1;
            load_page<HD>(c, __shfl(page, at, 64), g, col, grp, cur);
            while (true) {
                const int nx = todo ? __builtin_ctzll(todo) : at;
                load_page<HD>(c, __shfl(page, nx, 64), g, col, grp, nxt);
                add_page<HD>(pos + 1 - __shfl(idx, at, 64) * kPage, grp, qscale, qb, cur, m, l, o);
                if (!todo) break;
                todo &= todo - 1;
                at = nx;
                cur = nxt;
            }
        }
    }
    if (col < G) {
        if (grp == 0) { sm[w * kMaxGroup + col] = m; sl[w * kMaxGroup + col] = l; }
#pragma unroll
        for (int b = 0; b < HD / 16; ++b)
            *reinterpret_cast<f32x4*>(so + (w * G + col) * HD + 16 * b + 4 * grp) = o[b];
    }
    __syncthreads();
    join_waves<__bf16, HD, NW>(G, sm, sl, so, gate ? gate + r * ldg + static_cast<int64_t>(g) * G * HD : nullptr,
                               out + r * ldo + static_cast<int64_t>(g) * G * HD);
}

// fp32: the same split, on the vector units.  Scores with 4 lanes a key,
// outputs with one lane a channel; the heads one after another.
template <int HD, int NW>
__global__ void __launch_bounds__(64 * NW)
block_attend_f32(KvPages c, const int32_t* __restrict__ row_slot, const int32_t* __restrict__ positions,
                 const float* __restrict__ q, int64_t ldq, int G, const int32_t* __restrict__ sel_in, int top_k,
                 float qscale, const float* __restrict__ gate, int64_t ldg, float* __restrict__ out, int64_t ldo) {
    extern __shared__ __attribute__((aligned(16))) float so[];        // [NW][G][HD], then q [G][HD]
    __shared__ float sm[NW * kMaxGroup], sl[NW * kMaxGroup];
    float* lq = so + NW * G * HD;
    const int64_t r = blockIdx.x;
    const int g = blockIdx.y;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int pos = positions[r], slot = row_slot[r];
    const bool live = pos >= 0 && slot >= 0 && slot < c.max_slots && pos / kPage < c.max_pages;
    const int32_t* sel = sel_in + (r * c.n_kv + g) * top_k;
    const int32_t* row = c.page_table + static_cast<int64_t>(live ? slot : 0) * c.max_pages;
    for (int e = threadIdx.x; e < G * HD; e += 64 * NW) lq[e] = q[r * ldq + static_cast<int64_t>(g) * G * HD + e];
    for (int e = threadIdx.x; e < NW * G * HD; e += 64 * NW) so[e] = 0.f;
    if (threadIdx.x < NW * kMaxGroup) { sm[threadIdx.x] = -INFINITY; sl[threadIdx.x] = 0.f; }
    __syncthreads();
    constexpr int CK = HD / 4, CV = HD / 64;
    const int key = lane >> 2, part = lane & 3;
    if (live) {
        for (int e = w; e < top_k; e += NW) {
            const int idx = sel[e];
            if (idx < 0 || idx > pos / kPage) continue;
            const int page = row[idx];
            if (page < 0 || page >= c.num_pages) continue;
            const int nkeys = pos + 1 - idx * kPage;
            const int64_t base = (static_cast<int64_t>(page) * c.n_kv + g) * kPage * HD;
            const float* kp = static_cast<const float*>(c.k_pool) + base + key * HD + part * CK;
            const float* vp = static_cast<const float*>(c.v_pool) + base;
            float kr[CK], vr[CV][kPage];
#pragma unroll
            for (int i = 0; i < CK; ++i) kr[i] = kp[i];
#pragma unroll
            for (int j = 0; j < CV; ++j)
#pragma unroll
                for (int i = 0; i < kPage; ++i) vr[j][i] = i < nkeys ? vp[(lane + 64 * j) * kPage + i] : 0.f;
            for (int h = 0; h < G; ++h) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < CK; ++i) s = fmaf(kr[i], lq[h * HD + part * CK + i], s);
                s += __shfl_xor(s, 1, 64);
                s += __shfl_xor(s, 2, 64);
                s = key < nkeys ? s * qscale : -INFINITY;
                const float mo = sm[w * kMaxGroup + h], mn = fmaxf(mo, wave_max(s));
                const float ref = mn == -INFINITY ? 0.f : mn;
                const float corr = fast_exp2(mo - ref);
                const float p = fast_exp2(s - ref);
                float ps = part == 0 ? p : 0.f;
                ps = wave_sum(ps);
                sm[w * kMaxGroup + h] = mn;          // every lane the same value
                sl[w * kMaxGroup + h] = sl[w * kMaxGroup + h] * corr + ps;
#pragma unroll
                for (int j = 0; j < CV; ++j) {
                    float* dst = so + (w * G + h) * HD + lane + 64 * j;
                    float a = *dst * corr;
#pragma unroll
                    for (int i = 0; i < kPage; ++i) a = fmaf(__shfl(p, 4 * i, 64), vr[j][i], a);
                    *dst = a;
                }
            }
        }
    }
    __syncthreads();
    join_waves<float, HD, NW>(G, sm, sl, so, gate ? gate + r * ldg + static_cast<int64_t>(g) * G * HD : nullptr,
                              out + r * ldo + static_cast<int64_t>(g) * G * HD);
}

}  // namespace

static int score_chunks(const KvPages& c) { return (c.max_pages + kScorePages - 1) / kScorePages; }

int64_t block_select_ws(const KvPages& c, int64_t n_rows) {
    // 64-bit keys, 32-bit scores, bounds
    const int64_t row = c.n_kv * (static_cast<int64_t>(c.max_pages) * 12 + 4 * score_chunks(c));
    return n_rows * ((row + 15) / 16 * 16);
}

// LDS of a block's scores in the fused form: three or more blocks of a compute unit.
constexpr int kFusedBytes = 40 << 10;

void launch_block_select(const KvPages& c, const BlockRows& rows, int top_k, int sink, int local, int32_t* sel, void* ws,
                         int64_t ws_bytes, int cus, hipStream_t st) {
    const int G = rows.n_q / c.n_kv, gp = pow2_at_least(G), chunks = score_chunks(c);
    const int64_t eb = c.fmt == OUTLETS_FMT_F32 ? 4 : 2, row_bytes = block_select_ws(c, 1);
    // every row sees all it may read: no scores, no workspace
    const bool plain = c.max_pages <= top_k;
    const int slab = static_cast<int>(std::min<int64_t>(plain ? rows.n_rows : ws_bytes / row_bytes,
                                                        std::min(rows.n_rows, 32768)));     // (the grid's y)
    // Fused where a row's scores fit the LDS share and either the rows fill
    // the chip or the caches are short: otherwise few blocks read long caches.
    const bool fused = plain || (c.max_pages * 4 <= kFusedBytes &&
                                 (static_cast<int64_t>(rows.n_rows) * c.n_kv >= cus || c.max_pages <= kScorePages));
    int tile = 16 / gp;
    if (fused && !plain)
        while (tile > 1 && tile * c.max_pages * 4 > kFusedBytes) tile /= 2;
    for (int r0 = 0; r0 < rows.n_rows; r0 += slab) {
        const int n = std::min(slab, rows.n_rows - r0);
        const int64_t items = static_cast<int64_t>(n) * c.n_kv;
        uint64_t* keys = static_cast<uint64_t*>(ws);
        float* scores = plain ? nullptr : reinterpret_cast<float*>(keys + items * c.max_pages);
        const SelectArgs a{c,     rows.row_slot + r0, rows.positions + r0,
                           static_cast<const char*>(rows.q) + eb * rows.ldq * r0,
                           rows.ldq, n, G, top_k, sink, local, plain ? 1 : tile, keys, scores,
                           plain ? nullptr : scores + items * c.max_pages, sel + static_cast<int64_t>(r0) * c.n_kv * top_k};
#define OUTLETS_SELECT(T, HD, GP)                                                                                 \
    do {                                                                                                          \
        if (fused) {                                                                                              \
            hipLaunchKernelGGL((block_select_fused<T, HD, GP>), dim3(c.n_kv, n), dim3(kSelectThreads),              \
                               plain ? 0 : sizeof(float) * a.tile * c.max_pages, st, a);                            \
        } else {                                                                                                  \
            hipLaunchKernelGGL((block_scores<T, HD, GP>), dim3(c.n_kv, n, chunks), dim3(kSelectThreads), 0, st, a);   \
            OUTLETS_PICK(T, HD);                                                                                  \
        }                                                                                                         \
    } while (0)
#define OUTLETS_PICK(T, HD)                                                                                       \
    do {                                                                                                          \
        if (c.max_pages <= kPickLdsPages)                                                                         \
            hipLaunchKernelGGL((block_pick<T, HD, true>), dim3(c.n_kv, n), dim3(kPickThreads),                      \
                               sizeof(float) * c.max_pages, st, a, chunks);                                         \
        else                                                                                                      \
            hipLaunchKernelGGL((block_pick<T, HD, false>), dim3(c.n_kv, n), dim3(kPickThreads), 0, st, a, chunks);    \
    } while (0)
#define OUTLETS_SELECT_G(HD)                                                                                      \
    switch (gp) {                                                                                                 \
        case 1: OUTLETS_SELECT(__bf16, HD, 1); break;                                                             \
        case 2: OUTLETS_SELECT(__bf16, HD, 2); break;                                                             \
        case 4: OUTLETS_SELECT(__bf16, HD, 4); break;                                                             \
        case 8: OUTLETS_SELECT(__bf16, HD, 8); break;                                                             \
        default: OUTLETS_SELECT(__bf16, HD, 16); break;                                                           \
    }
        if (c.fmt == OUTLETS_FMT_F32) {
            if (c.hd == 128) OUTLETS_SELECT(float, 128, 1); else OUTLETS_SELECT(float, 64, 1);
        } else if (c.hd == 128) {
            OUTLETS_SELECT_G(128)
        } else {
            OUTLETS_SELECT_G(64)
        }
#undef OUTLETS_SELECT_G
#undef OUTLETS_PICK
#undef OUTLETS_SELECT
    }
}

int64_t block_attention_ws(const KvPages& c, int64_t n_rows, int n_q, int top_k, int cus) { return 0; }

void launch_block_attention(const KvPages& c, const BlockRows& r, const int32_t* sel, int top_k, const void* gate,
                            int64_t ldg, void* out, int64_t ldo, void* ws, int cus, hipStream_t st) {
    const int G = r.n_q / c.n_kv;
    const float qscale = 1.4426950408889634f / sqrtf(static_cast<float>(c.hd));
    constexpr int NW = 4;
    const dim3 grid(r.n_rows, c.n_kv), block(64 * NW);
#define OUTLETS_ATTEND(K, T, HD, LDS)                                                                            \
    hipLaunchKernelGGL((K<HD, NW>), grid, block, sizeof(float) * G * HD * (LDS), st, c, r.row_slot, r.positions,   \
                       static_cast<const T*>(r.q), r.ldq, G, sel, top_k, qscale, static_cast<const T*>(gate), ldg,  \
                       static_cast<T*>(out), ldo)
    if (c.fmt == OUTLETS_FMT_F32) {
        if (c.hd == 128) OUTLETS_ATTEND(block_attend_f32, float, 128, NW + 1);
        else OUTLETS_ATTEND(block_attend_f32, float, 64, NW + 1);
    } else {
        if (c.hd == 128) OUTLETS_ATTEND(block_attend_bf16, __bf16, 128, NW);
        else OUTLETS_ATTEND(block_attend_bf16, __bf16, 64, NW);
    }
#undef OUTLETS_ATTEND
}

}  // namespace outlets

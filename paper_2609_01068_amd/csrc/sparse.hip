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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Byte address for ds_bpermute: from lanes by rows of four to a product's
// order, row l % 16 and 16 bytes l / 16.
__device__ __forceinline__ int product_lane() {
    return 4 * (4 * (threadIdx.x & 15) + (threadIdx.x >> 4 & 3));
}
__device__ __forceinline__ u32x4 to_product(u32x4 x, int from) {
    u32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_ds_bpermute(from, x[e]);
    return y;
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------- scores
// Selection is made of comparisons of s_b = max over the group's heads of
// q_h . kbar_b, and its result is defined by the 64-bit scores.  They are not
// computed for every page: scores in 32 bits (matrix instructions for bf16)
// come with a bound on their error, one for all pages scored together.  A
// histogram of 256 equal bins between a row's extremes gives the border's bin.
// Where some page of that bin is closer to the border than the bound, all of the
// bin are scored again in 64 bits, or, past near_cap of them, all of it at once,
// through memory.  The first pass is then bound by reading the block keys: in the
// 512-row step (normal keys and queries, 260 candidate pages, 59 wanted) one row
// in nine scores two pages again.  Scores far from all others widen the bins:
// with one page at 30, 100 and 300 standard deviations of a request's scores
// the step takes 65, 185 and 392 us instead of 53, 445 prompt rows of 1,650
// pages 68, 301 and 570 instead of 61.
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
    int cap;               // tiles of up to so many pages are the fused form's, others the split form's
    int lds;               // scores of a row in LDS (fused form)
    int ld;                // scores of a row: max_pages, to a multiple of kPad
    uint64_t* keys;        // [rows, n_kv, ld]: 64-bit scores of crowded borders
    float* scores;         // [rows, n_kv, ld] (split form)
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
template <typename Args> __device__ __forceinline__ int block_rows(const Args& a, int r) {
    if (a.tile == 1) return 1;
    const int r0 = r / a.tile * a.tile, r1 = min(r0 + a.tile, a.n_rows);
    bool same = true;
    for (int i = r0 + 1; i < r1; ++i) same = same && a.row_slot[i] == a.row_slot[r0];
    if (!same) return 1;
    return r == r0 ? r1 - r0 : 0;
}

// Most pages that a row of r's tile sees, where the tile's rows share a slot,
// or that row r sees.
__device__ __forceinline__ int tile_pages(const SelectArgs& a, int r) {
    const int r0 = r / a.tile * a.tile, nr = block_rows(a, r0);
    if (nr == 1 && r != r0) return visible_pages(a, r);
    int most = 0;
    for (int j = 0; j < nr; ++j) most = max(most, visible_pages(a, r0 + j));
    return most;
}

constexpr int pow2_at_least(int g) { return g <= 1 ? 1 : g <= 2 ? 2 : g <= 4 ? 4 : g <= 8 ? 8 : 16; }

// Scores for rows r .. r + nr - 1 of one slot and KV head g, by one wave:
// sc[j * ld + b] of row j and page b (where it is a candidate), for `len` pages
// (at most 16 U, a multiple of 16) from p0 on, from p0 + step on, .. below p1.
// Returns the largest sum |q k| that this lane saw, as bits.
//
// bf16: v_mfma_f32_16x16x32_bf16 with the queries as A (rows: row j's head h
// at j GP + h, GP the group rounded up to a power of two with the last head
// repeated) and 16 pages as B; a lane then holds four heads of one page and
// the group's maximum takes at most two lane exchanges.  The same product of
// absolute values gives the bound.  A wave takes 16 U pages at a time: one
// coalesced read of their ids, then 4 U loads in flight (fused form, 512 rows:
// 62 us with U = 2, which leaves registers for more waves, 65 with 4; split
// form, 445 rows: 61 and 59).
template <int HD, int GP, int U>
__device__ __forceinline__ uint32_t score_pages_bf16(const SelectArgs& a, int r, int nr, int g, int p0, int len, int step,
                                                     int p1, float* sc, int64_t ld) {
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const __bf16* q = static_cast<const __bf16*>(a.q);
    const __bf16* keys = static_cast<const __bf16*>(a.c.block_keys);
    const int32_t* row = a.c.page_table + static_cast<int64_t>(a.row_slot[r]) * a.c.max_pages;
    auto ids = [&](int p) { return lane < len && p + lane < p1 ? row[p + lane] : -1; };
    int next = ids(p0);
    bf16x8 qf[HD / 32];
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
    const int from = product_lane();
    for (int p = p0; p < p1; p += step) {
        int id = next;
        next = ids(p + step);
        if (id >= a.c.num_pages) id = -1;
        u32x4 kf[U][HD / 32];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t page = max(__shfl(id, 16 * u + (lane >> 2), 64), 0);
            const __bf16* src = keys + (page * a.c.n_kv + g) * HD + 8 * (lane & 3);
#pragma unroll
            for (int b = 0; b < HD / 32; ++b) kf[u][b] = *reinterpret_cast<const u32x4*>(src + 32 * b);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (16 * u >= len || p + 16 * u >= p1) break;
            f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, m = s;
#pragma unroll
            for (int b = 0; b < HD / 32; ++b) {
                u32x4 x = to_product(kf[u][b], from);
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[b], __builtin_bit_cast(bf16x8, x), s, 0, 0, 0);
                x &= 0x7FFF7FFFu;
                const u32x4 qa = __builtin_bit_cast(u32x4, qf[b]) & 0x7FFF7FFFu;
                m = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qa), __builtin_bit_cast(bf16x8, x), m, 0, 0, 0);
            }
            const int b = p + 16 * u + col;
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
    return big;
}

// fp32: 16 lanes a page, on the vector units.
template <int HD>
__device__ __forceinline__ uint32_t score_pages_f32(const SelectArgs& a, int r, int nr, int g, int p0, int len, int step,
                                                    int p1, float* sc, int64_t ld) {
    constexpr int LP = 16, CH = HD / LP;
    const float* q = static_cast<const float*>(a.q);
    const float* keys = static_cast<const float*>(a.c.block_keys);
    const int32_t* row = a.c.page_table + static_cast<int64_t>(a.row_slot[r]) * a.c.max_pages;
    const int ln = threadIdx.x % LP;
    uint32_t big = 0;
    for (int j = 0; j < nr; ++j) {
        const int nb = visible_pages(a, r + j), hi = nb > a.top_k ? min(nb - a.local, p1) : 0;
        for (int p = p0; p < hi; p += step)
        for (int b = p + static_cast<int>(threadIdx.x & 63) / LP; b < min(p + len, hi); b += 64 / LP) {
            if (b < a.sink) continue;                // uniform over a page's lanes
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
    return big;
}

template <typename T, int HD, int GP, int U>
__device__ __forceinline__ uint32_t score_pages(const SelectArgs& a, int r, int nr, int g, int p0, int len, int step, int p1,
                                                float* sc, int64_t ld) {
    if constexpr (sizeof(T) == 2) return score_pages_bf16<HD, GP, U>(a, r, nr, g, p0, len, step, p1, sc, ld);
    else return score_pages_f32<HD>(a, r, nr, g, p0, len, step, p1, sc, ld);
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

// Order-preserving map of a score to an unsigned key above 0; -0 counts as +0
// and NaN as -infinity.
__device__ __forceinline__ uint64_t order_key(double s) {
    if (s != s) s = -__builtin_inf();
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
    return u ^ ((u >> 63) ? ~0ull : (1ull << 63));
}

// Candidates that are compared one with another: a selection by one wave
// keeps 64, by a block 256.
constexpr int near_cap(int nt) { return nt == 64 ? 64 : 256; }

// A selection runs on NT threads: a whole block, or one wave, whose LDS
// accesses are in order and need no barrier.
template <int NT>
__device__ __forceinline__ void group_sync() {
    if constexpr (NT > 64) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int NT>
struct PickShared {
    static constexpr int kNear = near_cap(NT);
    int hist[256];
    int red[NT / 64];
    float fred[NT / 64][2];
    int index[kNear];
    double exact[kNear];
    int bin, want, n, in, near;
    float t;
};

// Sum over the group, in every thread.
template <int NT>
__device__ __forceinline__ int block_sum(int a, PickShared<NT>& sh) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) a += __shfl_xor(a, o, 64);
    if (NT > 64 && (threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = a;
    group_sync<NT>();
    if (NT == 64) return a;
    a = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) a += sh.red[i];
    group_sync<NT>();
    return a;
}

// The histogram's bin (largest first) that holds the want-th entry: sh.bin,
// the rank within it in sh.want.
template <int NT>
__device__ __forceinline__ void find_bin(int want, PickShared<NT>& sh) {
    if (NT == 64 || threadIdx.x < 64) {
        const int lane = threadIdx.x & 63;
        int h[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += h[j] = sh.hist[255 - 4 * lane - j];
        int before = wave_inclusive(sum) - sum;
        if (before < want && before + sum >= want) {
            for (int j = 0; j < 4; ++j) {
                if (before + h[j] >= want) {
                    sh.bin = 255 - 4 * lane - j;
                    sh.want = want - before;
                    break;
                }
                before += h[j];
            }
        }
    }
    group_sync<NT>();
}

// The want-th largest of keys [lo, hi), by eight bits at a time; *left receives
// how many keys equal to it are wanted.
template <int NT>
__device__ __forceinline__ uint64_t radix_select(const uint64_t* keys, int lo, int hi, int want, int* left,
                                                 PickShared<NT>& sh) {
    const int tid = threadIdx.x % NT;
    uint64_t prefix = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += NT) sh.hist[i] = 0;
        group_sync<NT>();
        for (int i = lo + tid; i < hi; i += NT) {
            const uint64_t k = keys[i];
            if (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&sh.hist[(k >> shift) & 255], 1);
        }
        group_sync<NT>();
        find_bin<NT>(want, sh);
        prefix |= static_cast<uint64_t>(sh.bin) << shift;
        want = sh.want;
        group_sync<NT>();
    }
    *left = want;
    return prefix;
}

// 64-bit score of one page by 16 lanes; every one of them gets it.  Four
// heads' queries are in flight at a time.
template <typename T, int HD>
__device__ __forceinline__ double exact_score(const KvPages& c, const T* q, int G, int g, int page) {
    double s = -__builtin_inf();
    if (page < 0 || page >= c.num_pages) return s;
    constexpr int CH = HD / 16;
    const int at = (threadIdx.x & 15) * CH;
    const T* kb = static_cast<const T*>(c.block_keys) + (static_cast<int64_t>(page) * c.n_kv + g) * HD + at;
    T k[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) k[e] = kb[e];
    for (int h0 = 0; h0 < G; h0 += 4) {
        T x[4][CH];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < CH; ++e) x[j][e] = q[min(h0 + j, G - 1) * HD + at + e];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            double a = 0.0;
#pragma unroll
            for (int e = 0; e < CH; ++e) a = fma(to_f64(k[e]), to_f64(x[j][e]), a);
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) a += __shfl_xor(a, o, 64);
            s = a > s ? a : s;                       // NaN: never larger
        }
    }
    return s;
}

// Scores that a wave takes at a time; rows of scores are padded to it.
constexpr int kPad = 256;

// The scores of a row, dealt to the waves of a group in contiguous parts.
// Loops over them stay loops: a selection is a dozen short passes, and
// unrolled over scores held in registers their code did not fit the
// instruction cache (3,560 selections of 1,650 pages 35 -> 71 us).
template <int NT>
struct RowScores {
    float* sc;
    int first, end;            // the wave's pages, the last ones behind the row's

    __device__ __forceinline__ RowScores(float* scores, int nb) : sc(scores) {
        const int part = (nb + NT * 4 - 1) / (NT * 4) * kPad, padded = (nb + kPad - 1) / kPad * kPad;
        first = (threadIdx.x % NT >> 6) * part;
        end = min(first + part, padded);
    }
    // f(page, score) for every page of the wave's part, all lanes together; U
    // scores in flight (1 where the pass is rare)
    template <int U = 4, typename F> __device__ __forceinline__ void each(F f) const {
        for (int i = first + static_cast<int>(threadIdx.x & 63); i < end; i += 64 * U) {
            float v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = sc[i + 64 * u];
#pragma unroll
            for (int u = 0; u < U; ++u) f(i + 64 * u, v[u]);
        }
    }
};

// The selection of one row and KV head from its scores: pages below `lo`, from
// `hi` on and the `want` best between them, ascending.  By the NT threads of a
// group.
template <typename T, int HD, int NT>
__device__ void pick_row(const SelectArgs& a, int r, int g, int nb, float* sc, float bound, uint64_t* keys,
                         PickShared<NT>& sh) {
    const int tid = threadIdx.x % NT, lane = tid & 63, w = tid >> 6;
    constexpr int kNear = PickShared<NT>::kNear, NW = NT / 64;
    const int lo = a.sink, hi = nb - a.local, want = a.top_k - a.sink - a.local;
    int32_t* sel = a.sel + (static_cast<int64_t>(r) * a.c.n_kv + g) * a.top_k;
    const RowScores<NT> row(sc, nb);
    auto among = [&](int i) { return i >= lo && i < hi; };
    // NaN outside the candidates: no comparison takes them in, and the passes
    // need no other test (half their instructions were such tests)
    for (int i = tid; i < lo; i += NT) sc[i] = __builtin_nanf("");
    for (int i = hi + tid; i < (nb + kPad - 1) / kPad * kPad; i += NT) sc[i] = __builtin_nanf("");
    group_sync<NT>();
    const float d2 = bound * kScoreErr2 + kScoreErrAbs;
    float thr = INFINITY;                            // pages of at least this score are taken
    if (want > 0) {
        const bool bounded = d2 < INFINITY;          // not where a product overflows or is NaN
        float upper = 0.f, lower = 0.f;
        int need = want, crowd = hi - lo;            // of `crowd` pages near the border, `need` are taken
        if (bounded) {
            // the want-th largest score t, to one of 256 bins between the
            // extremes (of a linear scale: its bins hold few pages each)
            float mn = INFINITY, mx = -INFINITY;
            row.each([&](int, float s) {
                mx = fmaxf(mx, s);
                mn = fminf(mn, s == -INFINITY ? INFINITY : s);
            });
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                mx = fmaxf(mx, __shfl_xor(mx, o, 64));
                mn = fminf(mn, __shfl_xor(mn, o, 64));
            }
            if (lane == 0) { sh.fred[w][0] = mx; sh.fred[w][1] = mn; }
            for (int i = tid; i < 256; i += NT) sh.hist[i] = 0;
            if (tid == 0) sh.n = 0;
            group_sync<NT>();
#pragma unroll
            for (int i = 0; i < NW; ++i) { mx = fmaxf(mx, sh.fred[i][0]); mn = fminf(mn, sh.fred[i][1]); }
            const float scale = mx > mn ? 255.f / (mx - mn) : 0.f;
            auto bin = [&](float s) {                // nondecreasing in s
                return s > mn ? min(static_cast<int>((s - mn) * scale), 255) : 0;
            };
            row.each([&](int, float s) {
                if (s == s) atomicAdd(&sh.hist[bin(s)], 1);
            });
            group_sync<NT>();
            find_bin<NT>(want, sh);
            // that score t lies in bin B, in [lower + d2, upper - d2] (bin edges,
            // a hundredth of a bin apart to cover their rounding): pages above
            // t + d2 are in, pages below t - d2 are not, and both hold for
            // `upper` and `lower` (with d2 twice a score's error)
            const float B = static_cast<float>(sh.bin), width = (mx - mn) / 255.f;
            upper = mn + (B + 1.01f) * width + d2;
            lower = sh.bin == 0 ? -INFINITY : mn + (B - 0.01f) * width - d2;
            int in = 0;
            row.each([&](int i, float s) {
                in += s > upper;
                if (s >= lower && !(s > upper)) {
                    const int k = atomicAdd(&sh.n, 1);
                    if (k < kNear) sh.index[k] = i;
                }
            });
            need = want - block_sum<NT>(in, sh);
            crowd = sh.n;
        }
        if (bounded && need == crowd) {
            thr = lower;
        } else {
            // 64-bit scores decide where 32 bits do not, ties by the page index
            const T* q = static_cast<const T*>(a.q) + r * a.ldq + static_cast<int64_t>(g) * a.G * HD;
            const int32_t* table = a.c.page_table + static_cast<int64_t>(a.row_slot[r]) * a.c.max_pages;
            thr = bounded ? fmaxf(upper, -__FLT_MAX__) : 0.f;
            if (bounded && crowd <= kNear) {
                // t itself: the need-th largest of the crowd's 32-bit scores
                if (tid == 0) sh.in = sh.near = 0;
                for (int i = tid; i < crowd; i += NT) {
                    const float s = sc[sh.index[i]];
                    int above = 0;
                    for (int j = 0; j < crowd; ++j) {
                        const float x = sc[sh.index[j]];
                        above += x > s || (x == s && j < i);
                    }
                    if (above == need - 1) sh.t = s;
                }
                group_sync<NT>();
                const float t = sh.t;
                for (int i = tid; i < crowd; i += NT) {
                    const float s = sc[sh.index[i]];
                    if (s > t + d2) atomicAdd(&sh.in, 1);
                    else if (s >= t - d2) atomicAdd(&sh.near, 1);
                }
                group_sync<NT>();
                if (need - sh.in == sh.near) {       // no page that stays out is as near as the error
                    thr = t - d2;
                } else {
                    for (int i = tid / 16; i < crowd; i += NT / 16) {
                        const double s = exact_score<T, HD>(a.c, q, a.G, g, table[sh.index[i]]);
                        if (tid % 16 == 0) sh.exact[i] = s;
                    }
                    group_sync<NT>();
                    for (int i = tid; i < crowd; i += NT) {
                        const double s = sh.exact[i];
                        int above = 0;
                        for (int j = 0; j < crowd; ++j)
                            above += sh.exact[j] > s || (sh.exact[j] == s && sh.index[j] < sh.index[i]);
                        sc[sh.index[i]] = above < need ? INFINITY : -INFINITY;
                    }
                    group_sync<NT>();
                }
            } else {
                // keys of all candidates in memory, 0 for those that do not compete
                row.template each<1>([&](int i, float s) {
                    if (among(i)) keys[i] = !bounded || (s >= lower && !(s > upper));
                });
                __threadfence_block();
                group_sync<NT>();
                for (int i = lo + tid / 16; i < hi; i += NT / 16) {
                    if (!keys[i]) continue;
                    const double s = exact_score<T, HD>(a.c, q, a.G, g, table[i]);
                    if (tid % 16 == 0) keys[i] = order_key(s);
                }
                __threadfence_block();
                group_sync<NT>();
                int left;
                const uint64_t k = radix_select<NT>(keys, lo, hi, need, &left, sh);
                // ties in page order: first those of the waves before
                int ties = 0;
                row.template each<1>([&](int i, float) { ties += __popcll(__ballot(among(i) && keys[i] == k)); });
                if (lane == 0) sh.red[w] = ties;
                group_sync<NT>();
                ties = 0;
                for (int j = 0; j < w; ++j) ties += sh.red[j];
                row.template each<1>([&](int i, float) {
                    const bool mine = among(i) && keys[i] != 0;
                    const uint64_t x = mine ? keys[i] : 0, tb = __ballot(mine && x == k);
                    if (mine)
                        sc[i] = x > k || (x == k && ties + __popcll(tb & ((1ull << lane) - 1)) < left) ? INFINITY : -INFINITY;
                    ties += __popcll(tb);
                });
                group_sync<NT>();
            }
        }
    }
    if (want == 0) row.template each<1>([&](int i, float) { sc[i] = __builtin_nanf(""); });
    group_sync<NT>();
    for (int i = tid; i < lo; i += NT) sc[i] = INFINITY;
    for (int i = hi + tid; i < nb; i += NT) sc[i] = INFINITY;
    group_sync<NT>();
    // each wave lists its part, behind those of the waves before it
    int at = 0;
    if (NW > 1) {
        int n = 0;
        row.each([&](int, float s) { n += __popcll(__ballot(s >= thr)); });
        if (lane == 0) sh.red[w] = n;
        group_sync<NT>();
#pragma unroll
        for (int j = 0; j < NW; ++j) at += j < w ? sh.red[j] : 0;
    }
    row.each([&](int i, float s) {
        const uint64_t m = __ballot(s >= thr);
        if (s >= thr) sel[at + __builtin_amdgcn_mbcnt_hi(m >> 32, __builtin_amdgcn_mbcnt_lo(m, 0))] = i;
        at += __popcll(m);
    });
    group_sync<NT>();
}

// A row that reads every page it sees.
template <int NT>
__device__ __forceinline__ void pick_all(const SelectArgs& a, int r, int g, int nb) {
    int32_t* sel = a.sel + (static_cast<int64_t>(r) * a.c.n_kv + g) * a.top_k;
    for (int i = threadIdx.x % NT; i < a.top_k; i += NT) sel[i] = i < nb ? i : -1;
}

// Tables up to this many pages take the fused form (512 rows of 264 pages on
// average: 55 us, 86 split; 64 rows of 750: 30 and 32; 8 rows: 19 and 15).
constexpr int kFusedPages = 1024;
constexpr int kPickLdsPages = 12288; // padded scores of a row that the split form copies to LDS (48 KB)
constexpr int kUnit = 64;            // pages that a wave scores at a time

// A KV head's part of a block key (256 bytes at 128 channels) falls on few of
// an L2's channels, the same for every page, so an XCD that worked on one
// head would use a fraction of its L2: the grids below give each XCD every
// head (445 prompt rows of 1,650 pages, scores alone: 192 us by head, 75 us
// by row).
//
// Fused form: one block of four waves per KV head and row (or tile of rows),
// blocks i and i + 8, which share an XCD, taking the heads of one tile.
// Scores in LDS by all waves, then a wave per row selects (a wave per block,
// which waits for no other: 57 us against 55 for 512 rows).
template <typename T, int HD, int GP>
__global__ void __launch_bounds__(256)
block_select_fused(SelectArgs a) {
    constexpr int NW = 4;
    extern __shared__ float sc[];                    // [tile][lds]
    __shared__ PickShared<64> sh[NW];
    __shared__ uint32_t bound;
    const int w = threadIdx.x >> 6, ld = a.lds;
    const int x = blockIdx.x % 8, y = blockIdx.x / 8, g = y % a.c.n_kv;
    const int r = (y / a.c.n_kv * 8 + x) * a.tile + blockIdx.y;
    if (r >= a.n_rows) return;
    const int nr = block_rows(a, r);
    if (nr == 0) return;
    int most = 0;
    for (int j = 0; j < nr; ++j) most = max(most, visible_pages(a, r + j));
    if (most > a.cap) return;
    if (most > a.top_k) {                            // uniform over the block
        if (threadIdx.x == 0) bound = 0;
        __syncthreads();
        // equal shares of 16 pages; a wave's part begins where the last one's ends
        const int first = a.sink, end = most - a.local, tiles = (end - first + 15) / 16;
        const uint32_t big = score_pages<T, HD, GP, 2>(a, r, nr, g, first + 16 * (tiles * w / NW), 32, 32,
                                                    min(first + 16 * (tiles * (w + 1) / NW), end), sc, ld);
        if (big) atomicMax(&bound, big);
        __syncthreads();
    }
    for (int j = w; j < nr; j += NW) {
        const int nb = visible_pages(a, r + j);
        if (nb <= a.top_k) pick_all<64>(a, r + j, g, nb);
        else
            pick_row<T, HD, 64>(a, r + j, g, nb, sc + j * ld, __uint_as_float(bound),
                                a.keys + (static_cast<int64_t>(r + j) * a.c.n_kv + g) * a.ld, sh[w]);
    }
}

// Split form, for long tables: units of 64 pages dealt to gridDim.x waves (a
// multiple of 8), so that an XCD scores the same pages for all rows and heads
// and finds their block keys in its L2; then one group of threads per row and
// KV head selects: 1,024 where there are fewer groups than compute units (48
// of 3,750 to 8,192 pages: 14 us, 19 with 256, 46 with 64), 64 where there are
// four a compute unit (3,560 of 1,650 pages: 24 us, 34 with 256, 110 with
// 1,024), 256 between.
template <typename T, int HD, int GP>
__global__ void __launch_bounds__(64)
block_scores(SelectArgs a) {
    const int g = blockIdx.y, r = blockIdx.z, slices = gridDim.x;
    const int nr = block_rows(a, r);
    if (nr == 0) return;
    int most = 0;
    for (int j = 0; j < nr; ++j) most = max(most, visible_pages(a, r + j));
    if (most <= a.cap || most <= a.top_k) return;
    uint32_t big = score_pages<T, HD, GP, kUnit / 16>(a, r, nr, g, blockIdx.x * kUnit, kUnit, slices * kUnit, most - a.local,
                                          a.scores + (static_cast<int64_t>(r) * a.c.n_kv + g) * a.ld,
                                          static_cast<int64_t>(a.c.n_kv) * a.ld);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) big = max(big, __shfl_xor(big, o, 64));
    if (threadIdx.x < nr)
        a.bounds[(static_cast<int64_t>(r + threadIdx.x) * a.c.n_kv + g) * slices + blockIdx.x] = __uint_as_float(big);
}

template <typename T, int HD, int NT, bool LDS>
__global__ void __launch_bounds__(NT)
block_pick(SelectArgs a, int slices) {
    extern __shared__ float lds[];                   // [ld]
    __shared__ PickShared<NT> sh;
    __shared__ uint32_t bound;
    const int g = blockIdx.x, r = blockIdx.y, nb = visible_pages(a, r);
    if (a.cap >= 0 && tile_pages(a, r) <= a.cap) return;
    if (nb <= a.top_k) {
        pick_all<NT>(a, r, g, nb);
        return;
    }
    const int64_t item = static_cast<int64_t>(r) * a.c.n_kv + g;
    float* sc = a.scores + item * a.ld;
    if (threadIdx.x == 0) bound = 0;
    __syncthreads();
    if (LDS) {
        // eight loads in flight: other XCDs wrote the scores, each is a trip to memory
        for (int i0 = threadIdx.x; i0 < nb; i0 += 8 * NT) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = sc[min(i0 + k * NT, nb - 1)];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i0 + k * NT < nb) lds[i0 + k * NT] = v[k];
        }
    }
    for (int i = threadIdx.x; i < slices; i += NT) {
        const uint32_t b = __float_as_uint(a.bounds[item * slices + i]);
        if (b) atomicMax(&bound, b);
    }
    __syncthreads();
    uint64_t* keys = a.keys + item * a.ld;
    if constexpr (LDS) pick_row<T, HD, NT>(a, r, g, nb, lds, __uint_as_float(bound), keys, sh);
    else pick_row<T, HD, NT>(a, r, g, nb, sc, __uint_as_float(bound), keys, sh);
}

// ---------------------------------------------------------------- attention
// Largest query heads per KV head: the columns of a 16-wide MFMA.
constexpr int kMaxGroup = 16;

constexpr int kAttendWaves = 4;

// What the attention kernels share: the queries' rows, the selection and
// where the result goes: to `out`, or, where the entries of an item are split
// over gridDim.z blocks, each block's state to its record in `rec`.
struct AttendArgs {
    KvPages c;
    const int32_t* row_slot;
    const int32_t* positions;
    const void* q;
    int64_t ldq;
    int n_rows, G, top_k;
    int tile;              // rows taken together where they belong to one slot
    const int32_t* sel;
    float qscale;
    const void* gate;
    int64_t ldg;
    void* out;
    int64_t ldo;
    float* rec;            // [rows, n_kv, G, splits, HD + 2]: m, l, o
                           // (tile = 1)
};

// Output element e of an item from its running sum L and output O.  A row
// without keys gives zeros.
template <typename T, int HD>
__device__ __forceinline__ void put_output(const AttendArgs& a, int64_t r, int g, int e, float L, float O) {
    const int64_t col = static_cast<int64_t>(g) * a.G * HD + e;
    float y = L == 0.f ? 0.f : O / L;
    if (a.gate) y /= 1.f + fast_exp2(-1.4426950408889634f * to_f32(static_cast<const T*>(a.gate)[r * a.ldg + col]));
    static_cast<T*>(a.out)[r * a.ldo + col] = static_cast<T>(y);
}

// Joins the states (m, l, o) that the block's waves left in LDS, in wave order.
template <typename T, int HD>
__device__ __forceinline__ void join_waves(const AttendArgs& a, int64_t r, int g, const float* sm, const float* sl,
                                           const float* so) {
    constexpr int NW = kAttendWaves;
    for (int e = threadIdx.x; e < a.G * HD; e += 64 * NW) {
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
            O = fmaf(so[w * a.G * HD + e], f, O);
        }
        if (a.rec) {
            float* rec = a.rec + (((r * a.c.n_kv + g) * a.G + h) * gridDim.z + blockIdx.z) * (HD + 2);
            if (e % HD == 0) { rec[0] = M; rec[1] = L; }
            rec[2 + e % HD] = O;
        } else {
            put_output<T, HD>(a, r, g, e, L, O);
        }
    }
}

constexpr int kMaxSplits = 64;

// Joins the records of an item's splits, in order: one block per row and
// query head, one thread a channel.  Other XCDs wrote the records, so each
// read is a trip to memory: the weights in one, then eight outputs a trip.
template <typename T, int HD>
__global__ void __launch_bounds__(HD) join_splits(AttendArgs a, int splits) {
    const int64_t r = blockIdx.y;
    const int h = blockIdx.x, ch = threadIdx.x, lane = ch & 63;
    const float* rec = a.rec + (r * a.c.n_kv * a.G + h) * splits * (HD + 2);
    const float* mine = rec + min(lane, splits - 1) * (HD + 2);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = rec[min(k, splits - 1) * (HD + 2) + 2 + ch];
    const float m = mine[0], l = lane < splits ? mine[1] : 0.f;
    const float M = wave_max(l == 0.f ? -INFINITY : m);
    const float f = l == 0.f ? 0.f : fast_exp2(m - M);
    float L = 0.f, O = 0.f;
    for (int i = 0; i < splits; i += 8) {
        float next[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) next[k] = rec[min(i + 8 + k, splits - 1) * (HD + 2) + 2 + ch];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (i + k >= splits) break;
            const float w = __shfl(f, i + k, 64);
            L = fmaf(__shfl(l, i + k, 64), w, L);
            O = fmaf(v[k], w, O);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = next[k];
    }
    put_output<T, HD>(a, r, h / a.G, h % a.G * HD + ch, L, O);
}

// bf16: one workgroup per row and KV head (and split), whose waves take the
// entries of the row's list in turn, two pages A and B (32 keys) at a time:
// S = K Q^T by two v_mfma_f32_16x16x32_bf16 chains and O^T += V^T P^T by one
// such instruction per 16 channels.  The order of the keys in the products is
// free as long as P and V agree: row m of the first chain is token
// 8 (m / 4 % 2) + m % 4 of page m / 8, of the second the token four behind.
// Lane l (column l % 16, group l / 16) then holds, in its outputs, tokens
// 8 (group % 2) .. + 7 of page group / 2, which is its part of the B operand of
// the second product; its part of A is those tokens of one channel, 16
// bytes of the transposed value page.  No element changes lanes, and every
// load is 16 bytes a lane: with one page at a time the values came by 8, and
// rows that share pages waited for the L1's address path (219 cycles a page
// and compute unit; 445 rows of 4 slots 134 us, now 121; 509
// rows of their own 335 us, now 322).
// Softmax statistics in fp32; a probability enters the second product as the
// sum of two bf16 values, 2^-16 off at most: as one value, 2^-8 off, it was as
// large an error as the output's own rounding (one value and two, 509 rows of
// 64 pages: 320 and 320 us, 6 rows of 128: 13.8 and 14.3, 445 rows of 4 slots:
// 105 and 109).
// ONCE: the pages are not read again soon (rows of different slots):
// non-temporal loads, 509 rows of 64 pages 353 -> 335 us; where rows share
// pages they cost (445 rows of 4 slots: 241 -> 270 us).
template <bool ONCE> __device__ __forceinline__ u32x4 load16(const __bf16* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else return *reinterpret_cast<const u32x4*>(p);
}

template <int HD> struct KeyFrag { u32x4 x[2][HD / 32]; };
template <int HD> struct ValueFrag { u32x4 x[HD / 16]; };

// The keys of a pair.  ONCE: as the product takes them, lane l row l % 16 and
// 16 bytes l / 16.  Otherwise lane l holds 16 bytes l % 4 of row l / 4, and
// score_keys exchanges lanes: four neighbouring lanes then read 64
// neighbouring bytes, and a load takes the L1 17 cycles instead of 64 (445 rows
// of 4 slots 121 -> 99 us; 509 rows of their own wait for memory, 322 us
// without the exchange and 329 us with it).
template <int HD, bool ONCE>
__device__ __forceinline__ void load_keys(const KvPages& c, int page_a, int page_b, int g, int lane, KeyFrag<HD>& f) {
    const int m = ONCE ? lane & 15 : lane >> 2, chunk = ONCE ? lane >> 4 : lane & 3;
    const int64_t page = m >> 3 ? page_b : page_a;
    const __bf16* p = static_cast<const __bf16*>(c.k_pool) + (page * c.n_kv + g) * kPage * HD +
                      (8 * (m >> 2 & 1) + (m & 3)) * HD + 8 * chunk;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int b = 0; b < HD / 32; ++b) f.x[i][b] = load16<ONCE>(p + 4 * i * HD + 32 * b);
}

template <int HD, bool ONCE>
__device__ __forceinline__ void load_values(const KvPages& c, int page_a, int page_b, int g, int col, int grp,
                                            ValueFrag<HD>& f) {
    const int64_t page = grp >> 1 ? page_b : page_a;
    const __bf16* p = static_cast<const __bf16*>(c.v_pool) + (page * c.n_kv + g) * HD * kPage + col * kPage + 8 * (grp & 1);
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) f.x[b] = load16<ONCE>(p + 16 * kPage * b);
}

template <int HD, bool ONCE>
__device__ __forceinline__ void score_keys(const KeyFrag<HD>& f, const bf16x8* qb, float* s) {
    const int from = product_lane();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < HD / 32; ++b) {
            const u32x4 k = ONCE ? f.x[i][b] : to_product(f.x[i][b], from);
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), qb[b], x, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * i + e] = x[e];
    }
}

// Probabilities as the B operand of the second product: hi + lo.
struct Probs { bf16x8 hi, lo; };

// The running softmax (m, l, o) of each column with the lane's eight scores: of
// them the first `n` count (by column and page; 0 or less: none).
template <int HD>
__device__ __forceinline__ Probs add_scores(int n, float qscale, float* s, float& m, float& l, f32x4* o) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i >= n) s[i] = -INFINITY;
    float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    mx *= qscale;
    // the reference moves only when the keys exceed it by more than 8 (the
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
    Probs pb;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float p = fast_exp2(fmaf(s[i], qscale, nm));
        pb.hi[i] = static_cast<__bf16>(p);
        pb.lo[i] = static_cast<__bf16>(p - static_cast<float>(pb.hi[i]));
        ps += p;
    }
    ps += __shfl_xor(ps, 16, 64);
    ps += __shfl_xor(ps, 32, 64);
    l += ps;
    return pb;
}

// `part`: some page holds fewer than its 16 tokens, `n` of the lane's eight
// (what stands behind the newest token is not read).  `both`: the second parts
// of the probabilities too.
template <int HD>
__device__ __forceinline__ void add_values(const ValueFrag<HD>& f, bool part, int n, const Probs& pb, bool both, f32x4* o) {
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) {
        u32x4 x = f.x[b];
        if (part) {                                  // wave-uniform
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] &= (2 * e < n ? 0x0000FFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u);
        }
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), pb.hi, o[b], 0, 0, 0);
        if (both) o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), pb.lo, o[b], 0, 0, 0);
    }
}

// A wave's walk over the pages whose bit is set in `todo` (lane i: page
// `page`, index `idx` in the request), by pairs.  keys(idx) is how many tokens
// of page idx count for this lane's column, held(idx) how many it holds
// (wave-uniform).  The values of a pair are loaded while its scores are
// computed, the keys of the next one while its values are awaited.
template <int HD, bool ONCE, typename Keys, typename Held>
__device__ __forceinline__ void walk_pages(const KvPages& c, int g, uint64_t todo, int page, int idx, Keys keys, Held held,
                                           float qscale, const bf16x8* qb, bool both, float& m, float& l, f32x4* o) {
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    int a = 0, b = 0;
    bool two = false;
    auto next = [&]() {                              // the next pair, page A twice where there is one left
        a = __builtin_ctzll(todo);
        todo &= todo - 1;
        two = todo != 0;
        b = two ? __builtin_ctzll(todo) : a;
        todo &= todo - 1;
    };
    if (!todo) return;
    next();
    KeyFrag<HD> kf;
    int pa = __builtin_amdgcn_readlane(page, a), pb = __builtin_amdgcn_readlane(page, b);
    load_keys<HD, ONCE>(c, pa, pb, g, lane, kf);
    while (true) {
        ValueFrag<HD> vf;
        load_values<HD, ONCE>(c, pa, pb, g, col, grp, vf);
        float s[8];
        score_keys<HD, ONCE>(kf, qb, s);
        const int ia = __builtin_amdgcn_readlane(idx, a), ib = __builtin_amdgcn_readlane(idx, b);
        const int ha = held(ia), hb = two ? held(ib) : 0;
        const int ka = keys(ia), kb = two ? keys(ib) : 0;
        const bool more = todo != 0;
        if (more) {
            next();
            pa = __builtin_amdgcn_readlane(page, a);
            pb = __builtin_amdgcn_readlane(page, b);
            load_keys<HD, ONCE>(c, pa, pb, g, lane, kf);
        }
        const int half = 8 * (grp & 1);
        const Probs p = add_scores<HD>((grp >> 1 ? kb : ka) - half, qscale, s, m, l, o);
        add_values<HD>(vf, min(ha, hb) < kPage, (grp >> 1 ? hb : ha) - half, p, both, o);
        if (!more) break;
    }
}

// Query column `col` (of row r, head h of the group), or zeros.
template <int HD>
__device__ __forceinline__ void load_query(const AttendArgs& a, int64_t r, int g, int h, bool live, int grp, bf16x8* qb) {
    const __bf16* src = static_cast<const __bf16*>(a.q) + r * a.ldq + (static_cast<int64_t>(g) * a.G + h) * HD + 8 * grp;
#pragma unroll
    for (int b = 0; b < HD / 32; ++b) {
        uint4 x = *reinterpret_cast<const uint4*>(src + 32 * b);
        if (!live) x = make_uint4(0u, 0u, 0u, 0u);
        qb[b] = __builtin_bit_cast(bf16x8, x);
    }
}

// The slot's row of the page table, or null for a row that sees nothing.
__device__ __forceinline__ const int32_t* table_row(const AttendArgs& a, int64_t r) {
    const int pos = a.positions[r], slot = a.row_slot[r];
    const bool live = pos >= 0 && slot >= 0 && slot < a.c.max_slots && pos / kPage < a.c.max_pages;
    return live ? a.c.page_table + static_cast<int64_t>(slot) * a.c.max_pages : nullptr;
}

// Attention of one row (and split) by the block.  so: [NW][G][HD].
template <int HD, bool ONCE>
__device__ __forceinline__ void attend_row(const AttendArgs& a, int64_t r, int g, float* so, float* sm, float* sl) {
    constexpr int NW = kAttendWaves;
    const KvPages& c = a.c;
    const int G = a.G, top_k = a.top_k;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const int first = blockIdx.z * NW + w, turn = gridDim.z * NW;
    const int pos = a.positions[r];
    const int32_t* row = table_row(a, r);
    const int32_t* sel = a.sel + (r * c.n_kv + g) * top_k;
    bf16x8 qb[HD / 32];
    load_query<HD>(a, r, g, min(col, G - 1), col < G, grp, qb);
    float m, l;
    f32x4 o[HD / 16];
    // an infinite value times a second part that is 0 or negative is NaN or of the
    // other sign: a wave whose sums are not finite walks again with the first
    // parts alone
    for (bool both = true;; both = false) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < HD / 16; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int e0 = 0; row && e0 < top_k; e0 += 64 * turn) {
            // 64 entries of this wave, one a lane; entries that are no visible
            // page of the row are dropped here
            const int e = e0 + lane * turn + first;
            const int idx = e < top_k ? sel[e] : -1;
            int page = -1;
            if (idx >= 0 && idx <= pos / kPage) page = row[idx];
            if (page >= c.num_pages) page = -1;
            auto tokens = [&](int i) { return pos + 1 - i * kPage; };
            walk_pages<HD, ONCE>(c, g, __ballot(page >= 0), page, idx, tokens, tokens, a.qscale, qb, both, m, l, o);
        }
        bool finite = true;
#pragma unroll
        for (int b = 0; b < HD / 16; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) finite = finite && fabsf(o[b][e]) < INFINITY;
        if (!both || __all(finite || col >= G)) break;
    }
    if (col < G) {
        if (grp == 0) { sm[w * kMaxGroup + col] = m; sl[w * kMaxGroup + col] = l; }
#pragma unroll
        for (int b = 0; b < HD / 16; ++b)
            *reinterpret_cast<f32x4*>(so + (w * G + col) * HD + 16 * b + 4 * grp) = o[b];
    }
    __syncthreads();
    join_waves<__bf16, HD>(a, r, g, sm, sl, so);
}

// Attention of nr rows of one slot at once: the G heads of each in the columns
// of one MFMA, over the pages that any of the rows selects, read once.  A page
// weighs nothing in the columns of rows that do not select it.  Returns false,
// with nothing that counts written, where that is not the same as row by row:
// a list that names a page twice, or an output that is not finite (a value of a
// page that only other rows select may be infinite or NaN, and 0 times it is
// not 0).  The pages are taken in their order, whatever the order in which the
// rows' entries arrive, so that a call repeats its bits.  LDS: `buf` holds the
// pages' row masks and their list, then the states.
template <int HD>
__device__ __forceinline__ bool attend_tile(const AttendArgs& a, int64_t r, int nr, int g, float* buf, float* sm,
                                            float* sl) {
    constexpr int NW = kAttendWaves;
    __shared__ int listed[NW];
    const KvPages& c = a.c;
    const int G = a.G, tid = threadIdx.x;
    const int lane = tid & 63, w = tid >> 6, col = lane & 15, grp = lane >> 4;
    const int words = (c.max_pages + 1) / 2;
    uint32_t* mask = reinterpret_cast<uint32_t*>(buf);               // 16 bits a page: rows that select it
    int32_t* list = reinterpret_cast<int32_t*>(buf) + words;
    for (int i = tid; i < words; i += 64 * NW) mask[i] = 0;
    __syncthreads();
    bool twice = false;
    int last = -1;                                                   // newest position of the tile
    const int32_t* row = nullptr;
    for (int j = 0; j < nr; ++j) {
        const int32_t* tr = table_row(a, r + j);
        if (!tr) continue;
        row = tr;
        const int pos = a.positions[r + j];
        last = max(last, pos);
        const int32_t* sel = a.sel + ((r + j) * c.n_kv + g) * a.top_k;
        for (int e = tid; e < a.top_k; e += 64 * NW) {
            const int idx = sel[e];
            if (idx < 0 || idx > pos / kPage) continue;
            const uint32_t bit = 1u << (16 * (idx & 1) + j);
            const uint32_t was = atomicOr(&mask[idx >> 1], bit);
            twice = twice || (was & bit);
        }
    }
    if (__syncthreads_or(twice)) return false;
    // each wave lists its part of the words, behind those of the waves before it
    const int seen = min(words, last / (2 * kPage) + 1), part = (seen + 64 * NW - 1) / (64 * NW) * 64;
    const int end = min((w + 1) * part, seen);
    int n = 0;
    for (int i = w * part + lane; i - lane < end; i += 64) {
        const uint32_t x = i < end ? mask[i] : 0u;
        n += __popcll(__ballot(x & 0xFFFFu)) + __popcll(__ballot(x >> 16));
    }
    if (lane == 0) listed[w] = n;
    __syncthreads();
    n = 0;
    int at = 0;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
        at += v < w ? listed[v] : 0;
        n += listed[v];
    }
    for (int i = w * part + lane; i - lane < end; i += 64) {
        const uint32_t x = i < end ? mask[i] : 0u;
        const uint64_t even = __ballot(x & 0xFFFFu), odd = __ballot(x >> 16), below = (1ull << lane) - 1;
        int k = at + __popcll(even & below) + __popcll(odd & below);
        if (x & 0xFFFFu) list[k++] = 2 * i;
        if (x >> 16) list[k] = 2 * i + 1;
        at += __popcll(even) + __popcll(odd);
    }
    __syncthreads();
    const int j = min(col / G, nr - 1), h = col % G;
    const bool mine = col < nr * G;
    const int pos = mine && table_row(a, r + j) ? a.positions[r + j] : -1;
    bf16x8 qb[HD / 32];
    load_query<HD>(a, r + j, g, h, mine, grp, qb);
    float m = -INFINITY, l = 0.f;
    f32x4 o[HD / 16];
#pragma unroll
    for (int b = 0; b < HD / 16; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int e0 = 0; e0 < n; e0 += 64 * NW) {
        const int e = e0 + lane * NW + w;
        const int idx = e < n ? list[e] : -1;
        int page = idx >= 0 ? row[idx] : -1;
        if (page >= c.num_pages) page = -1;
        walk_pages<HD, false>(
            c, g, __ballot(page >= 0), page, idx,
            [&](int i) { return mask[i >> 1] >> (16 * (i & 1) + j) & 1u ? pos + 1 - i * kPage : 0; },
            [&](int i) { return last + 1 - i * kPage; }, a.qscale, qb, true, m, l, o);
    }
    __syncthreads();                                                 // the masks and the list are done with
    if (mine) {
        if (grp == 0) { sm[w * kMaxGroup + col] = m; sl[w * kMaxGroup + col] = l; }
#pragma unroll
        for (int b = 0; b < HD / 16; ++b)
            *reinterpret_cast<f32x4*>(buf + (w * nr * G + col) * HD + 16 * b + 4 * grp) = o[b];
    }
    __syncthreads();
    bool finite = true;
    for (int e = tid; e < nr * G * HD; e += 64 * NW) {
        const int x = e / HD;
        float M = -INFINITY;
#pragma unroll
        for (int v = 0; v < NW; ++v) M = fmaxf(M, sm[v * kMaxGroup + x]);
        float L = 0.f, O = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            // a wave none of whose pages the column selects still carries 0 V in o
            const float f = sl[v * kMaxGroup + x] == 0.f ? 0.f : fast_exp2(sm[v * kMaxGroup + x] - M);
            L = fmaf(sl[v * kMaxGroup + x], f, L);
            O = fmaf(buf[v * nr * G * HD + e], f, O);
        }
        finite = finite && fabsf(O) < INFINITY && fabsf(L) < INFINITY;
        put_output<__bf16, HD>(a, r + x / G, g, x % G * HD + e % HD, L, O);
    }
    return !__syncthreads_or(!finite);
}

// One block per KV head and row (or tile of rows of one slot, where `tile` is
// not 1).  KV heads are the fast axis of the grid: with eight of them, an XCD
// works on one and finds pages that rows share in its L2.
template <int HD, bool ONCE>
__global__ void __launch_bounds__(64 * kAttendWaves)
block_attend_bf16(AttendArgs a) {
    extern __shared__ __attribute__((aligned(16))) float buf[];
    __shared__ float sm[kAttendWaves * kMaxGroup], sl[kAttendWaves * kMaxGroup];
    // the tiles' first rows first: blocks with work that stand apart in the
    // grid, between empty ones, meet on a quarter of the compute units
    // (445 rows of 4 slots: 404 us, in this order 134 us)
    const int tiles = gridDim.y / a.tile;
    const int r = blockIdx.y % tiles * a.tile + blockIdx.y / tiles, g = blockIdx.x;
    if (r >= a.n_rows) return;
    const int nr = block_rows(a, r);
    if (nr == 0) return;
    if (nr > 1) {
        if (attend_tile<HD>(a, r, nr, g, buf, sm, sl)) return;
        for (int j = 0; j < nr; ++j) {
            attend_row<HD, false>(a, r + j, g, buf, sm, sl);
            __syncthreads();
        }
    } else {
        attend_row<HD, ONCE>(a, r, g, buf, sm, sl);
    }
}

// fp32: the same split, on the vector units.  Scores with 4 lanes a key,
// outputs with one lane a channel; the heads one after another.
template <int HD>
__global__ void __launch_bounds__(64 * kAttendWaves)
block_attend_f32(AttendArgs a) {
    constexpr int NW = kAttendWaves;
    extern __shared__ __attribute__((aligned(16))) float so[];        // [NW][G][HD], then q [G][HD]
    __shared__ float sm[NW * kMaxGroup], sl[NW * kMaxGroup];
    const KvPages& c = a.c;
    const float* q = static_cast<const float*>(a.q);
    const int64_t ldq = a.ldq;
    const int G = a.G, top_k = a.top_k;
    const float qscale = a.qscale;
    float* lq = so + NW * G * HD;
    const int64_t r = blockIdx.y;
    const int g = blockIdx.x;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int pos = a.positions[r], slot = a.row_slot[r];
    const bool live = pos >= 0 && slot >= 0 && slot < c.max_slots && pos / kPage < c.max_pages;
    const int32_t* sel = a.sel + (r * c.n_kv + g) * top_k;
    const int32_t* row = c.page_table + static_cast<int64_t>(live ? slot : 0) * c.max_pages;
    for (int e = threadIdx.x; e < G * HD; e += 64 * NW) lq[e] = q[r * ldq + static_cast<int64_t>(g) * G * HD + e];
    for (int e = threadIdx.x; e < NW * G * HD; e += 64 * NW) so[e] = 0.f;
    if (threadIdx.x < NW * kMaxGroup) { sm[threadIdx.x] = -INFINITY; sl[threadIdx.x] = 0.f; }
    __syncthreads();
    constexpr int CK = HD / 4, CV = HD / 64;
    const int key = lane >> 2, part = lane & 3;
    if (live) {
        for (int e = blockIdx.z * NW + w; e < top_k; e += gridDim.z * NW) {
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
                    float y = *dst * corr;
#pragma unroll
                    for (int i = 0; i < kPage; ++i) y = fmaf(__shfl(p, 4 * i, 64), vr[j][i], y);
                    *dst = y;
                }
            }
        }
    }
    __syncthreads();
    join_waves<float, HD>(a, r, g, sm, sl, so);
}

}  // namespace

// Waves that share a row's units in the split form: about three units each
// where the table is that long.
static int score_slices(const KvPages& c) { return 8 * std::max(1, (c.max_pages + kUnit - 1) / kUnit / 24); }

static int score_stride(const KvPages& c) { return (c.max_pages + kPad - 1) / kPad * kPad; }

int64_t block_select_ws(const KvPages& c, int64_t n_rows) {
    // 64-bit keys, 32-bit scores, bounds
    const int64_t row = c.n_kv * (static_cast<int64_t>(score_stride(c)) * 12 + 4 * score_slices(c));
    return n_rows * ((row + 15) / 16 * 16);
}

constexpr int kFusedBytes = 16 << 10;    // LDS of a block's scores in the fused form

void launch_block_select(const KvPages& c, const BlockRows& rows, int top_k, int sink, int local, int32_t* sel, void* ws,
                         int64_t ws_bytes, int cus, hipStream_t st) {
    const int G = rows.n_q / c.n_kv, gp = pow2_at_least(G);
    const int64_t eb = c.fmt == OUTLETS_FMT_F32 ? 4 : 2, row_bytes = block_select_ws(c, 1);
    // every row sees all it may read: no scores, no workspace
    const bool plain = c.max_pages <= top_k;
    const bool fused = plain || c.max_pages <= kFusedPages;
    // Long tables and many rows, more or less one of each slot (a decode step):
    // the rows whose caches are short take the fused form all the same
    // (8 heads of 512 rows of 264 pages at the mean, in tables of 2,048 and 8,192:
    // 90 and 158 us by the split form alone, 74 and 102 by both).  Few prompts'
    // rows beside many slots take it too, and find nothing in the fused form (445
    // rows of 4 of 512 slots: 66 us in tables of 2,049 pages, where 6 slots take
    // 64; 114 us in tables of 8,192).
    const bool both =
        !fused && rows.n_rows < 2 * c.max_slots && static_cast<int64_t>(rows.n_rows) * c.n_kv >= 4 * cus;
    // many rows are waves enough: fewer blocks for those with nothing to score
    // (the 512 rows in tables of 8,192: 115 us with 40 slices, 102 with 24, 97
    // with 16; with a quarter of them at 8,191 pages: 701, 710, 724)
    const int slices = both ? std::min(24, score_slices(c)) : score_slices(c);
    const int cap = plain ? c.max_pages : fused || both ? kFusedPages : -1;
    const int ld = score_stride(c), lds_row = std::min(ld, kFusedPages);
    // rows of one launch: the grid's z, and the threads of its x, which are
    // counted in 32 bits (fused form: 256 a row and KV head)
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(32768, (1 << 23) / c.n_kv));
    const int slab = static_cast<int>(
        std::min<int64_t>(plain ? rows.n_rows : ws_bytes / row_bytes, std::min<int64_t>(rows.n_rows, most)));
    int tile = plain ? 1 : 16 / gp;
    if (fused || both)
        while (tile > 1 && tile * lds_row * 4 > kFusedBytes) tile /= 2;
    for (int r0 = 0; r0 < rows.n_rows; r0 += slab) {
        const int n = std::min(slab, rows.n_rows - r0);
        const int64_t items = static_cast<int64_t>(n) * c.n_kv;
        uint64_t* keys = static_cast<uint64_t*>(ws);
        float* scores = plain ? nullptr : reinterpret_cast<float*>(keys + items * ld);
        const SelectArgs a{c,     rows.row_slot + r0, rows.positions + r0,
                           static_cast<const char*>(rows.q) + eb * rows.ldq * r0,
                           rows.ldq, n, G, top_k, sink, local, tile, cap, lds_row, ld, keys, scores,
                           plain ? nullptr : scores + items * ld, sel + static_cast<int64_t>(r0) * c.n_kv * top_k};
#define OUTLETS_SELECT(T, HD, GP)                                                                                 \
    do {                                                                                                          \
        const dim3 blocks((n + 8 * tile - 1) / (8 * tile) * 8 * c.n_kv, tile);                                    \
        const size_t lds = plain ? 0 : sizeof(float) * tile * lds_row;                                            \
        if (fused || both)                                                                                        \
            hipLaunchKernelGGL((block_select_fused<T, HD, GP>), blocks, dim3(256), lds, st, a);                   \
        if (!fused) {                                                                                             \
            hipLaunchKernelGGL((block_scores<T, HD, GP>), dim3(slices, c.n_kv, n), dim3(64), 0, st, a);           \
            if (items < cus) OUTLETS_PICK(T, HD, 1024);                                                           \
            else if (items < 4 * cus) OUTLETS_PICK(T, HD, 256);                                                   \
            else OUTLETS_PICK(T, HD, 64);                                                                         \
        }                                                                                                         \
    } while (0)
#define OUTLETS_PICK(T, HD, NT)                                                                                   \
    do {                                                                                                          \
        if (ld <= kPickLdsPages)                                                                                  \
            hipLaunchKernelGGL((block_pick<T, HD, NT, true>), dim3(c.n_kv, n), dim3(NT), sizeof(float) * ld, st,  \
                               a, slices);                                                                        \
        else                                                                                                      \
            hipLaunchKernelGGL((block_pick<T, HD, NT, false>), dim3(c.n_kv, n), dim3(NT), 0, st, a, slices);      \
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

// Blocks over which an item's entries are split: where there are fewer items
// than two blocks a compute unit, and as long as a wave has eight pages (six
// rows of 128 pages, 8 KV heads: 28 us on one block each, 17 us split and joined).
static int attend_splits(int64_t items, int top_k, int cus) {
    const int64_t fill = (2 * cus + items - 1) / std::max<int64_t>(items, 1);
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({fill, top_k / (8 * kAttendWaves), kMaxSplits})));
}

int64_t block_attention_ws(const KvPages& c, int64_t n_rows, int n_q, int top_k, int cus) {
    const int splits = attend_splits(n_rows * c.n_kv, top_k, cus);
    return splits == 1 ? 0 : n_rows * n_q * splits * (c.hd + 2) * static_cast<int64_t>(sizeof(float));
}

// Rows of one launch (the grid's y).
constexpr int kAttendRows = 32768;
constexpr int kTileBytes = 32 << 10;     // LDS of a tile's page masks and list

void launch_block_attention(const KvPages& c, const BlockRows& rows, const int32_t* sel, int top_k, const void* gate,
                            int64_t ldg, void* out, int64_t ldo, void* ws, int cus, hipStream_t st) {
    const int G = rows.n_q / c.n_kv;
    const int splits = attend_splits(static_cast<int64_t>(rows.n_rows) * c.n_kv, top_k, cus);
    const int64_t eb = c.fmt == OUTLETS_FMT_F32 ? 4 : 2;
    // rows taken together: as many as fill the 16 columns and whose page list
    // and masks fit the LDS that their states need (445 prompt rows, 4 together
    // in tables of up to 8,192 pages: 109 us; one by one in tables of 16,384: 244)
    int tile = c.fmt == OUTLETS_FMT_F32 || splits > 1 ? 1 : 16 / G;
    while (tile > 1 && 4 * ((c.max_pages + 1) / 2 + static_cast<int64_t>(tile) * top_k) > kTileBytes) tile /= 2;
    for (int r0 = 0; r0 < rows.n_rows; r0 += kAttendRows) {
        const int n = std::min(kAttendRows, rows.n_rows - r0);
        const AttendArgs a{c, rows.row_slot + r0, rows.positions + r0, static_cast<const char*>(rows.q) + eb * rows.ldq * r0,
                           rows.ldq, n, G, top_k, tile, sel + static_cast<int64_t>(r0) * c.n_kv * top_k,
                           1.4426950408889634f / sqrtf(static_cast<float>(c.hd)),
                           gate ? static_cast<const char*>(gate) + eb * ldg * r0 : nullptr, ldg,
                           static_cast<char*>(out) + eb * ldo * r0, ldo, splits == 1 ? nullptr : static_cast<float*>(ws)};
        const dim3 grid(c.n_kv, (n + tile - 1) / tile * tile, splits);
#define OUTLETS_ATTEND(K, T, HD, LDS)                                                                             \
    do {                                                                                                          \
        hipLaunchKernelGGL(K, grid, dim3(64 * kAttendWaves), LDS, st, a);                                         \
        if (splits > 1) hipLaunchKernelGGL((join_splits<T, HD>), dim3(rows.n_q, n), dim3(HD), 0, st, a, splits);     \
    } while (0)
        if (c.fmt == OUTLETS_FMT_F32) {
            const size_t lds = sizeof(float) * G * c.hd * (kAttendWaves + 1);
            if (c.hd == 128) OUTLETS_ATTEND(block_attend_f32<128>, float, 128, lds);
            else OUTLETS_ATTEND(block_attend_f32<64>, float, 64, lds);
        } else {
            const size_t lds = std::max<size_t>(sizeof(float) * tile * G * c.hd * kAttendWaves,
                                                tile > 1 ? 4 * ((c.max_pages + 1) / 2 + tile * top_k) : 0);
            if (splits > 1) {
                if (c.hd == 128) OUTLETS_ATTEND((block_attend_bf16<128, false>), __bf16, 128, lds);
                else OUTLETS_ATTEND((block_attend_bf16<64, false>), __bf16, 64, lds);
            } else {
                if (c.hd == 128) OUTLETS_ATTEND((block_attend_bf16<128, true>), __bf16, 128, lds);
                else OUTLETS_ATTEND((block_attend_bf16<64, true>), __bf16, 64, lds);
            }
        }
#undef OUTLETS_ATTEND
    }
}

}  // namespace outlets

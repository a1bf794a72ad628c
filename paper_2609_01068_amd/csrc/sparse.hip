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
// Order-preserving map of a score to an unsigned key; 0 is below every score.
// -0 counts as +0 and NaN as -infinity.
__device__ __forceinline__ uint64_t score_key(double s) {
    if (s != s) s = -__builtin_inf();
    s += 0.0;
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    return u ^ ((u >> 63) ? ~0ull : (1ull << 63));
}

// Pages whose scores one workgroup computes.
constexpr int kScorePages = 128;

// s_b = max over the group's heads of q_h . kbar_b, in 64 bits: a selection
// is made of comparisons, and with 64-bit sums of exact products scores that
// differ in the inputs do not tie or swap by the order of a sum.  Four lanes a
// page and head group.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
block_scores(KvPages c, int row0, const int32_t* __restrict__ row_slot, const int32_t* __restrict__ positions,
             const T* __restrict__ q, int64_t ldq, int G, int top_k, int sink, int local, int stride,
             uint64_t* __restrict__ keys) {
    extern __shared__ double lq[];                   // [G][HD]
    const int r = row0 + blockIdx.x, g = blockIdx.y, p0 = blockIdx.z * kScorePages;
    const int pos = positions[r], slot = row_slot[r];
    if (pos < 0 || slot < 0 || slot >= c.max_slots) return;
    const int nb = pos / kPage + 1;
    if (nb > c.max_pages || nb <= top_k) return;
    const int lo = max(p0, sink), hi = min(p0 + kScorePages, nb - local);
    if (lo >= hi) return;
    for (int e = threadIdx.x; e < G * HD; e += 256)
        lq[e] = to_f64(q[r * ldq + static_cast<int64_t>(g) * G * HD + e]);
    __syncthreads();
    constexpr int LP = 16, CH = HD / LP;             // lanes a page, channels a lane
    const int ln = threadIdx.x % LP;
    for (int b = p0 + threadIdx.x / LP; b < p0 + kScorePages; b += 256 / LP) {
        if (b < lo || b >= hi) continue;             // uniform over a page's lanes
        const int page = c.page_table[static_cast<int64_t>(slot) * c.max_pages + b];
        double s = -__builtin_inf();
        if (page >= 0 && page < c.num_pages) {
            const T* kb = static_cast<const T*>(c.block_keys) + (static_cast<int64_t>(page) * c.n_kv + g) * HD + ln * CH;
            double kd[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e) kd[e] = to_f64(kb[e]);
            for (int h = 0; h < G; ++h) {
                double a = 0.0;
#pragma unroll
                for (int e = 0; e < CH; ++e) a = fma(kd[e], lq[h * HD + ln * CH + e], a);
#pragma unroll
                for (int o = 1; o < LP; o <<= 1) a += __shfl_xor(a, o, 64);
                s = a > s ? a : s;                   // NaN: never larger
            }
        }
        if (ln == 0) keys[(static_cast<int64_t>(blockIdx.x) * c.n_kv + g) * stride + b] = score_key(s);
    }
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

// One workgroup per row and KV head: the m-th largest key by an eight-bit
// radix search, then the pages above it and the first ones equal to it, in
// page order.
__global__ void __launch_bounds__(256)
block_pick(KvPages c, int row0, const int32_t* __restrict__ row_slot, const int32_t* __restrict__ positions, int top_k,
           int sink, int local, int stride, const uint64_t* __restrict__ all_keys, int32_t* __restrict__ sel_out) {
    const int r = row0 + blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
    int32_t* sel = sel_out + (static_cast<int64_t>(r) * c.n_kv + g) * top_k;
    const int pos = positions[r], slot = row_slot[r];
    int nb = pos < 0 || slot < 0 || slot >= c.max_slots ? 0 : pos / kPage + 1;
    if (nb > c.max_pages) nb = 0;
    if (nb <= top_k) {
        for (int i = tid; i < top_k; i += 256) sel[i] = i < nb ? i : -1;
        return;
    }
    const uint64_t* keys = all_keys + (static_cast<int64_t>(blockIdx.x) * c.n_kv + g) * stride;
    const int lo = sink, hi = nb - local;
    int want = top_k - sink - local;                 // at most hi - lo
    __shared__ int hist[256];
    __shared__ uint64_t sh_prefix;
    __shared__ int sh_want;
    uint64_t prefix = 0;
    if (want > 0) {
        for (int shift = 56; shift >= 0; shift -= 8) {
            hist[tid] = 0;
            __syncthreads();
            for (int b = lo + tid; b < hi; b += 256) {
                const uint64_t key = keys[b];
                if (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255], 1);
            }
            __syncthreads();
            if (tid < 64) {                          // bins 255 - 4 tid .. 252 - 4 tid, largest first
                int h[4], sum = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += h[j] = hist[255 - 4 * tid - j];
                int before = wave_inclusive(sum) - sum;
                if (before < want && before + sum >= want) {
                    for (int j = 0; j < 4; ++j) {
                        if (before + h[j] >= want) {
                            sh_prefix = prefix | (static_cast<uint64_t>(255 - 4 * tid - j) << shift);
                            sh_want = want - before;
                            break;
                        }
                        before += h[j];
                    }
                }
            }
            __syncthreads();
            prefix = sh_prefix;
            want = sh_want;                          // how many of the keys equal to the prefix so far
        }
    }
    __shared__ int red[4][2];
    int done = 0, ties = 0;                          // pages written, equal keys seen
    for (int b0 = 0; b0 < nb; b0 += 256) {
        const int b = b0 + tid;
        bool take = b < nb && (b < lo || b >= hi), tie = false;
        if (b >= lo && b < hi && want > 0) {
            const uint64_t key = keys[b];
            take = key > prefix;
            tie = key == prefix;
        }
        const int w = tid >> 6, lane = tid & 63;
        const uint64_t below = (1ull << lane) - 1;
        const uint64_t tb = __ballot(tie);
        if (lane == 0) red[w][0] = __popcll(tb);
        __syncthreads();
        int t0 = ties;
        for (int i = 0; i < w; ++i) t0 += red[i][0];
        for (int i = 0; i < 4; ++i) ties += red[i][0];
        if (tie && t0 + __popcll(tb & below) < want) take = true;
        const uint64_t kb = __ballot(take);
        if (lane == 0) red[w][1] = __popcll(kb);
        __syncthreads();
        int k0 = done;
        for (int i = 0; i < w; ++i) k0 += red[i][1];
        for (int i = 0; i < 4; ++i) done += red[i][1];
        if (take) sel[k0 + __popcll(kb & below)] = b;
        __syncthreads();
    }
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

int64_t block_select_ws(const KvPages& c, int64_t n_rows) {
    return n_rows * c.n_kv * c.max_pages * static_cast<int64_t>(sizeof(uint64_t));
}

void launch_block_select(const KvPages& c, const BlockRows& r, int top_k, int sink, int local, int32_t* sel, void* ws,
                         int64_t ws_bytes, hipStream_t st) {
    const int G = r.n_q / c.n_kv;
    const int64_t row_bytes = block_select_ws(c, 1);
    const int slab = static_cast<int>(std::min<int64_t>(std::max<int64_t>(ws_bytes / row_bytes, 1), r.n_rows));
    uint64_t* keys = static_cast<uint64_t*>(ws);
    for (int r0 = 0; r0 < r.n_rows; r0 += slab) {
        const int n = std::min(slab, r.n_rows - r0);
        if (c.max_pages > top_k) {
            const dim3 grid(n, c.n_kv, (c.max_pages + kScorePages - 1) / kScorePages);
#define OUTLETS_SCORES(T, HD)                                                                                     \
    hipLaunchKernelGGL((block_scores<T, HD>), grid, dim3(256), sizeof(double) * G * HD, st, c, r0, r.row_slot,      \
                       r.positions, static_cast<const T*>(r.q), r.ldq, G, top_k, sink, local, c.max_pages, keys)
            if (c.fmt == OUTLETS_FMT_F32) {
                if (c.hd == 128) OUTLETS_SCORES(float, 128); else OUTLETS_SCORES(float, 64);
            } else {
                if (c.hd == 128) OUTLETS_SCORES(__bf16, 128); else OUTLETS_SCORES(__bf16, 64);
            }
#undef OUTLETS_SCORES
        }
        hipLaunchKernelGGL(block_pick, dim3(n, c.n_kv), dim3(256), 0, st, c, r0, r.row_slot, r.positions, top_k, sink,
                           local, c.max_pages, keys, sel);
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

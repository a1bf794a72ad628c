// Page tables kept on the GPU, and the write into the paged cache.
#include <algorithm>

#include "common.hpp"
#include "outlets.h"
#include "paged.hpp"

namespace outlets {

namespace {

constexpr int kAppendThreads = 1024;
// Calls up to these sizes run in one workgroup with their lists in LDS: one
// launch and no round trip through memory between its phases.
constexpr int kSmallReqs = 1024;
constexpr int kSmallRows = 4096;

__device__ __forceinline__ int wave_inclusive(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(v, o, 64);
        if (lane >= o) v += x;
    }
    return v;
}

// Exclusive prefix sums of a and b over the workgroup; *ta and *tb receive
// the totals.  Sums of page and token counts that passed the checks fit 31 bits.
__device__ __forceinline__ void block_scan2(int& a, int& b, int* ta, int* tb, int (*red)[2]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    constexpr int NW = kAppendThreads / 64;
    const int ia = wave_inclusive(a), ib = wave_inclusive(b);
    if (lane == 63) { red[w][0] = ia; red[w][1] = ib; }
    __syncthreads();
    int pa = 0, pb = 0, sa = 0, sb = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        if (i == w) { pa = sa; pb = sb; }
        sa += red[i][0];
        sb += red[i][1];
    }
    __syncthreads();
    a = pa + ia - a;
    b = pb + ib - b;
    *ta = sa;
    *tb = sb;
}

// Word i of the free bitmap, without bits behind the last page.
__device__ __forceinline__ uint32_t free_word(const PageState& s, int i) {
    const int left = s.num_pages - i * 32;
    return s.free_bits[i] & (left >= 32 ? ~0u : (1u << left) - 1u);
}

// What a row needs of its request.
struct AppendReq {
    int slot, old, base, cu;     // base: rank of its first new page
};

// Row r of an accepted call: its request by binary search over the first
// rows, its page from the table or, for a new page, from the list of pages
// taken (rank order), which is entered into the table by the page's first row.
__device__ __forceinline__ void append_row(const PageState& s, int r, int n_req, int T, const AppendReq* reqs,
                                           const int32_t* list, int32_t* slot_map, int32_t* positions,
                                           int32_t* row_slot) {
    int sm = -1, ps = -1, rs = -1;
    if (r < T) {
        int lo = 0, hi = n_req;              // the last request whose first row is <= r has rows
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (reqs[mid].cu <= r) lo = mid; else hi = mid;
        }
        const AppendReq q = reqs[lo];
        ps = q.old + (r - q.cu);
        rs = q.slot;
        const int idx = ps / kPage, have = (q.old + kPage - 1) / kPage;
        const int64_t at = static_cast<int64_t>(q.slot) * s.max_pages + idx;
        int page;
        if (idx < have) {
            page = s.page_table[at];
        } else {
            page = list[q.base + idx - have];
            if (ps % kPage == 0) s.page_table[at] = page;
        }
        sm = page < 0 ? -1 : page * kPage + ps % kPage;
    }
    slot_map[r] = sm;
    positions[r] = ps;
    row_slot[r] = rs;
}

// One workgroup: checks, prefix sums over the requests, and the lowest free
// pages by rank.  Lowest-first order is a prefix sum of the bitmap's
// population counts, so no list of free pages is kept between calls.  Bound
// by the latency of its few dependent passes (a call moves a few hundred KB
// at most).  SMALL: requests and pages in LDS and the rows here as well;
// otherwise both in `ws` and the rows by append_rows.
template <bool SMALL>
__global__ void __launch_bounds__(kAppendThreads)
pages_append(PageState s, int n_req, const int32_t* __restrict__ slots, const int32_t* __restrict__ new_tokens,
             int n_rows, int32_t* __restrict__ cu, int32_t* __restrict__ slot_map, int32_t* __restrict__ positions,
             int32_t* __restrict__ row_slot, int32_t* __restrict__ status, AppendReq* ws_reqs, int32_t* ws_list) {
    extern __shared__ uint32_t marks[];
    __shared__ int red[kAppendThreads / 64][2];
    __shared__ AppendReq l_reqs[SMALL ? kSmallReqs : 1];
    __shared__ int32_t l_list[SMALL ? kSmallRows : 1];
    AppendReq* reqs = SMALL ? l_reqs : ws_reqs;
    int32_t* list = SMALL ? l_list : ws_list;
    const int tid = threadIdx.x;
    const int mwords = (s.max_slots + 31) / 32, words = (s.num_pages + 31) / 32;

    // the bitmap's first words, while the requests are looked at (8,192 words:
    // 262,144 pages)
    constexpr int KEEP = 8;
    uint32_t kept[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const int i = k * kAppendThreads + tid;
        kept[k] = i < words ? free_word(s, i) : 0u;
    }
    for (int i = tid; i < mwords; i += kAppendThreads) marks[i] = 0;
    __syncthreads();

    // the requests
    int64_t T64 = 0, N64 = 0;
    bool bad = false;
    for (int c = 0; c < n_req; c += kAppendThreads) {
        const int i = c + tid;
        int slot = -1, t = 0, old = 0, need = 0;
        if (i < n_req) {
            slot = slots[i];
            if (slot >= 0 && slot < s.max_slots) {
                if (atomicOr(&marks[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1u) bad = true;
                t = new_tokens[i];
                old = s.seq_len[slot];
                if (t < 0 || old < 0 || old > s.max_seq_len || t > s.max_seq_len - old || t > n_rows) {
                    bad = true;
                    t = 0;
                }
                need = (old + t + kPage - 1) / kPage - (old + kPage - 1) / kPage;
            } else if (slot != -1) {
                bad = true;
            }
        }
        // a chunk's sums fit 31 bits: at most 1024 terms of n_rows <= kPageMaxRows
        if (__syncthreads_or(bad)) break;
        int tc = t, nc = need, tt, tn;
        block_scan2(tc, nc, &tt, &tn, red);
        if (T64 + tt > n_rows) { bad = true; break; }
        if (i < n_req) reqs[i] = AppendReq{slot, old, static_cast<int>(N64) + nc, static_cast<int>(T64) + tc};
        T64 += tt;
        N64 += tn;
    }
    const int any_bad = __syncthreads_or(bad);
    const int T = static_cast<int>(T64), N = static_cast<int>(N64);

    // free pages in all
    int cnt = 0;
#pragma unroll
    for (int k = 0; k < KEEP; ++k) cnt += __popc(kept[k]);
    for (int i = KEEP * kAppendThreads + tid; i < words; i += kAppendThreads) cnt += __popc(free_word(s, i));
    int zero = 0, n_free, dummy;
    block_scan2(cnt, zero, &n_free, &dummy, red);
    int done = 0;
    const int rc = any_bad ? OUTLETS_ERR_INVALID_ARG : (N > n_free ? OUTLETS_ERR_OUT_OF_PAGES : OUTLETS_OK);
    if (tid == 0) {
        status[0] = rc;
        status[1] = rc ? 0 : T;
        status[2] = rc ? 0 : N;
        status[3] = rc ? n_free : n_free - N;
    }
    if (rc) {
        for (int i = tid; i <= n_req; i += kAppendThreads) cu[i] = 0;
        if (SMALL)
            for (int r = tid; r < n_rows; r += kAppendThreads) slot_map[r] = positions[r] = row_slot[r] = -1;
        return;
    }

    // the N lowest free pages: ranks by prefix sums over the words, then a
    // lane per bit, so that neighbouring lanes store neighbouring ranks
    auto take = [&](int c, uint32_t w) {             // words c + tid
        int rank = __popc(w), z = 0, total;
        block_scan2(rank, z, &total, &dummy, red);
        rank += done;
        const int lane = tid & 63;
        const uint64_t some = __ballot(w != 0 && rank < N);
        const int last = some ? 63 - __builtin_clzll(some) : -1;
        for (int i = 0; i <= last; i += 2) {
            const int j = i + (lane >> 5), b = lane & 31;
            const uint32_t x = __shfl(w, j, 64);
            const int at = __shfl(rank, j, 64) + __popc(x & ((1u << b) - 1u));
            if ((x >> b & 1u) && at < N) list[at] = (c + (tid & ~63) + j) * 32 + b;
        }
        if (w && rank < N) {
            uint32_t left = 0;                       // all taken, or all but those from rank N on
            if (rank + __popc(w) > N) {
                left = w;
                for (int k = rank; k < N; ++k) left &= left - 1;
            }
            s.free_bits[c + tid] = left;
        }
        done += total;
    };
    uint32_t next = kept[0];
    for (int c = 0; c < words && done < N; c += kAppendThreads) {
        take(c, next);
        const int i = c + kAppendThreads + tid;
        next = i < words ? free_word(s, i) : 0u;
    }
    __syncthreads();
    for (int i = tid; i < n_req; i += kAppendThreads) {
        const AppendReq q = reqs[i];
        const int next = i + 1 < n_req ? reqs[i + 1].cu : T;
        cu[i] = q.cu;
        if (q.slot >= 0 && next > q.cu) s.seq_len[q.slot] = q.old + next - q.cu;
    }
    if (tid == 0) cu[n_req] = T;
    if (SMALL)
        for (int r = tid; r < n_rows; r += kAppendThreads)
            append_row(s, r, n_req, T, reqs, list, slot_map, positions, row_slot);
}

__global__ void __launch_bounds__(256)
append_rows(PageState s, int n_req, int n_rows, const AppendReq* __restrict__ reqs, const int32_t* __restrict__ list,
            const int32_t* __restrict__ status, int32_t* __restrict__ slot_map, int32_t* __restrict__ positions,
            int32_t* __restrict__ row_slot) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r < n_rows) append_row(s, r, n_req, status[1], reqs, list, slot_map, positions, row_slot);
}

// One block per request.  Every block checks all slots (a few KB), so that a
// refused call changes nothing and needs no launch of its own for the check.
constexpr int kReleaseThreads = 512;
__global__ void __launch_bounds__(kReleaseThreads)
pages_release(PageState s, int n, const int32_t* __restrict__ slots, int32_t* __restrict__ status) {
    extern __shared__ uint32_t marks[];
    const int mwords = (s.max_slots + 31) / 32;
    for (int i = threadIdx.x; i < mwords; i += kReleaseThreads) marks[i] = 0;
    __syncthreads();
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += kReleaseThreads) {
        const int slot = slots[i];
        if (slot >= 0 && slot < s.max_slots) {
            if (atomicOr(&marks[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1u) bad = true;
        } else if (slot != -1) {
            bad = true;
        }
    }
    bad = __syncthreads_or(bad);
    if (blockIdx.x == 0 && threadIdx.x == 0) status[0] = bad ? OUTLETS_ERR_INVALID_ARG : OUTLETS_OK;
    if (bad || static_cast<int>(blockIdx.x) >= n) return;
    const int slot = slots[blockIdx.x];
    if (slot < 0) return;
    const int len = min(max(s.seq_len[slot], 0), s.max_seq_len), held = (len + kPage - 1) / kPage;
    int32_t* row = s.page_table + static_cast<int64_t>(slot) * s.max_pages;
    for (int i = threadIdx.x; i < held; i += kReleaseThreads) {
        const int page = row[i];
        if (page >= 0 && page < s.num_pages) atomicOr(&s.free_bits[page >> 5], 1u << (page & 31));
        row[i] = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0) s.seq_len[slot] = 0;
}

__global__ void __launch_bounds__(256) pages_reset(PageState s) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, step = static_cast<int64_t>(gridDim.x) * 256;
    const int words = (s.num_pages + 31) / 32;
    for (int64_t j = i; j < words; j += step) {
        const int left = s.num_pages - static_cast<int>(j) * 32;
        s.free_bits[j] = left >= 32 ? ~0u : (1u << left) - 1u;
    }
    for (int64_t j = i; j < static_cast<int64_t>(s.max_slots) * s.max_pages; j += step) s.page_table[j] = -1;
    for (int64_t j = i; j < s.max_slots; j += step) s.seq_len[j] = 0;
}

// ---------------------------------------------------------------- cache write
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return static_cast<float>(x); }

// The mean of a page's keys of one channel: the 64-bit sum of 16 stored
// values in position order (exact where their exponents are at most 41 apart in
// bf16, 25 in fp32: 8 or 24 significant bits, and 4 for the sum, in 53), rounded
// to 32 bits and then to the storage format.
template <typename T> __device__ __forceinline__ T block_mean(double sum) {
    return static_cast<T>(static_cast<float>(sum * (1.0 / kPage)));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Calls of this many rows on take tiles of 32 rows, which look at fewer rows
// twice, and non-temporal stores (37,800 rows of 8 heads, 310 MB read and
// written: 88 us with tiles of 16 rows, 80 with 32, 66 with such stores; a copy
// of as many bytes takes 61; 4,000 rows 12.2 and 10.8 us, 1,000 rows 9.0 and
// 8.9); single rows need the workgroups of 16 (509 of them: 8.7 and 11.9).
constexpr int kBigWrite = 2048;

template <bool STREAM> __device__ __forceinline__ void put16(void* p, u32x4 x) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, static_cast<u32x4*>(p));
    else *static_cast<u32x4*>(p) = x;
}

// K and V of TR rows and one KV head.  Rows that follow each other in one
// page are a run; the workgroup that holds a run's first row writes all of
// it, so a prompt's value pages (transposed: [channel][token]) go out as
// whole 32-byte rows whatever the tile's alignment to pages.  Keys go from
// registers to their rows; values, and keys for the block keys, cross LDS,
// where a wave takes a run.  The keys of a page that a
// run completes are in LDS (this call's) or in the pool (earlier calls'), so
// its block key needs no second pass.  The launch's tiles start at row `first`.
template <typename T, int HD, int TR, bool VEC>
__global__ void __launch_bounds__(256)
cache_write(KvPages c, int64_t first, int n_rows, const int32_t* __restrict__ slot_map, const T* __restrict__ k, int64_t ldk,
            const T* __restrict__ v, int64_t ldv) {
    constexpr int EX = TR + kPage - 1;              // the last run may end behind the tile
    constexpr bool STREAM = TR > 16;
    constexpr int VE = VEC ? 16 / sizeof(T) : 1;    // elements of an access to k and v
    typedef T T2 __attribute__((ext_vector_type(2)));
    struct alignas(VE * sizeof(T)) Chunk { T e[VE]; };
    __shared__ int sm[EX + 1];                      // slot map of rows r0 - 1 ..
    __shared__ bool own[EX];                        // rows of runs that start in the tile
    constexpr int TE = 16 / sizeof(T);              // tokens of a 16-byte store to a value page
    constexpr int LD = HD + TE;                     // rows 4 banks apart: a store's tokens do not meet on one
    __shared__ __attribute__((aligned(16))) T lk[EX][LD];
    __shared__ __attribute__((aligned(16))) T lv[EX][LD];
    __shared__ int runs[TR], n_runs;
    // the heads of a tile on one XCD (blocks i and i + 8 share one): rows of
    // k and v stand far apart, so one head's parts meet on few L2 channels
    const int y = blockIdx.x / 8, g = y % c.n_kv, tid = threadIdx.x;
    const int64_t r0 = first + (y / c.n_kv * 8 + blockIdx.x % 8) * TR;
    if (r0 >= n_rows) return;
    const int limit = c.num_pages * kPage;
    if (tid == 0) n_runs = 0;
    for (int i = tid; i <= EX; i += 256) {
        const int64_t r = r0 - 1 + i;
        const int s = r >= 0 && r < n_rows ? slot_map[r] : -1;
        sm[i] = s >= 0 && s < limit ? s : -1;
    }
    __syncthreads();
    auto leads = [&](int i) {                        // row r0 + i starts a run
        const int s = sm[i + 1];
        return s >= 0 && (s % kPage == 0 || sm[i] != s - 1);
    };
    for (int i = tid; i < EX; i += 256) {
        if (i < TR && leads(i)) runs[atomicAdd(&n_runs, 1)] = i;
        int j = i;                                   // its run's first row, or one before the tile
        while (j >= 0 && sm[j + 1] >= 0 && !leads(j)) --j;
        own[i] = sm[i + 1] >= 0 && j >= 0 && j < TR;
    }
    __syncthreads();
    const int rows = static_cast<int>(min<int64_t>(EX, n_rows - r0));
    for (int e = tid; e < rows * (HD / VE); e += 256) {
        const int i = e / (HD / VE), ch = e % (HD / VE) * VE, s = sm[i + 1];
        if (!own[i]) continue;
        const int64_t r = r0 + i;
        const Chunk x = *reinterpret_cast<const Chunk*>(k + r * ldk + g * HD + ch);
        const Chunk y = *reinterpret_cast<const Chunk*>(v + r * ldv + g * HD + ch);
        T* kp = static_cast<T*>(c.k_pool) + ((static_cast<int64_t>(s / kPage) * c.n_kv + g) * kPage + s % kPage) * HD;
        if constexpr (VEC) put16<STREAM>(kp + ch, __builtin_bit_cast(u32x4, x));
        else *reinterpret_cast<Chunk*>(kp + ch) = x;
        *reinterpret_cast<Chunk*>(&lk[i][ch]) = x;
        *reinterpret_cast<Chunk*>(&lv[i][ch]) = y;
    }
    __syncthreads();
    const int lane = tid & 63, ch = lane * 2;
    for (int j = tid >> 6; j < n_runs; j += 4) {
        const int i0 = runs[j], s0 = sm[i0 + 1], off = s0 % kPage;
        int len = 1;
        while (off + len < kPage && i0 + len < EX && sm[i0 + len + 1] == s0 + len) ++len;
        const int64_t page = s0 / kPage, at = (page * c.n_kv + g) * HD;
        T* vp = static_cast<T*>(c.v_pool) + at * kPage;
        if (len == kPage) {
            // neighbouring lanes, neighbouring 16 bytes
            for (int e = lane; e < HD * kPage / TE; e += 64) {
                const int vc = e / (kPage / TE), t0 = e % (kPage / TE) * TE;
                alignas(16) T y[TE];
#pragma unroll
                for (int x = 0; x < TE; ++x) y[x] = lv[i0 + t0 + x][vc];
                put16<STREAM>(vp + e * TE, *reinterpret_cast<const u32x4*>(y));
            }
        } else {
            for (int x = 0; x < len; ++x)
                for (int vc = lane; vc < HD; vc += 64) vp[vc * kPage + off + x] = lv[i0 + x][vc];
        }
        if (ch >= HD) continue;
        if (c.block_keys && off + len == kPage) {
            // all loads of the keys that stand in the pool at once
            const T* kp = static_cast<const T*>(c.k_pool) + at * kPage + ch;
            T2 y[kPage];
#pragma unroll
            for (int x = 0; x < kPage; ++x) {
                if (x < off) y[x] = *reinterpret_cast<const T2*>(kp + x * HD);
                else y[x] = *reinterpret_cast<const T2*>(&lk[i0 + x - off][ch]);
            }
            double a = 0.0, b = 0.0;
#pragma unroll
            for (int x = 0; x < kPage; ++x) {
                a += static_cast<double>(to_f32(y[x][0]));
                b += static_cast<double>(to_f32(y[x][1]));
            }
            *reinterpret_cast<T2*>(static_cast<T*>(c.block_keys) + at + ch) = T2{block_mean<T>(a), block_mean<T>(b)};
        }
    }
}

// Workgroups of one launch; more go out in several (the threads of a grid's
// axis are counted in 32 bits).
constexpr int64_t kWriteBlocks = 1 << 20;

template <typename T>
void write_rows(const KvPages& c, int n_rows, const int32_t* slot_map, const void* k, int64_t ldk, const void* v,
                int64_t ldv, hipStream_t st) {
    const T* kk = static_cast<const T*>(k);
    const T* vv = static_cast<const T*>(v);
    const bool vec = (reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % 16 == 0 &&
                     (ldk * sizeof(T)) % 16 == 0 && (ldv * sizeof(T)) % 16 == 0;
    const bool big = n_rows >= kBigWrite && sizeof(T) == 2;
#define OUTLETS_WRITE(HD, TR, VEC)                                                                             \
    do {                                                                                                       \
        const int64_t row = 8 * static_cast<int64_t>(c.n_kv), per = std::max<int64_t>(1, kWriteBlocks / row);  \
        const int64_t tiles = (static_cast<int64_t>(n_rows) + 8 * TR - 1) / (8 * TR);    /* eight of them */   \
        for (int64_t t = 0; t < tiles; t += per)                                                               \
            hipLaunchKernelGGL((cache_write<T, HD, TR, VEC>), dim3(std::min(per, tiles - t) * row), dim3(256), 0, st, c, \
                               t * (8 * TR), n_rows, slot_map, kk, ldk, vv, ldv);                              \
    } while (0)
    if (c.hd == 128) {
        if (!vec) OUTLETS_WRITE(128, 16, false);
        else if (big) OUTLETS_WRITE(128, (sizeof(T) == 2 ? 32 : 16), true);
        else OUTLETS_WRITE(128, 16, true);
    } else {
        if (!vec) OUTLETS_WRITE(64, 16, false);
        else if (big) OUTLETS_WRITE(64, (sizeof(T) == 2 ? 32 : 16), true);
        else OUTLETS_WRITE(64, 16, true);
    }
#undef OUTLETS_WRITE
}

// Rows that end a page average its 16 keys: a wave looks at kKeyRows rows (a
// prompt's end one page among them) and takes those pages one after another,
// all of a page's keys in flight.
constexpr int kKeyRows = 16;

template <typename T, int HD>
__global__ void __launch_bounds__(64)
block_keys_kernel(KvPages c, int n_rows, const int32_t* __restrict__ row_slot, const int32_t* __restrict__ positions) {
    typedef T T2 __attribute__((ext_vector_type(2)));
    const int g = blockIdx.y, lane = threadIdx.x, r = blockIdx.x * kKeyRows + lane, ch = 2 * lane;
    int page = -1;
    if (lane < kKeyRows && r < n_rows) {
        const int pos = positions[r], slot = row_slot[r];
        if (pos >= 0 && pos % kPage == kPage - 1 && pos / kPage < c.max_pages && slot >= 0 && slot < c.max_slots)
            page = c.page_table[static_cast<int64_t>(slot) * c.max_pages + pos / kPage];
        if (page >= c.num_pages) page = -1;
    }
    for (uint64_t todo = __ballot(page >= 0); todo; todo &= todo - 1) {
        const int64_t at = (static_cast<int64_t>(__shfl(page, __builtin_ctzll(todo), 64)) * c.n_kv + g) * HD + ch;
        if (ch >= HD) continue;
        const T* kp = static_cast<const T*>(c.k_pool) + (at - ch) * kPage + ch;
        T2 y[kPage];
#pragma unroll
        for (int x = 0; x < kPage; ++x) y[x] = *reinterpret_cast<const T2*>(kp + x * HD);
        double a = 0.0, b = 0.0;
#pragma unroll
        for (int x = 0; x < kPage; ++x) {
            a += static_cast<double>(to_f32(y[x][0]));
            b += static_cast<double>(to_f32(y[x][1]));
        }
        *reinterpret_cast<T2*>(static_cast<T*>(c.block_keys) + at) = T2{block_mean<T>(a), block_mean<T>(b)};
    }
}

bool append_small(int n_req, int64_t n_rows) { return n_req <= kSmallReqs && n_rows <= kSmallRows; }

}  // namespace

void launch_pages_reset(const PageState& s, hipStream_t st) {
    const int64_t work = std::max<int64_t>(static_cast<int64_t>(s.max_slots) * s.max_pages, s.num_pages / 32 + 1);
    const int blocks = static_cast<int>(std::min<int64_t>((work + 255) / 256, 1024));
    hipLaunchKernelGGL(pages_reset, dim3(blocks), dim3(256), 0, st, s);
}

int64_t pages_append_ws(int n_req, int64_t n_rows) {
    return append_small(n_req, n_rows) ? 0 : 4 * static_cast<int64_t>(n_req) + n_rows;
}

void launch_pages_append(const PageState& s, int n_req, const int32_t* slots, const int32_t* new_tokens, int n_rows,
                         int32_t* cu, int32_t* slot_map, int32_t* positions, int32_t* row_slot, int32_t* status,
                         int32_t* ws, hipStream_t st) {
    const size_t marks = sizeof(uint32_t) * ((s.max_slots + 31) / 32);
    if (append_small(n_req, n_rows)) {
        hipLaunchKernelGGL((pages_append<true>), dim3(1), dim3(kAppendThreads), marks, st, s, n_req, slots, new_tokens,
                           n_rows, cu, slot_map, positions, row_slot, status, nullptr, nullptr);
        return;
    }
    AppendReq* reqs = reinterpret_cast<AppendReq*>(ws);
    int32_t* list = ws + 4 * static_cast<int64_t>(n_req);
    hipLaunchKernelGGL((pages_append<false>), dim3(1), dim3(kAppendThreads), marks, st, s, n_req, slots, new_tokens,
                       n_rows, cu, slot_map, positions, row_slot, status, reqs, list);
    if (n_rows > 0)
        hipLaunchKernelGGL(append_rows, dim3((n_rows + 255) / 256), dim3(256), 0, st, s, n_req, n_rows, reqs, list,
                           status, slot_map, positions, row_slot);
}

void launch_pages_release(const PageState& s, int n, const int32_t* slots, int32_t* status, hipStream_t st) {
    const size_t marks = sizeof(uint32_t) * ((s.max_slots + 31) / 32);
    hipLaunchKernelGGL(pages_release, dim3(std::max(n, 1)), dim3(kReleaseThreads), marks, st, s, n, slots, status);
}

void launch_cache_write(const KvPages& c, int n_rows, const int32_t* slot_map, const void* k, int64_t ldk,
                        const void* v, int64_t ldv, hipStream_t st) {
    if (n_rows <= 0) return;
    if (c.fmt == OUTLETS_FMT_F32) write_rows<float>(c, n_rows, slot_map, k, ldk, v, ldv, st);
    else write_rows<__bf16>(c, n_rows, slot_map, k, ldk, v, ldv, st);
}

void launch_block_keys(const KvPages& c, int n_rows, const int32_t* row_slot, const int32_t* positions,
                       hipStream_t st) {
    if (n_rows <= 0) return;
    const dim3 grid((n_rows + kKeyRows - 1) / kKeyRows, c.n_kv), block(64);
#define OUTLETS_KEYS(T, HD) \
    hipLaunchKernelGGL((block_keys_kernel<T, HD>), grid, block, 0, st, c, n_rows, row_slot, positions)
    if (c.fmt == OUTLETS_FMT_F32) {
        if (c.hd == 128) OUTLETS_KEYS(float, 128); else OUTLETS_KEYS(float, 64);
    } else {
        if (c.hd == 128) OUTLETS_KEYS(__bf16, 128); else OUTLETS_KEYS(__bf16, 64);
    }
#undef OUTLETS_KEYS
}

}  // namespace outlets

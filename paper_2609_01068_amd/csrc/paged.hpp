// Launch interface of the paged-cache operators (library-internal): page
// tables kept on the GPU, the write into the cache, the selection of pages by
// their block keys and the attention over selected pages.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace outlets {

constexpr int kPage = 16;          // tokens per KV page

// Device-resident page state (see outlets_page_state).
struct PageState {
    uint32_t* free_bits;
    int32_t* page_table;
    int32_t* seq_len;
    int32_t num_pages, max_slots, max_seq_len, max_pages;
};

// Largest slot count of a state: the repeat check marks slots in LDS, one bit each.
constexpr int kPageMaxSlots = 1 << 17;
// Most rows of one append: 1024 requests' sums then fit 31 bits.
constexpr int kPageMaxRows = 1 << 20;
// Most slots of one release: each of its blocks looks at all of them.
constexpr int kReleaseMax = 1 << 18;

void launch_pages_reset(const PageState& s, hipStream_t st);
// int32 entries of `ws` (0 where the whole call works in LDS).
int64_t pages_append_ws(int n_req, int64_t n_rows);
void launch_pages_append(const PageState& s, int n_req, const int32_t* slots, const int32_t* new_tokens, int n_rows,
                         int32_t* cu, int32_t* slot_map, int32_t* positions, int32_t* row_slot, int32_t* status,
                         int32_t* ws, hipStream_t st);
void launch_pages_release(const PageState& s, int n, const int32_t* slots, int32_t* status, hipStream_t st);

// A cache's device memory (see outlets_kv_pages).
struct KvPages {
    void* k_pool;
    void* v_pool;
    void* block_keys;
    const int32_t* page_table;
    int32_t fmt, n_kv, hd, num_pages, max_slots, max_pages;
};

void launch_cache_write(const KvPages& c, int n_rows, const int32_t* slot_map, const void* k, int64_t ldk,
                        const void* v, int64_t ldv, hipStream_t st);
// Block keys of the pages whose last token is one of the given rows, read
// from the key pool (the predict calls write K and V in other kernels).
void launch_block_keys(const KvPages& c, int n_rows, const int32_t* row_slot, const int32_t* positions, hipStream_t st);

// Rows of queries over a cache.
struct BlockRows {
    int32_t n_rows;
    const int32_t* row_slot;
    const int32_t* positions;
    const void* q;
    int64_t ldq;
    int32_t n_q;
};
int64_t block_select_ws(const KvPages& c, int64_t n_rows);       // bytes
void launch_block_select(const KvPages& c, const BlockRows& r, int top_k, int sink, int local, int32_t* sel, void* ws,
                         int64_t ws_bytes, int cus, hipStream_t st);
int64_t block_attention_ws(const KvPages& c, int64_t n_rows, int n_q, int top_k, int cus);    // bytes
void launch_block_attention(const KvPages& c, const BlockRows& r, const int32_t* sel, int top_k, const void* gate,
                            int64_t ldg, void* out, int64_t ldo, void* ws, int cus, hipStream_t st);

}  // namespace outlets

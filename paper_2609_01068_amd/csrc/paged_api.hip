// C ABI of the paged-cache operators: argument checks and launches on the
// caller's memory.  They keep nothing between calls and allocate nothing.
#include <hip/hip_runtime.h>

#include <atomic>
#include <string>

#include "error.hpp"
#include "outlets.h"
#include "paged.hpp"

using namespace outlets;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Makes `device` the current one for a call and puts the caller's back.
class DeviceGuard {
public:
    explicit DeviceGuard(int device) {
        err_ = hipGetDevice(&before_);
        if (err_ == hipSuccess && device != before_) {
            err_ = hipSetDevice(device);
            changed_ = err_ == hipSuccess;
        }
    }
    ~DeviceGuard() {
        if (changed_) (void)hipSetDevice(before_);
    }
    hipError_t error() const { return err_; }

private:
    hipError_t err_;
    int before_ = 0;
    bool changed_ = false;
};

// Runs a call's body with its device current; no C++ exception leaves.  An
// error that an earlier HIP call of the thread left unread is dropped, so that
// the check behind the body is about its launches alone.
template <typename F>
int guarded(int device, F&& body) noexcept {
    try {
        DeviceGuard dev(device);
        (void)hipGetLastError();
        if (dev.error() != hipSuccess)
            return fail(OUTLETS_ERR_HIP, std::string("device: ") + hipGetErrorString(dev.error()));
        body();
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return fail(OUTLETS_ERR_HIP, std::string("kernel launch: ") + hipGetErrorString(e));
        return OUTLETS_OK;
    } catch (...) {
        return OUTLETS_ERR_NOMEM;
    }
}

int bad(int rc, const char* why) noexcept {
    try {
        return fail(rc, why);
    } catch (...) {
        return rc;
    }
}

int check_state(const outlets_page_state* s) {
    if (!s) return bad(OUTLETS_ERR_INVALID_ARG, "null page state");
    if (s->num_pages < 1 || s->num_pages > INT32_MAX / kPage)
        return bad(OUTLETS_ERR_INVALID_ARG, "num_pages outside [1, (2^31 - 1) / 16]");
    if (s->max_slots < 1 || s->max_seq_len < 1 || s->max_seq_len > INT32_MAX - kPage)
        return bad(OUTLETS_ERR_INVALID_ARG, "max_slots and max_seq_len must be positive");
    if (s->max_slots > kPageMaxSlots) return bad(OUTLETS_ERR_UNSUPPORTED, "more than 131072 slots");
    if (s->device < 0) return bad(OUTLETS_ERR_INVALID_ARG, "negative device");
    if (!s->free_bits || !s->page_table || !s->seq_len) return bad(OUTLETS_ERR_INVALID_ARG, "null page state memory");
    return OUTLETS_OK;
}

PageState state_of(const outlets_page_state* s) {
    return PageState{s->free_bits, s->page_table, s->seq_len, s->num_pages, s->max_slots, s->max_seq_len,
                     (s->max_seq_len + kPage - 1) / kPage};
}

int check_cache(const outlets_kv_pages* c) {
    if (!c) return bad(OUTLETS_ERR_INVALID_ARG, "null cache");
    if (c->fmt != OUTLETS_FMT_F32 && c->fmt != OUTLETS_FMT_BF16)
        return bad(OUTLETS_ERR_UNSUPPORTED, "the cache format is F32 or BF16");
    if (c->head_dim != 64 && c->head_dim != 128) return bad(OUTLETS_ERR_UNSUPPORTED, "head_dim is 64 or 128");
    if (c->n_kv_heads < 1 || c->n_kv_heads > 65535) return bad(OUTLETS_ERR_INVALID_ARG, "n_kv_heads outside [1, 65535]");
    if (c->num_pages < 1 || c->num_pages > INT32_MAX / kPage)
        return bad(OUTLETS_ERR_INVALID_ARG, "num_pages outside [1, (2^31 - 1) / 16]");
    if (c->device < 0) return bad(OUTLETS_ERR_INVALID_ARG, "negative device");
    if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned16(c->block_keys))
        return bad(OUTLETS_ERR_UNSUPPORTED, "the pools must be 16-byte aligned");
    return OUTLETS_OK;
}

KvPages cache_of(const outlets_kv_pages* c) {
    return KvPages{c->k_pool,       c->v_pool,     c->block_keys, c->page_table, c->fmt,
                   c->n_kv_heads,   c->head_dim,   c->num_pages,  c->max_slots,  c->max_pages};
}

// Queries of a call over the cache's page table.
int check_rows(const outlets_kv_pages* c, int32_t n_rows, const int32_t* row_slot, const int32_t* positions,
               const void* q, int64_t q_stride, int32_t n_q) {
    if (!c->page_table || c->max_slots < 1 || c->max_pages < 1 || c->max_pages > INT32_MAX / kPage)
        return bad(OUTLETS_ERR_INVALID_ARG, "the cache has no page table");
    if (n_q < 1 || n_q % c->n_kv_heads != 0) return bad(OUTLETS_ERR_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads");
    if (n_q / c->n_kv_heads > 16) return bad(OUTLETS_ERR_UNSUPPORTED, "more than 16 query heads per KV head");
    if (n_rows < 0) return bad(OUTLETS_ERR_INVALID_ARG, "negative n_rows");
    if (n_rows == 0) return OUTLETS_OK;
    if (!row_slot || !positions || !q) return bad(OUTLETS_ERR_INVALID_ARG, "null rows");
    if (q_stride < static_cast<int64_t>(n_q) * c->head_dim) return bad(OUTLETS_ERR_INVALID_ARG, "q_stride below a row");
    return OUTLETS_OK;
}

bool vectors(const outlets_kv_pages* c, const void* p, int64_t stride) {
    return aligned16(p) && stride % (c->fmt == OUTLETS_FMT_F32 ? 4 : 8) == 0;
}

// Compute units of a device, asked for once.
int compute_units(int device) {
    static std::atomic<int> known[64];
    if (device < 64) {
        const int n = known[device].load(std::memory_order_relaxed);
        if (n) return n;
    }
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return 256;
    }
    if (device < 64) known[device].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace

extern "C" {

int outlets_pages_reset(const outlets_page_state* state, void* stream) {
    if (int rc = check_state(state)) return rc;
    return guarded(state->device, [&] { launch_pages_reset(state_of(state), static_cast<hipStream_t>(stream)); });
}

int64_t outlets_pages_append_workspace(int32_t n_req, int32_t n_rows) {
    return n_req < 0 || n_rows < 0 ? 0 : pages_append_ws(n_req, n_rows) * static_cast<int64_t>(sizeof(int32_t));
}

int outlets_pages_append(const outlets_page_state* state, int32_t n_req, const int32_t* slots,
                         const int32_t* new_tokens, int32_t n_rows, int32_t* cu_out, int32_t* slot_map_out,
                         int32_t* positions_out, int32_t* row_slot_out, int32_t* status_out, void* ws,
                         int64_t ws_bytes, void* stream) {
    if (int rc = check_state(state)) return rc;
    if (n_req < 0 || n_rows < 0) return bad(OUTLETS_ERR_INVALID_ARG, "negative n_req or n_rows");
    if (n_req > kPageMaxRows || n_rows > kPageMaxRows) return bad(OUTLETS_ERR_UNSUPPORTED, "more than 2^20 requests or rows");
    if ((n_req && (!slots || !new_tokens)) || !cu_out || !status_out ||
        (n_rows && (!slot_map_out || !positions_out || !row_slot_out)))
        return bad(OUTLETS_ERR_INVALID_ARG, "null argument");
    const int64_t need = outlets_pages_append_workspace(n_req, n_rows);
    if (need && (!ws || ws_bytes < need || !aligned16(ws)))
        return bad(OUTLETS_ERR_INVALID_ARG, "workspace missing, too small or not 16-byte aligned");
    return guarded(state->device, [&] {
        launch_pages_append(state_of(state), n_req, slots, new_tokens, n_rows, cu_out, slot_map_out, positions_out,
                            row_slot_out, status_out, static_cast<int32_t*>(ws), static_cast<hipStream_t>(stream));
    });
}

int outlets_pages_release(const outlets_page_state* state, int32_t n, const int32_t* slots, int32_t* status_out,
                          void* stream) {
    if (int rc = check_state(state)) return rc;
    if (n < 0) return bad(OUTLETS_ERR_INVALID_ARG, "negative n");
    if (n > kReleaseMax) return bad(OUTLETS_ERR_UNSUPPORTED, "more than 2^18 slots");
    if ((n && !slots) || !status_out) return bad(OUTLETS_ERR_INVALID_ARG, "null argument");
    return guarded(state->device, [&] {
        launch_pages_release(state_of(state), n, slots, status_out, static_cast<hipStream_t>(stream));
    });
}

int outlets_cache_write(const outlets_kv_pages* cache, int32_t n_rows, const int32_t* slot_map, const void* k,
                        int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
    if (int rc = check_cache(cache)) return rc;
    if (!cache->k_pool || !cache->v_pool) return bad(OUTLETS_ERR_INVALID_ARG, "the cache has no key or value pool");
    if (n_rows < 0) return bad(OUTLETS_ERR_INVALID_ARG, "negative n_rows");
    if (n_rows == 0) return OUTLETS_OK;
    if (!slot_map || !k || !v) return bad(OUTLETS_ERR_INVALID_ARG, "null argument");
    const int64_t width = static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim;
    if (k_stride < width || v_stride < width) return bad(OUTLETS_ERR_INVALID_ARG, "stride below a row");
    return guarded(cache->device, [&] {
        launch_cache_write(cache_of(cache), n_rows, slot_map, k, k_stride, v, v_stride,
                           static_cast<hipStream_t>(stream));
    });
}

int64_t outlets_block_select_workspace(const outlets_kv_pages* cache, int32_t n_rows) {
    if (check_cache(cache) || n_rows < 0 || cache->max_pages < 1) return 0;
    return block_select_ws(cache_of(cache), n_rows);
}

int outlets_block_select(const outlets_kv_pages* cache, int32_t n_rows, const int32_t* row_slot,
                         const int32_t* positions, const void* q, int64_t q_stride, int32_t n_q_heads, int32_t top_k,
                         int32_t sink, int32_t local, int32_t* sel_out, void* ws, int64_t ws_bytes, void* stream) {
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_rows(cache, n_rows, row_slot, positions, q, q_stride, n_q_heads)) return rc;
    if (!cache->block_keys) return bad(OUTLETS_ERR_INVALID_ARG, "the cache has no block keys");
    if (sink < 0 || local < 1 || top_k < 1 || static_cast<int64_t>(sink) + local > top_k)
        return bad(OUTLETS_ERR_INVALID_ARG, "needs sink >= 0, local >= 1 and sink + local <= top_k");
    if (n_rows == 0) return OUTLETS_OK;
    if (!sel_out) return bad(OUTLETS_ERR_INVALID_ARG, "null sel_out");
    if (cache->max_pages > top_k && (!ws || !aligned16(ws) || ws_bytes < block_select_ws(cache_of(cache), 1)))
        return bad(OUTLETS_ERR_INVALID_ARG, "workspace missing, below one row or not 16-byte aligned");
    const int cus = compute_units(cache->device);
    return guarded(cache->device, [&] {
        launch_block_select(cache_of(cache), BlockRows{n_rows, row_slot, positions, q, q_stride, n_q_heads}, top_k, sink,
                            local, sel_out, ws, ws_bytes, cus, static_cast<hipStream_t>(stream));
    });
}

int64_t outlets_block_attention_workspace(const outlets_kv_pages* cache, int32_t n_rows, int32_t n_q_heads,
                                          int32_t top_k) {
    if (check_cache(cache) || n_rows < 1 || n_q_heads < 1 || top_k < 1) return 0;
    return block_attention_ws(cache_of(cache), n_rows, n_q_heads, top_k, compute_units(cache->device));
}

int outlets_block_attention(const outlets_kv_pages* cache, int32_t n_rows, const int32_t* row_slot,
                            const int32_t* positions, const void* q, int64_t q_stride, int32_t n_q_heads,
                            const int32_t* sel, int32_t top_k, const void* gate, int64_t gate_stride, void* out,
                            int64_t out_stride, void* ws, int64_t ws_bytes, void* stream) {
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_rows(cache, n_rows, row_slot, positions, q, q_stride, n_q_heads)) return rc;
    if (!cache->k_pool || !cache->v_pool) return bad(OUTLETS_ERR_INVALID_ARG, "the cache has no key or value pool");
    if (top_k < 1) return bad(OUTLETS_ERR_INVALID_ARG, "top_k below 1");
    if (n_rows == 0) return OUTLETS_OK;
    if (!sel || !out) return bad(OUTLETS_ERR_INVALID_ARG, "null argument");
    const int64_t width = static_cast<int64_t>(n_q_heads) * cache->head_dim;
    if (out_stride < width || (gate && gate_stride < width)) return bad(OUTLETS_ERR_INVALID_ARG, "stride below a row");
    if (!vectors(cache, q, q_stride)) return bad(OUTLETS_ERR_UNSUPPORTED, "q rows must be 16-byte aligned");
    const int cus = compute_units(cache->device);
    const int64_t need = block_attention_ws(cache_of(cache), n_rows, n_q_heads, top_k, cus);
    if (need && (!ws || !aligned16(ws) || ws_bytes < need))
        return bad(OUTLETS_ERR_INVALID_ARG, "workspace missing, too small or not 16-byte aligned");
    return guarded(cache->device, [&] {
        launch_block_attention(cache_of(cache), BlockRows{n_rows, row_slot, positions, q, q_stride, n_q_heads}, sel,
                               top_k, gate, gate_stride, out, out_stride, ws, cus, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"

// The handle behind the C ABI and the checks that its entry points share.
#pragma once

#include <mutex>

#include "gva_rope.cuh"
#ifdef GVA_WITH_MMA
#include "gva_decode_mma.cuh"
#endif

struct gva_handle {
    gva_config cfg;
    int device;
    int sm_count;
    int smem_optin;          // max dynamic shared memory per block
    int smem_per_sm;         // shared memory of one SM
    float scale;             // softmax scale of gva_decode
    gva::RopeTable rope;
    gva::HeadRope head_rope; // rotation of gqa_append
    int last_num_splits;
    int last_kernel;
    int last_tile;
    int epoch;               // number of the last decode call on this handle (see kSync* in gva_common.cuh)
    int serial;              // number of this handle among all created in this process (see kHdrEpoch)
    int32_t *sync_base;      // device address of the sync arena on this handle's device
    int sync_off, sync_cap;  // the region of the arena in use (words)
    int n_regions;           // regions reserved so far (the earlier, smaller ones are kept until gva_destroy)
    int region_off[24], region_cap[24];
#ifdef GVA_WITH_MMA
    gva::MmaHostState mma;
#endif
};

namespace gva {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline int check_common(const gva_handle *h, int B, int max_seq_len, int num_splits) {
    if (!h) return GVA_ERR_INVALID_ARG;
    if (B < 0 || max_seq_len < 0 || num_splits < 0) return GVA_ERR_INVALID_ARG;
    if (B > 8192 || num_splits > 4096) return GVA_ERR_UNSUPPORTED;
    // total tiles must fit an int with headroom
    if ((long long)B * ((max_seq_len + 31) / 32 + 1) >= (1ll << 30)) return GVA_ERR_UNSUPPORTED;
    return GVA_OK;
}

// The device a call launches on has to be the handle's.
inline int check_device(const gva_handle *h) {
    int current = -1;
    if (cudaGetDevice(&current) != cudaSuccess) return GVA_ERR_CUDA;
    return current == h->device ? GVA_OK : GVA_ERR_INVALID_ARG;
}
inline int check_plain(const gva_handle *h, const gva_cache *cache) {
    if (!h || !cache) return GVA_ERR_INVALID_ARG;
    if (!cache->v_pool || (h->cfg.d_r > 0 && !cache->kr_pool)) return GVA_ERR_INVALID_ARG;
    if (cache->num_pages <= 0 || cache->max_pages_per_seq <= 0) return GVA_ERR_INVALID_ARG;
    if (!aligned(cache->v_pool, 16) || !aligned(cache->kr_pool, 16) || !aligned(cache->block_table, 4)) return GVA_ERR_INVALID_ARG;
    return check_device(h);
}
inline int launched(cudaError_t ce) {
    if (ce == cudaSuccess) return GVA_OK;
    (void)cudaGetLastError();
    return GVA_ERR_CUDA;
}

// Lets `fn` have `bytes` of dynamic shared memory on the handle's device; asked of the runtime once per kernel and device, not per call.
inline int allow_smem(const gva_handle *h, const void *fn, size_t bytes) {
    struct Entry { const void *fn; int device; size_t bytes; };
    static std::mutex lock;
    static Entry seen[256];
    static int n = 0;
    if (bytes <= 16 * 1024) return GVA_OK;               // every kernel may have 48 KB, its static shared memory (27 KB at most) included
    std::lock_guard<std::mutex> hold(lock);
    int i = 0;
    while (i < n && (seen[i].fn != fn || seen[i].device != h->device)) ++i;
    if (i < n && seen[i].bytes >= bytes) return GVA_OK;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return GVA_ERR_CUDA;
    }
    if (i < n) seen[i].bytes = bytes;
    else if (n < 256) seen[n++] = Entry{fn, h->device, bytes};
    return GVA_OK;
}

}  // namespace gva

// Internal launch interface of the attention half of a layer: norm and rotation, the 4-bit cache, attention.  As in
// itq3s_kernels.h the caller has checked every argument; a launcher enqueues on `stream` and returns 0, -2 or -6.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace itq3s {

constexpr uint32_t kFlagBadSlot = 32u;

// Attention: workgroups for `tiles` tiles of each of `units` heads of sequences.  A launch has less than 2^32 threads, and
// estimates of a sequence's rows may be far too high: a workgroup takes several tiles where there would be too many.
constexpr int64_t kMostUnits = 1LL << 22;
inline int64_t most_tiles(int64_t tiles, int64_t units) {
    const int64_t most = kMostUnits / units;
    return tiles < most ? tiles : most;
}

struct CacheView {
    unsigned char* data;
    int64_t pages;
    int page_blocks;  // blocks of 32 tokens a page
    int kv_heads, head_dim;
};

struct AppendCall {
    const void* Q;
    int64_t ldq;
    int q_heads;
    const void* K;
    int64_t ldk;
    const void* V;
    int64_t ldv, T;
    int in_f16, kv_heads, head_dim;
    const float *q_norm, *k_norm;
    float eps;
    const int32_t* positions;
    const double* freq;
    int rot, interleaved;
    float gain;
    void* Q_out;
    int64_t ldqo;
    void* K_out;
    int64_t ldko;
    int out_f16;
    CacheView cache;  // data null: none
    const int64_t* slots;
    uint32_t* flags;
};
int launch_append(const AppendCall& c, hipStream_t stream);

int launch_cache_read(const CacheView& cache, const int64_t* slots, int64_t T, void* K, int64_t ldk, void* V, int64_t ldv, int out_f16, uint32_t* flags,
                      hipStream_t stream);

struct CacheAttentionCall {
    const _Float16* Q;
    int64_t ldq, T;
    int q_heads;
    const int32_t *starts, *kv_lens, *pages;
    int64_t seqs, ld_pages, max_q, max_kv;
    CacheView cache;
    float scale;
    _Float16* out;
    int64_t ldo;
    void* workspace;
    uint32_t* flags;
};
// Scratch of a call with these sizes.
size_t cache_attention_bytes(int64_t T, int64_t seqs, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv);
int launch_cache_attention(const CacheAttentionCall& c, hipStream_t stream);

struct PromptCall {
    const _Float16 *Q, *K, *V;
    int64_t ldq, ldk, ldv, T;
    int q_heads, kv_heads, head_dim;
    const int32_t* starts;
    int64_t seqs, max_len;
    int causal;
    float scale;
    _Float16* out;
    int64_t ldo;
};
int launch_prompt_attention(const PromptCall& c, hipStream_t stream);

}  // namespace itq3s

// C-ABI entry points of the attention half of a layer (include/itq3s.h): argument validation on the host, then launches.
#include "../../include/itq3s.h"
#include "itq3s_attention.h"

#include <math.h>

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool head_dim_ok(int D) { return D == 64 || D == 128 || D == 256; }

// Rows of `heads` heads: pointer and stride.  Returns 0 or the error.
int rows_ok(const void* p, int64_t ld, int64_t heads, int D, size_t size) {
    if (ld < heads * D || ld > (1LL << 40)) return ITQ3S_ERR_SHAPE;
    if (!aligned(p, 16) || ld * (int64_t)size % 16 != 0) return ITQ3S_ERR_ALIGN;
    return 0;
}

int cache_ok(const itq3s_cache* c) {
    if (!c->data) return ITQ3S_ERR_NULL;
    if (itq3s_cache_bytes(c->pages, c->page_tokens, c->kv_heads, c->head_dim) == 0) return ITQ3S_ERR_SHAPE;
    return aligned(c->data, 128) ? 0 : ITQ3S_ERR_ALIGN;
}

itq3s::CacheView view(const itq3s_cache* c) {
    return itq3s::CacheView{static_cast<unsigned char*>(c->data), c->pages, c->page_tokens / 32, c->kv_heads, c->head_dim};
}

inline bool heads_ok(int q_heads, int kv_heads) {
    return q_heads > 0 && q_heads <= 65536 && kv_heads > 0 && kv_heads <= 1024 && q_heads % kv_heads == 0;
}

constexpr int64_t kMostRows = 1LL << 30, kMostBytes = 1LL << 48, kMostStride = 1LL << 23;
constexpr int64_t kMostAppended = 1LL << 24, kMostRead = 1LL << 28;  // tokens: a launch has less than 2^32 threads
constexpr float kMostScale = 1099511627776.f;  // 2^40: scores stay within fp32

}  // namespace

extern "C" {

size_t itq3s_cache_bytes(int64_t pages, int page_tokens, int kv_heads, int head_dim) {
    if (pages <= 0 || pages > 0x7fffffffLL || kv_heads <= 0 || kv_heads > 1024 || !head_dim_ok(head_dim)) return 0;
    if (page_tokens < 32 || page_tokens > 65536 || (page_tokens & (page_tokens - 1)) != 0) return 0;
    const int64_t page = (int64_t)kv_heads * (page_tokens / 32) * (32 * head_dim + 128);
    return pages <= kMostBytes / page ? (size_t)(pages * page) : 0;
}

int itq3s_rope_frequencies(int rot, double base, double factor, int64_t trained_tokens, double slow_turns, double fast_turns, double* freq) {
    if (!freq) return ITQ3S_ERR_NULL;
    if (rot < 2 || rot > 256 || rot % 2 != 0 || !(base > 0.0) || !(factor > 0.0) || !isfinite(base) || !isfinite(factor) || trained_tokens < 0) return ITQ3S_ERR_SHAPE;
    if (trained_tokens > 0 && (!(slow_turns >= 0.0) || !(fast_turns > slow_turns) || !isfinite(fast_turns))) return ITQ3S_ERR_SHAPE;
    for (int i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot);
        double keep = 0.0;  // of the frequency as it was trained
        if (trained_tokens > 0) {
            const double turns = (double)trained_tokens * f / 6.283185307179586477;
            keep = (turns - slow_turns) / (fast_turns - slow_turns);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        }
        freq[i] = keep * f + (1.0 - keep) * (f / factor);
    }
    return ITQ3S_OK;
}

int itq3s_cache_append(const void* Q, int64_t ldq, int q_heads, const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t T, int in_dtype, int kv_heads, int head_dim,
                       const float* q_norm, const float* k_norm, float eps, const int32_t* positions, const double* freq, int rot, int interleaved, float gain, void* Q_out,
                       int64_t ldqo, void* K_out, int64_t ldko, int out_dtype, const itq3s_cache* cache, const int64_t* slots, uint32_t* status_flags, void* stream) {
    if ((!Q && !K) || (Q && !Q_out) || (K && !K_out && !cache) || (V && !cache)) return ITQ3S_ERR_NULL;
    if (cache && (!K || !V || !slots)) return ITQ3S_ERR_NULL;
    if (rot != 0 && (!positions || !freq)) return ITQ3S_ERR_NULL;
    if (T <= 0 || T > kMostAppended || !head_dim_ok(head_dim) || kv_heads <= 0 || kv_heads > 1024 || (Q && (q_heads <= 0 || q_heads > 65536))) return ITQ3S_ERR_SHAPE;
    if (rot < 0 || rot > head_dim || rot % 16 != 0) return ITQ3S_ERR_SHAPE;
    if (!(eps >= 0.f) || !isfinite(eps) || !isfinite(gain)) return ITQ3S_ERR_SHAPE;
    if ((in_dtype != ITQ3S_F32 && in_dtype != ITQ3S_F16) || (out_dtype != ITQ3S_F32 && out_dtype != ITQ3S_F16)) return ITQ3S_ERR_DTYPE;
    const size_t in = in_dtype == ITQ3S_F16 ? 2 : 4, out = out_dtype == ITQ3S_F16 ? 2 : 4;
    int rc = 0;
    if (cache) {
        if ((rc = cache_ok(cache)) != 0) return rc;
        if (cache->kv_heads != kv_heads || cache->head_dim != head_dim) return ITQ3S_ERR_SHAPE;
        if (!aligned(slots, 8)) return ITQ3S_ERR_ALIGN;
    }
    if (Q && ((rc = rows_ok(Q, ldq, q_heads, head_dim, in)) != 0 || (rc = rows_ok(Q_out, ldqo, q_heads, head_dim, out)) != 0)) return rc;
    if (K && (rc = rows_ok(K, ldk, kv_heads, head_dim, in)) != 0) return rc;
    if (K && K_out && (rc = rows_ok(K_out, ldko, kv_heads, head_dim, out)) != 0) return rc;
    if (V && (rc = rows_ok(V, ldv, kv_heads, head_dim, in)) != 0) return rc;
    if ((q_norm && !aligned(q_norm, 16)) || (k_norm && !aligned(k_norm, 16)) || (rot != 0 && (!aligned(positions, 4) || !aligned(freq, 8))) ||
        (status_flags && !aligned(status_flags, 4)))
        return ITQ3S_ERR_ALIGN;
    itq3s::AppendCall c{};
    c.Q = Q, c.ldq = ldq, c.q_heads = q_heads, c.K = K, c.ldk = ldk, c.V = V, c.ldv = ldv, c.T = T, c.in_f16 = in_dtype == ITQ3S_F16, c.kv_heads = kv_heads, c.head_dim = head_dim;
    c.q_norm = q_norm, c.k_norm = k_norm, c.eps = eps, c.positions = positions, c.freq = freq, c.rot = rot, c.interleaved = interleaved != 0, c.gain = gain;
    c.Q_out = Q_out, c.ldqo = ldqo, c.K_out = K ? K_out : nullptr, c.ldko = ldko, c.out_f16 = out_dtype == ITQ3S_F16, c.slots = slots, c.flags = status_flags;
    if (cache) c.cache = view(cache);
    return itq3s::launch_append(c, static_cast<hipStream_t>(stream));
}

int itq3s_cache_read(const itq3s_cache* cache, const int64_t* slots, int64_t T, void* K_out, int64_t ldk, void* V_out, int64_t ldv, int out_dtype, uint32_t* status_flags,
                     void* stream) {
    if (!cache || !slots || !K_out || !V_out) return ITQ3S_ERR_NULL;
    int rc = cache_ok(cache);
    if (rc != 0) return rc;
    if (T <= 0 || T > kMostRead) return ITQ3S_ERR_SHAPE;
    if (out_dtype != ITQ3S_F32 && out_dtype != ITQ3S_F16) return ITQ3S_ERR_DTYPE;
    const size_t out = out_dtype == ITQ3S_F16 ? 2 : 4;
    if ((rc = rows_ok(K_out, ldk, cache->kv_heads, cache->head_dim, out)) != 0 || (rc = rows_ok(V_out, ldv, cache->kv_heads, cache->head_dim, out)) != 0) return rc;
    if (!aligned(slots, 8) || (status_flags && !aligned(status_flags, 4))) return ITQ3S_ERR_ALIGN;
    return itq3s::launch_cache_read(view(cache), slots, T, K_out, ldk, V_out, ldv, out_dtype == ITQ3S_F16, status_flags, static_cast<hipStream_t>(stream));
}

size_t itq3s_cache_attention_workspace_bytes(int64_t T, int64_t seqs, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv) {
    if (T <= 0 || !heads_ok(q_heads, kv_heads) || seqs <= 0 || seqs > itq3s::kMostUnits / kv_heads || T > kMostRows / (q_heads / kv_heads) || !head_dim_ok(head_dim) || max_q <= 0 || max_kv <= 0 ||
        max_kv > kMostRows)
        return 256;
    return itq3s::cache_attention_bytes(T, seqs, q_heads, kv_heads, head_dim, max_q < T ? max_q : T, max_kv);
}

int itq3s_cache_attention(const void* Q, int64_t ldq, int64_t T, int q_heads, const itq3s_cache* cache, const int32_t* q_starts, const int32_t* kv_lens, int64_t seqs,
                          const int32_t* pages, int64_t ld_pages, int64_t max_q, int64_t max_kv, float scale, void* out, int64_t ldo, void* workspace, size_t workspace_bytes,
                          uint32_t* status_flags, void* stream) {
    if (!Q || !cache || !q_starts || !kv_lens || !pages || !out) return ITQ3S_ERR_NULL;
    int rc = cache_ok(cache);
    if (rc != 0) return rc;
    if (!heads_ok(q_heads, cache->kv_heads) || T <= 0 || seqs <= 0 || seqs > itq3s::kMostUnits / cache->kv_heads ||
        T > kMostRows / (q_heads / cache->kv_heads))
        return ITQ3S_ERR_SHAPE;
    if (ld_pages <= 0 || ld_pages > kMostRows / cache->page_tokens || max_q <= 0 || max_kv <= 0 || max_kv > kMostRows || !(fabsf(scale) <= kMostScale)) return ITQ3S_ERR_SHAPE;
    if ((rc = rows_ok(Q, ldq, q_heads, cache->head_dim, 2)) != 0 || (rc = rows_ok(out, ldo, q_heads, cache->head_dim, 2)) != 0) return rc;
    if (!aligned(q_starts, 4) || !aligned(kv_lens, 4) || !aligned(pages, 4) || (status_flags && !aligned(status_flags, 4))) return ITQ3S_ERR_ALIGN;
    if (max_q > T) max_q = T;
    if (!workspace || workspace_bytes < itq3s::cache_attention_bytes(T, seqs, q_heads, cache->kv_heads, cache->head_dim, max_q, max_kv)) return ITQ3S_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return ITQ3S_ERR_ALIGN;
    const itq3s::CacheAttentionCall c{static_cast<const _Float16*>(Q), ldq, T, q_heads, q_starts, kv_lens, pages, seqs, ld_pages, max_q, max_kv, view(cache), scale,
                                      static_cast<_Float16*>(out), ldo, workspace, status_flags};
    return itq3s::launch_cache_attention(c, static_cast<hipStream_t>(stream));
}

int itq3s_prompt_attention(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t T, int q_heads, int kv_heads, int head_dim,
                           const int32_t* starts, int64_t seqs, int64_t max_len, int causal, float scale, void* out, int64_t ldo, void* stream) {
    if (!Q || !K || !V || !starts || !out) return ITQ3S_ERR_NULL;
    if (!heads_ok(q_heads, kv_heads) || !head_dim_ok(head_dim) || T <= 0 || T > kMostRows / (q_heads / kv_heads) || seqs <= 0 || seqs > itq3s::kMostUnits / kv_heads ||
        max_len <= 0 || !(fabsf(scale) <= kMostScale))
        return ITQ3S_ERR_SHAPE;
    int rc = 0;
    if ((rc = rows_ok(Q, ldq, q_heads, head_dim, 2)) != 0 || (rc = rows_ok(K, ldk, kv_heads, head_dim, 2)) != 0 || (rc = rows_ok(V, ldv, kv_heads, head_dim, 2)) != 0 ||
        (rc = rows_ok(out, ldo, q_heads, head_dim, 2)) != 0)
        return rc;
    if (ldk > kMostStride || ldv > kMostStride) return ITQ3S_ERR_SHAPE;
    if (!aligned(starts, 4)) return ITQ3S_ERR_ALIGN;
    const itq3s::PromptCall c{static_cast<const _Float16*>(Q), static_cast<const _Float16*>(K), static_cast<const _Float16*>(V), ldq, ldk, ldv, T, q_heads, kv_heads, head_dim,
                              starts, seqs, max_len < T ? max_len : T, causal != 0, scale, static_cast<_Float16*>(out), ldo};
    return itq3s::launch_prompt_attention(c, static_cast<hipStream_t>(stream));
}

}  // extern "C"

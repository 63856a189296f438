// Attention over the 4-bit cache: o = softmax(scale q k^T) v for the last rows of every sequence.
//
// With cached rows k = H (s c), v = H (s c) (H orthonormal, symmetric): q . k = s (H q) . c, and sum p v = H sum p s c.
// The kernel turns q once, works on digits, and turns the result back; keys and values are never reconstructed.
//
// A wavefront takes 32 tokens (a block of the cache, one contiguous piece of memory, loaded lane by lane as the operands
// want it) against 16 query rows a column tile -- the heads of a group times the sequence's new rows:
//   S^T = C_k (H q)^T   rows tokens, columns query rows; digits as fp16 integers, products exact, sums in fp32
//   O^T += C_v^T P'^T   with P' = exp2(y - m) s_v: the accumulator layout of S^T is the operand layout of P'^T
// Online softmax in base 2.  Steps of values go into P' and may be any fp16, so the reference m follows the largest
// y + exponent(s_v): P' stays within fp16 whatever the steps are, and l = sum exp2(y - m) in fp32 has the range to follow.
// m only moves when a row's weights would pass 2^8 (then O and l are scaled): a block costs no rescaling otherwise.
//
// Few rows: the wavefronts of a workgroup take blocks in turn and meet in LDS.  Many rows: each has its own rows.  A
// long context is split over workgroups besides; combine_kernel joins the parts.
#include "itq3s_attention.h"
#include "itq3s_cache.h"

namespace itq3s {

namespace {

constexpr float kNoRow = -1e30f;    // reference of a row that has seen nothing
constexpr float kHeadroom = 8.f;    // weights may reach 2^8 before the reference moves
constexpr int kExpBias = 14;        // s < 2^(E - 14) for an fp16 with exponent field E
constexpr int kMaxSplits = 256;

struct AttnArgs {
    const _Float16* Q;
    const int32_t *starts, *kv_lens, *pages;
    const unsigned char* data;
    _Float16* out;
    float *part, *ml;  // [splits][T * q_heads][D], [splits][T * q_heads][2]
    uint32_t* flags;
    int64_t ldq, ldo, ld_pages, T, pool;
    float scale;  // softmax scale * log2(e) / sqrt(D)
    int q_heads, kv_heads, group, seqs, tiles, splits, split_blocks, page_shift;
};

// A sequence: its rows among all query rows, its tokens in the cache, and how its blocks are split.
struct Seq {
    int64_t first;
    int rows, len, blocks, per_split, splits;
};
__device__ __forceinline__ Seq find_seq(const AttnArgs& a, int s) {
    Seq q;
    int64_t lo = a.starts[s], hi = a.starts[s + 1];
    lo = lo < 0 ? 0 : lo > a.T ? a.T : lo;
    hi = hi < lo ? lo : hi > a.T ? a.T : hi;
    q.first = lo;
    q.rows = (int)(hi - lo);
    int64_t len = a.kv_lens[s];
    const int64_t most = a.ld_pages << (a.page_shift + 5);
    if (len > most) {
        if (a.flags != nullptr && threadIdx.x == 0) atomicOr(a.flags, kFlagBadSlot);
        len = most;
    }
    q.len = len < 0 ? 0 : (int)len;
    q.blocks = (q.len + kCacheBlock - 1) / kCacheBlock;
    const int need = (q.blocks + a.splits - 1) / a.splits;
    q.per_split = need > a.split_blocks ? need : a.split_blocks;
    q.splits = (q.blocks + q.per_split - 1) / q.per_split;
    return q;
}

template <int D>
struct Block {
    uint32_t k[2][D / 32];
    u32x4 v[D / 64];
    u32x4 s[2];
    int base;  // its first token, beyond every sequence for a block that is not there
};

template <int D>
__device__ __forceinline__ void load_block(const AttnArgs& a, const int32_t* pages, int head, int b, Block<D>& o) {
    int page = pages[b >> a.page_shift];
    o.base = b * kCacheBlock;
    if ((uint32_t)page >= (uint64_t)a.pool) {
        if (a.flags != nullptr && lane_id() == 0) atomicOr(a.flags, kFlagBadSlot);
        page = 0;
        o.base = 0x7fffff00;
    }
    const unsigned char* const at = a.data + block_offset<D>(page, head, a.kv_heads, 1 << a.page_shift, b & ((1 << a.page_shift) - 1));
    const int lane = lane_id(), g = lane >> 4, r = lane & 15;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
        const unsigned char* const kp = at + (tt * 16 + r) * (D / 2) + g * (D / 8);
        if constexpr (D == 64) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(kp);
            o.k[tt][0] = w[0], o.k[tt][1] = w[1];
        } else {
#pragma unroll
            for (int i = 0; i < D / 128; ++i) {
                const u32x4 w = reinterpret_cast<const u32x4*>(kp)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) o.k[tt][4 * i + j] = w[j];
            }
        }
        o.s[tt] = *reinterpret_cast<const u32x4*>(at + 32 * D + 4 * (tt * 16 + 4 * g));
    }
#pragma unroll
    for (int h = 0; h < D / 64; ++h) o.v[h] = *reinterpret_cast<const u32x4*>(at + 16 * D + h * 1024 + lane * 16);
}

__device__ __forceinline__ half8 join(half2v a, half2v b, half2v c, half2v d) {
    return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The rotated queries of a column tile: lane (column l % 16, g = l / 16) holds channels (D/4) g .. (D/4) (g + 1) - 1, scaled by
// a power of two into fp16's best range; returns what scores have to be multiplied with.
template <int D>
__device__ __forceinline__ float load_queries(const _Float16* q, bool there, float scale, half8 (&f)[D / 32]) {
    float x[D / 4];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        half8 h = there ? reinterpret_cast<const half8*>(q)[i] : half8{};
#pragma unroll
        for (int j = 0; j < 8; ++j) x[8 * i + j] = (float)h[j];
    }
#pragma unroll
    for (int h = 1; h < D / 4; h *= 2)
#pragma unroll
        for (int j = 0; j < D / 4; ++j)
            if ((j & h) == 0) {
                const float u = x[j], v = x[j + h];
                x[j] = u + v;
                x[j + h] = u - v;
            }
    float most = 0.f;
#pragma unroll
    for (int m = 16; m <= 32; m *= 2) {
        const float sign = (lane_id() & m) != 0 ? -1.f : 1.f;
#pragma unroll
        for (int j = 0; j < D / 4; ++j) x[j] = __builtin_fmaf(sign, x[j], xor_lane_f32(x[j], m));
    }
#pragma unroll
    for (int j = 0; j < D / 4; ++j) most = __builtin_fmaxf(most, __builtin_fabsf(x[j]));
    most = __builtin_fmaxf(most, xor_lane_f32(most, 16));
    most = __builtin_fmaxf(most, xor_lane_f32(most, 32));
    const int e = __builtin_amdgcn_frexp_expf(most);  // 0 for 0, infinities and NaN
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] = (_Float16)__builtin_ldexpf(x[8 * i + j], -e);
    return __builtin_ldexpf(scale, e);
}

template <int D, int CT>
struct State {
    floatx4 o[D / 16][CT];
    float m[CT], l[CT];
};

template <int D, int CT>
__device__ __forceinline__ void attend(const Block<D>& b, const half8 (&q)[CT][D / 32], const float (&qs)[CT], const int (&see)[CT], int see_all, int len, State<D, CT>& st) {
    const int g = lane_id() >> 4;
    float kf[2][4], vf[2][4], ve[2][4];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = b.s[tt][i];
            kf[tt][i] = f16_bits_to_f32(w & 0xffffu);
            vf[tt][i] = f16_bits_to_f32(w >> 16);
            ve[tt][i] = (float)((w >> 26) & 31u);
        }
    const bool edge = b.base + kCacheBlock > see_all;
    if (edge) {  // what stands behind the sequence may be anything
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = b.base + tt * 16 + 4 * g + i < len;
                kf[tt][i] = in ? kf[tt][i] : 0.f;
                vf[tt][i] = in ? vf[tt][i] : 0.f;
            }
    }
    floatx4 s[2][CT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) s[tt][ct] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const uint32_t w = b.k[tt][i];
            const half8 k = join(low_pair(w), high_pair(w), low_pair(w >> 8), high_pair(w >> 8));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[tt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[ct][i], s[tt][ct], 0, 0, 0);
        }
    half8 p[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        float x[2][4], top = -__builtin_inff();
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[tt][i] = s[tt][ct][i] * kf[tt][i];
                if (edge) {
                    const bool seen = b.base + tt * 16 + 4 * g + i < see[ct];
                    x[tt][i] = seen ? x[tt][i] * qs[ct] : -__builtin_inff();
                } else {
                    x[tt][i] *= qs[ct];
                }
                top = __builtin_fmaxf(top, x[tt][i] + ve[tt][i]);
            }
        top -= (float)kExpBias;
        if (__builtin_amdgcn_ballot_w64(top > st.m[ct] + kHeadroom) != 0) {
            top = __builtin_fmaxf(top, xor_lane_f32(top, 16));
            top = __builtin_fmaxf(top, xor_lane_f32(top, 32));
            const float m = __builtin_fmaxf(st.m[ct], top), f = __builtin_amdgcn_exp2f(st.m[ct] - m);
            st.m[ct] = m;
            st.l[ct] *= f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st.o[c][ct] *= f;
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(x[tt][i] - st.m[ct]);
                st.l[ct] += e;
                p[ct][4 * tt + i] = (_Float16)(e * vf[tt][i]);
            }
    }
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
#pragma unroll
        for (int pp = 0; pp < 2; ++pp) {
            const uint32_t w0 = b.v[h][2 * pp], w1 = b.v[h][2 * pp + 1];
            const half8 lo = join(low_pair(w0), low_pair(w0 >> 8), low_pair(w1), low_pair(w1 >> 8));
            const half8 hi = join(high_pair(w0), high_pair(w0 >> 8), high_pair(w1), high_pair(w1 >> 8));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                st.o[4 * h + 2 * pp][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, p[ct], st.o[4 * h + 2 * pp][ct], 0, 0, 0);
                st.o[4 * h + 2 * pp + 1][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, p[ct], st.o[4 * h + 2 * pp + 1][ct], 0, 0, 0);
            }
        }
}

// The transform of O^T's columns: channel 16 c + 4 g + i in accumulator c, lane group g, element i.
template <int D, int CT>
__device__ __forceinline__ void turn_back(floatx4 (&o)[D / 16][CT], int ct) {
    const int lane = lane_id();
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        floatx4 v = o[c][ct];
        v = floatx4{v[0] + v[1], v[0] - v[1], v[2] + v[3], v[2] - v[3]};
        v = floatx4{v[0] + v[2], v[1] + v[3], v[0] - v[2], v[1] - v[3]};
#pragma unroll
        for (int m = 16; m <= 32; m *= 2) {
            const float sign = (lane & m) != 0 ? -1.f : 1.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(sign, v[i], xor_lane_f32(v[i], m));
        }
        o[c][ct] = v;
    }
#pragma unroll
    for (int h = 1; h < D / 16; h *= 2)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            if ((c & h) == 0) {
                const floatx4 u = o[c][ct], v = o[c + h][ct];
                o[c][ct] = u + v;
                o[c + h][ct] = u - v;
            }
}

// kOwn: every wavefront has 16 CT rows of its own; else the four of a workgroup share them and take blocks in turn.
template <int D, int CT, bool kOwn>
__global__ void __launch_bounds__(256) cache_attention_kernel(const AttnArgs a) {
    constexpr int kRows = 16 * CT;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), g = lane >> 4, col = lane & 15;
    // heads fastest: with eight heads each die keeps to one, and its cache to that head's blocks
    int id = blockIdx.x;
    const int head = id % a.kv_heads;
    id /= a.kv_heads;
    const int seq = id % a.seqs;
    id /= a.seqs;
    const int split = id / a.tiles;
    const Seq sq = find_seq(a, seq);
    if (split > 0 && split >= sq.splits) return;
    const int32_t* const pages = a.pages + (int64_t)seq * a.ld_pages;
    const int total = sq.rows * a.group;
    extern __shared__ floatx4 meet[];
    for (int tile = id % a.tiles; tile * (kOwn ? 4 : 1) * kRows < total; tile += a.tiles) {
        const int row0 = (kOwn ? tile * 4 + wave : tile) * kRows;
        State<D, CT> st;
        half8 q[CT][D / 32];
        float qs[CT];
        int see[CT];
        int64_t at[CT];  // row among T * q_heads
        bool there[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int row = row0 + ct * 16 + col;
            there[ct] = row < total;
            const int i = there[ct] ? row / a.group : 0, hq = head * a.group + (there[ct] ? row % a.group : 0);
            at[ct] = (sq.first + i) * a.q_heads + hq;
            const int v = sq.len - sq.rows + i + 1;
            see[ct] = there[ct] && v > 0 ? v : 0;
            qs[ct] = load_queries<D>(a.Q + (sq.first + i) * a.ldq + (int64_t)hq * D + g * (D / 4), there[ct], a.scale, q[ct]);
            st.m[ct] = kNoRow, st.l[ct] = 0.f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st.o[c][ct] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        // rows of the tile see between see_all and see_most places
        const int last = row0 + kRows < total ? row0 + kRows - 1 : total - 1;
        const int see_all = sq.len - sq.rows + (row0 < total ? row0 / a.group : 0) + 1;
        int see_most = row0 < total ? sq.len - sq.rows + last / a.group + 1 : 0;
        see_most = see_most < 0 ? 0 : see_most;
        int b = split * sq.per_split, end = b + sq.per_split;
        const int need = (see_most + kCacheBlock - 1) / kCacheBlock;
        end = end < need ? end : need;
        if (!kOwn) b += wave;
        constexpr int kStep = kOwn ? 1 : 4;
        if (b < end) {
            Block<D> now, next;
            load_block<D>(a, pages, head, b, now);
            for (; b < end; b += kStep) {
                load_block<D>(a, pages, head, b + kStep < end ? b + kStep : b, next);
                attend<D, CT>(now, q, qs, see, see_all, sq.len, st);
                now = next;
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            st.l[ct] += xor_lane_f32(st.l[ct], 16);
            st.l[ct] += xor_lane_f32(st.l[ct], 32);
        }
        if constexpr (!kOwn) {  // the other wavefronts' sums to the first
            floatx4* const mine = meet + (wave - 1) * (64 * (CT * D / 16 + CT));
            if (wave > 0) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) mine[(ct * (D / 16) + c) * 64 + lane] = st.o[c][ct];
                    mine[(CT * D / 16 + ct) * 64 + lane] = floatx4{st.m[ct], st.l[ct], 0.f, 0.f};
                }
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float m = st.m[ct], l[3], f[3];
                    const floatx4* other = meet + (CT * D / 16 + ct) * 64 + lane;
#pragma unroll
                    for (int w = 0; w < 3; ++w) {
                        const floatx4 v = other[w * (64 * (CT * D / 16 + CT))];
                        f[w] = v[0], l[w] = v[1];
                        m = __builtin_fmaxf(m, v[0]);
                    }
                    const float f0 = __builtin_amdgcn_exp2f(st.m[ct] - m);
                    st.m[ct] = m;
                    st.l[ct] *= f0;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) st.o[c][ct] *= f0;
#pragma unroll
                    for (int w = 0; w < 3; ++w) {
                        f[w] = __builtin_amdgcn_exp2f(f[w] - m);
                        st.l[ct] += l[w] * f[w];
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) st.o[c][ct] += meet[w * (64 * (CT * D / 16 + CT)) + (ct * (D / 16) + c) * 64 + lane] * f[w];
                    }
                }
            }
            __syncthreads();
            if (wave != 0) continue;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (sq.splits > 1) {
                const int64_t row = (int64_t)split * a.T * a.q_heads + at[ct];
                if (there[ct]) {
                    if (g == 0) {
                        a.ml[2 * row] = st.m[ct];
                        a.ml[2 * row + 1] = st.l[ct];
                    }
                    floatx4* const o = reinterpret_cast<floatx4*>(a.part + row * D);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) o[4 * c + g] = st.o[c][ct];
                }
            } else {
                turn_back<D, CT>(st.o, ct);
                const float f = st.l[ct] == 0.f ? 0.f : (float)(1.0 / kRootD<D>) / st.l[ct];
                if (there[ct]) {
                    _Float16* const o = a.out + at[ct] / a.q_heads * a.ldo + at[ct] % a.q_heads * D + 4 * g;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        const floatx4 v = st.o[c][ct] * f;
                        *reinterpret_cast<half4*>(o + 16 * c) = half4{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
                    }
                }
            }
        }
    }
}

// Joins the parts of rows whose sequence was split: a workgroup a row, D / 8 lanes a part.
template <int D>
__global__ void __launch_bounds__(256) combine_kernel(const AttnArgs a) {
    constexpr int kLanes = D / 8, kGroups = 256 / kLanes;
    __shared__ float weight[kMaxSplits];
    __shared__ float top[4], sum[4];
    __shared__ __align__(16) float meet[kGroups][D];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const Seq sq = find_seq(a, (int)blockIdx.x);
    if (sq.splits <= 1) return;
    const int64_t stride = a.T * a.q_heads;
    for (int64_t r = blockIdx.y; r < (int64_t)sq.rows * a.q_heads; r += gridDim.y) {
        const int64_t row = sq.first * a.q_heads + r;
        float m = kNoRow, l = 0.f;
        if (tid < sq.splits) {
            m = a.ml[2 * (tid * stride + row)];
            l = a.ml[2 * (tid * stride + row) + 1];
        }
        float most = m;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) most = __builtin_fmaxf(most, xor_lane_f32(most, x));
        if (lane == 0) top[wave] = most;
        __syncthreads();
        most = __builtin_fmaxf(__builtin_fmaxf(top[0], top[1]), __builtin_fmaxf(top[2], top[3]));
        const float w = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - most);
        weight[tid] = w;
        float part = l == 0.f ? 0.f : w * l;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) part += xor_lane_f32(part, x);
        if (lane == 0) sum[wave] = part;
        __syncthreads();
        const float total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        const int grp = tid / kLanes, ch = tid % kLanes * 8;
        float o[8] = {};
        for (int s = grp; s < sq.splits; s += kGroups) {
            const float f = weight[s];
            const floatx4* const p = reinterpret_cast<const floatx4*>(a.part + (s * stride + row) * D + ch);
            const floatx4 u = p[0], v = p[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                o[j] += f == 0.f ? 0.f : u[j] * f;
                o[4 + j] += f == 0.f ? 0.f : v[j] * f;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<floatx4*>(&meet[grp][ch + 4 * i]) = floatx4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
        __syncthreads();
        if (wave == 0) {
            float v[8] = {};
            for (int k = 0; k < kGroups; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += meet[k][ch + j];
            hadamard<D>(v);
            const float f = total == 0.f ? 0.f : (float)(1.0 / kRootD<D>) / total;
            half8 h;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (_Float16)(v[j] * f);
            if (lane < kLanes) *reinterpret_cast<half8*>(a.out + row / a.q_heads * a.ldo + row % a.q_heads * D + ch) = h;
        }
        __syncthreads();
    }
}

// How a call is cut up: CT column tiles of 16 rows a wavefront, own rows or shared ones, workgroups along rows and blocks.
struct Plan {
    int ct;
    bool own;
    int64_t tiles;
    int splits, split_blocks;
};
Plan plan_of(int64_t seqs, int q_heads, int kv_heads, int64_t max_q, int64_t max_kv) {
    Plan p;
    const int64_t rows = max_q * (q_heads / kv_heads);
    p.own = rows > 128;
    p.ct = rows <= 16 ? 1 : 2;
    const int64_t per = 16 * p.ct * (p.own ? 4 : 1);
    p.tiles = (rows + per - 1) / per;
    const int64_t blocks = (max_kv + kCacheBlock - 1) / kCacheBlock, units = seqs * kv_heads * p.tiles;
    // parts of at least four blocks (one a wavefront), and no more of them than about eight workgroups a compute unit
    int64_t per_split = (units * blocks + 2047) / 2048;
    per_split = per_split < 4 ? 4 : (per_split + 3) / 4 * 4;
    if (p.own && per_split < 16) per_split = 16;
    const int64_t least = (blocks + kMaxSplits - 1) / kMaxSplits;
    if (per_split < least) per_split = least;
    p.split_blocks = (int)per_split;
    p.splits = (int)((blocks + per_split - 1) / per_split);
    if (p.splits < 1) p.splits = 1;
    return p;
}

template <int D, int CT, bool kOwn>
int start(const AttnArgs& a, int64_t grid, hipStream_t st) {
    constexpr int kLds = kOwn ? 0 : 3 * 64 * (CT * D / 16 + CT) * 16;
    if constexpr (kLds > 65536) {
        static DeviceOnce once;
        if (!raise_lds_limit(once, reinterpret_cast<const void*>(&cache_attention_kernel<D, CT, kOwn>), kLds)) return -6;
    }
    cache_attention_kernel<D, CT, kOwn><<<dim3((unsigned)grid), dim3(256), kLds, st>>>(a);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

template <int D>
int start(const AttnArgs& a, const Plan& p, int64_t grid, int64_t max_q, hipStream_t st) {
    int rc;
    if (p.own) rc = start<D, 2, true>(a, grid, st);
    else if (p.ct == 1) rc = start<D, 1, false>(a, grid, st);
    else rc = start<D, 2, false>(a, grid, st);
    if (rc != 0 || p.splits <= 1) return rc;
    const int64_t rows = max_q * a.q_heads;
    combine_kernel<D><<<dim3((unsigned)a.seqs, (unsigned)(rows < 65535 ? rows : 65535)), dim3(256), 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

}  // namespace

size_t cache_attention_bytes(int64_t T, int64_t seqs, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv) {
    const Plan p = plan_of(seqs, q_heads, kv_heads, max_q, max_kv);
    if (p.splits <= 1) return 256;
    return (size_t)p.splits * (size_t)T * (size_t)q_heads * (size_t)(head_dim + 2) * 4 + 256;
}

int launch_cache_attention(const CacheAttentionCall& c, hipStream_t st) {
    const int G = c.q_heads / c.cache.kv_heads, D = c.cache.head_dim;
    const Plan p = plan_of(c.seqs, c.q_heads, c.cache.kv_heads, c.max_q, c.max_kv);
    AttnArgs a{};
    a.Q = c.Q, a.starts = c.starts, a.kv_lens = c.kv_lens, a.pages = c.pages, a.data = c.cache.data, a.out = c.out, a.flags = c.flags;
    a.part = static_cast<float*>(c.workspace);
    a.ml = a.part + (size_t)p.splits * (size_t)c.T * (size_t)c.q_heads * (size_t)D;
    a.ldq = c.ldq, a.ldo = c.ldo, a.ld_pages = c.ld_pages, a.T = c.T, a.pool = c.cache.pages;
    a.scale = (float)((double)c.scale * 1.44269504088896340736 / (D == 64 ? 8.0 : D == 128 ? 11.313708498984760390 : 16.0));
    a.q_heads = c.q_heads, a.kv_heads = c.cache.kv_heads, a.group = G, a.seqs = (int)c.seqs, a.tiles = (int)p.tiles, a.splits = p.splits, a.split_blocks = p.split_blocks;
    a.page_shift = __builtin_ctz((unsigned)c.cache.page_blocks);
    const int64_t grid = c.seqs * c.cache.kv_heads * p.tiles * p.splits;
    if (grid > 0x7fffffffLL) return -2;
    if (D == 64) return start<64>(a, p, grid, c.max_q, st);
    if (D == 128) return start<128>(a, p, grid, c.max_q, st);
    return start<256>(a, p, grid, c.max_q, st);
}

}  // namespace itq3s

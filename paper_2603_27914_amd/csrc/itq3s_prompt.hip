// Attention of whole prompts over their own keys and values in fp16: o = softmax(scale q k^T) v, causal or not, grouped
// heads, sequences of different lengths packed behind each other.
//
// A wavefront takes 32 or 64 query rows (a row: one head of one token; the heads of a group are neighbouring rows, so that a
// workgroup's keys serve them all) as columns of  S^T = K Q^T  and  O^T += V^T P^T.  With 32x32x16 products the accumulator of
// S^T leaves a lane, for its column, the tokens 16 k + 4 (l / 32) + {0..3, 8..11} of step k: taken as they stand they are the
// operand P^T of step k, if V^T comes with its tokens in the same order.  So weights never leave their lane, and only a
// row's maximum crosses to one other lane, when it moves by more than 2^8 (else the old reference is as good).
// Keys and values pass through LDS in tiles of 64 tokens, rows as in memory, 16-byte chunks permuted within a row
// against bank conflicts; V^T is read with the transposing LDS read.  The next tile is on its way to registers meanwhile.
#include "itq3s_attention.h"
#include "itq3s_cache.h"

namespace itq3s {

namespace {

constexpr float kNoRow = -1e30f;
constexpr float kHeadroom = 8.f;
template <int D>
constexpr int kTile = D <= 128 ? 64 : 32;  // tokens of a tile

struct PromptArgs {
    const _Float16 *Q, *K, *V;
    const int32_t* starts;
    _Float16* out;
    int64_t ldq, ldk, ldv, ldo;
    float scale;    // |softmax scale| * log2(e)
    _Float16 sign;  // the scale's sign, which the queries take (a scale of 0: 0, and any other scale)
    int q_heads, kv_heads, group, seqs, tiles, causal, T;
};

typedef short short4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ half4 read_turned(const _Float16* p) {
    typedef __attribute__((address_space(3))) short4v* lds_t;
    return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(short4v*)p));
}

// Where chunk c (eight channels) of row r of a tile stands: keys are read a row a lane, so rows shift by one; values four
// rows of two chunks at once, so rows shift by two.
template <int D>
__device__ __forceinline__ int k_at(int r, int c) { return (r * (D / 8) + (c ^ (r & (D / 8 < 16 ? D / 8 - 1 : 15)))) * 8; }
template <int D>
__device__ __forceinline__ int v_at(int r, int c) { return (r * (D / 8) + (c ^ ((2 * r) & (D / 8 < 16 ? D / 8 - 1 : 15)))) * 8; }

template <int D, int RT>
__global__ void __launch_bounds__(256) prompt_kernel(const PromptArgs a) {
    constexpr int kChunks = kTile<D> * D / 8 / 256;  // 16-byte chunks of a tile a thread moves
    __shared__ __align__(16) _Float16 ks[kTile<D> * D];
    __shared__ __align__(16) _Float16 vs[kTile<D> * D];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = lane_id(), hi = lane >> 5, col = lane & 31;
    int id = blockIdx.x;
    const int head = id % a.kv_heads;
    id /= a.kv_heads;
    const int seq = id % a.seqs;
    int64_t first = a.starts[seq], end = a.starts[seq + 1];
    first = first < 0 ? 0 : first > a.T ? a.T : first;
    end = end < first ? first : end > a.T ? a.T : end;
    const int len = (int)(end - first), total = len * a.group;
    constexpr int kRows = 128 * RT;
    const int count = (total + kRows - 1) / kRows;
    const _Float16* const kb = a.K + first * a.ldk + (int64_t)head * D;
    const _Float16* const vb = a.V + first * a.ldv + (int64_t)head * D;
    // the last rows have the most to see: they begin
    for (int tile = count - 1 - id / a.seqs; tile >= 0; tile -= a.tiles) {
        const int row0 = tile * kRows + wave * 32 * RT;
        half8 q[RT][D / 16];
        int see[RT];
        floatx16 o[D / 32][RT];
        float m[RT], l[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int row = row0 + 32 * t + col;
            const bool there = row < total;
            const int i = there ? row / a.group : 0, hq = head * a.group + (there ? row % a.group : 0);
            const half8* const p = reinterpret_cast<const half8*>(a.Q + (first + i) * a.ldq + (int64_t)hq * D + 8 * hi);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) q[t][k] = there ? p[2 * k] * a.sign : half8{};
            see[t] = !there ? 0 : a.causal ? i + 1 : len;
            m[t] = kNoRow, l[t] = 0.f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[c][t][x] = 0.f;
        }
        const int last_row = (tile + 1) * kRows < total ? (tile + 1) * kRows - 1 : total - 1;
        const int tokens = a.causal ? last_row / a.group + 1 : len;  // that the workgroup needs
        const int my_last = row0 + 32 * RT < total ? row0 + 32 * RT - 1 : total - 1;
        const int mine = row0 >= total ? 0 : a.causal ? my_last / a.group + 1 : len;  // that this wavefront needs
        const int all = row0 >= total ? 0 : a.causal ? row0 / a.group + 1 : len;      // that all of its rows see

        half8 kr[kChunks], vr[kChunks];
        auto load = [&](int t0) {
#pragma unroll
            for (int u = 0; u < kChunks; ++u) {
                const int x = tid + 256 * u, r = t0 + x / (D / 8), c = x % (D / 8);
                const bool in = r < len;  // rows behind the sequence are another's, or nothing: zeros
                const int64_t rr = in ? r : len - 1;
                kr[u] = *reinterpret_cast<const half8*>(kb + rr * a.ldk + 8 * c);
                vr[u] = *reinterpret_cast<const half8*>(vb + rr * a.ldv + 8 * c);
                if (!in) kr[u] = half8{}, vr[u] = half8{};
            }
        };
        load(0);
        for (int t0 = 0; t0 < tokens; t0 += kTile<D>) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kChunks; ++u) {
                const int x = tid + 256 * u, r = x / (D / 8), c = x % (D / 8);
                *reinterpret_cast<half8*>(ks + k_at<D>(r, c)) = kr[u];
                *reinterpret_cast<half8*>(vs + v_at<D>(r, c)) = vr[u];
            }
            __syncthreads();
            if (t0 + kTile<D> < tokens) load(t0 + kTile<D>);
            if (t0 >= mine) continue;
#pragma unroll
            for (int tt = 0; tt < kTile<D> / 32; ++tt) {
                floatx16 s[RT];
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[t][x] = 0.f;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const half8 kf = *reinterpret_cast<const half8*>(ks + k_at<D>(32 * tt + col, 2 * k + hi));
#pragma unroll
                    for (int t = 0; t < RT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, q[t][k], s[t], 0, 0, 0);
                }
                half8 p[RT][2];
                const bool edge = t0 + 32 * tt + 32 > all;
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if (edge) {
#pragma unroll
                        for (int x = 0; x < 16; ++x)
                            s[t][x] = t0 + 32 * tt + 8 * (x / 4) + 4 * hi + x % 4 < see[t] ? s[t][x] : -__builtin_inff();
                    }
                    float top = s[t][0];
#pragma unroll
                    for (int x = 1; x < 16; ++x) top = __builtin_fmaxf(top, s[t][x]);
                    top *= a.scale;
                    if (__builtin_amdgcn_ballot_w64(top > m[t] + kHeadroom) != 0) {
                        top = __builtin_fmaxf(top, xor_lane_f32(top, 32));
                        const float n = __builtin_fmaxf(m[t], top), f = __builtin_amdgcn_exp2f(m[t] - n);
                        m[t] = n;
                        l[t] *= f;
#pragma unroll
                        for (int c = 0; c < D / 32; ++c)
#pragma unroll
                            for (int x = 0; x < 16; ++x) o[c][t][x] *= f;
                    }
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][x], a.scale, -m[t]));
                        l[t] += e;
                        p[t][x / 8][x % 8] = (_Float16)e;
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        const int r = 32 * tt + 16 * k + 4 * hi + ((lane >> 2) & 3), ch = 32 * c + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                        const half4 u = read_turned(vs + v_at<D>(r, ch / 8) + (ch & 4)), w = read_turned(vs + v_at<D>(r + 8, ch / 8) + (ch & 4));
                        const half8 vf = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
#pragma unroll
                        for (int t = 0; t < RT; ++t) o[c][t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, p[t][k], o[c][t], 0, 0, 0);
                    }
            }
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            l[t] += xor_lane_f32(l[t], 32);
            const float f = l[t] == 0.f ? 0.f : 1.f / l[t];
            const int row = row0 + 32 * t + col;
            if (row < total) {
                _Float16* const out = a.out + (first + row / a.group) * a.ldo + (int64_t)(head * a.group + row % a.group) * D + 4 * hi;
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        *reinterpret_cast<half4*>(out + 32 * c + 8 * x) = half4{(_Float16)(o[c][t][4 * x] * f), (_Float16)(o[c][t][4 * x + 1] * f), (_Float16)(o[c][t][4 * x + 2] * f),
                                                                                (_Float16)(o[c][t][4 * x + 3] * f)};
            }
        }
    }
}

// Copies global -> LDS, 16 bytes a lane: lane l to lds + 16 l from its offset; zeros from beyond the descriptor's range.  (m0 is
// reserved and cannot be named as clobbered: nothing else in a kernel with these copies uses it, which a test reads from
// the assembly.  What the copies write, sync() orders for the compiler as well.)
__device__ __forceinline__ void copy_to_lds(u32x4 rsrc, int offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(rsrc));
}
__device__ __forceinline__ void sync_copies() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ u32x4 rows_descriptor(const _Float16* p, int64_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, (uint32_t)bytes, 0x00027000u};
}

// 64 rows a wavefront, two column tiles of 32, as a pipeline: while the matrix cores work on one column tile (the scores of the
// next 32 tokens, the products of these), the vector ALU makes weights of the other one's scores; the operands of
// the next 32 tokens come from LDS meanwhile.  One wavefront a SIMD (some 400 registers): the two halves of
// its own work fill both pipes, and an operand read from LDS serves 64 rows, which is what LDS can deliver.
template <int D>
struct Pipe {
    half8 q[2][D / 16];
    floatx16 o[2][D / 32], s[2];
    half8 p[2][2];
    half8 kf[D / 16], vf[2][D / 32];  // keys of the next 32 tokens, values of these
    float m[2], l[2];
    int see[2];
};

// A lane's places in a tile, in bytes: of the key chunk of step k in its row, of the value chunk of channel tile c in its row.
template <int D>
struct Places {
    uint32_t k[D / 16], v[D / 32];
};
template <int D>
__device__ __forceinline__ Places<D> find_places(int lane) {
    Places<D> p;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) p.k[k] = (uint32_t)k_at<D>(lane & 31, 2 * k + (lane >> 5)) * 2;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        const int r = 4 * (lane >> 5) + ((lane >> 2) & 3), ch = 32 * c + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        p.v[c] = (uint32_t)(v_at<D>(r, ch / 8) + (ch & 4)) * 2;
    }
    return p;
}
// (32 rows of a tile from `at` on; the permutation of a row's chunks repeats every 16 rows of keys, every 8 of values)
template <int D>
__device__ __forceinline__ half8 key_part(const unsigned char* at, const Places<D>& p, int k) {
    return *reinterpret_cast<const half8*>(at + p.k[k]);
}
template <int D>
__device__ __forceinline__ half8 value_part(const unsigned char* at, const Places<D>& p, int k, int c) {
    const half4 u = read_turned(reinterpret_cast<const _Float16*>(at + p.v[c] + 16 * k * D * 2)), w = read_turned(reinterpret_cast<const _Float16*>(at + p.v[c] + (16 * k + 8) * D * 2));
    return half8{u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
}

// Scores of tokens from t0 on, masked, against the row's reference: it moves where a weight would pass 2^8.
template <int D, int X>
__device__ __forceinline__ void set_reference(Pipe<D>& w, int t0, int all, float scale, int hi) {
    floatx16& s = w.s[X];
    if (t0 + 32 > all) {
        asm volatile("");  // (a branch stays one: few tiles are cut)
#pragma unroll
        for (int x = 0; x < 16; ++x) s[x] = t0 + 8 * (x / 4) + 4 * hi + x % 4 < w.see[X] ? s[x] : -__builtin_inff();
    }
    float top = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) top = __builtin_fmaxf(top, s[x]);
    top *= scale;
    if (__builtin_amdgcn_ballot_w64(top > w.m[X] + kHeadroom) != 0) {
        top = __builtin_fmaxf(top, xor_lane_f32(top, 32));
        const float n = __builtin_fmaxf(w.m[X], top), f = __builtin_amdgcn_exp2f(w.m[X] - n);
        w.m[X] = n;
        w.l[X] *= f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) w.o[X][c] *= f;
    }
}

// One half step: column tile X's scores of tokens t + 1 and products of tokens t on the matrix cores, the other one's weights on the
// vector ALU (of t for X = 0, of t + 1 for X = 1).  In the second half the operands of step t + 1 are read.
template <int D, int X>
__device__ __forceinline__ void half_step(Pipe<D>& w, const unsigned char* kn, const unsigned char* vn, const Places<D>& places, float scale) {
    constexpr int Y = 1 - X;
    floatx16 s;
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(w.kf[k], w.q[X][k], s, 0, 0, 0);
        if constexpr (X == 1) w.kf[k] = key_part<D>(kn, places, k);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            w.o[X][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w.vf[k][c], w.p[X][k], w.o[X][c], 0, 0, 0);
            if constexpr (X == 1) w.vf[k][c] = value_part<D>(vn, places, k, c);
        }
    const float m = w.m[Y];
    float l = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(w.s[Y][x], scale, -m));
        l += e;
        w.p[Y][x / 8][x % 8] = (_Float16)e;
    }
    w.l[Y] += l;
    w.s[X] = s;
    asm volatile("" : "+v"(w.p[Y][0]), "+v"(w.p[Y][1]), "+v"(w.l[Y]));  // (made here, beside the products, and not where they are used)
    // a matrix instruction (32 cycles), then what fits beside it
#pragma unroll
    for (int i = 0; i < 3 * D / 32; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (X == 1) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, X == 1 ? 5 : 4, 0);
    }
}

template <int D>
__global__ void __launch_bounds__(256, 1) prompt_pipe_kernel(const PromptArgs a) {
    constexpr int kChunks = kTile<D> * D / 8 / 256, kBuffers = 3;
    constexpr int kTileBytes = kTile<D> * D * 2, kValues = kBuffers * kTileBytes;
    extern __shared__ __align__(1024) unsigned char lds[];  // three tiles of keys, three of values
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = lane_id(), hi = lane >> 5, col = lane & 31;
    const Places<D> places = find_places<D>(lane);
    int id = blockIdx.x;
    const int head = id % a.kv_heads;
    id /= a.kv_heads;
    const int seq = id % a.seqs;
    int first = a.starts[seq], end = a.starts[seq + 1];
    first = first < 0 ? 0 : first > a.T ? a.T : first;
    end = end < first ? first : end > a.T ? a.T : end;
    const int len = end - first, total = len * a.group;
    constexpr int kRows = 256;
    const int count = (total + kRows - 1) / kRows;
    const _Float16* const kb = a.K + (int64_t)first * a.ldk + (int64_t)head * D;
    const _Float16* const vb = a.V + (int64_t)first * a.ldv + (int64_t)head * D;
    // the last rows have the most to see: they begin
    for (int tile = count - 1 - id / a.seqs; tile >= 0; tile -= a.tiles) {
        const int row0 = tile * kRows + wave * 64;
        const int last_row = (tile + 1) * kRows < total ? (tile + 1) * kRows - 1 : total - 1;
        const int tokens = a.causal ? last_row / a.group + 1 : len;  // that the workgroup needs
        const int my_last = row0 + 64 < total ? row0 + 63 : total - 1;
        const int mine = row0 >= total ? 0 : a.causal ? my_last / a.group + 1 : len;  // that this wavefront needs
        const int all = row0 >= total ? 0 : a.causal ? row0 / a.group + 1 : len;      // that all of its rows see
        const int steps = (mine + 31) / 32, rounds = (tokens + kTile<D> - 1) / kTile<D>;
        // thread x moves chunks x + 256 u of a tile: rows r + 256 / (D / 8) u, in a chunk's place the one that k_at, v_at put there
        const int r = tid / (D / 8), c = tid % (D / 8);
        const int k_off = (int)(r * a.ldk * 2) + (c ^ (r & (D / 8 < 16 ? D / 8 - 1 : 15))) * 16, v_off = (int)(r * a.ldv * 2) + (c ^ ((2 * r) & (D / 8 < 16 ? D / 8 - 1 : 15))) * 16;
        auto load = [&](int t0, int buffer) {  // (rows behind the sequence are another's, or nothing: zeros)
            const int rows = len - t0 < kTile<D> ? len - t0 : kTile<D>;
            const u32x4 kd = rows_descriptor(kb + t0 * a.ldk, rows > 0 ? ((rows - 1) * a.ldk + D) * 2 : 0);
            const u32x4 vd = rows_descriptor(vb + t0 * a.ldv, rows > 0 ? ((rows - 1) * a.ldv + D) * 2 : 0);
            const uint32_t to = lds_base + (uint32_t)(buffer * kTileBytes + wave * 1024);
#pragma unroll
            for (int u = 0; u < kChunks; ++u) {
                copy_to_lds(kd, k_off + (int)(u * (2048 / D) * 2 * a.ldk), to + u * 4096);
                copy_to_lds(vd, v_off + (int)(u * (2048 / D) * 2 * a.ldv), to + kValues + u * 4096);
            }
        };
        sync_copies();  // (the tiles before are read)
        load(0, 0);
        load(kTile<D>, 1);
        Pipe<D> w;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = row0 + 32 * t + col;
            const bool there = row < total;
            const int i = there ? row / a.group : 0, hq = head * a.group + (there ? row % a.group : 0);
            const half8* const p = reinterpret_cast<const half8*>(a.Q + (int64_t)(first + i) * a.ldq + (int64_t)hq * D + 8 * hi);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) w.q[t][k] = p[2 * k] * a.sign;
            w.see[t] = !there ? 0 : a.causal ? i + 1 : len;
            w.m[t] = kNoRow, w.l[t] = 0.f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int x = 0; x < 16; ++x) w.o[t][c][x] = 0.f;
        }
        sync_copies();
        if (steps > 0) {
            floatx16 s[2];
#pragma unroll
            for (int x = 0; x < 16; ++x) s[0][x] = s[1][x] = 0.f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const half8 f = key_part<D>(lds, places, k);
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, w.q[0][k], s[0], 0, 0, 0);
                s[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, w.q[1][k], s[1], 0, 0, 0);
                w.kf[k] = key_part<D>(lds + 64 * D, places, k);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int c = 0; c < D / 32; ++c) w.vf[k][c] = value_part<D>(lds + kValues, places, k, c);
            w.s[0] = s[0], w.s[1] = s[1];
            set_reference<D, 0>(w, 0, all, a.scale, hi);
            set_reference<D, 1>(w, 0, all, a.scale, hi);
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(w.s[0][x], a.scale, -w.m[0]));
                w.l[0] += e;
                w.p[0][x / 8][x % 8] = (_Float16)e;
            }
        }
        // Tile r + 1 is in LDS when round r begins: its steps 2 r and 2 r + 1 read keys up to 2 r + 3, values up to 2 r + 2.  What is
        // written in a round is tile r + 2, in the place of tile r - 1, which nobody has read since the last barrier.
        int buffer = 0;
        for (int r = 0; r < rounds; ++r) {
            const int after = buffer == 2 ? 0 : buffer + 1;
            load((r + 2) * kTile<D>, after == 2 ? 0 : after + 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = 2 * r + h;
                if (t < steps) {
                    half_step<D, 0>(w, nullptr, nullptr, places, a.scale);
                    set_reference<D, 0>(w, 32 * t + 32, all, a.scale, hi);
                    half_step<D, 1>(w, lds + after * kTileBytes + 64 * D * h, lds + kValues + (h == 0 ? buffer * kTileBytes + 64 * D : after * kTileBytes), places, a.scale);
                    set_reference<D, 1>(w, 32 * t + 32, all, a.scale, hi);
                }
            }
            sync_copies();
            buffer = after;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            w.l[t] += xor_lane_f32(w.l[t], 32);
            const float f = w.l[t] == 0.f ? 0.f : 1.f / w.l[t];
            const int row = row0 + 32 * t + col;
            if (row < total) {
                _Float16* const out = a.out + (int64_t)(first + row / a.group) * a.ldo + (int64_t)(head * a.group + row % a.group) * D + 4 * hi;
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const floatx16& o = w.o[t][c];
                        *reinterpret_cast<half4*>(out + 32 * c + 8 * x) = half4{(_Float16)(o[4 * x] * f), (_Float16)(o[4 * x + 1] * f), (_Float16)(o[4 * x + 2] * f), (_Float16)(o[4 * x + 3] * f)};
                    }
            }
        }
    }
}

template <int D>
int start(const PromptArgs& a, int64_t max_len, hipStream_t st) {
    // 64 rows a wavefront where that leaves every compute unit a workgroup, else 32
    const int64_t rows = max_len * a.group, units = (int64_t)a.seqs * a.kv_heads;
    const bool wide = D <= 128 && units * ((rows + 255) / 256) >= cu_count();
    PromptArgs b = a;
    const int64_t per = wide ? 256 : 128, tiles = (rows + per - 1) / per;
    if (units * tiles > 0x7fffffffLL) return -2;
    b.tiles = (int)tiles;
    const dim3 grid((unsigned)(units * tiles));
    if constexpr (D <= 128) {
        if (wide) {
            constexpr int kLds = 2 * 3 * kTile<D> * D * 2;
            if constexpr (kLds > 65536) {
                static DeviceOnce once;
                if (!raise_lds_limit(once, reinterpret_cast<const void*>(&prompt_pipe_kernel<D>), kLds)) return -6;
            }
            prompt_pipe_kernel<D><<<grid, dim3(256), kLds, st>>>(b);
            return hipGetLastError() == hipSuccess ? 0 : -6;
        }
    }
    prompt_kernel<D, 1><<<grid, dim3(256), 0, st>>>(b);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

}  // namespace

int launch_prompt_attention(const PromptCall& c, hipStream_t st) {
    PromptArgs a{};
    a.Q = c.Q, a.K = c.K, a.V = c.V, a.starts = c.starts, a.out = c.out;
    a.ldq = c.ldq, a.ldk = c.ldk, a.ldv = c.ldv, a.ldo = c.ldo, a.T = (int)c.T;
    a.scale = c.scale == 0.f ? 1.f : (float)(__builtin_fabs((double)c.scale) * 1.44269504088896340736);
    a.sign = (_Float16)(c.scale > 0.f ? 1.f : c.scale < 0.f ? -1.f : 0.f);
    a.q_heads = c.q_heads, a.kv_heads = c.kv_heads, a.group = c.q_heads / c.kv_heads, a.seqs = (int)c.seqs, a.causal = c.causal;
    if (c.head_dim == 64) return start<64>(a, c.max_len, st);
    if (c.head_dim == 128) return start<128>(a, c.max_len, st);
    return start<256>(a, c.max_len, st);
}

}  // namespace itq3s

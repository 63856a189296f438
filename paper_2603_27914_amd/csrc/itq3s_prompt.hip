// Attention of whole prompts over their own keys and values in fp16: o = softmax(scale q k^T) v, causal or not, grouped
// heads, sequences of different lengths packed behind each other.
//
// A wavefront takes 32 query rows (a row: one head of one token; the heads of a group are neighbouring rows, so that a
// workgroup's keys serve them all) as columns of  S^T = K Q^T  and  O^T += V^T P^T.  With 32x32x16 products the accumulator of
// S^T leaves a lane, for its column, the tokens 16 k + 4 (l / 32) + {0..3, 8..11} of step k: taken as they stand they are the
// operand P^T of step k, if V^T comes with its tokens in the same order.  So weights never leave their lane, and only a
// row's maximum crosses to one other lane, when it moves by more than 2^8 (else the old reference is as good).
//
// Tiles of 32 tokens are copied to LDS by the memory pipe, a tile ahead, rows as in memory, 16-byte chunks permuted within a
// row against bank conflicts (by the address that each lane copies from); V^T is read with the transposing LDS read.
// Few rows leave compute units with little: there two wavefronts share the tokens of the same rows and join in LDS.
// Many: three workgroups of four wavefronts a compute unit: nothing in a wavefront overlaps its products with its exponentials, the
// others do.  (One wavefront a SIMD with 64 rows, which reads LDS half as often, and its two halves interleaved by hand: 606
// us where this took 546, 8192 tokens, 32 query and 8 kv heads of 128.)  That takes 535 us by now, 1.03 PFLOP/s, where a matrix product
// of 8192 x 8192 x 8192 reaches 1.21; the matrix pipes are busy for 59 % of the time, the vector ALU for 47 %, and the clock is down
// to 1.66 GHz by what that draws.  Neither products nor softmax first (wavefront priorities) helped: 556 and 562 us where it was 554.
#include <type_traits>

#include "itq3s_attention.h"
#include "itq3s_cache.h"

namespace itq3s {

namespace {

constexpr float kNoRow = -1e30f;
constexpr float kHeadroom = 8.f;
constexpr float kFar = 4194304.f;  // 2^22: references beyond it are rounded by more than a weight's exponent takes
constexpr int kTile = 32;  // tokens of a tile

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
__device__ __forceinline__ half4 read_turned(const unsigned char* p) {
    typedef __attribute__((address_space(3))) short4v* lds_t;
    return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(short4v*)p));
}

// Chunk c (eight channels) of row r of a tile stands in chunk c ^ k_mix(r) (keys) or c ^ v_mix(r) (values) of its row.  Keys are read
// a row a lane, 16 rows at a time, values four rows of four chunks at a time: either way the 64 banks once.
template <int D>
__device__ __forceinline__ constexpr int k_mix(int r) { return D == 64 ? (r >> 1) & 7 : r & 15; }
template <int D>
__device__ __forceinline__ constexpr int v_mix(int r) { return D == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); }

// A lane's places in a tile, in bytes: of the key chunk of step 0 in its row, of the value chunk of channel tile 0 in its row.  The
// others differ from them in the bits of the chunk's number alone, which the permutations flip: by exclusive or.
template <int D>
__device__ __forceinline__ uint32_t key_place(int lane) {
    const int r = lane & 31;
    return (uint32_t)(r * D * 2 + ((lane >> 5) ^ k_mix<D>(r)) * 16);
}
template <int D>
__device__ __forceinline__ uint32_t value_place(int lane) {
    const int r = 4 * (lane >> 5) + ((lane >> 2) & 3), ch = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    return (uint32_t)(r * D * 2 + ((ch / 8) ^ v_mix<D>(r)) * 16 + (ch & 4) * 2);
}
template <int D>
__device__ __forceinline__ half8 key_part(const unsigned char* lds, uint32_t at, int k) {
    return *reinterpret_cast<const half8*>(lds + (at ^ (uint32_t)(32 * k)));
}
template <int D>
__device__ __forceinline__ half8 value_part(const unsigned char* lds, uint32_t at, int k, int c) {
    const unsigned char* const p = lds + (at ^ (uint32_t)(64 * c)) + 16 * k * D * 2;
    const half4 u = read_turned(p), w = read_turned(p + 8 * D * 2);
    return half8{u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
}

// A tile of values with zeros for those that are not finite, 16 bytes of 1024 a lane, and the first token that has one (none: one beyond all).
template <int D>
__device__ __forceinline__ int copy_finite_values(const unsigned char* tile, unsigned char* to) {
    int first = 1 << 30;
#pragma unroll 1
    for (int u = kTile * D * 2 / 1024 - 1; u >= 0; --u) {
        u32x4 v = *reinterpret_cast<const u32x4*>(tile + 1024 * u);
        bool finite = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool lo = (v[i] & 0x7c00u) != 0x7c00u, hi = (v[i] & 0x7c000000u) != 0x7c000000u;
            v[i] &= (lo ? 0xffffu : 0u) | (hi ? 0xffff0000u : 0u);
            finite = finite && lo && hi;
        }
        *reinterpret_cast<u32x4*>(to + 1024 * u) = v;
        const uint64_t bad = __builtin_amdgcn_ballot_w64(!finite);
        if (bad != 0) first = (u * 1024 + (int)__builtin_ctzll(bad) * 16) / (D * 2);
    }
    return first;
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

// Wavefronts a SIMD: what LDS has room for, three for 128 channels.
constexpr int waves_of_simd(int D, int waves, int parts) { return D == 64 ? 4 : parts == 2 ? (D == 128 ? 2 : 1) : D == 128 ? waves / 2 + waves / 4 : waves / 2; }

// kParts = 2: the wavefronts of one half take the tiles 0, 2, 4, ..., the others, with the same rows, 1, 3, 5, ..., and join in the end.
template <int D, int kWaves, int kParts>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(waves_of_simd(D, kWaves, kParts), waves_of_simd(D, kWaves, kParts)))) prompt_kernel(const PromptArgs a) {
    constexpr int kThreads = 64 * kWaves, kTokens = kTile * kParts, kChunks = kTokens * D / 8 / kThreads, kTileBytes = kTile * D * 2, kStepBytes = kParts * kTileBytes, kValues = 2 * kStepBytes;
    constexpr int kStep = kThreads * 8 / D;  // rows between a thread's chunks
    __shared__ __align__(1024) unsigned char lds[4 * kStepBytes];  // keys of two steps, values of two
    __shared__ int not_finite;                                     // some result of the workgroup's is not
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int part = kParts == 1 ? 0 : wave / (kWaves / kParts), group = kParts == 1 ? wave : wave % (kWaves / kParts);  // which tiles and which rows
    int id = blockIdx.x;
    const int head = id % a.kv_heads;
    id /= a.kv_heads;
    const int seq = id % a.seqs;
    int first = a.starts[seq], end = a.starts[seq + 1];
    first = first < 0 ? 0 : first > a.T ? a.T : first;
    end = end < first ? first : end > a.T ? a.T : end;
    const int len = end - first, total = len * a.group;
    constexpr int kRows = 32 * kWaves / kParts;
    const int count = (total + kRows - 1) / kRows;
    const _Float16* const kb = a.K + (int64_t)first * a.ldk + (int64_t)head * D;
    const _Float16* const vb = a.V + (int64_t)first * a.ldv + (int64_t)head * D;
    // The rows of a tile; with care for values that are not finite (see below).
    auto rows_of = [&](int tile, auto with_care) {
        constexpr bool careful = decltype(with_care)::value;
        int lane = lane_id();
        if constexpr (careful) asm volatile("" : "+v"(lane));  // (what hangs on it is not kept for this)
        const int tid = wave * 64 + lane, hi = lane >> 5, col = lane & 31;
        const uint32_t k_place = key_place<D>(lane) + part * kTileBytes, v_place = value_place<D>(lane) + kValues + part * kTileBytes;
        const int row0 = tile * kRows + group * 32, row = row0 + col;
        const int last_row = (tile + 1) * kRows < total ? (tile + 1) * kRows - 1 : total - 1;
        const int tokens = a.causal ? last_row / a.group + 1 : len;  // that the workgroup needs
        const int my_last = row0 + 32 < total ? row0 + 31 : total - 1;
        const int mine = row0 >= total ? 0 : a.causal ? my_last / a.group + 1 : len;  // that this wavefront needs
        const int all = row0 >= total ? 0 : a.causal ? row0 / a.group + 1 : len;      // that all of its rows see

        // thread x copies the chunks whose places are x, x + kThreads, ...: row r, then kStep rows on
        const int r = tid / (D / 8), c = tid % (D / 8);
        const int k_row = (int)(r * a.ldk * 2), v_row = (int)(r * a.ldv * 2), k_chunk = (c ^ k_mix<D>(r)) * 16, v_chunk = (c ^ v_mix<D>(r)) * 16;
        auto load = [&](int t0, int buffer) {  // (rows behind the sequence are another's, or nothing: zeros)
            const int rows = len - t0 < kTokens ? len - t0 : kTokens;
            const u32x4 kd = rows_descriptor(kb + t0 * a.ldk, rows > 0 ? ((rows - 1) * a.ldk + D) * 2 : 0);
            const u32x4 vd = rows_descriptor(vb + t0 * a.ldv, rows > 0 ? ((rows - 1) * a.ldv + D) * 2 : 0);
            const uint32_t to = lds_base + (uint32_t)(buffer * kStepBytes + wave * 1024);
#pragma unroll
            for (int u = 0; u < kChunks; ++u) {
                copy_to_lds(kd, k_row + (int)(u * kStep * 2 * a.ldk) + (k_chunk ^ k_mix<D>(u * kStep) * 16), to + u * kThreads * 16);
                copy_to_lds(vd, v_row + (int)(u * kStep * 2 * a.ldv) + (v_chunk ^ v_mix<D>(u * kStep) * 16), to + kValues + u * kThreads * 16);
            }
        };
        sync_copies();  // (the tiles before are read)
        load(0, 0);
        half8 q[D / 16];
        floatx16 o[D / 32];
        const bool there = row < total;
        const int i = there ? row / a.group : 0, hq = head * a.group + (there ? row % a.group : 0), see = !there ? 0 : a.causal ? i + 1 : len;
        // A row's reference is m + far * scale; one of them is 0.  m is a score's product with the scale, rounded, and a weight's exponent the
        // exact difference from it: that holds what the rounding left, of a score of 2^28 more than fp16 has.  So where a row passes
        // kFar its reference is its largest score before the scale, taken off the others before they are scaled.  room is how far
        // scores may be above m: kHeadroom, or minus infinity (every tile moves references) once a row of the wavefront is there.
        float m = kNoRow, far = 0.f, l = 0.f, room = kHeadroom;
        {
            const half8* const p = reinterpret_cast<const half8*>(a.Q + (int64_t)(first + i) * a.ldq + (int64_t)hq * D + 8 * hi);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) q[k] = p[2 * k] * a.sign;
        }
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int y = 0; y < 16; ++y) o[x][y] = 0.f;
        int buffer = 0;
        for (int step = 0; step < tokens; step += kTokens, buffer ^= 1) {
            sync_copies();  // this step's tiles are there, and the others' place is free
            if constexpr (!careful) {
                load(step + kTokens, buffer ^ 1);
            } else {
                load(step, buffer);
                sync_copies();
            }
            const int t0 = step + part * kTile;
            if (t0 >= mine) continue;
            const uint32_t ka = k_place + buffer * kStepBytes;
            uint32_t va = v_place + buffer * kStepBytes;
            if (careful && t0 + kTile > all) {
                // (all wavefronts that come here between two barriers write the same)
                unsigned char* const values = lds + kValues + part * kTileBytes + lane * 16;
                if (t0 + copy_finite_values<D>(values + buffer * kStepBytes, values + (buffer ^ 1) * kStepBytes) < see) l = __builtin_nanf("");
                va = v_place + (buffer ^ 1) * kStepBytes;
            }
            floatx16 s;
#pragma unroll
            for (int x = 0; x < 16; ++x) s[x] = 0.f;
            half8 next = key_part<D>(lds, ka, 0);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const half8 now = next;
                if (k + 1 < D / 16) next = key_part<D>(lds, ka, k + 1);
                // (where no other wavefront's products are there in the meantime, keys are read a product ahead)
                if constexpr (waves_of_simd(D, kWaves, kParts) == 1) __builtin_amdgcn_sched_barrier(0);
                s = __builtin_amdgcn_mfma_f32_32x32x16_f16(now, q[k], s, 0, 0, 0);
                if constexpr (waves_of_simd(D, kWaves, kParts) == 1) __builtin_amdgcn_sched_barrier(0);
            }
            if (t0 + kTile > all) {
                asm volatile("");  // (a branch stays one: few tiles are cut)
#pragma unroll
                for (int x = 0; x < 16; ++x) s[x] = t0 + 8 * (x / 4) + 4 * hi + x % 4 < see ? s[x] : -__builtin_inff();
            }
            float top = s[0];
#pragma unroll
            for (int x = 1; x < 16; ++x) top = __builtin_fmaxf(top, s[x]);
            if (__builtin_amdgcn_ballot_w64(top * a.scale > m + room) != 0) {
                top = __builtin_fmaxf(top, xor_lane_f32(top, 32));
                float n = __builtin_fmaxf(__builtin_fmaf(far, a.scale, m), top * a.scale), far_n = 0.f;
                if (room < 0.f || __builtin_amdgcn_ballot_w64(__builtin_fabsf(n) > kFar && n > 0.1f * kNoRow) != 0) {
                    asm volatile("");
                    room = -__builtin_inff();
                    if (__builtin_fabsf(n) > kFar && n > 0.1f * kNoRow) n = 0.f, far_n = far != 0.f ? __builtin_fmaxf(far, top) : top;
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[x] -= far_n;
                }
                const float f = __builtin_amdgcn_exp2f(__builtin_fmaf(far - far_n, a.scale, m - n));
                m = n, far = far_n;
                l *= f;
#pragma unroll
                for (int x = 0; x < D / 32; ++x) o[x] *= f;
            }
            half8 p[2];  // weights: fp16, at most 2^8, one rounding each; their sum in fp32
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x], a.scale, -m));
                l += e;
                p[x / 8][x % 8] = (_Float16)e;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int x = 0; x < D / 32; ++x) o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value_part<D>(lds, va, k, x), p[k], o[x], 0, 0, 0);
        }
        l += xor_lane_f32(l, 32);
        if constexpr (kParts == 2) {
            sync_copies();
            floatx4* const meet = reinterpret_cast<floatx4*>(lds) + group * ((D / 8 + 1) * 64) + lane;
            if (part == 1) {
#pragma unroll
                for (int x = 0; x < D / 32; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) meet[(4 * x + y) * 64] = floatx4{o[x][4 * y], o[x][4 * y + 1], o[x][4 * y + 2], o[x][4 * y + 3]};
                meet[D / 8 * 64] = floatx4{m, l, far, 0.f};
            }
            sync_copies();
            if (part == 0) {
                const floatx4 ml = meet[D / 8 * 64];
                const float d = __builtin_fmaf(far - ml[2], a.scale, m - ml[0]), f0 = __builtin_amdgcn_exp2f(d < 0.f ? d : 0.f), f1 = __builtin_amdgcn_exp2f(d > 0.f ? -d : 0.f);
                l = l * f0 + ml[1] * f1;
#pragma unroll
                for (int x = 0; x < D / 32; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const floatx4 v = meet[(4 * x + y) * 64];
#pragma unroll
                        for (int z = 0; z < 4; ++z) o[x][4 * y + z] = o[x][4 * y + z] * f0 + v[z] * f1;
                    }
            }
        }
        const float f = l == 0.f ? 0.f : 1.f / l;
        half2v zeros = half2v{(_Float16)0.f, (_Float16)0.f};
        asm volatile("" : "+s"(zeros));  // (for the compiler any number)
        float none = 0.f;                // unless a result is not finite
        if (there && part == 0) {
            _Float16* const out = a.out + (int64_t)(first + i) * a.ldo + (int64_t)hq * D + 4 * hi;
#pragma unroll
            for (int x = 0; x < D / 32; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const half4 h = half4{(_Float16)(o[x][4 * y] * f), (_Float16)(o[x][4 * y + 1] * f), (_Float16)(o[x][4 * y + 2] * f), (_Float16)(o[x][4 * y + 3] * f)};
                    *reinterpret_cast<half4*>(out + 32 * x + 8 * y) = h;
                    none = __builtin_amdgcn_fdot2(half2v{h[0], h[1]}, zeros, none, false);
                    none = __builtin_amdgcn_fdot2(half2v{h[2], h[3]}, zeros, none, false);
                }
        }
        if (!careful && a.causal && __builtin_amdgcn_ballot_w64(!(none == 0.f)) != 0) not_finite = 1;
    };
    not_finite = 0;
    // the last rows have the most to see: they begin
    const int last = count - 1 - id / a.seqs;
    for (int tile = last; tile >= 0; tile -= a.tiles) rows_of(tile, std::false_type());
    sync_copies();  // (the copies behind the last tile are into this workgroup's LDS)
    // A weight of 0 keeps a value from rows that do not see it, unless it is not finite.  So where results are not, the workgroup takes its rows
    // once more: in tiles that not all rows see, such values are zeros (a copy in the other step's place, so nothing is loaded ahead), and
    // the rows that do see one are no numbers.  (To look at values beforehand costs every prompt 1 to 10 %, to look at results 0 to 1.)
    if (__builtin_amdgcn_readfirstlane(not_finite) != 0)
        for (int tile = last; tile >= 0; tile -= a.tiles) rows_of(tile, std::true_type());
}

template <int D, int kWaves, int kParts>
int start(PromptArgs a, int64_t max_len, hipStream_t st) {
    constexpr int kRows = 32 * kWaves / kParts;
    const int64_t units = (int64_t)a.seqs * a.kv_heads, tiles = most_tiles((max_len * a.group + kRows - 1) / kRows, units), grid = tiles * units;
    a.tiles = (int)tiles;
    prompt_kernel<D, kWaves, kParts><<<dim3((unsigned)grid), dim3(64 * kWaves), 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}
template <int D>
int start(const PromptArgs& a, int64_t max_len, hipStream_t st) {
    // Workgroups of four wavefronts with rows of their own.  (There are rows for so many at most, whatever max_len says.)
    const int64_t tiles = (max_len * a.group + 127) / 128 * a.seqs, all = (int64_t)a.T * a.group / 128 + a.seqs, full = (tiles < all ? tiles : all) * a.kv_heads, cus = cu_count();
    // Where they are fewer than compute units (twice as many for 64 channels, whose LDS has room for more), the last rows' way through
    // their tokens is what a call takes: two wavefronts share it, if there are enough tokens to share.  us with four, two that share
    // rows' tokens (and two with rows of their own): 32 query and 8 kv heads of 128, one sequence of 60 tokens 8.0, 7.7 (7.0), 250
    // 12.0, 9.9 (11.1), 1000 30.0, 22.4 (28.6), 2000 53.0, 52.4 (56.5); 4 of 250 13.9, 13.6 (12.9); 16 and 4 heads of 64, 2000
    // tokens 37.8, 23.6 (37.5), 4000 68.8, 50.2 (69.4), 7 of 700 19.8, 20.5; 16 and 8 of 256, 2000 91.8, 67.8 (93.5), 4000 187, 216.
    // Without a mask every row's way is the same, and they have to fit at once, two for one, which 256 channels halve: 1000 tokens
    // 53.0, 36.0 (48.7), 1403 69.3, 80.5 (77.8).
    const bool enough = max_len >= 192 && max_len * cus >= 384 * full;
    if (enough && 2 * full <= (D == 64 ? 4 : D == 256 && !a.causal ? 1 : 2) * cus) return start<D, 4, 2>(a, max_len, st);
    // Else two wavefronts a workgroup where four would leave compute units without one.
    return full < cus && !enough ? start<D, 2, 1>(a, max_len, st) : start<D, 4, 1>(a, max_len, st);
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

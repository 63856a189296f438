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
// m only moves when a row's weights would pass 2^15 (then O and l are scaled, weights up to 2^7 again): a block costs no rescaling
// otherwise, and weights keep all of fp16's bits down to 2^-21 of a long row's largest.
// Of large scores the step's exponent is lost in m, and y - m holds what m's rounding left: from 2^25 on a weight could be beyond
// fp16.  So where a row passes 2^22 its reference is its largest score alone, before that is multiplied with the scale (State::far):
// the difference comes first, and a weight is at most a step of values.
//
// Few rows: the wavefronts of a workgroup take blocks in turn and meet in LDS.  Many rows: each has its own rows.  A
// long context is split over workgroups besides; combine_kernel joins the parts.
//
// What bounds it.  Few rows: the stream of blocks -- 16 sequences of 1500 to 2500 tokens, 32 heads of 128 with one row each, 138 MB, in
// 31 us, 4.5 TB/s (a copy: 5.2); one of 131072 tokens, 8 kv heads, in 25 us and 5 for the join.  A wavefront waits for memory
// for a third of its time there, and unpacking and softmax take the vector ALU for 40 %: more wavefronts (four a SIMD), or
// two blocks on their way at once, gain nothing.  Short contexts: a chain of loads (lengths and page, block, ...): 1000 tokens
// 10 us, where one token takes 7.  Many rows: the vector ALU and the matrix pipe, which share a SIMD's issue (66 and 33 %
// of it): 512 rows of 64 heads over 16500 tokens 350 us with its join, 778 TFLOP/s (once the clock has settled; the first calls take
// 40 more).  Unpacking once for four wavefronts into LDS saves a third of the vector instructions and took 345 to 385 us, other sizes 5 % more than
// this: it leaves room for few more wavefronts, and they wait for each other.  (The older of two workgroups on a unit takes 270 us, the younger
// 355; one of eight wavefronts that keep step takes as long.)
#include "itq3s_attention.h"
#include "itq3s_cache.h"

namespace itq3s {

namespace {

constexpr float kNoRow = -1e30f;    // reference of a row that has seen nothing
constexpr float kHeadroom = 8.f;    // weights may grow by 2^8 before the reference moves
constexpr float kFar = 4194304.f;   // 2^22: references beyond it are rounded by more than weights have room for
constexpr int kExpBias = 21;        // s < 2^(E - 14) for an fp16 with exponent field E; weights take 2^7 of what fp16 has above 2^8
constexpr int kMaxSplits = 256;

struct AttnArgs {
    const _Float16* Q;
    const int32_t *starts, *kv_lens, *pages;
    const unsigned char* data;
    _Float16* out;
    float *part, *ml;  // [splits][T * q_heads][D], [splits][T * q_heads][2]
    uint32_t* flags;
    int64_t ldq, ldo;
    float scale;  // softmax scale * log2(e) / sqrt(D)
    int q_heads, kv_heads, group, seqs, tiles, splits, split_blocks, page_shift, pool, page_units, T, ld_pages;
};

typedef const __attribute__((address_space(4))) int32_t* table_t;  // read through the scalar cache, beside the vector loads

// A sequence: its rows among all query rows, its tokens in the cache, and how its blocks are split.
struct Seq {
    int first, rows, len, blocks, per_split, splits;
};
__device__ __forceinline__ Seq find_seq(const AttnArgs& a, int s) {
    Seq q;
    const table_t starts = (table_t)(uintptr_t)a.starts, lens = (table_t)(uintptr_t)a.kv_lens;
    int lo = starts[s], hi = starts[s + 1];
    lo = lo < 0 ? 0 : lo > a.T ? a.T : lo;
    hi = hi < lo ? lo : hi > a.T ? a.T : hi;
    q.first = lo;
    q.rows = hi - lo;
    int len = lens[s];
    const int most = a.ld_pages << (a.page_shift + 5);  // at most 2^30
    if (len > most) {
        if (a.flags != nullptr && threadIdx.x == 0) atomicOr(a.flags, kFlagBadSlot);
        len = most;
    }
    q.len = len < 0 ? 0 : len;
    q.blocks = (q.len + kCacheBlock - 1) / kCacheBlock;
    const int need = (q.blocks + a.splits - 1) / a.splits;
    q.per_split = need > a.split_blocks ? need : a.split_blocks;
    q.splits = (q.blocks + q.per_split - 1) / q.per_split;
    return q;
}

// Across the 16-lane rows of a wavefront: sums and differences, sums, maxima of lanes l and l ^ kMask (16 or 32), by the
// instruction that swaps such rows between two registers: handed one value twice it gives every lane both rows' values.
template <int kMask>
__device__ __forceinline__ floatx2 both_rows(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    uint32_t even, odd;  // (scalars: a bit cast of a vector's element takes the first one)
    if constexpr (kMask == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        even = r[0], odd = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        even = r[0], odd = r[1];
    }
    return floatx2{__builtin_bit_cast(float, even), __builtin_bit_cast(float, odd)};
}
template <int kMask>
__device__ __forceinline__ float butterfly(float v, int lane) {
    const floatx2 r = both_rows<kMask>(v);
    return __builtin_fmaf((lane & kMask) != 0 ? -1.f : 1.f, r[1], r[0]);
}
__device__ __forceinline__ float sum_rows(float v) {
    floatx2 r = both_rows<16>(v);
    r = both_rows<32>(r[0] + r[1]);
    return r[0] + r[1];
}
__device__ __forceinline__ float max_rows(float v) {
    floatx2 r = both_rows<16>(v);
    r = both_rows<32>(__builtin_fmaxf(r[0], r[1]));
    return __builtin_fmaxf(r[0], r[1]);
}

// A block on its way to the matrix operands.
template <int D>
struct Block {
    uint32_t k[2][D / 32];
    u32x4 v[D / 64], s[2];
};

// Where a block is, and its first token: beyond every sequence for one that is not there.
typedef const __attribute__((address_space(1))) unsigned char* bytes_t;
struct Place {
    bytes_t at;
    int base;
};
template <int D>
__device__ __forceinline__ Place find_block(const AttnArgs& a, int page, int head, int b) {
    Place p;
    p.base = b * kCacheBlock;
    if ((uint32_t)page >= (uint32_t)a.pool) {
        if (a.flags != nullptr && lane_id() == 0) atomicOr(a.flags, kFlagBadSlot);
        page = 0;
        p.base = 0x7fffff00;
    }
    // in units of 128 bytes: a page's fit 32 bits
    constexpr uint32_t kUnits = kBlockBytes<D> / 128;
    const uint64_t units = (uint64_t)(uint32_t)page * (uint32_t)a.page_units + (uint32_t)(((head << a.page_shift) + (b & ((1 << a.page_shift) - 1))) * kUnits);
    // (one place for the wavefront: kept in scalar registers, which the products of 64 bits leave)
    const uint32_t low = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)units), high = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(units >> 32));
    p.at = (bytes_t)(uintptr_t)a.data + ((uint64_t)high << 32 | low) * 128;
    asm("" : "+s"(p.at));  // lanes add 32-bit offsets to it
    p.base = __builtin_amdgcn_readfirstlane(p.base);
    return p;
}
template <int D>
__device__ __forceinline__ void load_keys(bytes_t at, uint32_t (&k)[2][D / 32], int lane) {
    uint32_t off = (uint32_t)((lane & 15) * (D / 2) + (lane >> 4) * (D / 8));
    asm volatile("" : "+v"(off));  // (32 bits wide up to the load, which adds them to scalars)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
        if constexpr (D == 64) {
            const u32x2 w = *(const __attribute__((address_space(1))) u32x2*)(at + tt * 8 * D + off);
            k[tt][0] = w[0], k[tt][1] = w[1];
        } else {
#pragma unroll
            for (int i = 0; i < D / 128; ++i) {
                const u32x4 w = *(const __attribute__((address_space(1))) u32x4*)(at + tt * 8 * D + 16 * i + off);
#pragma unroll
                for (int j = 0; j < 4; ++j) k[tt][4 * i + j] = w[j];
            }
        }
    }
}
template <int D>
__device__ __forceinline__ void load_steps(bytes_t at, u32x4 (&s)[2], int lane) {
    uint32_t off = (uint32_t)(lane >> 4) * 16;
    asm volatile("" : "+v"(off));  // (32 bits wide up to the load, which adds them to scalars)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) s[tt] = *(const __attribute__((address_space(1))) u32x4*)(at + 32 * D + 64 * tt + off);
}
template <int D>
__device__ __forceinline__ void load_values(bytes_t at, u32x4 (&v)[D / 64], int lane) {
    uint32_t off = (uint32_t)lane * 16;
    asm volatile("" : "+v"(off));  // (32 bits wide up to the load, which adds them to scalars)
#pragma unroll
    for (int h = 0; h < D / 64; ++h) v[h] = *(const __attribute__((address_space(1))) u32x4*)(at + 16 * D + h * 1024 + off);
}

__device__ __forceinline__ half8 as_halves(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(half8, u32x4{a, b, c, d}); }

// Stored digits n = c + 8 of keys: in the mantissa of 1024 (nibbles 0 and 4 of a word or of the word a byte on) or of 64
// (nibbles 1 and 5).  What is too much, 1032 sum q of the first and 72 sum q of the second, is the accumulator's start.
// (Mask and mantissa are one instruction if one of the two constants is in a vector register.)
struct Mantissas {
    uint32_t low = 0x64006400u, high = 0x54005400u;
};
__device__ __forceinline__ half8 key_operand(uint32_t w, const Mantissas& m) {
    return as_halves((w & 0x000f000fu) | m.low, (w & 0x00f000f0u) | m.high, ((w >> 8) & 0x000f000fu) | m.low, ((w >> 8) & 0x00f000f0u) | m.high);
}
// Stored digits of values, as subnormal fp16: n 2^-24, or n 2^-20 for the upper nibbles, exactly what the matrix cores take them for.
// Where few rows share blocks, as digits c themselves: in the mantissa of 1024 or of 64, and 1032 or 72 off that.
__device__ __forceinline__ half8 value_operand_low(uint32_t u, uint32_t w) { return as_halves(u & 0x000f000fu, (u >> 8) & 0x000f000fu, w & 0x000f000fu, (w >> 8) & 0x000f000fu); }
__device__ __forceinline__ half8 value_operand_high(uint32_t u, uint32_t w) { return as_halves(u & 0x00f000f0u, (u >> 8) & 0x00f000f0u, w & 0x00f000f0u, (w >> 8) & 0x00f000f0u); }

__device__ __forceinline__ half8 centred_operand_low(uint32_t u, uint32_t w, const Mantissas& m) {
    const half8 offset = as_halves(0xe408e408u, 0xe408e408u, 0xe408e408u, 0xe408e408u);  // -1032
    return as_halves((u & 0x000f000fu) | m.low, ((u >> 8) & 0x000f000fu) | m.low, (w & 0x000f000fu) | m.low, ((w >> 8) & 0x000f000fu) | m.low) + offset;
}
__device__ __forceinline__ half8 centred_operand_high(uint32_t u, uint32_t w, const Mantissas& m) {
    const half8 offset = as_halves(0xd480d480u, 0xd480d480u, 0xd480d480u, 0xd480d480u);  // -72
    return as_halves((u & 0x00f000f0u) | m.high, ((u >> 8) & 0x00f000f0u) | m.high, (w & 0x00f000f0u) | m.high, ((w >> 8) & 0x00f000f0u) | m.high) + offset;
}

// The rotated queries of a wavefront's rows, as the products want them: lane (column l % 16, g = l / 16) holds channels
// (D/4) g .. (D/4) (g + 1) - 1, scaled by a power of two into fp16's best range, in kParts parts of fp16 (two leave no
// rounding to speak of).
template <int D, int CT>
struct Queries {
    half8 f[CT][D / 32];  // the first part; the second stays in LDS, where it is read once a block
    uint32_t row[CT];     // there, in bytes
    float start[CT];      // of the scores' accumulators
    float unit[CT];       // what scores are multiplied with, positive
};
// They are turned eight channels a lane, 512 / D rows a wavefront at a time, and change lanes through LDS: a row is kParts
// rows of fp16, start and unit, with 8 bytes more so that neighbouring rows begin in other banks.
template <int D, int kParts>
constexpr int kQueryPitch = kParts * 2 * D + 16;
template <int D, int kParts>
__device__ __forceinline__ void turn_query(half8 h8, bool there, float scale, unsigned char* row, int lane) {
    const int ch = lane % (D / 8) * 8;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = there ? (float)h8[j] : 0.f;
    hadamard<D>(x, lane);
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = __builtin_fmaxf(most, __builtin_fabsf(x[j]));
    most = row_max<D>(most);
    const int e = __builtin_amdgcn_frexp_expf(most);  // 0 for 0, infinities and NaN
    const float sign = scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f;
    float start = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __builtin_ldexpf(x[j], -e) * sign;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        half8 f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = (_Float16)x[j];
            x[j] -= (float)f[j];
            start = __builtin_fmaf((j & 2) == 0 ? -1032.f : -72.f, (float)f[j], start);  // key_operand's nibbles
        }
        *reinterpret_cast<half8*>(row + p * 2 * D + 2 * ch) = f;
    }
    start = row_sum<D>(start);
    if (ch == 0) *reinterpret_cast<floatx2*>(row + kParts * 2 * D) = floatx2{start, scale == 0.f ? 1.f : __builtin_ldexpf(__builtin_fabsf(scale), e)};
}
template <int D, int CT, int kParts>
__device__ __forceinline__ void load_queries(const unsigned char* lds, uint32_t row, int ct, Queries<D, CT>& q, int g) {
    q.row[ct] = row + (D / 2) * g;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) q.f[ct][i] = *reinterpret_cast<const half8*>(lds + row + (D / 2) * g + 16 * i);
    q.start[ct] = *reinterpret_cast<const float*>(lds + row + kParts * 2 * D);
    q.unit[ct] = *reinterpret_cast<const float*>(lds + row + kParts * 2 * D + 4);
}

// O^T in the units of value_operand: accumulators of even channel tiles times 2^24, of odd ones 2^20.  With digits n = c + 8 each has
// `eight` too much (of sum 8 P', in the even ones' units).  The matrix cores cut the sum of a product's terms, subnormal ones at the place of
// fp16's least normal number: a row of 131072 tokens comes out 6e-4 off.  So few rows, whose time is the memory's, have the digits c as
// ordinary fp16 (kCentred: 2.9e-4, nothing is cut; with 8 taken off subnormal ones 3.3e-4 in the same time), and many rows, whose
// time is the vector ALU's, do not (16500 tokens 4.5e-4, where it were 4.1e-4 and 4 to 12 % of time; queries in two parts
// 3.6e-4 and 399 us instead of 347; 2.1e-4 of each is the result's rounding to fp16).  Nor do sixteen wavefronts of a short
// sequence (3.0e-4 either way).
template <int D, int CT>
struct State {
    floatx4 o[D / 16][CT], eight[CT];
    float m[CT], l[CT];
    float far[CT];  // a row's reference is m + far * unit: one of them is 0, m where a score's size passes kFar
    float room;     // how far scores may be above m: kHeadroom, or minus infinity (every block moves references) once a row is there
};

template <int D, int CT, int kParts>
__device__ __forceinline__ void scores(const uint32_t (&k)[2][D / 32], const Mantissas& mant, const unsigned char* lds, const Queries<D, CT>& q, floatx4 (&s)[2][CT]) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) s[tt][ct] = floatx4{q.start[ct], q.start[ct], q.start[ct], q.start[ct]};
    uint32_t second = 2 * D;
    if constexpr (kParts == 2) asm volatile("" : "+v"(second));  // (read anew for every block)
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const half8 f = key_operand(k[tt][i], mant);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                s[tt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q.f[ct][i], s[tt][ct], 0, 0, 0);
                if constexpr (kParts == 2)
                    s[tt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, *reinterpret_cast<const half8*>(lds + q.row[ct] + second + 16 * i), s[tt][ct], 0, 0, 0);
            }
        }
}

__device__ __forceinline__ _Float16 half_of(uint32_t w, bool upper) { return __builtin_bit_cast(half2v, w)[upper ? 1 : 0]; }

template <int D, int CT, bool kCentred>
__device__ __forceinline__ void weights(const floatx4 (&s)[2][CT], u32x4 (&step)[2], int base, const Queries<D, CT>& q, const int (&see)[CT], int see_all, int len, State<D, CT>& st,
                                        half8 (&p)[CT], int g) {
    const bool edge = base + kCacheBlock > see_all;
    if (edge) {  // what stands behind the sequence may be anything
        asm volatile("");  // (keeps a branch a branch: most blocks are whole)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) step[tt][i] = base + tt * 16 + 4 * g + i < len ? step[tt][i] : 0u;
    }
    // A quarter of the upper byte of an fp16 is its exponent field and two bits more.  The lane's largest step stands for its eight:
    // that makes weights smaller than they could be by as much as the steps differ, which is taken up to 2^6.  Beyond that every token is looked at with its own.
    uint32_t most = 0, least = 0xffffffffu;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            most = most > step[tt][i] ? most : step[tt][i];
            least = least < step[tt][i] ? least : step[tt][i];
        }
    const float bias = __builtin_fmaf((float)(most >> 24), 0.25f, -(float)kExpBias);
    const bool apart = __builtin_amdgcn_ballot_w64((most >> 24) - (least >> 24) > 24u) != 0;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const float unit = q.unit[ct];
        float x[2][4], top = -__builtin_inff();
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[tt][i] = __builtin_fmaf(s[tt][ct][i], (float)half_of(step[tt][i], false), 0.f);
        if (edge) {
            asm volatile("");
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[tt][i] = base + tt * 16 + 4 * g + i < see[ct] ? x[tt][i] : -__builtin_inff();
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, x[tt][i]);
        top = __builtin_fmaf(top, unit, bias);
        if (apart) {
            asm volatile("");
            top = -__builtin_inff();
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, __builtin_fmaf((float)(step[tt][i] >> 24), 0.25f, x[tt][i] * unit));
            top -= (float)kExpBias;
        }
        if (__builtin_amdgcn_ballot_w64(top > st.m[ct] + st.room) != 0) {
            float m = __builtin_fmaxf(__builtin_fmaf(st.far[ct], unit, st.m[ct]), max_rows(top)), far = 0.f;
            if (st.room < 0.f || __builtin_amdgcn_ballot_w64(__builtin_fabsf(m) > kFar && m > 0.1f * kNoRow) != 0) {
                asm volatile("");
                st.room = -__builtin_inff();
                float most_x = -__builtin_inff();
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most_x = __builtin_fmaxf(most_x, x[tt][i]);
                most_x = max_rows(most_x);
                if (__builtin_fabsf(m) > kFar && m > 0.1f * kNoRow) m = 0.f, far = st.far[ct] != 0.f ? __builtin_fmaxf(st.far[ct], most_x) : most_x;
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[tt][i] -= far;
            }
            const float f = __builtin_amdgcn_exp2f(__builtin_fmaf(st.far[ct] - far, unit, st.m[ct] - m));
            st.m[ct] = m, st.far[ct] = far;
            st.l[ct] *= f;
            if constexpr (!kCentred) st.eight[ct] *= f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st.o[c][ct] *= f;
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tt][i], unit, -st.m[ct]));
                st.l[ct] += e;
                p[ct][4 * tt + i] = (_Float16)__builtin_fmaf(e, (float)half_of(step[tt][i], true), 0.f);
            }
    }
}

template <int D, int CT, bool kCentred>
__device__ __forceinline__ void products(const u32x4 (&v)[D / 64], const half8 (&p)[CT], const Mantissas& mant, State<D, CT>& st) {
    const half8 eight = as_halves(0x00080008u, 0x00080008u, 0x00080008u, 0x00080008u);
    if constexpr (!kCentred)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) st.eight[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight, p[ct], st.eight[ct], 0, 0, 0);
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
#pragma unroll
        for (int pp = 0; pp < 2; ++pp) {
            half8 lo, hi;
            if constexpr (kCentred) lo = centred_operand_low(v[h][2 * pp], v[h][2 * pp + 1], mant), hi = centred_operand_high(v[h][2 * pp], v[h][2 * pp + 1], mant);
            else lo = value_operand_low(v[h][2 * pp], v[h][2 * pp + 1]), hi = value_operand_high(v[h][2 * pp], v[h][2 * pp + 1]);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                st.o[4 * h + 2 * pp][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, p[ct], st.o[4 * h + 2 * pp][ct], 0, 0, 0);
                st.o[4 * h + 2 * pp + 1][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, p[ct], st.o[4 * h + 2 * pp + 1][ct], 0, 0, 0);
            }
        }
}

// The transform of O^T's columns: channel 16 c + 4 g + i in accumulator c, lane group g, element i.
template <int D, int CT>
__device__ __forceinline__ void turn_back(floatx4 (&o)[D / 16][CT], int ct, int lane) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        floatx4 v = o[c][ct];
        v = floatx4{v[0] + v[1], v[0] - v[1], v[2] + v[3], v[2] - v[3]};
        v = floatx4{v[0] + v[2], v[1] + v[3], v[0] - v[2], v[1] - v[3]};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = butterfly<32>(butterfly<16>(v[i], lane), lane);
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

// How the wavefronts of a workgroup share its rows and blocks.
enum class Share {
    blocks,  // 16 rows, all take blocks in turn
    tiles,   // 16 or 32 rows (64 if it has more than was said), as many as the sequence has: wavefronts of different rows take the same blocks at one time
    none     // 16 CT rows of its own a wavefront, every block
};

// LDS: the turned queries, of every wavefront or shared; in their place afterwards what the wavefronts have of shared rows: of each
// (channel tile, lane row) 16 columns of four channels, with a place left free behind them, then references and sums.
template <int D, int CT, int kWaves, Share kShare, int kParts>
struct Lds {
    static constexpr int kQueryRows = (kShare == Share::none ? kWaves : kShare == Share::tiles ? 4 : 1) * 16 * CT;
    static constexpr int kQueries = kQueryRows * kQueryPitch<D, kParts>;
    static constexpr int kPart = D / 4 * 17 + 8;  // floatx4
    static constexpr int kBytes = kShare == Share::none || kWaves * kPart * 16 < kQueries ? kQueries : kWaves * kPart * 16;
};

// Sums and maxima of lanes l and l ^ kMask, ... up to l ^ (kEnd / 2).
template <int kMask>
__device__ __forceinline__ float with_lane(float v, int which) {  // 0: sum, 1: maximum
    float a, b;
    if constexpr (kMask >= 16) {
        const floatx2 r = both_rows<kMask>(v);
        a = r[0], b = r[1];
    } else {
        a = v, b = row_xor<kMask>(v);
    }
    return which == 0 ? a + b : __builtin_fmaxf(a, b);
}
template <int kMask, int kEnd>
__device__ __forceinline__ float across(float v, int which) {
    if constexpr (kMask < kEnd) return across<2 * kMask, kEnd>(with_lane<kMask>(v, which), which);
    else return v;
}

template <int D, int CT, int kWaves, Share kShare, int kParts>
__global__ void __launch_bounds__(64 * kWaves, CT == 1 && D <= 128 ? 4 : 2) cache_attention_kernel(const AttnArgs a) {
    constexpr bool kOwn = kShare == Share::none, kCentred = !kOwn && kWaves < 16;
    typedef Lds<D, CT, kWaves, kShare, kParts> L;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // heads fastest: with eight heads each die keeps to one, and its cache to that head's blocks
    int id = blockIdx.x;
    const int head = id % a.kv_heads;
    id /= a.kv_heads;
    const int first_tile = id % a.tiles;  // tiles of one piece of the cache beside each other
    id /= a.tiles;
    const int seq = id % a.seqs, split = id / a.seqs;
    // The way to the first block is a chain of loads, each some hundred nanoseconds: the page of the block that this will most likely
    // be is read beside the sequence's lengths, and the block is on its way before the queries are turned.
    const table_t pages = (table_t)(uintptr_t)(a.pages + (int64_t)seq * a.ld_pages);
    const int likely = (split * a.split_blocks + (kOwn ? 0 : wave)) >> a.page_shift, likely_at = likely < a.ld_pages ? likely : a.ld_pages - 1;
    const int likely_page = pages[likely_at];
    const Seq sq = find_seq(a, seq);
    if (split > 0 && split >= sq.splits) return;
    const int total = sq.rows * a.group;
    // rows of a workgroup's tile, 16 (or a wavefront's own ones) times a power of two
    const int share = kShare != Share::tiles ? 0 : total > 32 ? 2 : total > 16 ? 1 : 0;
    const int tile_rows = kOwn ? kWaves * 16 * CT : 16 << share;
    const int first_row = kOwn ? wave * 16 * CT : (wave & ((1 << share) - 1)) * 16;  // of the wavefront within it
    const int take = kOwn ? 0 : wave >> share, step = kOwn ? 1 : kWaves >> share;    // which blocks
    extern __shared__ __align__(16) unsigned char lds[];
    floatx4* const meet = reinterpret_cast<floatx4*>(lds);
    for (int tile = first_tile; tile * tile_rows < total; tile += a.tiles) {
        int lane = lane_id();
        asm volatile("" : "+v"(lane));  // (nothing that hangs on it is kept from one tile to the next)
        const int g = lane >> 4, col = lane & 15;
        const int tile_row0 = tile * tile_rows, row0 = tile_row0 + first_row;
        // rows of the wavefront see between see_all and see_most places
        const int last = row0 + 16 * CT < total ? row0 + 16 * CT - 1 : total - 1;
        const int see_all = sq.len - sq.rows + (row0 < total ? row0 / a.group : 0) + 1;
        int see_most = row0 < total ? sq.len - sq.rows + last / a.group + 1 : 0;
        see_most = see_most < 0 ? 0 : see_most;
        int b = split * sq.per_split + take, end = split * sq.per_split + sq.per_split;
        const int need = (see_most + kCacheBlock - 1) / kCacheBlock;
        end = end < need ? end : need;
        int page = likely_page;
        if (b >= end) page = 0;
        else if ((b >> a.page_shift) != likely_at) page = pages[b >> a.page_shift];

        constexpr int kTurned = 512 / D;  // rows at a time
        // rows of the tile (of the wavefront) from r on, in the lanes' order: the row, whether it is there, its values
        auto query_row = [&](int r, bool& there) {
            const int row = (kOwn ? row0 : tile_row0) + r + lane / (D / 8);
            there = row < total;
            const int i = there ? row / a.group : 0, hq = head * a.group + (there ? row % a.group : 0);
            return *reinterpret_cast<const half8*>(a.Q + (int64_t)(sq.first + i) * a.ldq + (int64_t)hq * D + lane % (D / 8) * 8);
        };
        const int turn_rows = kOwn ? 16 * CT : tile_rows, turn_step = (kOwn ? 1 : kWaves) * kTurned;
        int r_turn = (kOwn ? 0 : wave) * kTurned;
        bool there_turn;
        half8 h_turn = query_row(r_turn < turn_rows ? r_turn : 0, there_turn);
        Block<D> r;
        Place now = find_block<D>(a, page, head, b < end ? b : 0);
        load_keys<D>(now.at, r.k, lane);
        load_steps<D>(now.at, r.s, lane);
        load_values<D>(now.at, r.v, lane);
        const uint32_t queries = kOwn ? wave * (16 * CT) * kQueryPitch<D, kParts> : 0;
#pragma unroll 1
        while (r_turn < turn_rows) {
            turn_query<D, kParts>(h_turn, there_turn, a.scale, lds + queries + (r_turn + lane / (D / 8)) * kQueryPitch<D, kParts>, lane);
            r_turn += turn_step;
            if (r_turn < turn_rows) h_turn = query_row(r_turn, there_turn);
        }
        __syncthreads();
        State<D, CT> st;
        st.room = kHeadroom;
        Queries<D, CT> q;
        int see[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int row = row0 + ct * 16 + col, v = sq.len - sq.rows + row / a.group + 1;
            see[ct] = row < total && v > 0 ? v : 0;
            load_queries<D, CT, kParts>(lds, queries + ((kOwn ? 0 : first_row) + ct * 16 + col) * kQueryPitch<D, kParts>, ct, q, g);
            st.m[ct] = kNoRow, st.l[ct] = st.far[ct] = 0.f;
            st.eight[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st.o[c][ct] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        Mantissas mant;
        asm volatile("" : "+v"(mant.low), "+v"(mant.high));
        if (b < end) {
            // What a block's part of the registers is done with is loaded for the next block at once: keys ahead by a softmax and a
            // product, values by two products' worth of other wavefronts.  The last block is loaded twice rather than branched round.
            int ahead = b + step < end ? b + step : b;
            page = pages[ahead >> a.page_shift];
            for (; b < end; b += step) {
                const Place next = find_block<D>(a, page, head, ahead);
                ahead = ahead + step < end ? ahead + step : ahead;
                page = pages[ahead >> a.page_shift];
                floatx4 s[2][CT];
                scores<D, CT, kParts>(r.k, mant, lds, q, s);
                __builtin_amdgcn_sched_barrier(0);
                load_keys<D>(next.at, r.k, lane);
                __builtin_amdgcn_sched_barrier(0);
                half8 p[CT];
                // (ahead of others' products: the vector ALU is what a unit has least of.  A chunk of 512 rows of 16500 tokens 365 -> 356 us)
                __builtin_amdgcn_s_setprio(1);
                weights<D, CT, kCentred>(s, r.s, now.base, q, see, see_all, sq.len, st, p, g);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(0);
                load_steps<D>(next.at, r.s, lane);
                __builtin_amdgcn_sched_barrier(0);
                products<D, CT, kCentred>(r.v, p, mant, st);
                __builtin_amdgcn_sched_barrier(0);
                load_values<D>(next.at, r.v, lane);
                __builtin_amdgcn_sched_barrier(0);
                now = next;
            }
        }
        // where the results go is read again from the arguments: it would stay in scalar registers all the way
        typedef const __attribute__((address_space(4))) AttnArgs* args_t;
        args_t late = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(late));
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            st.l[ct] = sum_rows(st.l[ct]);
            st.m[ct] = __builtin_fmaf(st.far[ct], q.unit[ct], st.m[ct]);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                if constexpr (!kCentred) {
                    st.o[c][ct] -= c % 2 == 0 ? st.eight[ct] : st.eight[ct] * 16.f;
                    st.o[c][ct] *= c % 2 == 0 ? 16777216.f : 1048576.f;
                }
            }
        }
        if constexpr (!kOwn) {
            // Every wavefront leaves its sums.  A row is joined by a wavefront, D / 8 lanes a part.
            static_assert(CT == 1, "one column tile");
            __syncthreads();
            floatx4* const mine = meet + wave * L::kPart;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) mine[(4 * c + g) * 17 + col] = st.o[c][0];
            if (g == 0) reinterpret_cast<floatx2*>(mine + D / 4 * 17)[col] = floatx2{st.m[0], st.l[0]};
            __syncthreads();
            constexpr int kLanes = D / 8, kGroups = 64 / kLanes;
            const int grp = lane / kLanes, ch = lane % kLanes * 8;
#pragma unroll 1
            for (int r0 = wave; r0 < tile_rows; r0 += kWaves) {
                const int row = tile_row0 + r0, r = r0 & 15;
                if (row >= total) break;
                float l = 0.f, o[8] = {}, most = kNoRow;
#pragma unroll 1
                for (int w = (r0 >> 4) + (grp << share); w < kWaves; w += kGroups << share) {
                    const floatx4* const part = meet + w * L::kPart;
                    const floatx2 ml = reinterpret_cast<const floatx2*>(part + D / 4 * 17)[r];
                    const float n = __builtin_fmaxf(most, ml[0]), f = __builtin_amdgcn_exp2f(most - n), h = __builtin_amdgcn_exp2f(ml[0] - n);
                    most = n;
                    l = l * f + ml[1] * h;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const floatx4 v = part[(ch / 4 + i) * 17 + r];
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[4 * i + j] = o[4 * i + j] * f + v[j] * h;
                    }
                }
                const float own = most;
                most = across<kLanes, 64>(most, 1);
                const float f = __builtin_amdgcn_exp2f(own - most);
                l = across<kLanes, 64>(l * f, 0);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = across<kLanes, 64>(o[j] * f, 0);
                const bool there = grp == 0;
                const int64_t token = sq.first + row / late->group;
                const int hq = head * late->group + row % late->group;
                if (sq.splits > 1) {
                    const int64_t part = ((int64_t)split * late->T + token) * late->q_heads + hq;
                    if (there) {
                        if (ch == 0) *reinterpret_cast<floatx2*>(late->ml + 2 * part) = floatx2{most, l};
                        floatx4* const to = reinterpret_cast<floatx4*>(late->part + part * D + ch);
                        to[0] = floatx4{o[0], o[1], o[2], o[3]};
                        to[1] = floatx4{o[4], o[5], o[6], o[7]};
                    }
                } else {
                    hadamard<D>(o, lane);
                    const float f = l == 0.f ? 0.f : (float)(1.0 / kRootD<D>) / l;
                    half8 h;
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[j] = (_Float16)(o[j] * f);
                    if (there) *reinterpret_cast<half8*>(late->out + token * late->ldo + (int64_t)hq * D + ch) = h;
                }
            }
            __syncthreads();
            continue;
        } else {
            __syncthreads();  // (the queries' place is written again)
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int row = row0 + ct * 16 + col;
            const bool there = row < total;
            const int64_t token = sq.first + row / late->group;
            const int hq = head * late->group + row % late->group;
            if (sq.splits > 1) {
                const int64_t part = ((int64_t)split * late->T + token) * late->q_heads + hq;
                if (there) {
                    if (g == 0) *reinterpret_cast<floatx2*>(late->ml + 2 * part) = floatx2{st.m[ct], st.l[ct]};
                    floatx4* const o = reinterpret_cast<floatx4*>(late->part + part * D);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) o[4 * c + g] = st.o[c][ct];
                }
            } else {
                turn_back<D, CT>(st.o, ct, lane);
                const float f = st.l[ct] == 0.f ? 0.f : (float)(1.0 / kRootD<D>) / st.l[ct];
                if (there) {
                    _Float16* const o = late->out + token * late->ldo + (int64_t)hq * D + 4 * g;
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

// Joins the parts of rows whose sequence was split: D / 8 lanes a part, `lanes` groups of them a row (a power of two up to a
// workgroup's), the groups of a row beside each other.  64 rows of 64 parts 5 us, of which a launch is half; 32768 rows of two, 34 MB,
// 9 us.
template <int D>
__global__ void __launch_bounds__(256) combine_kernel(const AttnArgs a, int groups_of_row) {
    constexpr int kLanes = D / 8, kGroups = 256 / kLanes;
    __shared__ __align__(16) float meet[kGroups][D + 4];
    const int tid = threadIdx.x, grp = tid / kLanes, ch = tid % kLanes * 8;
    const int mine = grp % groups_of_row, rows_at_once = kGroups / groups_of_row;
    const Seq sq = find_seq(a, (int)blockIdx.x);
    if (sq.splits <= 1) return;
    const int64_t stride = (int64_t)a.T * a.q_heads, all = (int64_t)sq.rows * a.q_heads;
    for (int64_t r0 = (int64_t)blockIdx.y * rows_at_once; r0 < all; r0 += (int64_t)gridDim.y * rows_at_once) {
        const int64_t r = r0 + grp / groups_of_row;
        const bool there = r < all;
        const int64_t row = (int64_t)sq.first * a.q_heads + (there ? r : all - 1);
        float m = kNoRow, l = 0.f, o[8] = {};
        // four parts at a time, all their loads before the first is used; parts that are not there weigh nothing
        for (int s0 = mine; s0 < sq.splits; s0 += 4 * groups_of_row) {
            floatx2 ml[4];
            floatx4 u[4], v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int s = s0 + k * groups_of_row < sq.splits ? s0 + k * groups_of_row : s0;
                ml[k] = *reinterpret_cast<const floatx2*>(a.ml + 2 * (s * stride + row));
                const floatx4* const p = reinterpret_cast<const floatx4*>(a.part + (s * stride + row) * D + ch);
                u[k] = p[0], v[k] = p[1];
            }
            float n = m;
#pragma unroll
            for (int k = 0; k < 4; ++k) n = __builtin_fmaxf(n, ml[k][0]);
            const float f = __builtin_amdgcn_exp2f(m - n);
            m = n;
            l *= f;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] *= f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float h = s0 + k * groups_of_row < sq.splits ? __builtin_amdgcn_exp2f(ml[k][0] - n) : 0.f;
                l += ml[k][1] * h;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o[j] += u[k][j] * h;
                    o[4 + j] += v[k][j] * h;
                }
            }
        }
        if (groups_of_row > 1) {
#pragma unroll
            for (int i = 0; i < 2; ++i) *reinterpret_cast<floatx4*>(&meet[grp][ch + 4 * i]) = floatx4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
            if (ch == 0) *reinterpret_cast<floatx2*>(&meet[grp][D]) = floatx2{m, l};
            __syncthreads();
            if (mine == 0) {
                for (int k = 1; k < groups_of_row; ++k) {
                    const float* const part = meet[grp + k];
                    const floatx2 ml = *reinterpret_cast<const floatx2*>(part + D);
                    const float n = __builtin_fmaxf(m, ml[0]), f = __builtin_amdgcn_exp2f(m - n), h = __builtin_amdgcn_exp2f(ml[0] - n);
                    m = n;
                    l = l * f + ml[1] * h;
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = o[j] * f + part[ch + j] * h;
                }
            }
            __syncthreads();
        }
        hadamard<D>(o);  // (all lanes: neighbouring groups exchange nothing)
        const float f = l == 0.f ? 0.f : (float)(1.0 / kRootD<D>) / l;
        half8 h;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = (_Float16)(o[j] * f);
        if (there && mine == 0) *reinterpret_cast<half8*>(a.out + row / a.q_heads * a.ldo + row % a.q_heads * D + ch) = h;
    }
}

// How a call is cut up.
struct Plan {
    Share share;
    bool wide;  // sixteen wavefronts share the blocks
    int64_t tiles;
    int splits, split_blocks;
};
Plan plan_of(int64_t T, int64_t seqs, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv) {
    Plan p;
    const int64_t group = q_heads / kv_heads, rows = max_q * group, all_rows = T * group, units = seqs * kv_heads, cus = cu_count();
    const int64_t blocks = (max_kv + kCacheBlock - 1) / kCacheBlock;
    // Rows of its own a wavefront: unpacks a block once for 32 rows and loads it four times as often as wavefronts that share it,
    // so it takes many rows -- of a sequence to fill a workgroup, and of all to fill the card -- or much to do for each.  us
    // with own rows and with shared blocks, 64 query and 8 kv heads of 128: 128 rows of 4000 tokens 58 and 46, 256 77 and 73, 512
    // 113 and 126; 128 rows of 16500 120 and 137, of 1000 37 and 25; 16 sequences of 2000 with 16 rows 56 and 57.
    const int64_t own = head_dim < 256 ? 128 : 64, most_rows = all_rows < rows * seqs ? all_rows : rows * seqs;
    const bool many = rows >= own && 2 * all_rows >= own * seqs && (most_rows * kv_heads >= 64 * cus || most_rows * kv_heads >= 8192 * cus / blocks);
    // Two tiles of 16 rows in one workgroup of eight wavefronts, or in two of four: us of ragged batches of up to 4 rows, 61 of up to 8000
    // tokens 81 and 102, 60 of 4000 50 and 56, 20 of 8000 43 and 52; of equal ones, 16 of 4000 39 and 32.  For more tiles: 60
    // of up to 9 rows 110 and 77, of 5 rows 79 and 60.
    p.share = many ? Share::none : rows > 16 && rows <= 32 ? Share::tiles : Share::blocks;
    const int64_t per = p.share == Share::none ? own : p.share == Share::tiles ? 32 : 16;
    p.tiles = most_tiles((rows + per - 1) / per, units);
    // Sixteen wavefronts share one short sequence, and no second launch joins parts.  us with them and with parts of four: one
    // sequence, 8 kv heads, of 120 tokens 8.7 and 8.2, 250 9.3 and 10.8, 1000 11.6 and 12.2, 2000 14.5 and 12.5; 8 of 2000
    // 14.7 and 15.8, of 4000 20.5 and 18.1; 32 of 6000 47 and 52; 48 of 250 16.3 and 16.2, of 120 15.1 and 9.9.
    p.wide = p.share == Share::blocks && rows <= 16 && head_dim <= 128 && blocks > 4 && units <= cus && blocks <= 32 + units * 256 / cus;
    // Else as many parts as give every unit two workgroups (three of Share::tiles, for their ragged batches: 81 us above, with two 89.  LDS
    // has room for two at a time with 128 channels, for one with 256: the third begins where one of short sequences has ended).
    // Four a unit, which also fit where a workgroup has four wavefronts, measured for 8 kv heads of 128: one sequence of
    // 131072 tokens 41.9 us, with two 40.7; 64 of 1000 23.9 and 18.9; one of 16000 20.7 and 16.2; 16 of 2500 with 32 heads
    // 40.2 and 36.7.  One a unit: 131072 tokens 45.8 us.  (Sequences have rows for so many tiles at most.)
    const int64_t all_tiles = kv_heads * (all_rows / per + seqs), some_tiles = units * p.tiles;
    const int64_t places = (p.share == Share::tiles ? 3 : 2) * cus, work = (all_tiles < some_tiles ? all_tiles : some_tiles) * blocks;
    int64_t per_split = p.wide ? blocks : (work + places - 1) / places;
    // Parts of own rows cost the most to join: 512 rows of 1000 tokens in parts of 16 blocks 54 us, of 32 (one part) 46, 200 rows of
    // 4000 83 and 72.  Shared ones: one row of 4000 tokens in parts of 2, 4 and 8 blocks 14.8, 13.1 and 13.2.
    const int64_t few = p.share == Share::none ? 32 : 4;
    if (per_split < few) per_split = few;
    const int64_t least = (blocks + kMaxSplits - 1) / kMaxSplits;
    if (per_split < least) per_split = least;
    p.split_blocks = (int)(per_split < blocks ? per_split : blocks);
    p.splits = (int)((blocks + p.split_blocks - 1) / p.split_blocks);
    return p;
}

template <int D, int CT, int kWaves, Share kShare, int kParts>
int start(const AttnArgs& a, int64_t grid, hipStream_t st) {
    constexpr int kLds = Lds<D, CT, kWaves, kShare, kParts>::kBytes;
    static_assert(kLds <= 160 * 1024, "LDS");
    if constexpr (kLds > 65536) {
        static DeviceOnce once;
        if (!raise_lds_limit(once, reinterpret_cast<const void*>(&cache_attention_kernel<D, CT, kWaves, kShare, kParts>), kLds)) return -6;
    }
    cache_attention_kernel<D, CT, kWaves, kShare, kParts><<<dim3((unsigned)grid), dim3(64 * kWaves), kLds, st>>>(a);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

template <int D>
int start(const AttnArgs& a, const Plan& p, int64_t grid, int64_t max_q, hipStream_t st) {
    int rc = 0;
    if (p.share == Share::none) rc = start<D, D == 256 ? 1 : 2, 4, Share::none, 1>(a, grid, st);
    else if (p.share == Share::tiles) rc = start<D, 1, 8, Share::tiles, 2>(a, grid, st);
    else {
        bool wide = false;
        if constexpr (D <= 128) wide = p.wide;
        if (!wide) rc = start<D, 1, 4, Share::blocks, 2>(a, grid, st);
        if constexpr (D <= 128)
            if (wide) rc = start<D, 1, 16, Share::blocks, 2>(a, grid, st);
    }
    if (rc != 0 || p.splits <= 1) return rc;
    int groups = 1;
    while (4 * groups < p.splits && groups < 2048 / D) groups *= 2;  // (four parts a group are one round of loads)
    const int64_t at_once = 2048 / D / groups, rows = (max_q * a.q_heads + at_once - 1) / at_once;
    combine_kernel<D><<<dim3((unsigned)a.seqs, (unsigned)(rows < 65535 ? rows : 65535)), dim3(256), 0, st>>>(a, groups);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

}  // namespace

size_t cache_attention_bytes(int64_t T, int64_t seqs, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv) {
    const Plan p = plan_of(T, seqs, q_heads, kv_heads, head_dim, max_q, max_kv);
    if (p.splits <= 1) return 256;
    return (size_t)p.splits * (size_t)T * (size_t)q_heads * (size_t)(head_dim + 2) * 4 + 256;
}

int launch_cache_attention(const CacheAttentionCall& c, hipStream_t st) {
    const int G = c.q_heads / c.cache.kv_heads, D = c.cache.head_dim;
    const Plan p = plan_of(c.T, c.seqs, c.q_heads, c.cache.kv_heads, D, c.max_q, c.max_kv);
    AttnArgs a{};
    a.Q = c.Q, a.starts = c.starts, a.kv_lens = c.kv_lens, a.pages = c.pages, a.data = c.cache.data, a.out = c.out, a.flags = c.flags;
    a.part = static_cast<float*>(c.workspace);
    a.ml = a.part + (size_t)p.splits * (size_t)c.T * (size_t)c.q_heads * (size_t)D;
    a.ldq = c.ldq, a.ldo = c.ldo, a.ld_pages = (int)c.ld_pages, a.T = (int)c.T, a.pool = (int)c.cache.pages;
    a.scale = (float)((double)c.scale * 1.44269504088896340736 / (D == 64 ? 8.0 : D == 128 ? 11.313708498984760390 : 16.0));
    if (__builtin_fabsf(a.scale) < 1e-30f) a.scale = 0.f;  // no score leaves 2^-40 then: all weights alike
    a.q_heads = c.q_heads, a.kv_heads = c.cache.kv_heads, a.group = G, a.seqs = (int)c.seqs, a.tiles = (int)p.tiles, a.splits = p.splits, a.split_blocks = p.split_blocks;
    a.page_units = c.cache.kv_heads * c.cache.page_blocks * (D / 4 + 1);  // of 128 bytes: at most 2^21 * 65
    a.page_shift = __builtin_ctz((unsigned)c.cache.page_blocks);
    const int64_t grid = c.seqs * c.cache.kv_heads * p.tiles * p.splits;
    if (D == 64) return start<64>(a, p, grid, c.max_q, st);
    if (D == 128) return start<128>(a, p, grid, c.max_q, st);
    return start<256>(a, p, grid, c.max_q, st);
}

}  // namespace itq3s

// Norm and position rotation of query and key heads, keys and values into the 4-bit cache, and back.
//
// A row is one head of one token, D values x.  Norm: x w / sqrt(mean x^2 + eps).  Rotation: pairs (a, b) of channels turn by
// the angle position * freq[i]: (a cos - b sin, b cos + a sin), times a gain.  Cache: w = H x with the orthonormal
// Walsh-Hadamard matrix of D points, step s = max|w| / 7.5 rounded to fp16, digit c = floor(w / s + 1/2) within -8..7;
// the row stands for H (s c).  The transform spreads an outlier channel over the row, so that one step serves it whole.
//
// What decides digits is computed in 64 bits (keys and values; the vector ALU issues a 64-bit addition at the rate of an
// unpacked 32-bit one), so that a digit depends on the definition alone and not on an order of summation or on a
// library's sine: with 32 bits some 1e-6 of the digits fall on the other side of their border.  Queries, which are
// only rounded, take 32 bits behind a 64-bit angle.
//
// A lane holds eight channels of a row: 8, 16 or 32 lanes a row, 8, 4 or 2 rows a wavefront.  The rows of one wavefront are heads of
// one token (a kilobyte of neighbouring memory an instruction; they share the sines, so each row of lanes works out its
// part of them) or, for values, neighbouring tokens (so that their bytes share words of memory).  A wavefront walks over
// heads with the sines that it has worked out once.
//
// Measured: 11385 tokens, 64 normed query heads and 8 kv heads of 128, half of each rotated, fp16 (440 MB) 99 us, 4.4 TB/s; the
// arithmetic in 64 bits takes the vector ALU for 72 % of that time, so neither the memory (a copy: 5.2 TB/s) nor the ALU
// is far away.  One token 4.4 us, most of it a launch and two loads that wait for each other (position, then row).
#include <type_traits>

#include "itq3s_attention.h"
#include "itq3s_cache.h"

namespace itq3s {

namespace {

// eight neighbouring values
__device__ __forceinline__ void load8(const _Float16* p, _Float16 (&v)[8]) {
    const half8 h = *reinterpret_cast<const half8*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = h[j];
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const floatx4 a = reinterpret_cast<const floatx4*>(p)[0], b = reinterpret_cast<const floatx4*>(p)[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
}
// To fp16 with one rounding.  From 64 bits by way of 32: what is below the upper 20 bits of the mantissa goes into the last of them
// (not zero: set), so the way there is exact and the border stays on its side.
__device__ __forceinline__ _Float16 to_half(float v) { return (_Float16)v; }
__device__ __forceinline__ _Float16 to_half(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t rest = (uint32_t)u, upper = (uint32_t)(u >> 32) | (rest < 1u ? rest : 1u);
    return (_Float16)(float)__builtin_bit_cast(double, (uint64_t)upper << 32);
}
template <typename R>
__device__ __forceinline__ void store8(_Float16* p, const R (&v)[8]) {
    half8 h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = to_half(v[j]);
    *reinterpret_cast<half8*>(p) = h;
}
template <typename R>
__device__ __forceinline__ void store8(float* p, const R (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<floatx4*>(p)[i] = floatx4{(float)v[4 * i], (float)v[4 * i + 1], (float)v[4 * i + 2], (float)v[4 * i + 3]};
}

// sine and cosine in 64 bits: the angle less the nearest multiple of pi/2 (pi/2 in two parts, products by fused
// multiply-add: exact to 1e-17 for the 2^31 positions there are), then the Taylor series, whose first left-out terms are
// (pi/4)^19 / 19! = 8e-20 and (pi/4)^18 / 18! = 2e-18.
__device__ __forceinline__ void turn(double angle, double& c, double& s) {
    const double n = __builtin_rint(angle * 0.63661977236758134308);
    double r = __builtin_fma(n, -1.5707963267948965580, angle);
    r = __builtin_fma(n, -6.1232339957367660359e-17, r);
    const double z = r * r;
    double a = 1.0 / 355687428096000.0, b = 1.0 / 20922789888000.0;  // 17!, 16!
    a = __builtin_fma(a, z, -1.0 / 1307674368000.0), b = __builtin_fma(b, z, -1.0 / 87178291200.0);
    a = __builtin_fma(a, z, 1.0 / 6227020800.0), b = __builtin_fma(b, z, 1.0 / 479001600.0);
    a = __builtin_fma(a, z, -1.0 / 39916800.0), b = __builtin_fma(b, z, -1.0 / 3628800.0);
    a = __builtin_fma(a, z, 1.0 / 362880.0), b = __builtin_fma(b, z, 1.0 / 40320.0);
    a = __builtin_fma(a, z, -1.0 / 5040.0), b = __builtin_fma(b, z, -1.0 / 720.0);
    a = __builtin_fma(a, z, 1.0 / 120.0), b = __builtin_fma(b, z, 1.0 / 24.0);
    a = __builtin_fma(a, z, -1.0 / 6.0), b = __builtin_fma(b, z, -0.5);
    const double sn = __builtin_fma(r * z, a, r), cs = __builtin_fma(z, b, 1.0);
    const int q = (int)__builtin_fma(-4.0, __builtin_floor(n * 0.25), n);
    s = (q & 1) ? cs : sn;
    c = (q & 1) ? sn : cs;
    if (q & 2) s = -s;
    if ((q + 1) & 2) c = -c;
}

struct AppendArgs {
    const void *Q, *K, *V;
    void *Q_out, *K_out;
    const float *q_norm, *k_norm;
    const int32_t* positions;
    const double* freq;
    unsigned char* data;
    const int64_t* slots;
    uint32_t* flags;
    int64_t ldq, ldk, ldv, ldqo, ldko, T, slots_end;
    int q_heads, kv_heads, rot, interleaved;
    float eps, gain;
    int page_blocks;                  // blocks of 32 tokens a page
    int q_step, k_step, v_step;       // heads that a wavefront walks over
    int64_t groups;                   // of neighbouring tokens, whose values a wavefront takes
    int64_t k_jobs, v_jobs, q_jobs;   // wavefronts
    int few_are_kv, few_blocks, period;  // workgroups of keys and values (or of queries), one among so many while there are any
};

template <int D>
struct Rows {
    static constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    __device__ static __forceinline__ int row() { return lane_id() / kLanes; }
    __device__ static __forceinline__ int channel() { return lane_id() % kLanes * 8; }
};

// What a lane's channels and their partners are multiplied with: cosines and sines (pairs of channels have theirs in common where
// they are interleaved) times gain and the norm's weights.
template <typename R>
struct Turns {
    R own[8], other[8];
};
template <int D, typename R>
__device__ __forceinline__ void find_turns(const AppendArgs& a, int64_t token, int ch, bool turned, const float* norm, Turns<R>& t) {
    const int half = a.rot / 2;
    const bool upper = ch >= half;
    const int mate = turned && !a.interleaved ? (upper ? ch - half : ch + half) : ch;
    float w[8], wm[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = wm[j] = 1.f;
    if (norm != nullptr) {
        load8(norm + ch, w);
        load8(norm + mate, wm);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) t.own[j] = (R)1, t.other[j] = (R)0;
    if (a.rot != 0) {
        const double pos = (double)a.positions[token], gain = (double)a.gain;
        const int first = !turned ? 0 : a.interleaved ? ch / 2 : upper ? ch - half : ch;  // (lanes that do not turn work on a frequency that is there)
        // the rows of lanes have a token in common, and the same channels: each works out a part
        constexpr int kPart = 8 / Rows<D>::kRows;
        R pc[kPart], ps[kPart];
#pragma unroll
        for (int j = 0; j < kPart; ++j) {
            const int k = Rows<D>::row() * kPart + j;
            double c, s;
            turn(pos * a.freq[first + (a.interleaved ? k / 2 : k)], c, s);
            pc[j] = (R)(c * gain), ps[j] = (R)(s * gain);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int from = j / kPart * Rows<D>::kLanes + lane_id() % Rows<D>::kLanes;
            t.own[j] = __shfl(pc[j % kPart], from, 64), t.other[j] = __shfl(ps[j % kPart], from, 64);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool second = a.interleaved ? j % 2 == 1 : upper;  // of its pair
            t.other[j] = !turned ? (R)0 : second ? t.other[j] : -t.other[j];
            t.own[j] = turned ? t.own[j] : (R)1;
        }
    }
    if (norm != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t.own[j] = t.own[j] * (R)w[j];
            t.other[j] = t.other[j] * (R)(a.interleaved ? w[j ^ 1] : wm[j]);
        }
    }
}

// One row through norm and rotation.  Partners' values come as they are: the norm's factor is the row's, and waits for the end.
template <int D, typename R, typename In>
__device__ __forceinline__ void norm_and_turn(const AppendArgs& a, const In (&x)[8], bool normed, int partner, const Turns<R>& t, R (&y)[8]) {
    R f = (R)1;
    if (normed) {
        R sum = (R)0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = __builtin_elementwise_fma((R)x[j], (R)x[j], sum);
        sum = row_sum<D>(sum);
        f = (R)1 / __builtin_elementwise_sqrt(sum * (R)(1.0 / D) + (R)a.eps);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (R)x[j] * t.own[j];
    if (a.rot != 0) {
        R other[8];
        if (a.interleaved) {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = (R)x[j ^ 1];
        } else if constexpr (std::is_same<In, _Float16>::value) {  // two values a word
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint32_t mine = (uint32_t)__builtin_bit_cast(uint16_t, x[j]) | (uint32_t)__builtin_bit_cast(uint16_t, x[j + 1]) << 16;
                const uint32_t got = (uint32_t)__shfl((int)mine, partner, 64);
                other[j] = (R)__builtin_bit_cast(_Float16, (uint16_t)got);
                other[j + 1] = (R)__builtin_bit_cast(_Float16, (uint16_t)(got >> 16));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = (R)__shfl(x[j], partner, 64);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __builtin_elementwise_fma(other[j], t.other[j], y[j]);
    }
    if (normed) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = y[j] * f;
    }
}

// One row into the cache: transform, step, digits.  Rows without a slot do everything but the stores.
template <int D>
__device__ __forceinline__ void quantize_row(const AppendArgs& a, double (&v)[8], int64_t slot, bool live, int head, bool is_value) {
    hadamard<D>(v);
    double most = 0.0;
    bool finite = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        finite = finite && __builtin_fabs(v[j]) <= 1.7976931348623157e308;
        most = __builtin_fmax(most, __builtin_fabs(v[j]));
    }
    most = row_max<D>(finite ? most : __builtin_inf());
    const bool bad = !(most <= 1.7976931348623157e308);
    const float s32 = (float)(most * (1.0 / (7.5 * kRootD<D>)));
    const bool sat = s32 > 65504.f;
    _Float16 s = (_Float16)(sat ? 65504.f : s32);
    if (bad) s = (_Float16)0.f;
    const double step = (double)(float)s * kRootD<D>, inv = step > 0.0 ? 1.0 / step : 0.0;
    int d[8];
    // The nearest whole number, from the low bits of w / step + 1.5 2^52; it is right where the remainder stays clear of half a step, and
    // the number within 32 bits: it is unless the step was cut to fp16's largest.
    constexpr double kWhole = 6755399441055744.0;
    double rest = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const double q = __builtin_fma(v[j], inv, kWhole);
        rest = __builtin_fmax(rest, __builtin_fabs(__builtin_fma(kWhole - q, step, v[j])));
        d[j] = __double2loint(q);
    }
    if (__builtin_amdgcn_ballot_w64(sat || !(rest < step * (0.5 - 0x1p-40))) != 0) {  // such a row, a border or a step of 0 in the wavefront
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // floor(w / step + 1/2): by the reciprocal, then set right by the remainder, whose sign is exact
            double q = __builtin_floor(__builtin_fma(v[j], inv, 0.5));
            const double r = __builtin_fma(-q, step, v[j]);
            if (r >= 0.5 * step) q += 1.0;
            if (r < -0.5 * step) q -= 1.0;
            d[j] = step > 0.0 ? (int)__builtin_fmin(__builtin_fmax(q, -8.0), 7.0) : 0;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = (d[j] < -8 ? -8 : d[j] > 7 ? 7 : d[j]) + 8;
    const int lane = lane_id(), ch = Rows<D>::channel();
    if (a.flags != nullptr && live && ch == 0 && (bad || sat)) atomicOr(a.flags, bad ? kFlagNonFinite : kFlagScaleSat);
    const int t = (int)(slot & 31);
    const int64_t block = slot >> 5;
    unsigned char* const base = a.data + block_offset<D>(block / a.page_blocks, head, a.kv_heads, a.page_blocks, (int)(block % a.page_blocks));
    if (!is_value) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) w |= (uint32_t)d[j] << (4 * ((j >> 1) + 4 * (j & 1)));
        if (live) *reinterpret_cast<uint32_t*>(base + t * (D / 2) + ch / 2) = w;
    } else {
        // channels c and c + 16 of a group of 32 share a byte: lanes l and l ^ 2 hold them, each makes four of the bytes
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) w |= (uint32_t)d[j] << (4 * j);
        const uint32_t o = (uint32_t)row_xor_i32<2>((int)w);
        const bool upper = (lane & 2) != 0;
        const uint32_t lo = upper ? o >> 16 : w, hi = upper ? w >> 16 : o;
        const int p = ch / 32, c = (ch & 8) + (upper ? 4 : 0);
        unsigned char* const at = base + 16 * D + value_byte(t, p, c);
        if (live) {
#pragma unroll
            for (int j = 0; j < 4; ++j) at[16 * j] = (unsigned char)(((lo >> (4 * j)) & 15u) | ((hi >> (4 * j)) & 15u) << 4);
        }
    }
    if (live && ch == 0) *reinterpret_cast<_Float16*>(base + 32 * D + 4 * t + (is_value ? 2 : 0)) = s;
}

// One wavefront: its token's rows (of values: its tokens') for heads h0 .. h1 - 1 of the queries (what 0), the keys (1) or the values (2).
template <int D, typename In, typename Out, int kWhat>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int64_t group, int h0, int h1) {
    typedef typename std::conditional<kWhat == 0, float, double>::type R;
    const int row = Rows<D>::row(), ch = Rows<D>::channel();
    constexpr bool by_token = kWhat == 2;
    const int64_t token = by_token ? group * Rows<D>::kRows + row : group;
    const bool here = token < a.T;
    const int64_t tok = here ? token : a.T - 1;
    const int64_t ld = kWhat == 0 ? a.ldq : kWhat == 1 ? a.ldk : a.ldv;
    const In* const src = static_cast<const In*>(kWhat == 0 ? a.Q : kWhat == 1 ? a.K : a.V) + tok * ld + ch;
    Out* const dst = kWhat == 2 ? nullptr : static_cast<Out*>(kWhat == 0 ? a.Q_out : a.K_out);
    const int64_t ldo = kWhat == 0 ? a.ldqo : a.ldko;
    const bool cached = kWhat != 0 && a.data != nullptr;
    int64_t slot = 0;
    bool live = false;
    if (cached) {
        slot = a.slots[tok];
        live = here && slot >= 0 && slot < a.slots_end;
        if (here && slot >= a.slots_end && ch == 0 && a.flags != nullptr) atomicOr(a.flags, kFlagBadSlot);
        if (!live) slot = 0;
    }
    const int step = by_token ? 1 : Rows<D>::kRows;
    const int heads = kWhat == 0 ? a.q_heads : a.kv_heads;
    // kBatch rows are on their way while as many are worked on
    constexpr int kBatch = kWhat == 0 ? 4 : 2;
    auto head_of = [&](int hb) { return by_token ? hb : hb + row; };
    In x[kBatch][8], next[kBatch][8];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        const int h = head_of(h0 + b * step);
        load8(src + (int64_t)(h < heads ? h : heads - 1) * D, x[b]);
    }
    const int half = a.rot / 2;
    const bool turned = kWhat != 2 && ch < a.rot;
    const int partner = lane_id() + (turned ? (ch < half ? half : -half) : 0) / 8;
    const float* const norm = kWhat == 0 ? a.q_norm : kWhat == 1 ? a.k_norm : nullptr;
    Turns<R> t;
    if constexpr (kWhat != 2) find_turns<D, R>(a, tok, ch, turned, norm, t);
    for (int hb = h0; hb < h1; hb += kBatch * step) {
        if (hb + kBatch * step < h1) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int h = head_of(hb + (kBatch + b) * step);
                load8(src + (int64_t)(h < heads ? h : heads - 1) * D, next[b]);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (hb + b * step >= h1) break;
            const int h = head_of(hb + b * step);
            R y[8];
            if constexpr (kWhat == 2) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = (R)x[b][j];
            } else {
                norm_and_turn<D>(a, x[b], norm != nullptr, partner, t, y);
                if (dst != nullptr && here && h < h1) store8(dst + tok * ldo + (int64_t)h * D + ch, y);
            }
            if constexpr (kWhat != 0) {
                if (cached) quantize_row<D>(a, y, slot, live && h < h1, h < heads ? h : 0, kWhat == 2);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[b][j] = next[b][j];
    }
}

template <int D, typename In, typename Out>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a) {
    // Workgroups of keys and values, which compute, and of queries, which move memory, run side by side: the fewer ones are spread
    // among the others.
    const int b = blockIdx.x, turn = b / a.period, before = turn + (b % a.period != 0 ? 1 : 0);
    const bool few = b % a.period == 0 && turn < a.few_blocks, kv = few == (a.few_are_kv != 0);
    const int64_t block = few ? turn : b - (before < a.few_blocks ? before : a.few_blocks);
    int64_t job = block * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (!kv) {
        if (job < a.q_jobs) {
            const int h0 = (int)(job / a.T) * a.q_step;
            append_rows<D, In, Out, 0>(a, job % a.T, h0, h0 + a.q_step < a.q_heads ? h0 + a.q_step : a.q_heads);
        }
        return;
    }
    if (job < a.k_jobs) {
        const int h0 = (int)(job / a.T) * a.k_step;
        append_rows<D, In, Out, 1>(a, job % a.T, h0, h0 + a.k_step < a.kv_heads ? h0 + a.k_step : a.kv_heads);
        return;
    }
    job -= a.k_jobs;
    if (job < a.v_jobs) {
        const int h0 = (int)(job / a.groups) * a.v_step;
        append_rows<D, In, Out, 2>(a, job % a.groups, h0, h0 + a.v_step < a.kv_heads ? h0 + a.v_step : a.kv_heads);
        return;
    }
}

// ---- read

struct ReadArgs {
    const unsigned char* data;
    const int64_t* slots;
    void *K, *V;
    uint32_t* flags;
    int64_t ldk, ldv, T, slots_end;
    int kv_heads, page_blocks;
};

// The transform of a row of digits: sums of at most 256 * 8 = 2^11 in fp16, so every step is exact.  Pairs (2i, 2i + 1).
template <int D>
__device__ __forceinline__ void hadamard_digits(half2v (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = half2v{v[i][0], v[i][0]} + half2v{v[i][1], -v[i][1]};
#pragma unroll
    for (int h = 1; h < 4; h *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((i & h) == 0) {
                const half2v a = v[i], b = v[i + h];
                v[i] = a + b;
                v[i + h] = a - b;
            }
    const int lane = lane_id();
#define ITQ3S_STAGE(m)                                                                                                    \
    if constexpr ((m) < D / 8) {                                                                                          \
        const _Float16 sign = (lane & (m)) != 0 ? (_Float16)-1.f : (_Float16)1.f;                                         \
        _Pragma("unroll") for (int i = 0; i < 4; ++i)                                                                     \
            v[i] = half2v{sign, sign} * v[i] + __builtin_bit_cast(half2v, row_xor_i32<(m)>(__builtin_bit_cast(int, v[i]))); \
    }
    ITQ3S_STAGE(1) ITQ3S_STAGE(2) ITQ3S_STAGE(4) ITQ3S_STAGE(8) ITQ3S_STAGE(16)
#undef ITQ3S_STAGE
}

// Eight digits' sums times a factor, rounded once to the type (fp16: by the instruction that multiplies).
__device__ __forceinline__ void store_scaled(_Float16* p, const half2v (&v)[4], float f) {
    half8 h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = (_Float16)__builtin_fmaf((float)v[j >> 1][j & 1], f, 0.f);
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, h), reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store_scaled(float* p, const half2v (&v)[4], float f) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        __builtin_nontemporal_store(floatx4{(float)v[2 * i][0] * f, (float)v[2 * i][1] * f, (float)v[2 * i + 1][0] * f, (float)v[2 * i + 1][1] * f}, reinterpret_cast<floatx4*>(p) + i);
}

// Value bytes of a row's eight channels from `lane`'s first, as four words of two digits (to shift): the byte of channel c and of
// c + 16 is one.
__device__ __forceinline__ void value_pairs(const unsigned char* at, int shift, half2v (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = low_pair((((uint32_t)at[32 * j] | (uint32_t)at[32 * j + 16] << 16) >> shift) & 0x000f000fu);
}

// A workgroup reads 32 listed rows of one head.  Key words go straight to their lanes; of the values, whose bytes lie eight
// tokens beside each other, whole blocks go through LDS: listed rows are mostly neighbours, so 32 of them lie in one block or
// two.  Where they do not, a lane gathers its eight bytes from memory.
// Memory bounds it, the stores before all (fp16: 0.52 bytes in, 2 out a value; stored past the caches, nothing reads them
// soon): 32768 tokens of 8 heads of 128, 169 MB, 33 us, 5.1 TB/s where a copy reaches 5.2.  The vector ALU is busy for 76 % of it.
template <int D, typename Out>
__global__ void __launch_bounds__(256) read_kernel(const ReadArgs a) {
    constexpr int kRows = Rows<D>::kRows, kChunks = D, kHalf = 1024 + 64;  // 16-byte chunks of a block's values; LDS bytes of 64 channels
    __shared__ __align__(16) unsigned char values[2 * (D / 64) * kHalf];
    const int head = blockIdx.y;
    const int64_t first = (int64_t)blockIdx.x * 32;
    const int tid = threadIdx.x, wave = tid >> 6, lane = lane_id();
    auto place_of = [&](int64_t block) {
        return a.data + block_offset<D>(block / a.page_blocks, head, a.kv_heads, a.page_blocks, (int)(block % a.page_blocks));
    };
    // every wavefront looks over the list (the lower half of its lanes does)
    const int64_t mine = first + (lane & 31);
    const int64_t listed = mine < a.T ? a.slots[mine] : -1;
    const bool ours = listed >= 0 && listed < a.slots_end;
    if (listed >= a.slots_end && tid < 32 && head == 0 && a.flags != nullptr) atomicOr(a.flags, kFlagBadSlot);
    const int64_t my_block = ours ? listed >> 5 : -1;
    const uint64_t some = __builtin_amdgcn_ballot_w64(ours);
    int64_t two[2] = {0, 0};
    two[0] = two[1] = some != 0 ? __shfl(my_block, __builtin_ctzll(some), 64) : 0;
    const uint64_t others = __builtin_amdgcn_ballot_w64(ours && my_block != two[0]);
    if (others != 0) two[1] = __shfl(my_block, __builtin_ctzll(others), 64);
    const bool near = __builtin_amdgcn_ballot_w64(ours && my_block != two[0] && my_block != two[1]) == 0;
    // a lane's rows, and what of them does not go through LDS
    constexpr int kRounds = 8 / kRows;
    const int row = Rows<D>::row(), ch = Rows<D>::channel();
    uint32_t kw[kRounds], steps[kRounds];
    int at[kRounds];  // its value bytes in LDS
    bool live[kRounds];
#pragma unroll
    for (int n = 0; n < kRounds; ++n) {
        int64_t slot = __shfl(listed, wave * 8 + n * kRows + row, 64);
        live[n] = slot >= 0 && slot < a.slots_end;
        if (!live[n]) slot = two[0] << 5;
        const int t = (int)(slot & 31), byte = value_byte(t, ch / 32, ch & 8);
        const unsigned char* const base = place_of(slot >> 5);
        kw[n] = *reinterpret_cast<const uint32_t*>(base + t * (D / 2) + ch / 2);
        steps[n] = *reinterpret_cast<const uint32_t*>(base + 32 * D + 4 * t);
        at[n] = ((slot >> 5) == two[0] ? 0 : (D / 64) * kHalf) + byte / 1024 * kHalf + byte % 1024;
    }
    if (near) {
#pragma unroll
        for (int u = 0; u < (2 * kChunks + 255) / 256; ++u) {
            const int x = tid + 256 * u, which = x / kChunks, chunk = x % kChunks;
            if (which == 0 || (which == 1 && others != 0))
                *reinterpret_cast<u32x4*>(values + which * (D / 64) * kHalf + chunk / 64 * kHalf + chunk % 64 * 16) =
                    reinterpret_cast<const u32x4*>(place_of(which == 0 ? two[0] : two[1]) + 16 * D)[chunk];
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kRounds; ++n) {
        const int i = wave * 8 + n * kRows + row, shift = (ch & 16) != 0 ? 4 : 0;
        const int64_t token = first + i;
        half2v k[4] = {low_pair(kw[n]), high_pair(kw[n]), low_pair(kw[n] >> 8), high_pair(kw[n] >> 8)};
        half2v v[4];
        if (near) {
            value_pairs(values + at[n], shift, v);
        } else {
            int64_t slot = __shfl(listed, i, 64);  // (all lanes: a row's entry may be with one of a row that is not there)
            if (!live[n]) slot = two[0] << 5;
            value_pairs(place_of(slot >> 5) + 16 * D + value_byte((int)(slot & 31), ch / 32, ch & 8), shift, v);
        }
        hadamard_digits<D>(k);
        hadamard_digits<D>(v);
        const float root = (float)(1.0 / kRootD<D>);
        const float ks = live[n] ? f16_bits_to_f32(steps[n] & 0xffffu) * root : 0.f, vs = live[n] ? f16_bits_to_f32(steps[n] >> 16) * root : 0.f;
        if (token < a.T) {
            store_scaled(static_cast<Out*>(a.K) + token * a.ldk + (int64_t)head * D + ch, k, ks);
            store_scaled(static_cast<Out*>(a.V) + token * a.ldv + (int64_t)head * D + ch, v, vs);
        }
    }
}

template <int D, typename In, typename Out>
int start_append(const AppendArgs& a, int64_t blocks, hipStream_t st) {
    append_kernel<D, In, Out><<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? 0 : -6;
}
template <int D>
int start_append(const AppendArgs& a, int64_t blocks, int in_f16, int out_f16, hipStream_t st) {
    if (in_f16) return out_f16 ? start_append<D, _Float16, _Float16>(a, blocks, st) : start_append<D, _Float16, float>(a, blocks, st);
    return out_f16 ? start_append<D, float, _Float16>(a, blocks, st) : start_append<D, float, float>(a, blocks, st);
}

}  // namespace

int launch_append(const AppendCall& c, hipStream_t st) {
    const int rows = 512 / c.head_dim;  // of a wavefront
    AppendArgs a{};
    a.Q = c.Q, a.K = c.K, a.V = c.V, a.Q_out = c.Q_out, a.K_out = c.K_out;
    a.q_norm = c.q_norm, a.k_norm = c.k_norm, a.positions = c.positions, a.freq = c.freq, a.slots = c.slots, a.flags = c.flags;
    a.ldq = c.ldq, a.ldk = c.ldk, a.ldv = c.ldv, a.ldqo = c.ldqo, a.ldko = c.ldko, a.T = c.T;
    a.q_heads = c.Q != nullptr ? c.q_heads : 0, a.kv_heads = c.kv_heads, a.rot = c.rot, a.interleaved = c.interleaved, a.eps = c.eps, a.gain = c.gain;
    a.data = c.cache.data, a.page_blocks = c.cache.data != nullptr ? c.cache.page_blocks : 1;
    a.slots_end = c.cache.data != nullptr ? c.cache.pages * c.cache.page_blocks * kCacheBlock : 0;
    // Values: neighbouring tokens in a wavefront.  (Heads of one token as for keys are no better for one token, and worse for many: 10000
    // tokens, 32 heads of 128 203 us instead of 198.)
    a.groups = (c.T + rows - 1) / rows;
    // Heads that a wavefront walks over: more of them share the sines, fewer make more wavefronts.  8 a unit are plenty (us with 4, 8 and
    // 16, 64 and 8 heads of 128: 500 tokens 15.5, 17.1 and 18.2, 1000 22.0, 20.1 and 22.1, 2000 40.8, 30.3 and 29.6), and 32
    // of the short ones of values (11385 tokens, 64 and 8 heads of 128: 8, 4, 2 and 1 heads 116, 114, 106 and 118 us).
    auto heads_of = [&](int heads, int step, int64_t groups, int plenty) {
        while (step < heads && groups * ((heads + 2 * step - 1) / (2 * step)) >= plenty * (int64_t)cu_count()) step *= 2;
        return step;
    };
    a.q_step = heads_of(a.q_heads, rows, c.T, 8), a.k_step = heads_of(c.kv_heads, rows, c.T, 8), a.v_step = heads_of(c.kv_heads, 1, a.groups, 32);
    a.k_jobs = c.K != nullptr ? c.T * ((c.kv_heads + a.k_step - 1) / a.k_step) : 0;
    a.v_jobs = c.V != nullptr ? a.groups * ((c.kv_heads + a.v_step - 1) / a.v_step) : 0;
    a.q_jobs = a.q_heads > 0 ? c.T * ((a.q_heads + a.q_step - 1) / a.q_step) : 0;
    const int64_t kv_blocks = (a.k_jobs + a.v_jobs + 3) / 4, q_blocks = (a.q_jobs + 3) / 4, blocks = kv_blocks + q_blocks;
    if (blocks > 0x7fffffffLL) return -2;
    a.few_are_kv = kv_blocks <= q_blocks, a.few_blocks = (int)(a.few_are_kv ? kv_blocks : q_blocks);
    a.period = a.few_blocks > 0 ? (int)(blocks / a.few_blocks) : 1;
    if (c.head_dim == 64) return start_append<64>(a, blocks, c.in_f16, c.out_f16, st);
    if (c.head_dim == 128) return start_append<128>(a, blocks, c.in_f16, c.out_f16, st);
    return start_append<256>(a, blocks, c.in_f16, c.out_f16, st);
}

int launch_cache_read(const CacheView& cache, const int64_t* slots, int64_t T, void* K, int64_t ldk, void* V, int64_t ldv, int out_f16, uint32_t* flags, hipStream_t st) {
    const ReadArgs a{cache.data, slots, K, V, flags, ldk, ldv, T, cache.pages * cache.page_blocks * kCacheBlock, cache.kv_heads, cache.page_blocks};
    const dim3 grid((unsigned)((T + 31) / 32), (unsigned)cache.kv_heads);
    if (cache.head_dim == 64) {
        if (out_f16) read_kernel<64, _Float16><<<grid, dim3(256), 0, st>>>(a);
        else read_kernel<64, float><<<grid, dim3(256), 0, st>>>(a);
    } else if (cache.head_dim == 128) {
        if (out_f16) read_kernel<128, _Float16><<<grid, dim3(256), 0, st>>>(a);
        else read_kernel<128, float><<<grid, dim3(256), 0, st>>>(a);
    } else {
        if (out_f16) read_kernel<256, _Float16><<<grid, dim3(256), 0, st>>>(a);
        else read_kernel<256, float><<<grid, dim3(256), 0, st>>>(a);
    }
    return hipGetLastError() == hipSuccess ? 0 : -6;
}

}  // namespace itq3s

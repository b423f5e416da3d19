// One wave's attention of up to sixteen query columns over blocks of key and value rows, with a running maximum and sum.
// The rows come straight from memory into the operands of the matrix instructions, whole rows at a time, and nothing
// crosses lanes but the maximum:
//
//   logits    S^T = K Q^T: lane (c = lane % 16, j = lane / 16) ends up with column c of four consecutive rows of every tile.
//             Which key is which row of a tile is free: register e of lane group j is key 4 e + j of a tile of sixteen.
//   weights   p = 2^(s - m): what the lane holds is its operand of the second product as it is.
//   output    O^T = V^T P^T: the lane loads features c D / 16 ... of its own eight (four) value rows, so that one load is four whole
//             rows behind one another, and pairs the bf16 of two rows up by byte permutes; the t-th product yields the features
//             D / 16 * i + t, i = 0 ... 15.  (With keys 8 j + e of 32 instead, a load is four rows 2 KB apart, which are in two of the
//             sixteen channels of the cache.)
//
// Outputs are fp32, so bf16 weights are the sum of three bf16: twice the upper half of what is left of a float, shrunk a little
// first so that no term is zero (zero times an infinite value is NaN, the weight times it is infinite), then the rest, which
// rounding leaves within 2^-21 of the weight.  Logits, maxima and sums are fp32.
#pragma once

#include "device_utils.h"

namespace uncomp {

// a float's upper sixteen bits: a bf16, cut
__device__ __forceinline__ float upper_half(float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); }

constexpr float kLog2eA = 1.4426950408889634f, kLn2A = 0.6931471805599453f;

// maximum / sum over the four lanes (of the four rows of sixteen) that share a column
__device__ __forceinline__ float column_max(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// The reference that exponentials are taken against: the maximum, or zero while nothing has been seen (a maximum of -inf
// would turn logits of -inf into NaN instead of no weight).
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

template <int N>
struct Words { uint32_t w[N]; };
template <int N>
__device__ __forceinline__ Words<N> load_words(const void* p) {
    Words<N> r;
    if constexpr (N == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else {
        static_assert(N == 2, "two or four words");
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        r.w[0] = v.x; r.w[1] = v.y;
    }
    return r;
}

// row of a tile that register e of lane group j holds
__device__ __forceinline__ int row_of(int e, int j) { return 4 * e + j; }

template <typename T, int D>
struct WaveAttend;

// ---- bf16: blocks of 32 keys ---------------------------------------------------------------------------------------
template <int D>
struct WaveAttend<bf16_bits, D> {
    static constexpr int kBlock = 32, kPerLane = 8, kSteps = D / 32, kVw = D / 16;
    struct Keys { Words<4> w[2][kSteps]; };
    struct Values { Words<kVw / 2> w[8]; };
    bf16x8_t q[kSteps];
    f32x4_t o[kVw];
    float m, l;                        // running maximum (base 2), this lane's share of the running sum

    __device__ __forceinline__ void reset() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int t = 0; t < kVw; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    // qrow: the lane's column's query row, or NULL for a column that is not there
    __device__ __forceinline__ void load_query(const bf16_bits* qrow, int lane) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const Words<4> w = qrow != nullptr ? load_words<4>(qrow + 32 * s + 8 * (lane >> 4)) : Words<4>{{0u, 0u, 0u, 0u}};
            q[s] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
    // feature of product t that row i of its outputs is (t a multiple of four: of the four products from t on, four features on)
    static __device__ __forceinline__ int feature(int i, int t) { return kVw * i + t; }
    static __device__ __forceinline__ int key_row(int lane, int tile) { return 16 * tile + row_of(lane & 3, (lane & 15) >> 2); }
    static __device__ __forceinline__ int value_row(int lane, int e) { return 16 * (e >> 2) + row_of(e & 3, lane >> 4); }
    // tile0, tile1: the first rows of the block's two tiles
    static __device__ __forceinline__ void load_keys(Keys& k, int lane, const bf16_bits* tile0, const bf16_bits* tile1) {
        const int at = key_row(lane, 0) * D + 8 * (lane >> 4);
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) k.w[a][s] = load_words<4>((a ? tile1 : tile0) + (at + 32 * s));
    }
    static __device__ __forceinline__ void load_values(Values& v, int lane, const bf16_bits* tile0, const bf16_bits* tile1) {
        const int at = value_row(lane, 0) * D + kVw * (lane & 15);
#pragma unroll
        for (int e = 0; e < 8; ++e) v.w[e] = load_words<kVw / 2>((e < 4 ? tile0 : tile1) + (at + 4 * (e & 3) * D));
    }
    // one row in another's place, in the lanes that hold it: row `at` of the block
    static __device__ __forceinline__ void put_key(Keys& k, int lane, int at, const bf16_bits* row) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const Words<4> w = load_words<4>(row + 32 * s + 8 * (lane >> 4));
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) k.w[a][s].w[i] = key_row(lane, a) == at ? w.w[i] : k.w[a][s].w[i];
        }
    }
    static __device__ __forceinline__ void put_value(Values& v, int lane, int at, const bf16_bits* row) {
        const Words<kVw / 2> w = load_words<kVw / 2>(row + kVw * (lane & 15));
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < kVw / 2; ++i) v.w[e].w[i] = value_row(lane, e) == at ? w.w[i] : v.w[e].w[i];
    }
    static __device__ __forceinline__ void clear_value(Values& v, int e) {
#pragma unroll
        for (int i = 0; i < kVw / 2; ++i) v.w[e].w[i] = 0u;
    }
    __device__ __forceinline__ void logits(const Keys& k, float scale2, float (&s)[kPerLane]) const {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            f32x4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < kSteps; ++t)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k.w[a][t]), q[t], c, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * a + e] = c[e] * scale2;
        }
    }
    // the t-th product's value operand
    static __device__ __forceinline__ bf16x8_t value_operand(const Values& v, int t) {
        Words<4> a;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            a.w[e] = __builtin_amdgcn_perm(v.w[2 * e + 1].w[t >> 1], v.w[2 * e].w[t >> 1], (t & 1) ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(bf16x8_t, a);
    }
    __device__ __forceinline__ void add_values(const Values& v, const float (&p)[kPerLane]) {
        constexpr float kShrink = 1.f - 0x1p-8f;
        bf16x8_t w[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = upper_half(p[e] * kShrink), b = upper_half((p[e] - a) * kShrink);
            w[0][e] = (__bf16)a;
            w[1][e] = (__bf16)b;
            w[2][e] = (__bf16)((p[e] - a) - b);
        }
#pragma unroll
        for (int t = 0; t < kVw; ++t) {
            const bf16x8_t a = value_operand(v, t);
#pragma unroll
            for (int i = 0; i < 3; ++i) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[i], o[t], 0, 0, 0);
        }
    }
};

// ---- fp32: blocks of 16 keys ---------------------------------------------------------------------------------------
template <int D>
struct WaveAttend<float, D> {
    static constexpr int kBlock = 16, kPerLane = 4, kSteps = D / 16, kVw = D / 16;
    struct Keys { f32x4_t w[kSteps]; };
    struct Values { f32x4_t w[4][kVw / 4]; };
    f32x4_t q[kSteps];
    f32x4_t o[kVw];
    float m, l;

    __device__ __forceinline__ void reset() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int t = 0; t < kVw; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void load_query(const float* qrow, int lane) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            q[s] = qrow != nullptr ? *reinterpret_cast<const f32x4_t*>(qrow + 16 * s + 4 * (lane >> 4)) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    // sixteen lanes load 256 bytes of a row behind one another
    static __device__ __forceinline__ int feature(int i, int t) { return 64 * (t >> 2) + 4 * i + (t & 3); }
    static __device__ __forceinline__ int key_row(int lane, int) { return row_of(lane & 3, (lane & 15) >> 2); }
    static __device__ __forceinline__ int value_row(int lane, int e) { return row_of(e, lane >> 4); }
    static __device__ __forceinline__ void load_key(Keys& k, int lane, const float* row) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) k.w[s] = *reinterpret_cast<const f32x4_t*>(row + 16 * s + 4 * (lane >> 4));
    }
    static __device__ __forceinline__ void load_keys(Keys& k, int lane, const float* tile0, const float*) {
        load_key(k, lane, tile0 + key_row(lane, 0) * D);
    }
    // e: which of the lane's rows
    static __device__ __forceinline__ void load_value(Values& v, int lane, int e, const float* row) {
#pragma unroll
        for (int i = 0; i < kVw / 4; ++i) v.w[e][i] = *reinterpret_cast<const f32x4_t*>(row + feature(lane & 15, 4 * i));
    }
    static __device__ __forceinline__ void load_values(Values& v, int lane, const float* tile0, const float*) {
#pragma unroll
        for (int e = 0; e < 4; ++e) load_value(v, lane, e, tile0 + value_row(lane, e) * D);
    }
    static __device__ __forceinline__ void put_key(Keys& k, int lane, int at, const float* row) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const f32x4_t w = *reinterpret_cast<const f32x4_t*>(row + 16 * s + 4 * (lane >> 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) k.w[s][i] = key_row(lane, 0) == at ? w[i] : k.w[s][i];
        }
    }
    static __device__ __forceinline__ void put_value(Values& v, int lane, int at, const float* row) {
#pragma unroll
        for (int i = 0; i < kVw / 4; ++i) {
            const f32x4_t w = *reinterpret_cast<const f32x4_t*>(row + feature(lane & 15, 4 * i));
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int x = 0; x < 4; ++x) v.w[e][i][x] = value_row(lane, e) == at ? w[x] : v.w[e][i][x];
        }
    }
    // value rows from n on are zeros (what lies there is nobody's)
    static __device__ __forceinline__ void clear_values(Values& v, int lane, int n) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (value_row(lane, e) >= n)
#pragma unroll
                for (int i = 0; i < kVw / 4; ++i) v.w[e][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    static __device__ __forceinline__ void clear_value(Values& v, int e) {
#pragma unroll
        for (int i = 0; i < kVw / 4; ++i) v.w[e][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void logits(const Keys& k, float scale2, float (&s)[kPerLane]) const {
        f32x4_t c[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};        // two chains of products
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.w[t][e], q[t][e], c[e & 1], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = (c[0][e] + c[1][e]) * scale2;
    }
    __device__ __forceinline__ void add_values(const Values& v, const float (&p)[kPerLane]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < kVw; ++t) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.w[e][t >> 2][t & 3], p[e], o[t], 0, 0, 0);
    }
    static __device__ __forceinline__ bool values_finite(const Values& v) {
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < kVw; ++i) bad |= (__float_as_uint(v.w[e][i >> 2][i & 3]) & 0x7f800000u) == 0x7f800000u;
        return !bad;
    }
};

// The running maximum takes a block's logits in: s becomes the weights, sums and outputs are brought to the new reference.  That
// follows the maximum when it has grown by more than a factor of 2^8 of the weights: until then they are at most 2^8, which
// floats hold as precisely as what is below one.
template <typename A>
__device__ __forceinline__ void take_logits(A& a, float (&s)[A::kPerLane]) {
    float top = s[0];
#pragma unroll
    for (int e = 1; e < A::kPerLane; ++e) top = fmaxf(top, s[e]);
    top = column_max(top);
    if (__any(top > a.m + 8.f)) {
        const float m_new = fmaxf(a.m, top);
        const float f = __builtin_amdgcn_exp2f(a.m - reference(m_new));
        a.l *= f;
#pragma unroll
        for (int t = 0; t < A::kVw; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) a.o[t][i] *= f;
        a.m = m_new;
    }
    const float ref = reference(a.m);
#pragma unroll
    for (int e = 0; e < A::kPerLane; ++e) {
        s[e] = __builtin_amdgcn_exp2f(s[e] - ref);
        a.l += s[e];
    }
}

// The second product of a block in which some columns do not see some rows.  A weight of zero keeps finite values out, but zero
// times infinity or NaN is NaN: with such values about, the rows are taken one at a time and the columns that do not see one keep
// what they had.  sees(row of the block): whether the lane's column does.
template <typename A, typename F>
__device__ __forceinline__ void add_masked_values(A& a, const typename A::Values& v, const float (&p)[A::kPerLane], int lane, F&& sees) {
    if (!__any(!A::values_finite(v))) {
        a.add_values(v, p);
        return;
    }
#pragma unroll 1
    for (int row = 0; row < 4 * A::kPerLane; ++row) {
        const int e = row % A::kPerLane;
        typename A::Values one = v;
        float pe[A::kPerLane];
#pragma unroll
        for (int f = 0; f < A::kPerLane; ++f) {
            pe[f] = f == e ? p[f] : 0.f;
            if (f != e || (lane >> 4) != row / A::kPerLane) A::clear_value(one, f);
        }
        f32x4_t before[A::kVw];
#pragma unroll
        for (int t = 0; t < A::kVw; ++t) before[t] = a.o[t];
        a.add_values(one, pe);
        const bool seen = sees(row_of(e, row / A::kPerLane));
#pragma unroll
        for (int t = 0; t < A::kVw; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) a.o[t][i] = seen ? a.o[t][i] : before[t][i];
    }
}

}  // namespace uncomp

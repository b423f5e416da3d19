// Causal attention over whole prompts: grouped heads, packed or padded sequences, queries that continue earlier keys.
// Query row i of a sequence of nq queries and nk keys sees the keys j <= nk - nq + i.  Softmax in base 2 with a running maximum
// and sum, one pass over the keys; the natural-log normalisers go out beside the rows.
//
// The G query heads of a KV head are columns of the same products: column c of a sequence is query c / G, head c % G, so that
// keys and values are fetched once for all of them and short prompts still fill the columns.
#include "common.h"
#include "attend_wave.h"

namespace uncomp {

namespace {

struct Seq {
    int64_t q0, k0;      // element offsets of the first query / key row (sequence stride included)
    int nq, nk;
};

__device__ __forceinline__ void rows_of(const AttnRows& r, int s, int* first, int* n) {
    int f = r.first != nullptr ? r.first[s] : 0;
    f = f < 0 ? 0 : (f > r.rows ? r.rows : f);
    int64_t m = r.len != nullptr ? (int64_t)r.len[s] : r.first != nullptr ? (int64_t)r.first[s + 1] - f : (int64_t)r.rows;
    m = m < 0 ? 0 : (m > r.rows - f ? r.rows - f : m);
    *first = f;
    *n = (int)m;
}

// Work item number `rank` of the tiles of all sequences, those with most keys first (a workgroup that starts late then has little
// to do; equal ones in order of their sequence).  A tile is `tile` columns; its keys are counted in blocks of 64.  The tiles of a
// sequence see ever more keys, so how many see at least x blocks is a subtraction, and x is found by bisection, 64 sequences at a time.
// Returns whether there is such a tile; called by whole waves, the same for all lanes.
struct Tile {
    int seq, tile, q_first, nq, k_first, nk;
};
__device__ __forceinline__ bool find_tile(const PrefillArgs& a, int tile, int64_t rank, Tile* out) {
    const int lane = threadIdx.x & 63;
    auto seq_of = [&](int s, int* qf, int* nq, int* kf, int* nk) {
        *qf = *nq = *kf = *nk = 0;
        if (s < a.n_seq) {
            rows_of(a.q, s, qf, nq);
            rows_of(a.k, s, kf, nk);
        }
    };
    auto tiles_of = [&](int nq) { return (nq * a.G + tile - 1) / tile; };
    // tiles of a sequence that see at least x blocks
    auto at_least = [&](int nq, int nk, int x) {
        const int n = tiles_of(nq);
        if (x <= 0) return n;
        const int need = 64 * (x - 1) + 1;                 // keys
        if (nk < need) return 0;
        const int row = need - (nk - nq);                  // the sequence's row that is the first to see them, counted from one
        const int first = row <= 1 ? 0 : (int)((int64_t)(row - 1) * a.G / tile);
        return first < n ? n - first : 0;
    };
    auto wave_total = [](int v) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        return v;
    };
    int qf, nq, kf, nk;
    if (a.n_seq <= 64) {
        seq_of(lane, &qf, &nq, &kf, &nk);
        const int n = tiles_of(nq);
        if (rank >= wave_total(n)) return false;
        int most = (nk + 63) / 64;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, 64));
        int lo = 0, hi = most + 1;                         // at least lo blocks: more than rank tiles; at least hi: not
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (wave_total(at_least(nq, nk, mid)) > rank) lo = mid;
            else hi = mid;
        }
        const int more = at_least(nq, nk, hi), with = at_least(nq, nk, lo) - more;
        int before = with;                                 // tiles of exactly lo blocks in the sequences up to this one
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(before, o, 64);
            if (lane >= o) before += u;
        }
        const int at = (int)rank - wave_total(more);
        const int x = __ffsll(__ballot(before > at)) - 1;
        out->tile = __shfl(n - more - before + at, x, 64);      // its tiles of lo blocks end where those of more begin
        out->seq = x;
        out->q_first = __shfl(qf, x, 64);
        out->nq = __shfl(nq, x, 64);
        out->k_first = __shfl(kf, x, 64);
        out->nk = __shfl(nk, x, 64);
        return true;
    }
    // many sequences: in their order
    for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
        seq_of(s0 + lane, &qf, &nq, &kf, &nk);
        const int n = tiles_of(nq);
        int sum = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(sum, o, 64);
            if (lane >= o) sum += u;
        }
        const unsigned long long has = __ballot(sum > rank);
        if (has != 0) {
            const int x = __ffsll(has) - 1;
            out->tile = __shfl(n - sum + (int)rank, x, 64);
            out->seq = s0 + x;
            out->q_first = __shfl(qf, x, 64);
            out->nq = __shfl(nq, x, 64);
            out->k_first = __shfl(kf, x, 64);
            out->nk = __shfl(nk, x, 64);
            return true;
        }
        rank -= __shfl(sum, 63, 64);
    }
    return false;
}

constexpr int kWaveCols = 64;      // columns of a workgroup of the wave kernel: sixteen a wave

}  // namespace

// Sixteen columns per wave, keys straight from memory.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_wave_kernel(PrefillArgs a) {
    using A = WaveAttend<T, D, sizeof(T) == 4>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4;
    const int G = a.G;
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);
    const int h = blockIdx.x % a.H;
    Tile w;
    if (!find_tile(a, kWaveCols, blockIdx.x / a.H, &w)) return;
    const int s = w.seq, q_first = w.q_first, nq = w.nq, k_first = w.k_first, nk = w.nk;
    const int off = nk - nq;
    const int c0 = w.tile * kWaveCols + 16 * wave, last_col = nq * G - 1;
    if (c0 > last_col) return;
    const int col = c0 + (lane & 15), cc = col > last_col ? last_col : col;
    const int qi = cc / G, head = h * G + cc % G;
    const int lim = off + qi;                                         // last key this column sees
    const int all = off + c0 / G;                                     // keys up to here are seen by every column
    const int end = min(nk, off + min(c0 + 15, last_col) / G + 1);
    const T* Q = static_cast<const T*>(a.Q) + s * a.q.ss + head * a.q.sh + (int64_t)(q_first + qi) * a.q.sr;
    const T* K = static_cast<const T*>(a.K) + s * a.k.ss + h * a.k.sh + (int64_t)k_first * a.k.sr;
    const T* V = static_cast<const T*>(a.V) + s * a.v.ss + h * a.v.sh + (int64_t)k_first * a.v.sr;
    A at;
    at.reset();
    at.load_query(Q, lane);
    for (int r0 = 0; r0 < end; r0 += A::kBlock) {
        typename A::Rows rows;
        float p[A::kPerLane];
        A::load(rows, lane, [&](int r) { return K + min(r0 + r, nk - 1) * a.k.sr; }, [&](int r) { return V + min(r0 + r, nk - 1) * a.v.sr; });
        at.logits(rows, scale2, p);
        if (r0 + A::kBlock - 1 <= all) {
            take_logits(at, p);
            at.add_values(rows, p);
        } else {
            A::clear_values(rows, lane, nk - r0);
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e)
                if (r0 + A::value_row(lane, e) > lim) p[e] = -INFINITY;
            take_logits(at, p);
            add_masked_values(at, rows, p, lane, [&](int r) { return r0 + r <= lim; });
        }
    }
    const float l = column_sum(at.l);
    if (col <= last_col) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* O = static_cast<T*>(a.out) + s * a.o.ss + head * a.o.sh + (int64_t)(q_first + qi) * a.o.sr;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = A::kVw * (4 * j + i);
            if constexpr (sizeof(T) == 2) {
                typedef __bf16 out_t __attribute__((ext_vector_type(A::kVw)));
                out_t v;
#pragma unroll
                for (int t2 = 0; t2 < A::kVw; ++t2) v[t2] = (__bf16)(at.o[t2][i] * inv);
                *reinterpret_cast<out_t*>(O + d) = v;
            } else {
#pragma unroll
                for (int t2 = 0; t2 < A::kVw; t2 += 4)
                    *reinterpret_cast<f32x4_t*>(O + d + t2) =
                        f32x4_t{at.o[t2][i] * inv, at.o[t2 + 1][i] * inv, at.o[t2 + 2][i] * inv, at.o[t2 + 3][i] * inv};
            }
        }
        if (a.lse != nullptr && j == 0)
            a.lse[s * a.lse_ss + head * a.lse_sh + q_first + qi] = l == 0.f ? -INFINITY : (at.m + log2f(l)) * kLn2A;
    }
}

// ---- bf16 tiles ------------------------------------------------------------------------------------------------------
// NW waves of 32 columns each over tiles of 64 keys that the workgroup stages through LDS (two buffers, one barrier a tile; the
// next tile's rows wait in registers, the one after is on its way).
//   S^T = K Q^T  (32 x 32 x 16): keys are rows, so a lane has one column and its softmax stays in the lane but for one exchange;
//                accumulator register r of half h = lane / 32 is key 8 (r / 4) + 4 h + r % 4 of a block of 32;
//   O^T = V^T P^T: sixteen keys a product, slots 4 h ... of both halves of eight: the weights are the operand as they lie, and
//                the values come out of LDS through the transposing read (lane i of sixteen fetches four features of key i / 4 and
//                receives four keys of feature i).
// Rows in LDS have their 16-byte pieces exchanged by a pattern of the row, so that sixteen rows at one piece (keys) and
// four rows at four pieces (values) both lie in different banks.
namespace {
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTileKeys = 64;

template <int D>
__device__ __forceinline__ int piece_swap(int row) {
    return D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
}
__device__ __forceinline__ s16x4_t read_transposed(const unsigned char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)p);
}
// rows of a sequence from `row` on, readable up to its last (zeros behind it)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const bf16_bits* first, int64_t stride, int row, int n, int D) {
    const int left = n - row;
    const int64_t bytes = left <= 0 ? 0 : ((int64_t)(left - 1) * stride + D) * 2;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_bits*>(first + (int64_t)row * stride), 0,
                                             bytes > 0x7fffffff ? 0x7fffffff : (int)bytes, 0x00027000);
}
}  // namespace

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void prefill_tile_kernel(PrefillArgs a) {
    constexpr int kThreads = 64 * NW, kCols = 32 * NW, kRowBytes = D * 2, kPieces = D / 8, kTileBytes = kTileKeys * kRowBytes;
    constexpr int kMine = kTileKeys * kPieces / kThreads, kSteps = D / 16, kBlocks = D / 32;
    __shared__ __align__(16) unsigned char lds[2][2][kTileBytes];        // [buffer][keys, values]
    __shared__ int not_finite[2];                                         // tile (from one) in the buffer whose values are not all finite
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, c = lane & 31;
    const int G = a.G, h = blockIdx.x % a.H;
    Tile w;
    if (!find_tile(a, kCols, blockIdx.x / a.H, &w)) return;
    const int nk = __builtin_amdgcn_readfirstlane(w.nk), nq = __builtin_amdgcn_readfirstlane(w.nq), s = __builtin_amdgcn_readfirstlane(w.seq);
    const int off = nk - nq, last_col = nq * G - 1;
    const int c_wg = __builtin_amdgcn_readfirstlane(w.tile) * kCols, c_wave = c_wg + 32 * wave;
    const int col = c_wave + c, cc = min(col, last_col);
    const int qi = cc / G, head = h * G + cc % G;
    const int lim = off + qi;                                             // last key the lane's column sees
    const int wave_end = min(nk, off + min(c_wave + 31, last_col) / G + 1);      // keys that any of the wave's columns sees
    const int wg_all = off + c_wg / G, wg_end = min(nk, off + min(c_wg + kCols - 1, last_col) / G + 1);
    const int n_tiles = wg_end <= 0 ? 0 : (wg_end + kTileKeys - 1) / kTileKeys;
    const int n_whole = wg_all < 0 ? 0 : min(nk, wg_all + 1) / kTileKeys;            // tiles that all columns see all of
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);
    const int q_first = __builtin_amdgcn_readfirstlane(w.q_first), k_first = __builtin_amdgcn_readfirstlane(w.k_first);
    const bf16_bits* Q = static_cast<const bf16_bits*>(a.Q) + s * a.q.ss + head * a.q.sh + (int64_t)(q_first + qi) * a.q.sr;
    const bf16_bits* K = static_cast<const bf16_bits*>(a.K) + s * a.k.ss + h * a.k.sh + (int64_t)k_first * a.k.sr;
    const bf16_bits* V = static_cast<const bf16_bits*>(a.V) + s * a.v.ss + h * a.v.sh + (int64_t)k_first * a.v.sr;

    bf16x8_t q[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) q[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(Q + 16 * i + 8 * half));

    // staging: pieces of 16 bytes, consecutive threads along a row
    u32x4_t kp[kMine], vp[kMine];
    int put[kMine], k_off[kMine], v_off[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int p = tid + i * kThreads, row = p / kPieces, piece = p % kPieces;
        put[i] = row * kRowBytes + (piece ^ piece_swap<D>(row)) * 16;
        k_off[i] = row * (int)a.k.sr * 2 + piece * 16;
        v_off[i] = row * (int)a.v.sr * 2 + piece * 16;
    }
    auto fetch_keys = [&](int tile) __attribute__((always_inline)) {
        const auto rows = rows_from(K, a.k.sr, tile * kTileKeys, nk, D);
#pragma unroll
        for (int i = 0; i < kMine; ++i) kp[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rows, k_off[i], 0, 0));
    };
    auto fetch_values = [&](int tile) __attribute__((always_inline)) {
        const auto rows = rows_from(V, a.v.sr, tile * kTileKeys, nk, D);
#pragma unroll
        for (int i = 0; i < kMine; ++i) vp[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rows, v_off[i], 0, 0));
    };
    auto stage_keys = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) *reinterpret_cast<u32x4_t*>(&lds[buf][0][put[i]]) = kp[i];
    };
    auto stage_values = [&](int buf, int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) *reinterpret_cast<u32x4_t*>(&lds[buf][1][put[i]]) = vp[i];
        if (tile >= n_whole) {                                            // only tiles that some column does not see all of ask for it
            bool bad = false;
#pragma unroll
            for (int i = 0; i < kMine; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) bad |= (vp[i][e] & 0x7f80u) == 0x7f80u || (vp[i][e] & 0x7f800000u) == 0x7f800000u;
            if (bad) not_finite[buf] = tile + 1;
        }
    };

    f32x16_t o[kBlocks], z[2];                                            // output; logits of two blocks of 32 keys
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) o[b] = f32x16_t{};
    float m = -INFINITY, l = 0.f;                                         // maximum of the unscaled logits; this half's share of the sum

    const int k_row = c * kRowBytes, k_swap = piece_swap<D>(c);
    const int i16 = lane & 15, v_row = 4 * half + (i16 >> 2);
    auto key_operand = [&](int buf, int b, int i) __attribute__((always_inline)) {
        const unsigned char* at = lds[buf][0] + 32 * b * kRowBytes + k_row + (((2 * i + half) ^ k_swap) << 4);
        return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at));
    };
    auto value_operand = [&](int buf, int st, int b) __attribute__((always_inline)) {                    // keys 16 st ... of the tile, features of block b
        s16x4_t v[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int piece = 4 * b + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1), row = v_row + 8 * x;
            v[x] = read_transposed(lds[buf][1] + (16 * st + row) * kRowBytes + (piece ^ piece_swap<D>(row)) * 16 + (i16 & 1) * 8);
        }
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto logits = [&](int buf, int b, f32x16_t& to) __attribute__((always_inline)) {
        to = f32x16_t{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_operand(buf, b, i), q[i], to, 0, 0, 0);
    };
    auto follow = [&](const f32x16_t& z) __attribute__((always_inline)) {
        float top = z[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, z[r]);
        const auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1]));
        // The reference follows the maximum when that has grown by more than a factor of 2^8 of the weights: until then they are
        // at most 2^8, which floats and bf16 hold as precisely as what is below one.
        if (__any(top > m + 8.f / scale2)) {
            const float m_new = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f((m - reference(m_new)) * scale2);
            l *= f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= f;
            m = m_new;
        }
    };
    auto weights = [&](const f32x16_t& z, bf16x8_t (&p)[2]) __attribute__((always_inline)) {
        const float ref = reference(m) * scale2;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(z[r], scale2, -ref));
            sum[r & 1] += e;
            p[r >> 3][r & 7] = (__bf16)e;
        }
        l += sum[0] + sum[1];
    };
    // what the column does not see among 32 keys from k0 on
    auto mask = [&](f32x16_t& z, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (k0 + 8 * (r >> 2) + 4 * half + (r & 3) > lim) z[r] = -INFINITY;
    };
    auto add_values = [&](int buf, int blk, const bf16x8_t (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_operand(buf, 2 * blk + st, b), p[st], o[b], 0, 0, 0);
    };
    // Zero times infinity or NaN is NaN: the keys are taken one at a time, and columns that do not see one keep what they had.
    auto add_values_one_by_one = [&](int buf, int blk, const bf16x8_t (&p)[2], int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll 1
            for (int k = 0; k < 16; ++k) {                                // key 16 st + k: half k / 4 % 2, slot k % 4 + 4 (k / 8)
                const int slot = (k & 3) + 4 * (k >> 3);
                const bool here = half == ((k >> 2) & 1), seen = k0 + 16 * st + k <= lim;
                u32x4_t one = __builtin_bit_cast(u32x4_t, p[st]), keep;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    keep[e] = here && (slot >> 1) == e ? ((slot & 1) ? 0xffff0000u : 0xffffu) : 0u;
                    one[e] &= keep[e];
                }
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    u32x4_t v = __builtin_bit_cast(u32x4_t, value_operand(buf, 2 * blk + st, b));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] &= keep[e];
                    const f32x16_t next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, one),
                                                                                   o[b], 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[b][r] = seen ? next[r] : o[b][r];
                }
            }
    };
    // One turn of the loop, in units of 32 keys: the outputs of a tile's two units, the weights of its second and of the next tile's
    // first, the logits of the next tile's two.  A unit's logits are made beside the weights of the one before and its maximum
    // beside the outputs of that one, so that the matrix cores and the vector unit have independent work.  All reads of a
    // tile's keys, and of its values, lie between two barriers: keys one tile ahead of the values.
    bf16x8_t p[2];
    auto turn = [&](auto BUF, auto MASKED, int tile) __attribute__((always_inline)) {
        constexpr int buf = decltype(BUF)::value;
        constexpr bool masked = decltype(MASKED)::value;
        __syncthreads();
        stage_keys(buf);                                                  // tile + 2
        fetch_keys(tile + 3);
        stage_values(buf ^ 1, tile + 1);
        fetch_values(tile + 2);
        const int k0 = tile * kTileKeys;
        if (masked && k0 >= wave_end) return;
        const bool odd_values = masked && not_finite[buf] == tile + 1;
        if (odd_values) add_values_one_by_one(buf, 0, p, k0);
        else add_values(buf, 0, p);
        if constexpr (masked) mask(z[1], k0 + 32);
        follow(z[1]);
        logits(buf ^ 1, 0, z[0]);
        weights(z[1], p);
        if (odd_values) add_values_one_by_one(buf, 1, p, k0 + 32);
        else add_values(buf, 1, p);
        if constexpr (masked) mask(z[0], k0 + 64);
        follow(z[0]);
        logits(buf ^ 1, 1, z[1]);
        weights(z[0], p);
    };

    if (n_tiles > 0) {
        using I0 = std::integral_constant<int, 0>;
        using I1 = std::integral_constant<int, 1>;
        if (tid < 2) not_finite[tid] = 0;
        __syncthreads();
        fetch_keys(0);
        fetch_values(0);
        stage_keys(0);
        stage_values(0, 0);
        fetch_keys(1);
        fetch_values(1);
        stage_keys(1);
        fetch_keys(2);
        __syncthreads();
        logits(0, 0, z[0]);
        mask(z[0], 0);
        follow(z[0]);
        logits(0, 1, z[1]);
        weights(z[0], p);
        int tile = 0;
        for (; tile + 2 < n_whole; tile += 2) {
            turn(I0{}, std::false_type{}, tile);
            turn(I1{}, std::false_type{}, tile + 1);
        }
        for (; tile < n_tiles; tile += 2) {
            turn(I0{}, std::true_type{}, tile);
            if (tile + 1 < n_tiles) turn(I1{}, std::true_type{}, tile + 1);
        }
    }
    const auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(other[0]) + __uint_as_float(other[1]);
    if (col <= last_col) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16_bits* O = static_cast<bf16_bits*>(a.out) + s * a.o.ss + head * a.o.sh + (int64_t)(q_first + qi) * a.o.sr;
        typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                bf16x4_t v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[b][r + e] * inv);
                *reinterpret_cast<bf16x4_t*>(O + 32 * b + 2 * r + 4 * half) = v;
            }
        if (a.lse != nullptr && half == 0)
            a.lse[s * a.lse_ss + head * a.lse_sh + q_first + qi] = l == 0.f ? -INFINITY : (m * scale2 + log2f(l)) * kLn2A;
    }
}

size_t prefill_attention_bytes(int, int, int, int, int, int) { return 0; }

namespace {
// most tiles that the sequences can have: whole ones, and one broken one each
int64_t most_tiles(const PrefillArgs& a, int tile) {
    const int64_t cols = (int64_t)a.q.rows * a.G;
    return a.q.first != nullptr ? cols / tile + a.n_seq : (cols + tile - 1) / tile * a.n_seq;
}
template <int D, int NW>
hipError_t prefill_tiles(const PrefillArgs& a, const Env& env) {
    env.begin("prefill_tile");
    prefill_tile_kernel<D, NW><<<(unsigned)(most_tiles(a, 32 * NW) * a.H), 64 * NW, 0, env.s>>>(a);
    env.end();
    return hipGetLastError();
}
template <typename T, int D>
hipError_t prefill_of(const PrefillArgs& a, const Env& env) {
    if constexpr (sizeof(T) == 2) {
        const bool near = a.k.sr < 1 << 22 && a.v.sr < 1 << 22;      // 64 rows span less than 2 GiB
        if (near && !env.force_alu) return prefill_tiles<D, 8>(a, env);
    }
    const int64_t grid = most_tiles(a, kWaveCols) * a.H;
    env.begin("prefill_wave");
    prefill_wave_kernel<T, D><<<(unsigned)grid, 256, 0, env.s>>>(a);
    env.end();
    return hipGetLastError();
}
}  // namespace

hipError_t launch_prefill_attention(const PrefillArgs& a, uncomp_dtype dt, int D, char*, size_t, const Env& env) {
    if (dt == UNCOMP_BF16) return D == 128 ? prefill_of<bf16_bits, 128>(a, env) : prefill_of<bf16_bits, 64>(a, env);
    return D == 128 ? prefill_of<float, 128>(a, env) : prefill_of<float, 64>(a, env);
}

}  // namespace uncomp

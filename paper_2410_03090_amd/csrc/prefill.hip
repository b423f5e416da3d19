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
// Returns whether there is such a tile; called by whole waves, the same for all lanes.  blocks: those of all tiles (a tile sees
// about the mean of its sequence's first and last), 0 with more than 64 sequences, which are taken in their order.
constexpr int kRanked = 64;
struct Tile {
    int seq, tile, q_first, nq, k_first, nk;
    int64_t blocks;
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
    auto wave_total = [](auto v) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        return v;
    };
    int qf, nq, kf, nk;
    out->blocks = 0;
    if (a.n_seq == 1) {                                    // nothing to look for: its last tile sees most
        seq_of(0, &qf, &nq, &kf, &nk);
        const int n = tiles_of(nq), first = max(0, min(nk, nk - nq + (tile - 1) / a.G + 1));
        *out = Tile{0, n - 1 - (int)rank, qf, nq, kf, nk, n * ((int64_t)first + nk) / 128};
        return rank < n;
    }
    if (a.n_seq <= kRanked) {
        seq_of(lane, &qf, &nq, &kf, &nk);
        const int n = tiles_of(nq);
        if (rank >= wave_total(n)) return false;
        if (a.n_split > 1) {
            const int first = max(0, min(nk, nk - nq + (tile - 1) / a.G + 1));
            out->blocks = wave_total(n * ((int64_t)first + nk) / 128);
        }
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
    // many sequences: in their order, found among the sums of their tiles, 64 places of a range at a time
    int begin = 0, n = a.n_seq;                                           // the sequence is one of these
    if (rank >= a.sums[n - 1]) return false;
    while (n > 1) {
        const int step = (n + 63) / 64, end = min((lane + 1) * step, n);
        const int x = __ffsll(__ballot(a.sums[begin + end - 1] > rank)) - 1;
        begin += x * step;
        n = min(step, n - x * step);
    }
    rows_of(a.q, begin, &qf, &nq);
    rows_of(a.k, begin, &kf, &nk);
    const int64_t sum = a.sums[begin];
    *out = Tile{begin, tiles_of(nq) - (int)(sum - rank), qf, nq, kf, nk, 0};
    return true;
}

constexpr int kWaveCols = 64;      // columns of a workgroup of the fp32 kernel: sixteen a wave

// What a tile of columns sees, and the part of it that one workgroup takes.  Where few tiles, or a few long ones, would leave much of
// the chip idle, tiles are cut into parts of whole blocks of 64 keys, each about the target-th of all blocks but no fewer than
// kLeastBlocks: a part leaves its outputs in fp32, and joining them takes as long as about that many blocks (fp32: two).  One layer of 8
// KV heads, 4 query heads each, uncut and cut (us): 1 query on 20000 keys 387 / 42, 64 on 8000 203 / 49, 512 on 16000 399 / 150, a prompt of
// 3000 101 / 99.
// Key numbers below are counted from the part's first.
constexpr int kLeastBlocks = 12, kLeastBlocksF32 = 2;
__host__ __device__ inline int parts_of(int64_t blocks, int64_t all_blocks, int target, int least, int most) {
    int64_t share = (all_blocks + target - 1) / target;
    share = share < least ? least : share;
    const int64_t n = (blocks + share / 2) / share;                       // to the nearest: not a second round for a little more than a share
    return n < 1 ? 1 : n > most ? most : (int)n;
}
struct Part {
    int s, h, q_first, nq, last_col, c0;     // sequence, KV head, its rows, last column, the tile's first
    int shift, keys;                         // first key of the part (of the sequence's), keys in it
    int off;                                 // column of row i sees keys up to off + i
    int n_parts;
};
// Workgroups are numbered by head first (eight KV heads are one per XCD, whose L2 then holds that head's rows alone), then by
// tile, then by part, the last part first: what is cut starts before the short tiles, and those without a part are on every XCD.
__device__ __forceinline__ bool find_part(const PrefillArgs& a, int tile, Part* p, int item, int part) {
    const int h = item % a.H;
    Tile w;
    if (!find_tile(a, tile, item / a.H, &w)) return false;
    const auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int nk = uniform(w.nk), nq = uniform(w.nq);
    p->s = uniform(w.seq);
    p->h = h;
    p->q_first = uniform(w.q_first);
    p->nq = nq;
    p->last_col = nq * a.G - 1;
    p->c0 = uniform(w.tile) * tile;
    const int off = nk - nq, seen = min(nk, off + min(p->c0 + tile - 1, p->last_col) / a.G + 1);
    const int blocks = seen <= 0 ? 0 : (seen + 63) / 64;
    const int n = a.n_split == 1 ? 1 : parts_of(blocks, w.blocks * a.H, a.target, a.least, a.n_split);
    const int per = (blocks + n - 1) / n;
    p->n_parts = per == 0 ? 1 : (blocks + per - 1) / per;
    p->shift = min(part * per, blocks) * 64;
    p->keys = min(min(per, blocks - p->shift / 64) * 64, nk - p->shift);
    p->off = off - p->shift;
    p->shift += uniform(w.k_first);
    return part < p->n_parts;
}
__device__ __forceinline__ bool find_part(const PrefillArgs& a, int tile, Part* p) {
    return find_part(a, tile, p, blockIdx.x % a.items, a.n_split - 1 - blockIdx.x / a.items);
}
// where a part's unnormalised outputs and (maximum in base 2, sum) go
__device__ __forceinline__ int64_t part_row(const PrefillArgs& a, int tile, int col) {
    return ((int64_t)a.n_split * a.items - a.items - blockIdx.x + 2 * (blockIdx.x % a.items)) * tile + col;      // [part][item][column]
}

}  // namespace

// Sums of the sequences' tiles, for many of them.  One workgroup, a run of sequences a thread.
__global__ __launch_bounds__(1024) void prefill_sums_kernel(AttnRows q, int n_seq, int G, int tile, int64_t* __restrict__ sums) {
    __shared__ int64_t wave_s[16];
    const int tid = threadIdx.x, lane = tid & 63, run = (n_seq + 1023) / 1024, begin = min(n_seq, tid * run), end = min(n_seq, begin + run);
    const auto tiles = [&](int s) {
        int first, n;
        rows_of(q, s, &first, &n);
        return (n * G + tile - 1) / tile;
    };
    int64_t mine = 0;
    for (int s = begin; s < end; ++s) mine += tiles(s);
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(sum, o, 64);
        if (lane >= o) sum += u;
    }
    if (lane == 63) wave_s[tid >> 6] = sum;
    __syncthreads();
    sum -= mine;
    for (int x = 0; x < tid >> 6; ++x) sum += wave_s[x];
    for (int s = begin; s < end; ++s) {
        sum += tiles(s);
        sums[s] = sum;
    }
}

// ---- fp32 ------------------------------------------------------------------------------------------------------------
// Sixteen columns per wave, rows straight from memory into the operands: the fp32 matrix cores take 2048 cycles for sixteen rows of
// 128 features, which no fetch through the caches outlasts.  The next block's keys are on their way from the moment this one's
// logits are there, the values from the block's start.
template <int D>
__global__ __launch_bounds__(256) void prefill_f32_kernel(PrefillArgs a) {
    using A = WaveAttend<float, D>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4;
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);
    Part w;
    if (!find_part(a, kWaveCols, &w)) return;
    const int c0 = w.c0 + 16 * wave;
    if (c0 > w.last_col) return;
    const int col = c0 + (lane & 15), cc = min(col, w.last_col);
    const int qi = cc / a.G, head = w.h * a.G + cc % a.G;
    const int lim = min(w.off + qi, w.keys - 1);                          // last key the lane's column sees
    const int all = min(w.off + c0 / a.G, w.keys - 1);                    // keys up to here are seen by every column
    const int end = min(w.off + min(c0 + 15, w.last_col) / a.G + 1, w.keys);
    const float* Q = static_cast<const float*>(a.Q) + w.s * a.q.ss + head * a.q.sh + (int64_t)(w.q_first + qi) * a.q.sr;
    const float* K = static_cast<const float*>(a.K) + w.s * a.k.ss + w.h * a.k.sh + (int64_t)w.shift * a.k.sr;
    const float* V = static_cast<const float*>(a.V) + w.s * a.v.ss + w.h * a.v.sh + (int64_t)w.shift * a.v.sr;
    A at;
    at.reset();
    at.load_query(Q, lane);
    typename A::Keys keys;
    typename A::Values values;
    // a block's first row is uniform, the lane's rows 32-bit offsets from there; behind the last row that one is read again
    const int k_row = A::key_row(lane, 0), k_at = k_row * (int)a.k.sr;
    int v_at[A::kPerLane];
#pragma unroll
    for (int e = 0; e < A::kPerLane; ++e) v_at[e] = A::value_row(lane, e) * (int)a.v.sr;
    const auto fetch_keys = [&](int r0) __attribute__((always_inline)) {
        const float* first = K + (int64_t)min(r0, w.keys - 1) * a.k.sr;
        if (r0 + A::kBlock <= w.keys) A::load_key(keys, lane, first + k_at);
        else A::load_key(keys, lane, first + max(0, min(k_row, w.keys - 1 - r0)) * (int)a.k.sr);
    };
    const auto fetch_values = [&](int r0) __attribute__((always_inline)) {
        const float* first = V + (int64_t)r0 * a.v.sr;
        if (r0 + A::kBlock <= w.keys)
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e) A::load_value(values, lane, e, first + v_at[e]);
        else
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e) A::load_value(values, lane, e, first + min(A::value_row(lane, e), w.keys - 1 - r0) * (int)a.v.sr);
    };
    if (end > 0) fetch_keys(0);
    for (int r0 = 0; r0 < end; r0 += A::kBlock) {
        fetch_values(r0);
        float p[A::kPerLane];
        at.logits(keys, scale2, p);
        fetch_keys(r0 + A::kBlock);
        if (r0 + A::kBlock - 1 <= all) {
            take_logits(at, p);
            at.add_values(values, p);
        } else {
            A::clear_values(values, lane, w.keys - r0);
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e)
                if (r0 + A::value_row(lane, e) > lim) p[e] = -INFINITY;
            take_logits(at, p);
            add_masked_values(at, values, p, lane, [&](int r) { return r0 + r <= lim; });
        }
    }
    const float l = column_sum(at.l);
    if (col > w.last_col) return;
    if (w.n_parts > 1) {
        const int64_t row = part_row(a, kWaveCols, col - w.c0);
        float* acc = a.part_acc + row * D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < A::kVw; t += 4)
                *reinterpret_cast<f32x4_t*>(acc + A::feature(4 * j + i, t)) = f32x4_t{at.o[t][i], at.o[t + 1][i], at.o[t + 2][i], at.o[t + 3][i]};
        if (j == 0) a.part_ml[row] = make_float2(at.m, l);
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    float* O = static_cast<float*>(a.out) + w.s * a.o.ss + head * a.o.sh + (int64_t)(w.q_first + qi) * a.o.sr;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < A::kVw; t += 4)
            *reinterpret_cast<f32x4_t*>(O + A::feature(4 * j + i, t)) =
                f32x4_t{at.o[t][i] * inv, at.o[t + 1][i] * inv, at.o[t + 2][i] * inv, at.o[t + 3][i] * inv};
    if (a.lse != nullptr && j == 0)
        a.lse[w.s * a.lse_ss + head * a.lse_sh + w.q_first + qi] = l == 0.f ? -INFINITY : (at.m + log2f(l)) * kLn2A;
}

// Joins the parts of a tile's columns, sixteen columns a workgroup, four features a lane.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_join_kernel(PrefillArgs a, int tile) {
    constexpr int kLanes = D / 4, kPer = 256 / kLanes;
    const int groups = tile / 16, item = blockIdx.x / groups;
    Part w;
    if (!find_part(a, tile, &w, item, 0) || w.n_parts == 1) return;
    for (int i = threadIdx.x / kLanes; i < 16; i += kPer) {
        const int in_tile = (blockIdx.x % groups) * 16 + i, col = w.c0 + in_tile, d = (threadIdx.x % kLanes) * 4;
        if (col > w.last_col) continue;
        const int64_t row = (int64_t)item * tile + in_tile, next = (int64_t)a.items * tile;
        float m = -INFINITY;
        for (int p = 0; p < w.n_parts; ++p) m = fmaxf(m, a.part_ml[row + p * next].x);
        float l = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < w.n_parts; ++p) {
            const float2 ml = a.part_ml[row + p * next];
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.part_acc + (row + p * next) * D + d);
            const float f = __builtin_amdgcn_exp2f(ml.x - reference(m));
            l = fmaf(f, ml.y, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = ml.y == 0.f ? o[e] : fmaf(f, v[e], o[e]);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int qi = col / a.G, head = w.h * a.G + col % a.G;
        T* O = static_cast<T*>(a.out) + w.s * a.o.ss + head * a.o.sh + (int64_t)(w.q_first + qi) * a.o.sr + d;
        if constexpr (sizeof(T) == 2) {
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            *reinterpret_cast<bf16x4_t*>(O) = bf16x4_t{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
        } else {
            *reinterpret_cast<f32x4_t*>(O) = o * inv;
        }
        if (a.lse != nullptr && d == 0)
            a.lse[w.s * a.lse_ss + head * a.lse_sh + w.q_first + qi] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2A;
    }
}

// ---- bf16 tiles ------------------------------------------------------------------------------------------------------
// NW waves of 32 columns each over tiles of 64 keys that the workgroup stages through LDS (two buffers, one barrier a tile; its keys
// are on their way two turns ahead, its values one).
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
// 16 bytes a lane from `offset` into LDS, behind one another from `to` on (uniform).  (The host's compiler does not know the size.)
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t rows, unsigned char* to, int offset) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
#endif
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
__global__ __launch_bounds__(64 * NW, D == 64 ? 3 : 2) void prefill_tile_kernel(PrefillArgs a) {
    constexpr int kThreads = 64 * NW, kCols = 32 * NW, kRowBytes = D * 2, kPieces = D / 8, kTileBytes = kTileKeys * kRowBytes;
    constexpr int kMine = kTileKeys * kPieces / kThreads, kSteps = D / 16, kBlocks = D / 32;
    // two buffers each, by names of their own: the compiler waits for loads that are on their way to a buffer before reads of that one only
    __shared__ __align__(16) unsigned char keys0[kTileBytes], keys1[kTileBytes], values0[kTileBytes], values1[kTileBytes];
    __shared__ int not_finite[2];                                         // tile (from one) in the buffer whose values are not all finite
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, c = lane & 31;
    const int G = a.G;
    Part w;
    if (!find_part(a, kCols, &w)) return;
    const int c_wave = w.c0 + 32 * wave, col = c_wave + c, cc = min(col, w.last_col);
    const int qi = cc / G, head = w.h * G + cc % G, nk = w.keys;
    const int lim = min(w.off + qi, nk - 1);                              // last key the lane's column sees
    const int wave_end = min(nk, w.off + min(c_wave + 31, w.last_col) / G + 1);      // keys that any of the wave's columns sees
    const int wg_all = min(w.off + w.c0 / G, nk - 1);
    const int n_tiles = nk <= 0 ? 0 : (nk + kTileKeys - 1) / kTileKeys;
    const int n_whole = wg_all < 0 ? 0 : (wg_all + 1) / kTileKeys;        // tiles that all columns see all of
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);
    const bf16_bits* Q = static_cast<const bf16_bits*>(a.Q) + w.s * a.q.ss + head * a.q.sh + (int64_t)(w.q_first + qi) * a.q.sr;
    const bf16_bits* K = static_cast<const bf16_bits*>(a.K) + w.s * a.k.ss + w.h * a.k.sh + (int64_t)w.shift * a.k.sr;
    const bf16_bits* V = static_cast<const bf16_bits*>(a.V) + w.s * a.v.ss + w.h * a.v.sh + (int64_t)w.shift * a.v.sr;

    bf16x8_t q[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) q[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(Q + 16 * i + 8 * half));

    // staging: pieces of 16 bytes straight into LDS, 64 behind one another by a wave's instruction; which piece of a row goes where is
    // decided by what each lane fetches
    int k_off[kMine], v_off[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int p = tid + i * kThreads, row = p / kPieces, piece = (p % kPieces) ^ piece_swap<D>(row);
        k_off[i] = row * (int)a.k.sr * 2 + piece * 16;
        v_off[i] = row * (int)a.v.sr * 2 + piece * 16;
    }
    auto stage_keys = [&](int buf, int tile) __attribute__((always_inline)) {
        const auto rows = rows_from(K, a.k.sr, tile * kTileKeys, nk, D);
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            load_to_lds(rows, &(buf ? keys1 : keys0)[(i * kThreads + wave * 64) * 16], k_off[i]);
    };
    auto stage_values = [&](int buf, int tile) __attribute__((always_inline)) {
        const auto rows = rows_from(V, a.v.sr, tile * kTileKeys, nk, D);
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            load_to_lds(rows, &(buf ? values1 : values0)[(i * kThreads + wave * 64) * 16], v_off[i]);
    };
    // whether a tile's values are all finite: asked where some column does not see all of it
    auto check_values = [&](int buf, int tile) __attribute__((always_inline)) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(&(buf ? values1 : values0)[(i * kThreads + tid) * 16]);
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= (v[e] & 0x7f80u) == 0x7f80u || (v[e] & 0x7f800000u) == 0x7f800000u;
        }
        if (bad) not_finite[buf] = tile + 1;
    };

    f32x16_t o[kBlocks], z[2];                                            // output; logits of two blocks of 32 keys
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) o[b] = f32x16_t{};
    float m = -INFINITY, l = 0.f;                                         // maximum of the unscaled logits; this half's share of the sum

    const int k_row = c * kRowBytes, k_swap = piece_swap<D>(c);
    const int i16 = lane & 15, v_row = 4 * half + (i16 >> 2);
    auto key_operand = [&](int buf, int b, int i) __attribute__((always_inline)) {
        const unsigned char* at = (buf ? keys1 : keys0) + 32 * b * kRowBytes + k_row + (((2 * i + half) ^ k_swap) << 4);
        return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at));
    };
    auto value_operand = [&](int buf, int st, int b) __attribute__((always_inline)) {                    // keys 16 st ... of the tile, features of block b
        s16x4_t v[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int piece = 4 * b + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1), row = v_row + 8 * x;
            v[x] = read_transposed((buf ? values1 : values0) + (16 * st + row) * kRowBytes + (piece ^ piece_swap<D>(row)) * 16 + (i16 & 1) * 8);
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
    // The weights are rounded to bf16, the width of the values that they multiply: half a step is 2^-8 of a weight, as much as the rounding of the result
    // is of that, and the roundings of many keys mostly cancel.  (Relative error against 64 bits, 8192 rows: 0.0020, of which the result's own rounding
    // is 0.0016.  Three bf16 a weight, as the paged step has, would double the matrix instructions.)  Their sum is that of the unrounded ones.
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
    auto arrived = [&]() __attribute__((always_inline)) {                 // what all waves have asked for is in LDS
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    bf16x8_t p[2];
    auto turn = [&](auto BUF, auto MASKED, int tile) __attribute__((always_inline)) {
        constexpr int buf = decltype(BUF)::value;
        constexpr bool masked = decltype(MASKED)::value;
        arrived();
        stage_keys(buf, tile + 2);
        stage_values(buf ^ 1, tile + 1);
        if constexpr (masked) {
            check_values(buf, tile);
            __syncthreads();
        }
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
        stage_keys(0, 0);
        stage_values(0, 0);
        stage_keys(1, 1);
        arrived();
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
    if (w.n_parts > 1) {
        if (col > w.last_col) return;
        const int64_t row = part_row(a, kCols, col - w.c0);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4_t*>(a.part_acc + row * D + 32 * b + 2 * r + 4 * half) = f32x4_t{o[b][r], o[b][r + 1], o[b][r + 2], o[b][r + 3]};
        if (half == 0) a.part_ml[row] = make_float2(m * scale2, l);
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (a.lse != nullptr && half == 0 && col <= w.last_col)
        a.lse[w.s * a.lse_ss + head * a.lse_sh + w.q_first + qi] = l == 0.f ? -INFINITY : (m * scale2 + log2f(l)) * kLn2A;
    // a lane's four features are eight bytes: whole rows are put together in the buffers, a wave's 32 in a part of its own
    arrived();
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    constexpr int kFit = kTileBytes / (32 * kRowBytes);
    unsigned char* mine = (wave / kFit == 0 ? keys0 : wave / kFit == 1 ? keys1 : wave / kFit == 2 ? values0 : values1) + wave % kFit * 32 * kRowBytes;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            bf16x4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[b][r + e] * inv);
            *reinterpret_cast<bf16x4_t*>(mine + c * kRowBytes + ((4 * b + r / 4) ^ (c & (kPieces - 1))) * 16 + 8 * half) = v;
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    bf16_bits* O = static_cast<bf16_bits*>(a.out) + w.s * a.o.ss + (int64_t)w.q_first * a.o.sr;
    const int64_t to = head * a.o.sh + qi * a.o.sr;
#pragma unroll
    for (int i = 0; i < kPieces / 2; ++i) {
        const int row = i * (64 / kPieces) + lane / kPieces, piece = lane % kPieces;
        const int64_t at = __shfl(to, row);
        if (c_wave + row <= w.last_col)
            *reinterpret_cast<u32x4_t*>(O + at + 8 * piece) = *reinterpret_cast<const u32x4_t*>(mine + row * kRowBytes + (piece ^ (row & (kPieces - 1))) * 16);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
namespace {
struct Plan {
    int tile;            // columns of a workgroup
    int n_split, target, least;
    int64_t items;       // tiles of all KV heads, at most
    size_t acc_off, bytes;
};
// 64-wide heads take tiles of 128 columns, three workgroups a CU: as much work for the vector unit comes with half the products, and
// several that do not wait for each other fill it better.  8 KV heads of 4 query heads, us, of 8192 rows: one workgroup of 256 columns a CU 357, two of
// 128 347, three 322 (of 1024 rows 28.5, 22.3 and 23).  Three leave a wave 168 registers: 11 more wait in scratch memory outside the loop.
// 128-wide ones take tiles of 256, which read keys and values half as often, unless a sequence has not as many columns, or its keys are soon
// through (what comes before and after them then counts, and another workgroup fills it), or they would not fill the chip.  256 / 128, us, 8
// KV heads of 4 query heads: 16 sequences of 1 query on 20000 keys 341 / 199, 256 prompts of 128 rows 280 / 248, 32 of 1024 455 / 444, 1 of 1024
// 35.6 / 29.0, 1 of 2048 66.5 / 67.6, 32 of 2048 1354 / 1408, 4 times 512 on 16000 484 / 519; of 1 query head, 1 of 4096 98 / 70, 4 of 4096 152 / 166.
constexpr int kShortKeys = 1536;
int tile_of(bool f32, bool q_packed, bool k_packed, int n_seq, int H, int G, int D, int q_rows, int k_rows) {
    if (f32) return kWaveCols;
    const int64_t cols = (int64_t)q_rows * G / (q_packed ? n_seq : 1), keys = k_rows / (k_packed ? n_seq : 1);      // of a sequence, on the average
    const int64_t tiles = (cols + 255) / 256 * n_seq * H;
    return D == 64 || cols <= 128 || keys <= kShortKeys || (tiles < 256 && keys < 2 * cols / G) ? 128 : 256;
}
Plan plan(int tile, bool packed, int n_seq, int H, int G, int D, int q_rows, int k_rows) {
    const int64_t cols = (int64_t)q_rows * G;
    Plan p;
    p.tile = tile;
    const bool f32 = tile == kWaveCols;
    p.target = tile == 256 ? 256 : f32 || D == 128 ? 512 : 768;                       // workgroups that run at a time
    p.least = f32 ? kLeastBlocksF32 : kLeastBlocks;
    // most tiles that the sequences can have: whole ones, and one broken one each
    p.items = (packed ? cols / p.tile + n_seq : (cols + p.tile - 1) / p.tile * n_seq) * H;
    // as if the rows were one sequence's; how they are divided only the device knows
    const int64_t most = ((int64_t)k_rows + 63) / 64, first = (k_rows > q_rows ? (int64_t)k_rows - q_rows : 0) / 64;
    p.n_split = n_seq > kRanked ? 1 : parts_of(most, p.items * (first + most + 1) / 2, p.target, p.least, 64);
    p.acc_off = align_up((size_t)p.items * p.n_split * p.tile * sizeof(float2), 256);
    p.bytes = n_seq > kRanked ? (size_t)n_seq * sizeof(int64_t) : p.n_split == 1 ? 0 : p.acc_off + (size_t)p.items * p.n_split * p.tile * D * sizeof(float);
    return p;
}
Plan plan(const PrefillArgs& a, bool f32, int D) {
    // starts alone do not make sequences share the rows: with a stride between them each may have all of q_rows (left-padded batches)
    const bool packed = a.q.first != nullptr && a.q.ss == 0 && a.o.ss == 0, k_packed = a.k.first != nullptr && a.k.ss == 0 && a.v.ss == 0;
    return plan(tile_of(f32, packed, k_packed, a.n_seq, a.H, a.G, D, a.q.rows, a.k.rows), packed, a.n_seq, a.H, a.G, D, a.q.rows, a.k.rows);
}
}  // namespace

size_t prefill_attention_bytes(int n_seq, int H, int G, int D, int q_rows, int k_rows) {
    size_t most = 0;
    for (int tile : {kWaveCols, 128, 256})
        for (bool packed : {false, true}) {
            const size_t b = plan(tile, packed, n_seq, H, G, D, q_rows, k_rows).bytes;
            most = b > most ? b : most;
        }
    return most;
}

bool prefill_attention_fits(const PrefillArgs& a, uncomp_dtype dt, int D) { return plan(a, dt == UNCOMP_F32, D).items * 512 <= 0xffffffffLL; }
size_t prefill_attention_takes(const PrefillArgs& a, uncomp_dtype dt, int D, size_t ws_bytes) {
    const size_t bytes = plan(a, dt == UNCOMP_F32, D).bytes;
    return a.n_seq > kRanked || bytes <= ws_bytes ? bytes : 0;           // (no room for parts: whole tiles)
}

namespace {
template <int D>
hipError_t prefill_of(PrefillArgs a, bool f32, char* ws, size_t ws_bytes, const Env& env) {
    Plan p = plan(a, f32, D);
    if (p.bytes > ws_bytes) p.n_split = 1;                               // no room for parts: whole tiles
    if (a.n_seq > kRanked) {
        a.sums = reinterpret_cast<int64_t*>(ws);
        env.begin("prefill_sums");
        prefill_sums_kernel<<<1, 1024, 0, env.s>>>(a.q, a.n_seq, a.G, p.tile, a.sums);
        env.end();
    }
    a.n_split = p.n_split;
    a.target = p.target;
    a.least = p.least;
    a.items = (unsigned)p.items;
    a.part_ml = reinterpret_cast<float2*>(ws);
    a.part_acc = reinterpret_cast<float*>(ws + p.acc_off);
    const unsigned grid = (unsigned)(p.items * p.n_split);
    if (f32) {
        env.begin("prefill_f32");
        prefill_f32_kernel<D><<<grid, 256, 0, env.s>>>(a);
        env.end();
    } else {
        env.begin("prefill_tile");
        if (p.tile == 128) prefill_tile_kernel<D, 4><<<grid, 256, 0, env.s>>>(a);
        else if constexpr (D == 128) prefill_tile_kernel<D, 8><<<grid, 512, 0, env.s>>>(a);
        env.end();
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_split == 1) return e;
    env.begin("prefill_join");
    if (f32) prefill_join_kernel<float, D><<<(unsigned)(p.items * p.tile / 16), 256, 0, env.s>>>(a, p.tile);
    else prefill_join_kernel<bf16_bits, D><<<(unsigned)(p.items * p.tile / 16), 256, 0, env.s>>>(a, p.tile);
    env.end();
    return hipGetLastError();
}
}  // namespace

hipError_t launch_prefill_attention(const PrefillArgs& a, uncomp_dtype dt, int D, char* ws, size_t ws_bytes, const Env& env) {
    return D == 128 ? prefill_of<128>(a, dt == UNCOMP_F32, ws, ws_bytes, env) : prefill_of<64>(a, dt == UNCOMP_F32, ws, ws_bytes, env);
}

}  // namespace uncomp

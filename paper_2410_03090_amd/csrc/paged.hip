// The paged cache: rows of every KV head live in pages of a common pool, named by the head's own table, so that heads with
// different budgets hold what they need.  Row r of head h is row r % page of page table[h][r / page].
//
//   append   rows of dense caches join (paged_reserve_kernel: how many fit; paged_copy_kernel)
//   step     one new token joins, its queries attend over the rows, weights accumulate (paged_head_kernel: a head by one workgroup;
//            paged_attend_kernel, paged_finish_kernel: in parts; paged_list_kernel: which heads, where there are both)
//   evict    the rows of least accumulated weight leave (paged_select_wave_kernel, paged_select_kernel with paged_key_kernel for long
//            tables, paged_move_kernel)
#include "common.h"
#include "attend_wave.h"

namespace uncomp {

namespace {

constexpr int kAttendThreads = 256, kAttendWaves = kAttendThreads / 64;
constexpr int kFinishThreads = 256, kFinishRows = 1024;
constexpr int kFinishWgs = 8192;                      // about the most workgroups for rows, whatever room the tables have
constexpr int kSplitAim = 768;                        // workgroups of the attention of few heads: three a CU
constexpr int kLeastShare = 128;                      // rows of a workgroup, at least: a block a wave
// One workgroup a head, with logits that leave room for two workgroups on a CU, takes about 8 us and 1 more for every 125 rows, whatever the
// number of heads; parts of heads and their join 12 and 1 for every 15500 rows of all heads.  One workgroup / parts, us, heads of G 4, tables
// full to three quarters on the average: 8 heads of 300 rows 8.4 / 11.9, of 700 11.1 / 11.9, of 1016 13.6 / 12.0, of 2736 29 / 13; 48 of 1016
// 14.2 / 15.0; 110 of 2736 31.4 / 30.9; 256 of 300 9.8 / 19.1, of 2736 49 / 57; 500 of 2736 109 / 136.  A row of floats takes twice as long: 48
// heads of 700 21.9 / 16.6, 256 of 1000 37.8 / 46.3.
constexpr int kHeadsWorth = 124, kRowsWorth = 80000;
// Where tables of many heads have room for more rows than LDS, the heads that hold few enough for three workgroups take the one form and the rest
// the other.  All heads in parts / so, us, heads of G 4 with tables for 8192 and 20480 rows: 600 of 350 - 700 rows 72 / 45, 5120 of them
// 641 / 293, 600 of 1500 - 3000 181 / 165, 600 of 3000 - 6000 (a few of them short) 327 / 415, 600 of 10000 - 20000 1012 / 1042.
constexpr int kManyHeads = 512;
constexpr size_t kHeadLaunchLds = 76 * 1024, kShortHeadLds = 50 * 1024;
constexpr int kSelectThreads = 1024, kSelectKeys = 32768;                        // threads of a selection, keys that it holds in LDS
constexpr int kWaveSelectHeads = 512, kWaveSelectRows = 32;                      // heads from which a wave takes more rows, its most a lane

__device__ __forceinline__ int head_rows(const PagedCache& c, int h) {
    const int cap = c.max_pages << c.shift;
    const int n = c.len[h];
    return n < 0 ? 0 : (n > cap ? cap : n);
}
__device__ __forceinline__ bool page_ok(const PagedCache& c, int id) { return (unsigned)id < (unsigned)c.n_pages; }
// pool row of row r of head h, -1 where the page is none
__device__ __forceinline__ int64_t pool_row(const PagedCache& c, int h, int r) {
    const int id = c.table[(int64_t)h * c.max_pages + (r >> c.shift)];
    return page_ok(c, id) ? ((int64_t)id << c.shift) + (r & ((1 << c.shift) - 1)) : -1;
}

// entry of row r of head h in the workspace's arrays (of a head with all its pages)
template <bool POOL>
__device__ __forceinline__ int64_t row_entry(const PagedCache& c, int h, int r) {
    return POOL ? pool_row(c, h, r) : (int64_t)h * (c.max_pages << c.shift) + r;
}

}  // namespace

// ---- append ----------------------------------------------------------------------------------------------------------
// Rows that join head h: as many as are offered, fit the table and have pages up to the first that has none.
__global__ __launch_bounds__(256) void paged_reserve_kernel(PagedCache c, const int32_t* __restrict__ rows_in, int rows, int2* __restrict__ fit) {
    const int h = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (h >= c.n_heads) return;
    const int n = head_rows(c, h), cap = c.max_pages << c.shift;
    int want = rows_in != nullptr ? rows_in[h] : rows;
    want = want < 0 ? 0 : (want > rows ? rows : want);
    want = want > cap - n ? cap - n : want;
    int got = want;
    if (want > 0) {
        const int first = n >> c.shift, last = (n + want - 1) >> c.shift;
        for (int p0 = first; p0 <= last; p0 += 64) {
            const int p = p0 + lane;
            const bool bad = p <= last && !page_ok(c, c.table[(int64_t)h * c.max_pages + p]);
            const unsigned long long any = __ballot(bad);
            if (any != 0) {
                const int at = (p0 + __ffsll(any) - 1) << c.shift;
                got = at > n ? at - n : 0;
                break;
            }
        }
    }
    if (lane == 0) {
        fit[h] = make_int2(n, got);
        c.len[h] = n + got;
    }
}

// 64 rows of one head per workgroup; a row's K and V are copied 16 bytes a lane.
__global__ __launch_bounds__(256) void paged_copy_kernel(PagedCache c, const char* __restrict__ K, const char* __restrict__ V,
                                                         const int32_t* __restrict__ idx, const float* __restrict__ cum, int64_t head_bytes,
                                                         int64_t row_bytes, int rows, int row_size, int n_chunks, const int2* __restrict__ fit) {
    const int h = blockIdx.x / n_chunks, r0 = (blockIdx.x % n_chunks) * 64;
    const int2 f = fit[h];
    const int end = min(f.y, r0 + 64);
    const int lanes = row_size / 16, per = 256 / lanes, piece = (threadIdx.x % lanes) * 16;
    for (int r = r0 + threadIdx.x / lanes; r < end; r += per) {
        const int64_t to = pool_row(c, h, f.x + r) * row_size + piece, from = h * head_bytes + r * row_bytes + piece;
        *reinterpret_cast<uint4*>(static_cast<char*>(c.K) + to) = *reinterpret_cast<const uint4*>(K + from);
        *reinterpret_cast<uint4*>(static_cast<char*>(c.V) + to) = *reinterpret_cast<const uint4*>(V + from);
    }
    const int r = r0 + threadIdx.x;
    if (threadIdx.x < 64 && r < end) {
        const int64_t to = pool_row(c, h, f.x + r);
        c.idx[to] = idx[(int64_t)h * rows + r];
        c.cum[to] = cum != nullptr ? cum[(int64_t)h * rows + r] : 0.f;
    }
}

// ---- one token -------------------------------------------------------------------------------------------------------
namespace {

// What the queries of one head attend to: its rows and, where it joins, the new token behind them.
struct HeadRows {
    int n, n1;
    bool joins;
};
__device__ __forceinline__ HeadRows rows_of_head(const PagedCache& c, int h, bool has_new) {
    HeadRows r;
    r.n = head_rows(c, h);
    r.joins = has_new && r.n < (c.max_pages << c.shift) &&
              page_ok(c, c.table[(int64_t)h * c.max_pages + min(r.n >> c.shift, c.max_pages - 1)]);
    r.n1 = r.n + (r.joins ? 1 : 0);
    return r;
}

// One wave's share of a head: whole blocks of rows from `first` on, `step` rows apart, up to `end`, and the block of the head's last rows if
// it falls to this wave (tail).  keep(row, logits): the lane's column's logits of its rows of the block that begins with `row`, in base 2.
// A block's keys are on their way from the time the logits of the one before are there, its values from the time that one's have
// been added, its pages two blocks ahead.
template <typename T, int D, typename F>
__device__ __forceinline__ void attend_rows(WaveAttend<T, D>& a, const PagedCache& c, int h, const HeadRows& hr, const T* kn, const T* vn, int first,
                                            int step, int end, bool tail, int lane, F&& keep) {
    using A = WaveAttend<T, D>;
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);
    const int32_t* table = c.table + (int64_t)h * c.max_pages;
    const T* K = static_cast<const T*>(c.K);
    const T* V = static_cast<const T*>(c.V);
    const int in_page = (1 << c.shift) - 1, last = c.max_pages - 1;
    // the pages of a block's two tiles (the same one unless pages hold sixteen rows); the pool's first is read in the place of one that is none
    struct Pages {
        int id[2];
        __device__ __forceinline__ bool ok(const PagedCache& c, int tile) const { return page_ok(c, id[tile]); }
    };
    const auto pages_of = [&](int r0) __attribute__((always_inline)) {
        Pages p;
        p.id[0] = table[min(r0 >> c.shift, last)];
        p.id[1] = A::kBlock > 16 && c.shift == 4 ? table[min((r0 >> 4) + 1, last)] : p.id[0];
        return p;
    };
    const auto tile_at = [&](const T* pool, const Pages& p, int r0, int tile) __attribute__((always_inline)) {
        return pool + (((int64_t)(p.ok(c, tile) ? p.id[tile] : 0) << c.shift) + ((r0 + 16 * tile) & in_page)) * D;
    };
    typename A::Keys keys;
    typename A::Values values;
    const auto load_keys = [&](const Pages& p, int r0) __attribute__((always_inline)) { A::load_keys(keys, lane, tile_at(K, p, r0, 0), tile_at(K, p, r0, 1)); };
    const auto load_values = [&](const Pages& p, int r0) __attribute__((always_inline)) {
        A::load_values(values, lane, tile_at(V, p, r0, 0), tile_at(V, p, r0, 1));
    };
    const auto block = [&](int r0, float (&s)[A::kPerLane]) __attribute__((always_inline)) {
        keep(r0, s);
        take_logits(a, s);
        a.add_values(values, s);
    };
    if (tail) {
        const int r0 = hr.n / A::kBlock * A::kBlock;
        const Pages p = pages_of(r0);
        load_keys(p, r0);
        load_values(p, r0);
        if (hr.joins) {
            A::put_key(keys, lane, hr.n - r0, kn);
            A::put_value(values, lane, hr.n - r0, vn);
        }
        float s[A::kPerLane];
        a.logits(keys, scale2, s);
#pragma unroll
        for (int e = 0; e < A::kPerLane; ++e) {
            const int r = r0 + A::value_row(lane, e);
            const bool has = (r < hr.n && p.ok(c, e >> 2)) || (hr.joins && r == hr.n);
            s[e] = has ? s[e] : -INFINITY;
            if (!has) A::clear_value(values, e);
        }
        block(r0, s);
    }
    if (first >= end) return;
    // behind the last block its own rows are fetched once more, from the caches; nobody reads what they bring
    const auto after = [&](int r0) __attribute__((always_inline)) { return r0 + step < end ? r0 + step : r0; };
    Pages p = pages_of(first), next = pages_of(after(first));
    load_keys(p, first);
    __builtin_amdgcn_sched_barrier(0);                                    // in this order: the wait for the keys leaves the values on their way
    load_values(p, first);
    for (int r0 = first; r0 < end; r0 += step) {
        float s[A::kPerLane];
        a.logits(keys, scale2, s);
        const int r1 = after(r0);
        load_keys(next, r1);
        if (!p.ok(c, 0) || !p.ok(c, 1))
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e)
                if (!p.ok(c, e >> 2)) {
                    s[e] = -INFINITY;
                    A::clear_value(values, e);
                }
        block(r0, s);
        load_values(next, r1);
        p = next;
        next = pages_of(after(r1));
    }
}

template <typename T, int D>
__device__ __forceinline__ void write_new_row(const PagedCache& c, int h, int n, const T* kn, const T* vn, const int32_t* pos, int threads) {
    constexpr int kPieces = D * sizeof(T) / 16;
    const int64_t at = pool_row(c, h, n);
    const int t = threadIdx.x % threads;
    if (t < kPieces) reinterpret_cast<uint4*>(static_cast<T*>(c.K) + at * D)[t] = reinterpret_cast<const uint4*>(kn)[t];
    else if (t < 2 * kPieces) reinterpret_cast<uint4*>(static_cast<T*>(c.V) + at * D)[t - kPieces] = reinterpret_cast<const uint4*>(vn)[t - kPieces];
    if (t == 0) {
        c.idx[at] = pos[h];
        c.len[h] = n + 1;
    }
}

// Where N rows of head h, `step` apart, are in the pool (-1: not there), and their cumulative scores, that of row n being zero.  All loads are
// made, from row 0 of the pool where there is none, so that they do not wait for one another.
template <int N>
struct RowPlaces {
    int64_t at[N];
    float cum[N];
    __device__ __forceinline__ void fetch(const PagedCache& c, int h, int first, int step, int n, int n1) {
        int id[N];
#pragma unroll
        for (int i = 0; i < N; ++i) id[i] = c.table[(int64_t)h * c.max_pages + min((first + i * step) >> c.shift, c.max_pages - 1)];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = first + i * step;
            const bool has = r < n1 && page_ok(c, id[i]);
            at[i] = ((int64_t)(has ? id[i] : 0) << c.shift) + (has ? r & ((1 << c.shift) - 1) : 0);
            cum[i] = c.cum[at[i]];
            if (!has) at[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) cum[i] = first + i * step < n ? cum[i] : 0.f;
    }
};

// Logits lie query head by query head, `stride` rows each; those of columns that are not there are zeros, which norm gives no weight.
template <int GT>
struct RowLogits {
    float s[GT];
    __device__ __forceinline__ void load(const float* logits, int64_t stride) {
#pragma unroll
        for (int g = 0; g < GT; ++g) s[g] = logits[g * stride];
    }
    // sum over the query heads of the row's weights
    __device__ __forceinline__ float weight(const float2* norm) const {
        float inc = 0.f;
#pragma unroll
        for (int g = 0; g < GT; ++g) inc = fmaf(__builtin_amdgcn_exp2f(s[g] - norm[g].x), norm[g].y, inc);
        return inc;
    }
};

}  // namespace

// GT: bound on the query heads per KV head.
// Many heads, or short ones: one workgroup per head does all of the step (some: if it has fewer than `stride` rows).  The logits stay in LDS until
// the sums are known; then every row's weights go to
// its cum, and the waves' outputs are joined in the same LDS.
template <typename T, int D, int GT>
__global__ __launch_bounds__(kAttendThreads, 3) void paged_head_kernel(PagedCache c, const T* __restrict__ q, const T* __restrict__ k_new,
                                                                    const T* __restrict__ v_new, const int32_t* __restrict__ pos, int G,
                                                                    int stride, bool some, float* __restrict__ out) {
    using A = WaveAttend<T, D>;
    extern __shared__ float dyn[];                                        // logits [GT][stride], then outputs [waves][G][D]
    __shared__ float ml_s[kAttendWaves][16][2];
    const int h = spread_head(blockIdx.x, gridDim.x), lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, j = lane >> 4;
    if (some && head_rows(c, h) >= stride) return;
    const T* kn = k_new + (int64_t)h * D;
    const T* vn = v_new + (int64_t)h * D;
    A a;
    a.reset();
    a.load_query(col < G ? q + ((int64_t)h * G + col) * D : nullptr, lane);
    const HeadRows hr = rows_of_head(c, h, k_new != nullptr);
    const int n1 = hr.n1, blocks = hr.n / A::kBlock;
    attend_rows<T, D>(a, c, h, hr, kn, vn, A::kBlock * wave, A::kBlock * kAttendWaves, blocks * A::kBlock,
                      n1 > blocks * A::kBlock && blocks % kAttendWaves == wave, lane, [&](int r, const float (&s)[A::kPerLane]) {
        if (col < GT)
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e) dyn[col * stride + r + A::value_row(lane, e)] = col < G ? s[e] : 0.f;
    });
    const float l = column_sum(a.l);
    if (j == 0) {
        ml_s[wave][col][0] = a.m;
        ml_s[wave][col][1] = l;
    }
    // four rows a thread at a time, what lies in memory fetched ahead of the sums
    constexpr int kRows = 4;
    RowPlaces<kRows> places;
    places.fetch(c, h, threadIdx.x, kAttendThreads, hr.n, n1);
    __shared__ float2 norm[16];
    __syncthreads();
    if (threadIdx.x < 16) {
        float m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int x = 0; x < kAttendWaves; ++x) m = fmaxf(m, ml_s[x][threadIdx.x][0]);
        const float ref = reference(m);
#pragma unroll
        for (int x = 0; x < kAttendWaves; ++x) sum = fmaf(__builtin_amdgcn_exp2f(ml_s[x][threadIdx.x][0] - ref), ml_s[x][threadIdx.x][1], sum);
        norm[threadIdx.x] = make_float2(ref, sum == 0.f || (int)threadIdx.x >= G ? 0.f : 1.f / sum);
    }
    __syncthreads();
    for (int r0 = threadIdx.x; r0 < n1; r0 += kRows * kAttendThreads) {
        if (r0 >= kRows * kAttendThreads) places.fetch(c, h, r0, kAttendThreads, hr.n, n1);
        RowLogits<GT> row[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) row[i].load(dyn + min(r0 + i * kAttendThreads, stride - 1), stride);
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (places.at[i] >= 0) c.cum[places.at[i]] = places.cum[i] + row[i].weight(norm);
    }
    if (hr.joins) write_new_row<T, D>(c, h, hr.n, kn, vn, pos, kAttendThreads);
    if (out == nullptr) return;
    __syncthreads();
    if (col < G) {
        const float f = __builtin_amdgcn_exp2f(a.m - norm[col].x) * norm[col].y;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < A::kVw; t += 4)
                *reinterpret_cast<f32x4_t*>(dyn + (wave * G + col) * D + A::feature(4 * j + i, t)) =
                    f32x4_t{a.o[t][i] * f, a.o[t + 1][i] * f, a.o[t + 2][i] * f, a.o[t + 3][i] * f};
    }
    __syncthreads();
    for (int e = 4 * threadIdx.x; e < G * D; e += 4 * kAttendThreads) {
        f32x4_t o = *reinterpret_cast<const f32x4_t*>(dyn + e);
#pragma unroll
        for (int x = 1; x < kAttendWaves; ++x) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(dyn + x * G * D + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += v[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) out[(int64_t)h * G * D + e + i] = o[i];
    }
}

// The heads of at least `least` rows, in order, and their rows.  One workgroup, a run of heads a thread.  (Before any length changes.)
__global__ __launch_bounds__(1024) void paged_list_kernel(PagedCache c, int least, PagedStepPlan p, char* ws) {
    __shared__ int count_s[16];
    __shared__ int64_t rows_s[16];
    int64_t* total = reinterpret_cast<int64_t*>(ws + p.list_off);
    int32_t* list = reinterpret_cast<int32_t*>(total + 1);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int run = (c.n_heads + 1023) / 1024, begin = min(c.n_heads, tid * run), end = min(c.n_heads, begin + run);
    int mine = 0;
    int64_t rows = 0;
    for (int h = begin; h < end; ++h) {
        const int n = head_rows(c, h);
        mine += n >= least;
        rows += n >= least ? n + 1 : 0;
    }
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(sum, o, 64);
        if (lane >= o) sum += u;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) rows += __shfl_xor(rows, o, 64);
    if (lane == 63) count_s[wave] = sum;
    if (lane == 63) rows_s[wave] = rows;
    __syncthreads();
    int at = sum - mine;
    for (int x = 0; x < wave; ++x) at += count_s[x];
    for (int h = begin; h < end; ++h)
        if (head_rows(c, h) >= least) list[1 + at++] = h;
    if (tid == 1023) {
        list[0] = at;
        int64_t t = 0;
        for (int x = 0; x < 16; ++x) t += rows_s[x];
        *total = t;
    }
}

// The rows of few long heads, or of the listed ones, are dealt to about as many workgroups as run at a time, whatever the heads' lengths: as many parts
// of a head as it has shares of all rows, begun ones included, and all of one size.  Part number -> head and part of it, from the
// lengths, 64 of them at a time.
struct HeadPart {
    int h, part, n_parts;
};
template <bool LISTED>
__device__ __forceinline__ bool find_head_part(const PagedCache& c, const PagedStepPlan& p, const char* ws, int wg, HeadPart* out) {
    const int lane = threadIdx.x & 63;
    const int64_t* listed = reinterpret_cast<const int64_t*>(ws + p.list_off);
    const int32_t* list = reinterpret_cast<const int32_t*>(listed + 1);
    const int n_heads = LISTED ? list[0] : c.n_heads;
    int64_t total = 0;
    if (LISTED) {
        if (wg >= p.n_split + n_heads) return false;
        total = *listed;
    } else {
        for (int h = lane; h < c.n_heads; h += 64) total += head_rows(c, h) + 1;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    }
    // (at most one row more than a head can have, which is then one part: never more parts than n_split and a broken one a head)
    int share = (int)max((int64_t)kLeastShare, min((total + p.n_split - 1) / p.n_split, ((int64_t)1 << 26) + 1));
    if (share < 4 * kLeastShare) share = (share + kLeastShare - 1) / kLeastShare * kLeastShare;      // as many blocks for every wave, where they are few
    for (int h0 = 0; h0 < n_heads; h0 += 64) {
        const int i = min(h0 + lane, n_heads - 1), h = LISTED ? list[1 + i] : i;
        const int parts = h0 + lane < n_heads ? head_rows(c, h) / share + 1 : 0;
        int sum = parts;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(sum, o, 64);
            if (lane >= o) sum += u;
        }
        const unsigned long long has = __ballot(sum > wg);
        if (has != 0) {
            const int x = __builtin_amdgcn_readfirstlane(__ffsll(has) - 1);
            out->h = __builtin_amdgcn_readlane(h, x);
            out->n_parts = __builtin_amdgcn_readlane(parts, x);
            out->part = wg - (__builtin_amdgcn_readlane(sum, x) - out->n_parts);
            return true;
        }
        wg -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// One part of one head's rows per workgroup, its blocks dealt to the waves in turn.  Leaves the part's maximum, sum and output
// (joined by the finishing kernel) and every row's logits.
template <typename T, int D, int GT, bool LISTED>
__global__ __launch_bounds__(kAttendThreads, 3) void paged_attend_kernel(PagedCache c, const T* __restrict__ q, const T* __restrict__ k_new,
                                                                      const T* __restrict__ v_new, int G, PagedStepPlan p, char* ws) {
    using A = WaveAttend<T, D>;
    extern __shared__ float o_s[];                                        // [waves][G][D]
    __shared__ float ml_s[kAttendWaves][16][2];
    constexpr int kLine = A::kBlock + 4;
    __shared__ __align__(16) float line_s[kAttendWaves][GT * kLine];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, j = lane >> 4;
    constexpr int kStep = A::kBlock * kAttendWaves;
    HeadPart hp;
    if (!find_head_part<LISTED>(c, p, ws, blockIdx.x, &hp)) return;
    const int h = hp.h;
    A a;
    a.reset();
    a.load_query(col < G ? q + ((int64_t)h * G + col) * D : nullptr, lane);
    const HeadRows hr = rows_of_head(c, h, k_new != nullptr);
    const int size = (hr.n / hp.n_parts + A::kBlock) / A::kBlock * A::kBlock;                 // whole blocks, together more than n rows
    const int begin = hp.part * size, end = begin + size, blocks = hr.n / A::kBlock;
    const bool tail = hr.n1 > blocks * A::kBlock && blocks * A::kBlock >= begin && blocks * A::kBlock < end;
    float* logits = reinterpret_cast<float*>(ws + p.logit_off) + (p.by_pool ? 0 : (int64_t)h * GT * p.rows);
    attend_rows<T, D>(a, c, h, hr, k_new + (int64_t)h * D, v_new + (int64_t)h * D, begin + A::kBlock * wave, kStep, min(end, blocks * A::kBlock),
                      tail && (blocks - begin / A::kBlock) % kAttendWaves == wave, lane, [&](int r, const float (&s)[A::kPerLane]) {
        // a wave's logits change places in LDS (in the order its instructions have there) for stores of whole pieces of 16 bytes
        float* mine = line_s[wave];
        if (col < GT)
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e) mine[col * kLine + A::value_row(lane, e)] = col < G ? s[e] : 0.f;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < (GT * A::kBlock + 255) / 256; ++i) {
            const int x = 4 * (lane + 64 * i), g = x / A::kBlock, in = x % A::kBlock;
            if (g >= GT) continue;
            int64_t to = (int64_t)g * p.rows + r + in;
            if (p.by_pool) {
                const int page = (r + in) >> c.shift;                        // (a block may reach behind the table)
                const int id = page < c.max_pages ? c.table[(int64_t)h * c.max_pages + page] : -1;
                if (!page_ok(c, id)) continue;
                to = (((int64_t)id * GT + g) << c.shift) + ((r + in) & ((1 << c.shift) - 1));
            }
            *reinterpret_cast<f32x4_t*>(logits + to) = *reinterpret_cast<const f32x4_t*>(mine + g * kLine + in);
        }
        __builtin_amdgcn_wave_barrier();
    });
    // the waves' parts, then the workgroup's
    const float l = column_sum(a.l);
    if (j == 0) {
        ml_s[wave][col][0] = a.m;
        ml_s[wave][col][1] = l;
    }
    __syncthreads();
    float m = ml_s[0][col][0];
#pragma unroll
    for (int x = 1; x < kAttendWaves; ++x) m = fmaxf(m, ml_s[x][col][0]);
    const float ref = reference(m);
    if (col < G) {
        const float f = __builtin_amdgcn_exp2f(a.m - ref);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < A::kVw; t += 4)
                *reinterpret_cast<f32x4_t*>(o_s + (wave * G + col) * D + A::feature(4 * j + i, t)) =
                    f32x4_t{a.o[t][i] * f, a.o[t + 1][i] * f, a.o[t + 2][i] * f, a.o[t + 3][i] * f};
    }
    if (threadIdx.x < (unsigned)G) {
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < kAttendWaves; ++x) sum = fmaf(__builtin_amdgcn_exp2f(ml_s[x][col][0] - ref), ml_s[x][col][1], sum);
        reinterpret_cast<float2*>(ws + p.ml_off)[(int64_t)blockIdx.x * G + col] = make_float2(m, sum);
    }
    __syncthreads();
    float* acc = reinterpret_cast<float*>(ws + p.acc_off) + (int64_t)blockIdx.x * G * D;
    for (int e = 4 * threadIdx.x; e < G * D; e += 4 * kAttendThreads) {
        f32x4_t o = *reinterpret_cast<const f32x4_t*>(o_s + e);
#pragma unroll
        for (int x = 1; x < kAttendWaves; ++x) o += *reinterpret_cast<const f32x4_t*>(o_s + x * G * D + e);
        *reinterpret_cast<f32x4_t*>(acc + e) = o;
    }
    if (hp.part == 0 && threadIdx.x == 0) reinterpret_cast<int4*>(ws + p.head_off)[h] = make_int4(hr.n, hr.n1, blockIdx.x, hp.n_parts);
}

// Joins the parts.  The first n_chunks workgroups of a head take 1024 rows at a time and add their weights to cum; the rest take a share
// of the outputs, several threads to four features of them; the first also writes the new row.
template <typename T, int D, int GT, bool POOL>
__device__ __forceinline__ void finish_task(const PagedCache& c, const T* k_new, const T* v_new, const int32_t* pos, int G, int n_chunks, int n_join,
                                            const PagedStepPlan& p, const char* ws, float* out, int h, int task, float2* norm, f32x4_t* sum_s) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int4 head = reinterpret_cast<const int4*>(ws + p.head_off)[h];
    const int n = head.x, n1 = head.y, n_parts = head.w;
    const float2* ml = reinterpret_cast<const float2*>(ws + p.ml_off) + (int64_t)head.z * G;
    const bool rows = task < n_chunks;
    if (rows && task * kFinishRows >= n1 && task > 0) return;
    // what does not wait for the sums: this thread's rows
    constexpr int kRows = kFinishRows / kFinishThreads;
    RowPlaces<kRows> places;
    RowLogits<GT> row[kRows];
    const float* logits = reinterpret_cast<const float*>(ws + p.logit_off) + (POOL ? 0 : (int64_t)h * GT * p.rows);
    const auto fetch = [&](int first) __attribute__((always_inline)) {
        if (!POOL)
#pragma unroll
            for (int i = 0; i < kRows; ++i) row[i].load(logits + min(first + i * kFinishThreads, p.rows - 1), p.rows);
        places.fetch(c, h, first, kFinishThreads, n, n1);
        if (POOL)
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t at = places.at[i] < 0 ? 0 : places.at[i], mask = (1 << c.shift) - 1;
                row[i].load(logits + (at & ~mask) * GT + (at & mask), mask + 1);
            }
    };
    if (rows) fetch(task * kFinishRows + threadIdx.x);
    // maximum and sum of every query head, a wave each
    if (threadIdx.x < 16) norm[threadIdx.x] = make_float2(0.f, 0.f);
    __syncthreads();
    for (int g = wave; g < G; g += kFinishThreads / 64) {
        float m = -INFINITY, l = 0.f;
        for (int s = lane; s < n_parts; s += 64) m = fmaxf(m, ml[s * G + g].x);
        m = wave_max(m);
        const float ref = reference(m);
        for (int s = lane; s < n_parts; s += 64) l = fmaf(__builtin_amdgcn_exp2f(ml[s * G + g].x - ref), ml[s * G + g].y, l);
        l = wave_sum(l);
        if (lane == 0) norm[g] = make_float2(ref, l == 0.f ? 0.f : 1.f / l);
    }
    __syncthreads();
    if (rows) {
        for (int first = task * kFinishRows;;) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (places.at[i] >= 0) c.cum[places.at[i]] = places.cum[i] + row[i].weight(norm);
            first += n_chunks * kFinishRows;
            if (first >= n1) break;
            fetch(first + threadIdx.x);
        }
        if (task == 0 && n1 > n) write_new_row<T, D>(c, h, n, k_new + (int64_t)h * D, v_new + (int64_t)h * D, pos, kFinishThreads);
        return;
    }
    const float* acc = reinterpret_cast<const float*>(ws + p.acc_off) + (int64_t)head.z * G * D;
    const int quads = (G * D / 4 + n_join - 1) / n_join, groups = kFinishThreads / quads;      // (n_join: quads <= the workgroup's threads)
    const int quad = (task - n_chunks) * quads + threadIdx.x % quads, group = threadIdx.x / quads;
    const bool has = group < groups && quad < G * D / 4;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    if (has) {
        const int g = quad * 4 / D;
#pragma unroll 4
        for (int s = group; s < n_parts; s += groups) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(acc + (int64_t)s * G * D + quad * 4);
            const float2 w = ml[s * G + g];
            const float f = __builtin_amdgcn_exp2f(w.x - norm[g].x);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = w.y == 0.f ? o[i] : fmaf(f, v[i], o[i]);
        }
    }
    sum_s[threadIdx.x] = o;
    __syncthreads();
    if (has && group == 0) {
        for (int x = 1; x < groups; ++x) o += sum_s[x * quads + threadIdx.x];
        float* to = out + (int64_t)h * G * D + quad * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = o[i] * norm[quad * 4 / D].y;
    }
}

template <typename T, int D, int GT, bool POOL, bool LISTED>
__global__ __launch_bounds__(kFinishThreads) void paged_finish_kernel(PagedCache c, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                                      const int32_t* __restrict__ pos, int G, int n_chunks, int n_join,
                                                                      PagedStepPlan p, const char* __restrict__ ws, float* __restrict__ out) {
    __shared__ float2 norm[16];
    __shared__ f32x4_t sum_s[kFinishThreads];
    const int per = n_chunks + n_join;
    if constexpr (LISTED) {
        const int32_t* list = reinterpret_cast<const int32_t*>(reinterpret_cast<const int64_t*>(ws + p.list_off) + 1);
        for (int task = blockIdx.x, end = list[0] * per; task < end; task += gridDim.x) {
            finish_task<T, D, GT, POOL>(c, k_new, v_new, pos, G, n_chunks, n_join, p, ws, out, list[1 + task / per], task % per, norm, sum_s);
            __syncthreads();
        }
    } else {
        finish_task<T, D, GT, POOL>(c, k_new, v_new, pos, G, n_chunks, n_join, p, ws, out, blockIdx.x / per, blockIdx.x % per, norm, sum_s);
    }
}

// ---- eviction --------------------------------------------------------------------------------------------------------
// Rows leave in the order of (accumulated weight, position, row).  A row's key is its weight as an unsigned number of the same
// order; the key of the last one to leave is searched for, and only where equal keys lie on both sides of the cut the same is
// done with their positions, and with equal positions in row order.  The i-th gap before the new end is then paired with the i-th survivor
// behind it, as rows of the pool, and another kernel moves the rows.
namespace {
constexpr uint32_t kStays = 0xffffffffu, kLacks = kStays - 1;      // the keys of a row that may not leave, and of one without a page: above every other

__device__ __forceinline__ uint32_t weight_key(float f) { return f != f ? kLacks - 1 : order_key(f); }
__device__ __forceinline__ uint32_t row_key(const PagedCache& c, int64_t at, int64_t newest) {
    const int64_t from = at >= 0 ? at : 0;
    const float f = c.cum[from];
    const int32_t place = c.idx[from];
    return at < 0 ? kLacks : place <= newest ? weight_key(f) : kStays;
}
__device__ __forceinline__ uint32_t position_key(int32_t p) { return (uint32_t)p ^ 0x80000000u; }

// how many rows a head has to give up, were they all old enough
__device__ __forceinline__ int rows_over(int n, int budget, int w) {
    const int b = max(budget, w);
    return n > b ? n - b : 0;
}

// sum of v over the threads before this one, and over all
__device__ __forceinline__ int block_scan(int v, int* buf, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(s, o, 64);
        if (lane >= o) s += u;
    }
    __syncthreads();
    if (lane == 63) buf[wave] = s;
    __syncthreads();
    int before = 0, t = 0;
#pragma unroll
    for (int i = 0; i < kSelectThreads / 64; ++i) {
        if (i < wave) before += buf[i];
        t += buf[i];
    }
    *total = t;
    return before + s - v;
}

// The `want` smallest of the keys that each(f) hands to f (at least `want`): a histogram over what is left of their range, its bin that holds
// the last of them the next range.  cut: the key of the last; left: how many keys equal to it are among them (INT_MAX: all).
struct Cut {
    uint32_t key;
    int left;
};
constexpr int kAll = 0x7fffffff;
// the round's end, the same for whoever searches: `before` keys lie below bin `bin` of 1 << shift, `here` in it
__device__ __forceinline__ bool narrow(uint32_t& lo, uint32_t& hi, int shift, int bin, int before, int here, int& want, Cut* cut) {
    want -= before;
    lo += (uint32_t)bin << shift;
    if (hi - lo >= 1u << shift) hi = lo + ((1u << shift) - 1u);
    *cut = Cut{hi, here == want ? kAll : want};
    return here == want || shift == 0;
}
__device__ __forceinline__ int shift_of(uint32_t lo, uint32_t hi, int bits) {
    const int n = hi == lo ? 0 : 32 - __clz((int)(hi - lo));
    return n > bits ? n - bits : 0;
}

// by one wave: 256 bins of its own in LDS, four a lane
template <typename F>
__device__ __forceinline__ Cut last_of_smallest_wave(F&& each, int want, int* hist) {
    const int lane = threadIdx.x & 63;
    const auto in_order = []() {                                          // a wave's LDS instructions run in order; the compiler's too, from here to there
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    uint32_t lo = 0xffffffffu, hi = 0u;
    each([&](uint32_t k) {
        lo = min(lo, k);
        hi = max(hi, k);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
    }
    Cut cut;
    while (true) {
        const int shift = shift_of(lo, hi, 8);
        reinterpret_cast<int4*>(hist)[lane] = make_int4(0, 0, 0, 0);
        in_order();
        each([&](uint32_t k) {
            if (k >= lo && k <= hi) atomicAdd(&hist[(k - lo) >> shift], 1);
        });
        in_order();
        const int4 h = reinterpret_cast<const int4*>(hist)[lane];
        const int mine = (h.x + h.y) + (h.z + h.w);
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(sum, o, 64);
            if (lane >= o) sum += u;
        }
        // the lane whose four bins hold the want-th key, and the bin among them
        const int x = __ffsll(__ballot(sum >= want)) - 1;
        int before = sum - mine, bin = 4 * lane, here = h.x;
        if (before + here < want) { before += here; here = h.y; ++bin; }
        if (before + here < want) { before += here; here = h.z; ++bin; }
        if (before + here < want) { before += here; here = h.w; ++bin; }
        if (narrow(lo, hi, shift, __builtin_amdgcn_readlane(bin, x), __builtin_amdgcn_readlane(before, x), __builtin_amdgcn_readlane(here, x), want, &cut))
            return cut;
        in_order();
    }
}

// by the workgroup: a bin a thread
template <typename F>
__device__ Cut last_of_smallest(F&& each, int want, int* hist, int* buf, uint32_t* range, int* pick) {
    const int tid = threadIdx.x;
    uint32_t lo = 0xffffffffu, hi = 0u;
    each([&](uint32_t k) {
        lo = min(lo, k);
        hi = max(hi, k);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
    }
    if (tid == 0) {
        range[0] = 0xffffffffu;
        range[1] = 0u;
    }
    __syncthreads();
    if ((tid & 63) == 0) {
        atomicMin(&range[0], lo);
        atomicMax(&range[1], hi);
    }
    __syncthreads();
    lo = range[0];
    hi = range[1];
    Cut cut;
    while (true) {
        const int shift = shift_of(lo, hi, 10);
        hist[tid] = 0;
        __syncthreads();
        each([&](uint32_t k) {
            if (k >= lo && k <= hi) atomicAdd(&hist[(k - lo) >> shift], 1);
        });
        __syncthreads();
        int total;
        const int here = hist[tid], before = block_scan(here, buf, &total);
        if (before < want && before + here >= want) {
            pick[0] = tid;
            pick[1] = before;
            pick[2] = here;
        }
        __syncthreads();
        const bool done = narrow(lo, hi, shift, pick[0], pick[1], pick[2], want, &cut);
        __syncthreads();
        if (done) return cut;
    }
}
}  // namespace

// Short heads (at most 64 R rows): a wave per head with every row's key in a register; nobody waits for anybody.  Whole evictions, us: 5120 heads
// of 1016 rows, 6 % leaving, 132 (274 with the cut found bit by bit, by counts of the keys below it).  By a wave and by
// a workgroup per head: 8 heads of 1900 rows 46 / 29, 256 heads 62 / 48, 2000 heads 118 / 202.
// Where tables of many heads have room for more, the short heads are seen to first (5120 heads of 700 rows, room for 8192, 119; all by workgroups 259).
template <int R, bool POOL>
__global__ __launch_bounds__(256, R <= 16 ? 4 : 5) void paged_select_wave_kernel(PagedCache c, const int32_t* __restrict__ budget, const int32_t* __restrict__ pos,
                                                                int w, PagedEvictPlan p, char* ws, int32_t* __restrict__ evicted) {
    __shared__ __align__(16) int hist_s[4][256];
    const int lane = threadIdx.x & 63, wg = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (wg >= c.n_heads) return;
    const int h = spread_head(wg, c.n_heads), n = head_rows(c, h), over = rows_over(n, budget[h], w);
    const int64_t newest = (int64_t)pos[h] - w;
    if (n > 64 * R) return;                                               // a workgroup's
    int2* pairs = reinterpret_cast<int2*>(ws + p.pair_off);
    const int32_t* table = c.table + (int64_t)h * c.max_pages;
    const int in_page = (1 << c.shift) - 1;
    int drop = 0, gaps = 0;
    if (over > 0) {
        uint32_t key[R];
        const auto place_of = [&](int r) { return c.idx[pool_row(c, h, r)]; };
        int may = 0;
        unsigned long long lacking = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) key[i] = table[min((64 * i + lane) >> c.shift, c.max_pages - 1)];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int r = 64 * i + lane, id = (int)key[i];
            const bool there = r < n && page_ok(c, id);
            lacking |= __ballot(r < n && !there);
            const int at = there ? (id << c.shift) + (r & in_page) : 0;
            const float f = c.cum[at];
            key[i] = c.idx[at] <= newest ? weight_key(f) : kStays;
            key[i] = there ? key[i] : kStays;
            may += __builtin_popcountll(__ballot(key[i] != kStays));
            if (R > 16 && i % (R / 2) == R / 2 - 1) __builtin_amdgcn_sched_barrier(0);
        }
        drop = lacking != 0 ? 0 : min(over, may);
        // (many rows: their numbers are made anew, or those above and the addresses from them would stay in registers all the way, which then hold
        // three waves in the place of five: 5120 heads of 1016 rows 146 us, not 132)
        int late = lane;
        if constexpr (R > 16) asm volatile("" : "+v"(late));
        uint32_t leaves = 0;                                              // bit i: row 64 i + lane
        if (drop > 0) {
            int* hist = hist_s[threadIdx.x >> 6];
            Cut cut = last_of_smallest_wave([&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < R; ++i)
                    if (key[i] != kStays) f(key[i]);
            }, drop, hist);
#pragma unroll
            for (int i = 0; i < R; ++i) leaves |= key[i] < cut.key || (cut.left == kAll && key[i] == cut.key) ? 1u << i : 0u;
            if (cut.left != kAll) {
                // of the rows with the last key the lowest positions, of those at the last position the first rows
                uint32_t place[R];
#pragma unroll
                for (int i = 0; i < R; ++i) place[i] = key[i] == cut.key ? position_key(place_of(64 * i + late)) : 0u;
                Cut last = last_of_smallest_wave([&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        if (key[i] == cut.key) f(place[i]);
                }, cut.left, hist);
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const bool tied = key[i] == cut.key, same = tied && place[i] == last.key;
                    const unsigned long long m = __ballot(same);
                    if ((tied && place[i] < last.key) || (same && __builtin_popcountll(m & ((1ull << lane) - 1)) < last.left)) leaves |= 1u << i;
                    if (last.left != kAll) last.left -= __builtin_popcountll(m);          // below zero from here on (signed, as the builtin's counts are)
                }
            }
        }
        const int stay = n - drop;
        int movers = 0;
        if constexpr (R > 16) asm volatile("" : "+v"(late));
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int r = 64 * i + late;
            const bool out = leaves >> i & 1, gap = out && r < stay, mover = !out && r >= stay && r < n;
            const unsigned long long g = __ballot(gap), m = __ballot(mover), lower = (1ull << lane) - 1;
            if (gap) pairs[row_entry<POOL>(c, h, gaps + __builtin_popcountll(g & lower))].x = (int)pool_row(c, h, r);
            if (mover) pairs[row_entry<POOL>(c, h, movers + __builtin_popcountll(m & lower))].y = (int)pool_row(c, h, r);
            gaps += __builtin_popcountll(g);
            movers += __builtin_popcountll(m);
            if (R > 16) __builtin_amdgcn_sched_barrier(0);
        }
        if (lane == 0 && drop > 0) c.len[h] = stay;
    }
    if (lane == 0) {
        if (evicted != nullptr) evicted[h] = drop;
        reinterpret_cast<int32_t*>(ws + p.count_off)[h] = gaps;
    }
}

// Keys of tables that do not fit in LDS, 1024 rows of a head at a time.
__global__ __launch_bounds__(256) void paged_key_kernel(PagedCache c, const int32_t* __restrict__ budget, const int32_t* __restrict__ pos, int w,
                                                        PagedEvictPlan p, int n_chunks, char* ws) {
    const int h = blockIdx.x / n_chunks, n = head_rows(c, h);
    if (rows_over(n, budget[h], w) == 0) return;
    const int64_t newest = (int64_t)pos[h] - w;
    uint32_t* key = reinterpret_cast<uint32_t*>(ws + p.key_off);
    for (int first = blockIdx.x % n_chunks * 1024 + threadIdx.x; first < n; first += n_chunks * 1024)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = first + 256 * i;
            if (r >= n) continue;
            const int64_t at = pool_row(c, h, r), to = p.by_pool ? at : (int64_t)h * p.rows + r;
            if (to >= 0) key[to] = row_key(c, at, newest);
        }
}

// Longer heads: a workgroup per head, keys in LDS where they fit and from the workspace otherwise, four at a time.
template <bool POOL>
__global__ __launch_bounds__(kSelectThreads) void paged_select_kernel(PagedCache c, const int32_t* __restrict__ budget, const int32_t* __restrict__ pos,
                                                                      int w, PagedEvictPlan p, int least, char* ws, int32_t* __restrict__ evicted) {
    extern __shared__ __align__(16) uint32_t key_s[];
    __shared__ int hist[kSelectThreads];
    __shared__ int buf[kSelectThreads / 64];
    __shared__ uint32_t range[2];
    __shared__ int pick[3];
    const int h = spread_head(blockIdx.x, gridDim.x), tid = threadIdx.x;
    const int n = head_rows(c, h), over = rows_over(n, budget[h], w);
    if (n < least) return;                                                // a wave has seen to it
    const int64_t newest = (int64_t)pos[h] - w;
    int2* pairs = reinterpret_cast<int2*>(ws + p.pair_off);
    const bool in_lds = p.keys_in_lds;
    const uint32_t* key_m = reinterpret_cast<const uint32_t*>(ws + p.key_off) + (POOL ? 0 : (int64_t)h * p.rows);
    if (in_lds && over > 0) {
#pragma unroll 4
        for (int r = tid; r < n; r += kSelectThreads) key_s[r] = row_key(c, pool_row(c, h, r), newest);
        __syncthreads();
    }
    const auto four = [&](int r) __attribute__((always_inline)) {
        if (in_lds) return *reinterpret_cast<const uint4*>(key_s + r);
        if (!POOL) return *reinterpret_cast<const uint4*>(key_m + r);
        const int64_t at = pool_row(c, h, r);
        return at < 0 ? make_uint4(kLacks, kLacks, kLacks, kLacks) : *reinterpret_cast<const uint4*>(key_m + at);
    };
    // f(row, key) of every row from `begin` to `end`, `step` rows between fours
    const auto each_key = [&](int begin, int end, int step, auto&& f) __attribute__((always_inline)) {
        for (int r = begin; r < end; r += step) {
            const uint4 k = four(r);
            f(r, k.x);
            if (r + 1 < end) f(r + 1, k.y);
            if (r + 2 < end) f(r + 2, k.z);
            if (r + 3 < end) f(r + 3, k.w);
        }
    };
    int may = 0, lacking = 0;
    if (over > 0) {
        each_key(4 * tid, n, 4 * kSelectThreads, [&](int, uint32_t k) {
            may += k < kLacks;
            lacking += k == kLacks;
        });
        block_scan(may, buf, &may);
        block_scan(lacking, buf, &lacking);
    }
    const int drop = lacking > 0 ? 0 : min(over, may);
    if (tid == 0) {
        if (evicted != nullptr) evicted[h] = drop;
        if (drop == 0) reinterpret_cast<int32_t*>(ws + p.count_off)[h] = 0;
    }
    if (drop == 0) return;
    __syncthreads();
    const Cut cut = last_of_smallest([&](auto&& f) {
        each_key(4 * tid, n, 4 * kSelectThreads, [&](int, uint32_t k) {
            if (k < kLacks) f(k);
        });
    }, drop, hist, buf, range, pick);
    const bool ties = cut.left != kAll;                                   // some of the rows with the last key stay
    const auto place_of = [&](int r) { return position_key(c.idx[pool_row(c, h, r)]); };
    Cut last{0u, kAll};
    if (ties)
        last = last_of_smallest([&](auto&& f) {
            each_key(4 * tid, n, 4 * kSelectThreads, [&](int r, uint32_t k) {
                if (k == cut.key) f(place_of(r));
            });
        }, cut.left, hist, buf, range, pick);
    // Every thread takes a run of rows behind one another: one scan of the threads' counts says where its gaps and survivors go.
    const int stay = n - drop, run = ((n + kSelectThreads - 1) / kSelectThreads + 3) & ~3, begin = min(n, tid * run), end = min(n, begin + run);
    int same = 0;                                                         // rows before the run with the last key and the last position
    if (last.left != kAll) {
        each_key(begin, end, 4, [&](int r, uint32_t k) { same += k == cut.key && place_of(r) == last.key; });
        int total;
        same = block_scan(same, buf, &total);
    }
    const auto each_row = [&](auto&& gap, auto&& mover) __attribute__((always_inline)) {
        int seen = same;
        each_key(begin, end, 4, [&](int r, uint32_t k) {
            bool out = k <= cut.key;
            if (ties && k == cut.key) {
                const uint32_t place = place_of(r);
                out = place < last.key || (place == last.key && seen++ < last.left);
            }
            if (out && r < stay) gap(r);
            if (!out && r >= stay) mover(r);
        });
    };
    int gaps = 0, movers = 0, total;
    each_row([&](int) { ++gaps; }, [&](int) { ++movers; });
    int to = block_scan(gaps, buf, &total);
    if (tid == 0) {
        reinterpret_cast<int32_t*>(ws + p.count_off)[h] = total;
        c.len[h] = stay;
    }
    int from = block_scan(movers, buf, &total);
    each_row([&](int r) { pairs[row_entry<POOL>(c, h, to++)].x = (int)pool_row(c, h, r); },
             [&](int r) { pairs[row_entry<POOL>(c, h, from++)].y = (int)pool_row(c, h, r); });
}

// Moves the paired rows: 16 bytes a lane of K and of V, four pairs at a time.  (Three of the four pieces of K wait in scratch memory, 48 bytes a lane
// out and in again: a third of what the kernel writes.)
template <bool POOL>
__global__ __launch_bounds__(256) void paged_move_kernel(PagedCache c, int row_size, int n_chunks, PagedEvictPlan p, const char* __restrict__ ws) {
    const int h = spread_head(blockIdx.x / n_chunks, c.n_heads);
    const int2* pairs = reinterpret_cast<const int2*>(ws + p.pair_off);
    const int n = reinterpret_cast<const int32_t*>(ws + p.count_off)[h];
    const int lanes = row_size / 16, per = 256 / lanes, piece = (threadIdx.x % lanes) * 16;
    char* K = static_cast<char*>(c.K);
    char* V = static_cast<char*>(c.V);
    constexpr int kAhead = 4;
    const int step = n_chunks * per;
    for (int i0 = (blockIdx.x % n_chunks) * per + threadIdx.x / lanes; i0 < n; i0 += kAhead * step) {
        int2 m[kAhead];
        uint4 k[kAhead], v[kAhead];
        int32_t idx[kAhead];
        float cum[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) m[i] = pairs[row_entry<POOL>(c, h, min(i0 + i * step, n - 1))];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t from = m[i].y;
            k[i] = *reinterpret_cast<const uint4*>(K + from * row_size + piece);
            v[i] = *reinterpret_cast<const uint4*>(V + from * row_size + piece);
            idx[i] = c.idx[from];
            cum[i] = c.cum[from];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i0 + i * step >= n) continue;
            const int64_t to = m[i].x;
            *reinterpret_cast<uint4*>(K + to * row_size + piece) = k[i];
            *reinterpret_cast<uint4*>(V + to * row_size + piece) = v[i];
            if (piece == 0) {
                c.idx[to] = idx[i];
                c.cum[to] = cum[i];
            }
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
namespace {
int heads_bound(int G) { return G <= 4 ? 4 : G <= 8 ? 8 : 16; }
// LDS of the one-workgroup step: logits, and later the waves' outputs
size_t head_step_lds(int G, int D, int rows) {
    const size_t logits = (size_t)rows * heads_bound(G) * sizeof(float), outputs = (size_t)kAttendWaves * G * D * sizeof(float);
    return logits > outputs ? logits : outputs;
}
}  // namespace

PagedStepPlan plan_paged_step(bool f32, int n_heads, int G, int D, int rows, int64_t pool_rows) {
    PagedStepPlan p{};
    p.rows = (rows + 31) / 32 * 32;                                       // whole blocks are written
    const bool fits = head_step_lds(G, D, p.rows) <= kHeadLaunchLds;
    if (n_heads >= kManyHeads || (fits && (int64_t)p.rows * (f32 ? 2 : 1) * (kHeadsWorth - n_heads) <= kRowsWorth)) {
        p.split = !fits;
        p.head_rows = p.split ? (int)(kShortHeadLds / (heads_bound(G) * sizeof(float))) / 32 * 32 : p.rows;
        if (!p.split) return p;
    }
    p.split = true;
    const int64_t units = (int64_t)n_heads * ((rows + kLeastShare - 1) / kLeastShare);
    // broken parts count half: together about as many as run at a time; of more heads than that, several rounds
    const int aim = n_heads < kManyHeads ? kSplitAim - n_heads / 2 : 4 * kSplitAim;
    p.n_split = (int)(units < aim ? units : aim);
    const size_t parts = (size_t)p.n_split + n_heads;                     // every head may end with a broken one
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    p.by_pool = 2 * pool_rows < (int64_t)n_heads * p.rows;
    p.list_off = take(sizeof(int64_t) + ((size_t)n_heads + 1) * sizeof(int32_t));
    p.head_off = take((size_t)n_heads * sizeof(int4));
    p.ml_off = take(parts * G * sizeof(float2));
    p.acc_off = take(parts * G * D * sizeof(float));
    p.logit_off = take((size_t)(p.by_pool ? pool_rows : (int64_t)n_heads * p.rows) * heads_bound(G) * sizeof(float));
    p.bytes = off;
    return p;
}

PagedEvictPlan plan_paged_evict(int n_heads, int rows, int64_t pool_rows) {
    PagedEvictPlan p{};
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    p.rows = rows;
    p.by_pool = rows > 64 * kWaveSelectRows && 2 * pool_rows < (int64_t)n_heads * rows;
    const size_t entries = p.by_pool ? pool_rows : (int64_t)n_heads * rows;
    p.keys_in_lds = rows <= kSelectKeys;
    p.count_off = take((size_t)n_heads * sizeof(int32_t));
    p.pair_off = take(entries * sizeof(int2));
    p.key_off = take(p.keys_in_lds ? 0 : entries * sizeof(uint32_t));
    p.bytes = off;
    return p;
}

size_t paged_append_bytes(int n_heads) { return (size_t)n_heads * sizeof(int2); }

hipError_t launch_paged_append(const PagedCache& c, const void* K, const void* V, const int32_t* idx, const float* cum, const int32_t* rows_in,
                               int rows, int64_t head_bytes, int64_t row_bytes, int row_size, char* ws, const Env& env) {
    int2* fit = reinterpret_cast<int2*>(ws);
    env.begin("paged_reserve");
    paged_reserve_kernel<<<(c.n_heads + 3) / 4, 256, 0, env.s>>>(c, rows_in, rows, fit);
    env.end();
    const int n_chunks = (rows + 63) / 64;
    env.begin("paged_copy");
    paged_copy_kernel<<<c.n_heads * n_chunks, 256, 0, env.s>>>(c, static_cast<const char*>(K), static_cast<const char*>(V), idx, cum, head_bytes,
                                                               row_bytes, rows, row_size, n_chunks, fit);
    env.end();
    return hipGetLastError();
}

namespace {
template <typename T, int D, int GT>
hipError_t step_of(const PagedCache& c, const void* q, const void* k_new, const void* v_new, const int32_t* pos, int G, const PagedStepPlan& p,
                   char* ws, float* out, const Env& env) {
    const T* kn = static_cast<const T*>(k_new);
    const T* vn = static_cast<const T*>(v_new);
    if (p.split && p.head_rows > 0) {
        env.begin("paged_list");
        paged_list_kernel<<<1, 1024, 0, env.s>>>(c, p.head_rows, p, ws);
        env.end();
    }
    if (p.head_rows > 0) {
        env.begin("paged_head");
        paged_head_kernel<T, D, GT><<<c.n_heads, kAttendThreads, head_step_lds(G, D, p.head_rows), env.s>>>(c, static_cast<const T*>(q), kn, vn, pos,
                                                                                                            G, p.head_rows, p.split, out);
        env.end();
    }
    if (!p.split) return hipGetLastError();
    const bool listed = p.head_rows > 0;
    env.begin("paged_attend");
    const auto attend = listed ? paged_attend_kernel<T, D, GT, true> : paged_attend_kernel<T, D, GT, false>;
    attend<<<p.n_split + c.n_heads, kAttendThreads, (size_t)kAttendWaves * G * D * sizeof(float), env.s>>>(c, static_cast<const T*>(q), kn, vn, G, p, ws);
    env.end();
    // a workgroup joins up to 64 KiB of partial outputs, of at most as many quads as it has threads; 16 quads, if heads are listed: one may have all
    // parts
    const int n_chunks = (p.rows + kFinishRows - 1) / kFinishRows, most_chunks = listed ? 128 : kFinishWgs / c.n_heads + 1;
    const int chunks = min(n_chunks, most_chunks), n_parts = (p.n_split + c.n_heads - 1) / c.n_heads;
    int n_join = listed ? G * D / 64 : (int)(((int64_t)n_parts * G * D * 4 + 65535) / 65536);
    n_join = max(n_join, (G * D / 4 + kFinishThreads - 1) / kFinishThreads);
    if (out == nullptr) n_join = 0;
    const int64_t tasks = (int64_t)c.n_heads * (chunks + n_join);
    env.begin("paged_finish");
    const auto finish = p.by_pool ? listed ? paged_finish_kernel<T, D, GT, true, true> : paged_finish_kernel<T, D, GT, true, false>
                                  : listed ? paged_finish_kernel<T, D, GT, false, true> : paged_finish_kernel<T, D, GT, false, false>;
    finish<<<(int)(listed ? min(tasks, (int64_t)kFinishWgs) : tasks), kFinishThreads, 0, env.s>>>(c, kn, vn, pos, G, chunks, n_join, p, ws, out);
    env.end();
    return hipGetLastError();
}

// calls f with the kernels' types: element, head width, bound on the query heads
template <typename F>
hipError_t with_types(uncomp_dtype dt, int D, int G, F&& f) {
    const auto bound = [&](auto t, auto d) {
        if (G <= 4) return f(t, d, std::integral_constant<int, 4>{});
        if (G <= 8) return f(t, d, std::integral_constant<int, 8>{});
        return f(t, d, std::integral_constant<int, 16>{});
    };
    const auto width = [&](auto t) { return D == 128 ? bound(t, std::integral_constant<int, 128>{}) : bound(t, std::integral_constant<int, 64>{}); };
    return dt == UNCOMP_BF16 ? width(bf16_bits{}) : width(float{});
}
}  // namespace

hipError_t init_paged_kernels() {
    for (uncomp_dtype dt : {UNCOMP_BF16, UNCOMP_F32})
        for (int D : {64, 128})
            for (int G : {4, 8, 16}) {
                const hipError_t e = with_types(dt, D, G, [](auto t, auto d, auto g) {
                    return allow_dynamic_lds(reinterpret_cast<const void*>(paged_head_kernel<decltype(t), decltype(d)::value, decltype(g)::value>),
                                             kHeadLaunchLds);
                });
                if (e != hipSuccess) return e;
            }
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(paged_select_kernel<false>), kSelectKeys * sizeof(uint32_t));
    return e != hipSuccess ? e : allow_dynamic_lds(reinterpret_cast<const void*>(paged_select_kernel<true>), kSelectKeys * sizeof(uint32_t));
}

hipError_t launch_paged_step(const PagedCache& c, const void* q, const void* k_new, const void* v_new, uncomp_dtype dt, const int32_t* pos, int G,
                             int D, const PagedStepPlan& p, char* ws, float* out, const Env& env) {
    return with_types(dt, D, G, [&](auto t, auto d, auto g) {
        return step_of<decltype(t), decltype(d)::value, decltype(g)::value>(c, q, k_new, v_new, pos, G, p, ws, out, env);
    });
}

hipError_t launch_paged_evict(const PagedCache& c, const int32_t* budget, const int32_t* pos, int w, int row_size, const PagedEvictPlan& p, char* ws,
                              int32_t* evicted, const Env& env) {
    env.begin("paged_select");
    const int rows = c.max_pages << c.shift;
    const unsigned by_wave = (unsigned)(c.n_heads + 3) / 4;
    const auto wave_form = [&](auto r, auto pool) {
        paged_select_wave_kernel<decltype(r)::value, decltype(pool)::value><<<by_wave, 256, 0, env.s>>>(c, budget, pos, w, p, ws, evicted);
    };
    constexpr std::false_type kTable{};
    constexpr std::true_type kPool{};
    constexpr std::integral_constant<int, kWaveSelectRows> kMost{};
    const bool many = c.n_heads > kWaveSelectHeads;
    const int least = many ? 64 * kWaveSelectRows : 64 * 16;              // rows up to which a wave per head is the faster form
    if (rows <= 64 * 8) wave_form(std::integral_constant<int, 8>{}, kTable);
    else if (rows <= 64 * 16) wave_form(std::integral_constant<int, 16>{}, kTable);
    else if (rows <= 64 * 24 && rows <= least) wave_form(std::integral_constant<int, 24>{}, kTable);
    else if (rows <= least) wave_form(kMost, kTable);
    else {
        if (many) p.by_pool ? wave_form(kMost, kPool) : wave_form(kMost, kTable);
        if (!p.keys_in_lds) {
            const int most = (rows + 1023) / 1024, n_chunks = min(most, (4096 + c.n_heads - 1) / c.n_heads);
            paged_key_kernel<<<c.n_heads * n_chunks, 256, 0, env.s>>>(c, budget, pos, w, p, n_chunks, ws);
        }
        const auto select = p.by_pool ? paged_select_kernel<true> : paged_select_kernel<false>;
        select<<<c.n_heads, kSelectThreads, p.keys_in_lds ? (size_t)(rows + 3) / 4 * 16 : 0, env.s>>>(c, budget, pos, w, p, many ? least + 1 : 0, ws, evicted);
    }
    env.end();
    int n_chunks = 2048 / c.n_heads;
    const int most = (rows / 2 + 31) / 32;
    n_chunks = n_chunks < 1 ? 1 : (n_chunks > most ? most : n_chunks);
    env.begin("paged_move");
    const auto move = p.by_pool ? paged_move_kernel<true> : paged_move_kernel<false>;
    move<<<c.n_heads * n_chunks, 256, 0, env.s>>>(c, row_size, n_chunks, p, ws);
    env.end();
    return hipGetLastError();
}

}  // namespace uncomp

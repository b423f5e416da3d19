// The paged cache: rows of every KV head live in pages of a common pool, named by the head's own table, so that heads with
// different budgets hold what they need.  Row r of head h is row r % page of page table[h][r / page].
//
//   append   rows of dense caches join (paged_reserve_kernel: how many fit; paged_copy_kernel)
//   step     one new token joins, its queries attend over the rows, weights accumulate (paged_attend_kernel, paged_finish_kernel)
//   evict    the rows of least accumulated weight leave (paged_select_kernel, paged_move_kernel)
#include "common.h"
#include "attend_wave.h"

namespace uncomp {

namespace {

constexpr int kAttendThreads = 256, kAttendWaves = kAttendThreads / 64;
constexpr int kFinishThreads = 256, kFinishRows = 1024;
constexpr int kSelectThreads = 1024;

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

template <int BYTES>
__device__ __forceinline__ void copy_bytes(const char* src, char* dst) {
    if constexpr (BYTES == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(src);
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
        copy_bytes<16>(K + from, reinterpret_cast<char*>(c.K) + to);
        copy_bytes<16>(V + from, reinterpret_cast<char*>(c.V) + to);
    }
    const int r = r0 + threadIdx.x;
    if (threadIdx.x < 64 && r < end) {
        const int64_t to = pool_row(c, h, f.x + r);
        c.idx[to] = idx[(int64_t)h * rows + r];
        c.cum[to] = cum != nullptr ? cum[(int64_t)h * rows + r] : 0.f;
    }
}

// ---- one token -------------------------------------------------------------------------------------------------------
// One part of one head's rows per workgroup, its blocks dealt to the waves in turn.  Leaves the part's maximum, sum and output
// (joined by the finishing kernel) and every row's logits.
template <typename T, int D>
__global__ __launch_bounds__(kAttendThreads) void paged_attend_kernel(PagedCache c, const T* __restrict__ q, const T* __restrict__ k_new,
                                                                      const T* __restrict__ v_new, int G, int n_split, PagedStepPlan p, char* ws) {
    using A = WaveAttend<T, D>;
    constexpr int kVw = A::kVw;
    __shared__ float o_s[kAttendWaves][16][D];
    __shared__ float ml_s[kAttendWaves][16][2];
    const int h = blockIdx.x / n_split, part = blockIdx.x % n_split;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, j = lane >> 4;
    const int n = head_rows(c, h), cap = c.max_pages << c.shift;
    const bool joins = k_new != nullptr && n < cap && pool_row(c, h, n) >= 0;
    const int n1 = n + (joins ? 1 : 0);
    constexpr int kStep = A::kBlock * kAttendWaves;
    const int chunk = ((n1 + n_split - 1) / n_split + kStep - 1) / kStep * kStep;
    const int64_t begin64 = (int64_t)part * chunk;
    const int begin = begin64 > n1 ? n1 : (int)begin64, end = min(n1, begin + chunk);
    const int32_t* table = c.table + (int64_t)h * c.max_pages;
    const T* K = static_cast<const T*>(c.K);
    const T* V = static_cast<const T*>(c.V);
    const T* kn = k_new + (int64_t)h * D;
    const T* vn = v_new + (int64_t)h * D;
    float* logits = reinterpret_cast<float*>(ws + p.logit_off) + (int64_t)h * p.rows * G;
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);

    A a;
    a.reset();
    a.load_query(col < G ? q + ((int64_t)h * G + col) * D : nullptr, lane);
    const int in_page = (1 << c.shift) - 1;
    for (int r0 = begin + A::kBlock * wave; r0 < end; r0 += kStep) {
        // a block lies in one page, or in two where pages hold sixteen rows
        const int id0 = table[r0 >> c.shift];
        const int id1 = A::kBlock > 16 && r0 + 16 < n ? table[(r0 + 16) >> c.shift] : id0;
        const bool ok0 = page_ok(c, id0), ok1 = page_ok(c, id1);
        auto row_of = [&](int r) -> int64_t {
            const int id = r < 16 ? id0 : id1;
            return ((int64_t)id << c.shift) + ((r0 + r) & in_page);
        };
        typename A::Keys keys;
        typename A::Values values;
        float s[A::kPerLane];
        const bool whole = r0 + A::kBlock <= n && ok0 && ok1;
        if (whole) {
            A::load_keys(keys, lane, [&](int r) { return K + row_of(r) * D; });
            A::load_values(values, lane, [&](int r) { return V + row_of(r) * D; });
            a.logits(keys, scale2, s);
        } else {
            // rows behind the last, rows without a page (the pool's first row is read in their place) and the new token
            auto there = [&](int r) { return r0 + r < n ? (r < 16 ? ok0 : ok1) : joins && r0 + r == n; };
            A::load_keys(keys, lane, [&](int r) { return !there(r) ? K : r0 + r == n ? kn : K + row_of(r) * D; });
            A::load_values(values, lane, [&](int r) { return !there(r) ? V : r0 + r == n ? vn : V + row_of(r) * D; });
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e)
                if (!there(A::value_row(lane, e))) A::clear_value(values, e);
            a.logits(keys, scale2, s);
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e)
                if (!there(A::value_row(lane, e))) s[e] = -INFINITY;
        }
        if (col < G) {
#pragma unroll
            for (int e = 0; e < A::kPerLane; ++e) {
                const int r = r0 + A::value_row(lane, e);
                if (r < n1) logits[(int64_t)r * G + col] = s[e];
            }
        }
        take_logits(a, s);
        a.add_values(values, s);
    }
    // the waves' parts, then the workgroup's
    const float l = column_sum(a.l);
    if (j == 0) {
        ml_s[wave][col][0] = a.m;
        ml_s[wave][col][1] = l;
    }
#pragma unroll
    for (int t = 0; t < kVw; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o_s[wave][col][kVw * (4 * j + i) + t] = a.o[t][i];
    __syncthreads();
    float* acc = reinterpret_cast<float*>(ws + p.acc_off) + ((int64_t)h * n_split + part) * G * D;
    float* ml = reinterpret_cast<float*>(ws + p.ml_off) + ((int64_t)h * n_split + part) * G * 2;
    for (int e = threadIdx.x; e < G * D; e += kAttendThreads) {
        const int g = e / D, d = e % D;
        float m = ml_s[0][g][0];
#pragma unroll
        for (int x = 1; x < kAttendWaves; ++x) m = fmaxf(m, ml_s[x][g][0]);
        const float ref = reference(m);
        float sum = 0.f, out = 0.f;
#pragma unroll
        for (int x = 0; x < kAttendWaves; ++x) {
            const float f = __builtin_amdgcn_exp2f(ml_s[x][g][0] - ref);
            sum = fmaf(f, ml_s[x][g][1], sum);
            out = fmaf(f, o_s[x][g][d], out);
        }
        acc[e] = out;
        if (d == 0) {
            ml[2 * g] = m;
            ml[2 * g + 1] = sum;
        }
    }
    if (part == 0 && threadIdx.x == 0) reinterpret_cast<int2*>(ws + p.head_off)[h] = make_int2(n, n1);
}

// 1024 rows of one head per workgroup: the parts' maxima and sums are joined, every row's weights added to its cum.  The first
// workgroup of a head also joins the outputs and writes the new row.
template <typename T, int D>
__global__ __launch_bounds__(kFinishThreads) void paged_finish_kernel(PagedCache c, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                                      const int32_t* __restrict__ pos, int G, int n_split, int n_chunks,
                                                                      PagedStepPlan p, const char* __restrict__ ws, float* __restrict__ out) {
    __shared__ float2 norm[16];
    const int h = blockIdx.x / n_chunks, chunk = blockIdx.x % n_chunks;
    const int2 nn = reinterpret_cast<const int2*>(ws + p.head_off)[h];
    const int n = nn.x, n1 = nn.y;
    const float* ml = reinterpret_cast<const float*>(ws + p.ml_off) + (int64_t)h * n_split * G * 2;
    const float* acc = reinterpret_cast<const float*>(ws + p.acc_off) + (int64_t)h * n_split * G * D;
    if (threadIdx.x < (unsigned)G) {
        float m = -INFINITY, l = 0.f;
        for (int s = 0; s < n_split; ++s) {
            const float ms = ml[(s * G + threadIdx.x) * 2], ls = ml[(s * G + threadIdx.x) * 2 + 1];
            const float top = fmaxf(m, ms), ref = reference(top);
            l = l * __builtin_amdgcn_exp2f(m - ref) + ls * __builtin_amdgcn_exp2f(ms - ref);
            m = top;
        }
        norm[threadIdx.x] = make_float2(reference(m), l == 0.f ? 0.f : 1.f / l);
    }
    __syncthreads();
    const float* logits = reinterpret_cast<const float*>(ws + p.logit_off) + (int64_t)h * p.rows * G;
    for (int r = chunk * kFinishRows + threadIdx.x; r < min(n1, (chunk + 1) * kFinishRows); r += kFinishThreads) {
        const int64_t at = pool_row(c, h, r);
        if (at < 0) continue;
        float w = r < n ? c.cum[at] : 0.f;
        float inc = 0.f;
        for (int g = 0; g < G; ++g) inc = fmaf(__builtin_amdgcn_exp2f(logits[(int64_t)r * G + g] - norm[g].x), norm[g].y, inc);
        c.cum[at] = w + inc;
    }
    if (chunk != 0) return;
    if (out != nullptr)
        for (int e = threadIdx.x; e < G * D; e += kFinishThreads) {
            const int g = e / D;
            float o = 0.f;
            for (int s = 0; s < n_split; ++s) o = fmaf(acc[(int64_t)s * G * D + e], __builtin_amdgcn_exp2f(ml[(s * G + g) * 2] - norm[g].x), o);
            out[(int64_t)h * G * D + e] = o * norm[g].y;
        }
    if (n1 > n) {
        const int64_t at = pool_row(c, h, n);
        T* K = static_cast<T*>(c.K);
        T* V = static_cast<T*>(c.V);
        for (int d = threadIdx.x; d < D; d += kFinishThreads) {
            K[at * D + d] = k_new[(int64_t)h * D + d];
            V[at * D + d] = v_new[(int64_t)h * D + d];
        }
        if (threadIdx.x == 0) {
            c.idx[at] = pos[h];
            c.len[h] = n1;
        }
    }
}

// ---- eviction --------------------------------------------------------------------------------------------------------
namespace {
// Rows leave in the order of (accumulated weight, position, row).  A NaN counts as more than any number.
__device__ __forceinline__ uint32_t weight_key(float f) { return f != f ? 0xffffffffu : order_key(f); }
__device__ __forceinline__ uint32_t position_key(int32_t p) { return (uint32_t)p ^ 0x80000000u; }

__device__ __forceinline__ int block_sum(int v, int* buf) {
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[wave] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int i = 0; i < kSelectThreads / 64; ++i) t += buf[i];
    return t;
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
}  // namespace

// One workgroup per head finds the rows that leave (radix selection over the 64 bits of weight and position, eight at a time, then
// the row among equals) and pairs the i-th gap before the new end with the i-th survivor behind it.
__global__ __launch_bounds__(kSelectThreads) void paged_select_kernel(PagedCache c, const int32_t* __restrict__ budget, const int32_t* __restrict__ pos,
                                                                      int w, PagedEvictPlan p, char* ws, int32_t* __restrict__ evicted) {
    __shared__ int hist[256];
    __shared__ int buf[kSelectThreads / 64];
    __shared__ int pick[2];
    const int h = blockIdx.x, tid = threadIdx.x;
    const int n = head_rows(c, h);
    const int64_t newest = (int64_t)pos[h] - w;
    const int b = max(budget[h], w);
    int2* pairs = reinterpret_cast<int2*>(ws + p.pair_off) + (int64_t)h * p.pairs;
    int32_t* n_pairs = reinterpret_cast<int32_t*>(ws + p.count_off) + h;
    // an entry's order, all ones (above every one that may leave) where it may not
    auto key_of = [&](int r) -> unsigned long long {
        const int64_t at = pool_row(c, h, r);
        if (at < 0 || c.idx[at] > newest) return ~0ull;
        return (unsigned long long)weight_key(c.cum[at]) << 32 | position_key(c.idx[at]);
    };
    int may = 0;
    if (n > b)
        for (int r = tid; r < n; r += kSelectThreads) {
            const int64_t at = pool_row(c, h, r);
            may += at >= 0 && c.idx[at] <= newest;
        }
    may = block_sum(may, buf);
    const int drop = n > b ? min(n - b, may) : 0;
    if (tid == 0) {
        if (evicted != nullptr) evicted[h] = drop;
        *n_pairs = 0;
    }
    if (drop == 0) return;
    // the drop-th smallest key: its prefix grows by eight bits a round; `left` of the keys with that prefix leave
    unsigned long long prefix = 0;
    int left = drop;
    for (int bit = 56; bit >= 0; bit -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int r = tid; r < n; r += kSelectThreads) {
            const int64_t at = pool_row(c, h, r);
            if (at < 0 || c.idx[at] > newest) continue;
            const unsigned long long k = key_of(r);
            if (bit == 56 || k >> (bit + 8) == prefix >> (bit + 8)) atomicAdd(&hist[(k >> bit) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int sum = 0, d = 0;
            while (d < 255 && sum + hist[d] < left) sum += hist[d++];
            pick[0] = d;
            pick[1] = sum;
        }
        __syncthreads();
        prefix |= (unsigned long long)pick[0] << bit;
        left -= pick[1];
        __syncthreads();
    }
    // gaps and survivors, in row order
    const int stay = n - drop;
    int gaps = 0, movers = 0, equal = 0;
    for (int r0 = 0; r0 < n; r0 += kSelectThreads) {
        const int r = r0 + tid;
        bool leaves = false, same = false;
        if (r < n) {
            const int64_t at = pool_row(c, h, r);
            if (at >= 0 && c.idx[at] <= newest) {
                const unsigned long long k = key_of(r);
                leaves = k < prefix;
                same = k == prefix;
            }
        }
        int total;
        const int e = block_scan(same, buf, &total);
        if (same && equal + e < left) leaves = true;
        equal += total;
        const bool gap = leaves && r < stay, mover = r < n && !leaves && r >= stay;
        const int g = block_scan(gap, buf, &total);
        if (gap) pairs[gaps + g].x = r;
        gaps += total;
        const int m = block_scan(mover, buf, &total);
        if (mover) pairs[movers + m].y = r;
        movers += total;
    }
    if (tid == 0) {
        *n_pairs = gaps;
        c.len[h] = stay;
    }
}

__global__ __launch_bounds__(256) void paged_move_kernel(PagedCache c, int row_size, int n_chunks, PagedEvictPlan p, const char* __restrict__ ws) {
    const int h = blockIdx.x / n_chunks;
    const int2* pairs = reinterpret_cast<const int2*>(ws + p.pair_off) + (int64_t)h * p.pairs;
    const int n = reinterpret_cast<const int32_t*>(ws + p.count_off)[h];
    const int lanes = row_size / 16, per = 256 / lanes, piece = (threadIdx.x % lanes) * 16;
    char* K = static_cast<char*>(c.K);
    char* V = static_cast<char*>(c.V);
    for (int i = (blockIdx.x % n_chunks) * per + threadIdx.x / lanes; i < n; i += n_chunks * per) {
        const int2 m = pairs[i];
        const int64_t to = pool_row(c, h, m.x), from = pool_row(c, h, m.y);
        if (to < 0 || from < 0) continue;
        copy_bytes<16>(K + from * row_size + piece, K + to * row_size + piece);
        copy_bytes<16>(V + from * row_size + piece, V + to * row_size + piece);
        if (piece == 0) {
            c.idx[to] = c.idx[from];
            c.cum[to] = c.cum[from];
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
PagedStepPlan plan_paged_step(int n_heads, int G, int D, int rows) {
    PagedStepPlan p{};
    const int blocks = (rows + 127) / 128;
    int split = (1024 + n_heads - 1) / n_heads;
    split = split > blocks ? blocks : split;
    p.n_split = split < 1 ? 1 : (split > 256 ? 256 : split);
    p.rows = rows;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    p.head_off = take((size_t)n_heads * sizeof(int2));
    p.ml_off = take((size_t)n_heads * p.n_split * G * 2 * sizeof(float));
    p.acc_off = take((size_t)n_heads * p.n_split * G * D * sizeof(float));
    p.logit_off = take((size_t)n_heads * rows * G * sizeof(float));
    p.bytes = off;
    return p;
}

PagedEvictPlan plan_paged_evict(int n_heads, int rows) {
    PagedEvictPlan p{};
    p.pairs = rows / 2 + 1;
    p.count_off = 0;
    p.pair_off = align_up((size_t)n_heads * sizeof(int32_t), 256);
    p.bytes = p.pair_off + (size_t)n_heads * p.pairs * sizeof(int2);
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
template <typename T, int D>
hipError_t step_of(const PagedCache& c, const void* q, const void* k_new, const void* v_new, const int32_t* pos, int G, const PagedStepPlan& p,
                   char* ws, float* out, const Env& env) {
    env.begin("paged_attend");
    paged_attend_kernel<T, D><<<c.n_heads * p.n_split, kAttendThreads, 0, env.s>>>(
        c, static_cast<const T*>(q), static_cast<const T*>(k_new), static_cast<const T*>(v_new), G, p.n_split, p, ws);
    env.end();
    const int n_chunks = (p.rows + kFinishRows - 1) / kFinishRows;
    env.begin("paged_finish");
    paged_finish_kernel<T, D><<<c.n_heads * n_chunks, kFinishThreads, 0, env.s>>>(c, static_cast<const T*>(k_new), static_cast<const T*>(v_new), pos, G,
                                                                                p.n_split, n_chunks, p, ws, out);
    env.end();
    return hipGetLastError();
}
}  // namespace

hipError_t launch_paged_step(const PagedCache& c, const void* q, const void* k_new, const void* v_new, uncomp_dtype dt, const int32_t* pos, int G,
                             int D, const PagedStepPlan& p, char* ws, float* out, const Env& env) {
    if (dt == UNCOMP_BF16)
        return D == 128 ? step_of<bf16_bits, 128>(c, q, k_new, v_new, pos, G, p, ws, out, env)
                        : step_of<bf16_bits, 64>(c, q, k_new, v_new, pos, G, p, ws, out, env);
    return D == 128 ? step_of<float, 128>(c, q, k_new, v_new, pos, G, p, ws, out, env) : step_of<float, 64>(c, q, k_new, v_new, pos, G, p, ws, out, env);
}

hipError_t launch_paged_evict(const PagedCache& c, const int32_t* budget, const int32_t* pos, int w, int row_size, const PagedEvictPlan& p, char* ws,
                              int32_t* evicted, const Env& env) {
    env.begin("paged_select");
    paged_select_kernel<<<c.n_heads, kSelectThreads, 0, env.s>>>(c, budget, pos, w, p, ws, evicted);
    env.end();
    int n_chunks = 2048 / c.n_heads;
    const int most = (p.pairs + 31) / 32;
    n_chunks = n_chunks < 1 ? 1 : (n_chunks > most ? most : n_chunks);
    env.begin("paged_move");
    paged_move_kernel<<<c.n_heads * n_chunks, 256, 0, env.s>>>(c, row_size, n_chunks, p, ws);
    env.end();
    return hipGetLastError();
}

}  // namespace uncomp

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

constexpr int kTileCols = 64;      // columns of a workgroup: sixteen a wave

}  // namespace

// Sixteen columns per wave, keys straight from memory.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_wave_kernel(PrefillArgs a) {
    using A = WaveAttend<T, D, sizeof(T) == 4>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4;
    const int G = a.G;
    const float scale2 = kLog2eA * (D == 128 ? 0.08838834764831845f : 0.125f);
    // work item -> (KV head, sequence, tile), tiles counted over the sequences in order
    for (int64_t item = blockIdx.x;; item += gridDim.x) {
        const int h = (int)(item % a.H);
        int64_t t = item / a.H;
        int s = 0, tile = -1, q_first = 0, nq = 0;
        for (int s0 = 0; s0 < a.n_seq && tile < 0; s0 += 64) {
            int f = 0, n = 0;
            if (s0 + lane < a.n_seq) rows_of(a.q, s0 + lane, &f, &n);
            const int tiles = (n * G + kTileCols - 1) / kTileCols;
            int sum = tiles;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int u = __shfl_up(sum, o, 64);
                if (lane >= o) sum += u;
            }
            const unsigned long long has = __ballot(t < sum);
            if (has != 0) {
                const int x = __ffsll(has) - 1;
                s = s0 + x;
                q_first = __shfl(f, x, 64);
                nq = __shfl(n, x, 64);
                tile = (int)t - __shfl(sum - tiles, x, 64);
            } else {
                t -= __shfl(sum, 63, 64);
            }
        }
        if (tile < 0) return;
        int k_first, nk;
        rows_of(a.k, s, &k_first, &nk);
        const int off = nk - nq;
        const int c0 = tile * kTileCols + 16 * wave, last_col = nq * G - 1;
        if (c0 > last_col) continue;
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
            float w[A::kPerLane];
            A::load(rows, lane, [&](int r) { return K + min(r0 + r, nk - 1) * a.k.sr; }, [&](int r) { return V + min(r0 + r, nk - 1) * a.v.sr; });
            at.logits(rows, scale2, w);
            if (r0 + A::kBlock - 1 <= all) {
                take_logits(at, w);
                at.add_values(rows, w);
            } else {
                A::clear_values(rows, lane, nk - r0);
#pragma unroll
                for (int e = 0; e < A::kPerLane; ++e)
                    if (r0 + A::value_row(lane, e) > lim) w[e] = -INFINITY;
                take_logits(at, w);
                add_masked_values(at, rows, w, lane, [&](int r) { return r0 + r <= lim; });
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
}

size_t prefill_attention_bytes(int, int, int, int, int, int) { return 0; }

namespace {
// most tiles that the sequences can have: whole ones, and one broken one each
int64_t most_tiles(const PrefillArgs& a, int tile) {
    const int64_t cols = (int64_t)a.q.rows * a.G;
    return a.q.first != nullptr ? cols / tile + a.n_seq : (cols + tile - 1) / tile * a.n_seq;
}
template <typename T, int D>
hipError_t prefill_of(const PrefillArgs& a, const Env& env) {
    int64_t grid = most_tiles(a, kTileCols) * a.H;
    if (grid > 1 << 30) grid = 1 << 30;
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

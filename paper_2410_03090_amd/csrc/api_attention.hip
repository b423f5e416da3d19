// C interface, prompt attention and the paged cache: argument checks, workspace carving and kernel launches, as in api.hip.
#include "api_common.h"

using namespace uncomp;

namespace {

// The context's device is current while a call launches, whatever the caller's is, and before it makes the caller's stream wait for the
// side stream: the default stream (NULL) is the current device's.
class OnDevice {
public:
    explicit OnDevice(int device) {
        err = hipGetDevice(&prev_);
        if (err == hipSuccess && prev_ != device) {
            err = hipSetDevice(device);
            changed_ = err == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed_) (void)hipSetDevice(prev_);
    }
    hipError_t err;

private:
    int prev_ = 0;
    bool changed_ = false;
};

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool known_dtype(uncomp_dtype t) { return t == UNCOMP_BF16 || t == UNCOMP_F32; }

// Strides of (sequence, head, row): whole 32-byte (bf16: 16-byte) units, none negative
bool strides_ok(const int64_t s[3], int D) {
    return s[0] >= 0 && s[1] >= 0 && s[2] >= D && (s[0] & 7) == 0 && (s[1] & 7) == 0 && (s[2] & 7) == 0;
}

constexpr int64_t kMostThreads = 0xffffffffLL;      // of a launch, in all
constexpr int64_t kMostColumns = 1 << 30, kNoPool = INT64_MAX / 4;

// The workspace starts at offset 0: scores' key ranges are overwritten, side-stream work of an earlier call may still use it.
// (With the context's device current.)
uncomp_status take_workspace(uncomp_ctx* ctx, const char* who, size_t need, void* stream) {
    if (need > ctx->ws_bytes)
        return fail(ctx, UNCOMP_ERR_WORKSPACE, "%s: needs %zu workspace bytes, context has %zu", who, need, ctx->ws_bytes);
    if (need == 0) return UNCOMP_OK;
    ctx->key_range.ptr = nullptr;
    return uncomp_join(ctx, stream);
}

uncomp_status check_paged(uncomp_ctx* ctx, const char* who, const uncomp_paged_cache* c, PagedCache* v) {
    if (c == nullptr) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: null cache", who);
    if (c->K_pages == nullptr || c->V_pages == nullptr || c->idx_pages == nullptr || c->cum_pages == nullptr || c->table == nullptr ||
        c->len == nullptr)
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: null pointer in the cache", who);
    if (c->n_heads <= 0 || c->n_pages <= 0 || c->max_pages <= 0)
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: sizes must be positive", who);
    if (!known_dtype(c->dtype)) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: dtype", who);
    if (c->D != 64 && c->D != 128) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: D must be 64 or 128", who);
    int shift = 4;
    while (shift < 8 && (1 << shift) != c->page) ++shift;
    if ((1 << shift) != c->page) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: pages hold 16, 32, 64, 128 or 256 rows", who);
    if ((int64_t)c->max_pages * c->page > 1 << 26) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: more than 2^26 rows per head", who);
    if ((int64_t)c->n_pages * c->page > 0x7fffffffLL) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 rows in the pool", who);
    if ((int64_t)c->n_heads * 1024 > kMostThreads) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: too many heads", who);
    if (!aligned16(c->K_pages) || !aligned16(c->V_pages)) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: 16-byte aligned pages required", who);
    if (!aligned4(c->idx_pages) || !aligned4(c->cum_pages) || !aligned4(c->table) || !aligned4(c->len))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: misaligned pointer in the cache", who);
    *v = PagedCache{c->K_pages, c->V_pages, c->idx_pages, c->cum_pages, c->table, c->len, c->n_heads, c->n_pages, shift, c->max_pages};
    return UNCOMP_OK;
}

int row_bytes_of(const uncomp_paged_cache* c) { return c->D * (c->dtype == UNCOMP_BF16 ? 2 : 4); }

}  // namespace

extern "C" {

size_t uncomp_prefill_attention_workspace_bytes(int n_seq, int H, int G, int D, int q_rows, int k_rows) {
    if (n_seq <= 0 || H <= 0 || G <= 0 || q_rows <= 0 || k_rows <= 0) return 0;
    return prefill_attention_bytes(n_seq, H, G, D, q_rows, k_rows);
}

uncomp_status uncomp_prefill_attention(uncomp_ctx* ctx, const void* Q, const void* K, const void* V, uncomp_dtype dtype, int n_seq, int H,
                                       int G, int D, int q_rows, int k_rows, const int32_t* q_first, const int32_t* q_len,
                                       const int32_t* k_first, const int32_t* k_len, const int64_t q_strides[3],
                                       const int64_t k_strides[3], const int64_t v_strides[3], void* out, const int64_t out_strides[3],
                                       float* lse_out, const int64_t lse_strides[2], void* stream) {
    const char* who = "prefill_attention";
    if (ctx == nullptr) return UNCOMP_ERR_INVALID_ARG;
    if (Q == nullptr || K == nullptr || V == nullptr || out == nullptr || q_strides == nullptr || k_strides == nullptr ||
        v_strides == nullptr || out_strides == nullptr)
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (lse_out != nullptr && lse_strides == nullptr) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: lse_out needs lse_strides", who);
    if (n_seq <= 0 || H <= 0 || G <= 0 || q_rows <= 0 || k_rows <= 0)
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: sizes must be positive", who);
    if (!known_dtype(dtype)) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: dtype", who);
    if (D != 64 && D != 128) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: D must be 64 or 128", who);
    if ((int64_t)q_rows * G > kMostColumns || k_rows > kMostColumns || n_seq > 1 << 16 || H > 1 << 20)
        return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: problem too large", who);
    if (!strides_ok(q_strides, D) || !strides_ok(k_strides, D) || !strides_ok(v_strides, D) || !strides_ok(out_strides, D))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements, none negative, row strides >= D", who);
    if (k_strides[2] >= 1 << 24 || v_strides[2] >= 1 << 24) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: row strides below 2^24 elements", who);
    if (lse_out != nullptr && (lse_strides[0] < 0 || lse_strides[1] < 0))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: negative lse stride", who);
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(out) || !aligned4(lse_out) || !aligned4(q_first) || !aligned4(q_len) ||
        !aligned4(k_first) || !aligned4(k_len))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: 16-byte aligned Q, K, V and out required", who);
    PrefillArgs a{};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.out = out;
    a.lse = lse_out;
    a.n_seq = n_seq;
    a.H = H;
    a.G = G;
    a.q = AttnRows{q_first, q_len, q_rows, q_strides[0], q_strides[1], q_strides[2]};
    a.k = AttnRows{k_first, k_len, k_rows, k_strides[0], k_strides[1], k_strides[2]};
    a.v = AttnRows{k_first, k_len, k_rows, v_strides[0], v_strides[1], v_strides[2]};
    a.o = AttnRows{q_first, q_len, q_rows, out_strides[0], out_strides[1], out_strides[2]};
    if (lse_out != nullptr) {
        a.lse_ss = lse_strides[0];
        a.lse_sh = lse_strides[1];
    }
    if (!prefill_attention_fits(a, dtype, D)) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: problem too large", who);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return hip_fail(ctx, on.err, who);
    uncomp_status st = take_workspace(ctx, who, prefill_attention_takes(a, dtype, D, ctx->ws_bytes), stream);
    if (st != UNCOMP_OK) return st;
    hipError_t e = launch_prefill_attention(a, dtype, D, ctx->ws, ctx->ws_bytes, Env{static_cast<hipStream_t>(stream), &ctx->prof, ctx->force_alu});
    if (e != hipSuccess) return hip_fail(ctx, e, "prefill_attention: launch");
    return UNCOMP_OK;
}

size_t uncomp_paged_workspace_bytes(int n_heads, int G, int D, int rows) {
    if (n_heads <= 0 || G <= 0 || D <= 0 || rows <= 0) return 0;
    size_t need = paged_append_bytes(n_heads);                           // (the step of floats needs workspace wherever that of bf16 does)
    const size_t step = plan_paged_step(true, n_heads, G, D, rows, kNoPool).bytes, evict = plan_paged_evict(n_heads, rows, kNoPool).bytes;
    need = need > step ? need : step;
    return need > evict ? need : evict;
}

uncomp_status uncomp_paged_append(uncomp_ctx* ctx, const uncomp_paged_cache* cache, const void* K, const void* V, const int32_t* idx,
                                  const float* cum, const int32_t* n_rows, int rows, const int64_t strides[2], void* stream) {
    const char* who = "paged_append";
    if (ctx == nullptr) return UNCOMP_ERR_INVALID_ARG;
    PagedCache c;
    uncomp_status st = check_paged(ctx, who, cache, &c);
    if (st != UNCOMP_OK) return st;
    if (K == nullptr || V == nullptr || idx == nullptr || strides == nullptr) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (rows <= 0) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: sizes must be positive", who);
    if (strides[0] < 0 || strides[1] < cache->D || (strides[0] & 7) || (strides[1] & 7))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements, none negative, row stride >= D", who);
    if (!aligned16(K) || !aligned16(V) || !aligned4(idx) || !aligned4(cum) || !aligned4(n_rows))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: 16-byte aligned K and V required", who);
    if ((int64_t)c.n_heads * (((int64_t)rows + 63) / 64) * 256 > kMostThreads) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: problem too large", who);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return hip_fail(ctx, on.err, who);
    st = take_workspace(ctx, who, paged_append_bytes(c.n_heads), stream);
    if (st != UNCOMP_OK) return st;
    const int row_size = row_bytes_of(cache), elem = row_size / cache->D;
    hipError_t e = launch_paged_append(c, K, V, idx, cum, n_rows, rows, strides[0] * elem, strides[1] * elem, row_size, ctx->ws,
                                       Env{static_cast<hipStream_t>(stream), &ctx->prof, ctx->force_alu});
    if (e != hipSuccess) return hip_fail(ctx, e, "paged_append: launch");
    return UNCOMP_OK;
}

uncomp_status uncomp_paged_step(uncomp_ctx* ctx, const uncomp_paged_cache* cache, const void* q, int G, const void* k_new,
                                const void* v_new, const int32_t* pos, float* out, void* stream) {
    const char* who = "paged_step";
    if (ctx == nullptr) return UNCOMP_ERR_INVALID_ARG;
    PagedCache c;
    uncomp_status st = check_paged(ctx, who, cache, &c);
    if (st != UNCOMP_OK) return st;
    if (q == nullptr) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((k_new == nullptr) != (v_new == nullptr) || (k_new == nullptr) != (pos == nullptr))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: k_new, v_new and pos must be given together", who);
    if (G < 1 || G > 16) return fail(ctx, UNCOMP_ERR_UNSUPPORTED, "%s: need 1 <= G <= 16", who);
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned4(pos) || !aligned4(out))
        return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: 16-byte aligned q, k_new and v_new required", who);
    const int rows = c.max_pages << c.shift;
    const PagedStepPlan p = plan_paged_step(cache->dtype == UNCOMP_F32, c.n_heads, G, cache->D, rows, (int64_t)c.n_pages << c.shift);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return hip_fail(ctx, on.err, who);
    st = take_workspace(ctx, who, p.bytes, stream);
    if (st != UNCOMP_OK) return st;
    hipError_t e = launch_paged_step(c, q, k_new, v_new, cache->dtype, pos, G, cache->D, p, ctx->ws, out,
                                     Env{static_cast<hipStream_t>(stream), &ctx->prof, ctx->force_alu});
    if (e != hipSuccess) return hip_fail(ctx, e, "paged_step: launch");
    return UNCOMP_OK;
}

uncomp_status uncomp_paged_evict(uncomp_ctx* ctx, const uncomp_paged_cache* cache, const int32_t* budget, const int32_t* pos, int w,
                                 int32_t* evicted, void* stream) {
    const char* who = "paged_evict";
    if (ctx == nullptr) return UNCOMP_ERR_INVALID_ARG;
    PagedCache c;
    uncomp_status st = check_paged(ctx, who, cache, &c);
    if (st != UNCOMP_OK) return st;
    if (budget == nullptr || pos == nullptr) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (w < 0) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: w must not be negative", who);
    if (!aligned4(budget) || !aligned4(pos) || !aligned4(evicted)) return fail(ctx, UNCOMP_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    const PagedEvictPlan p = plan_paged_evict(c.n_heads, c.max_pages << c.shift, (int64_t)c.n_pages << c.shift);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return hip_fail(ctx, on.err, who);
    st = take_workspace(ctx, who, p.bytes, stream);
    if (st != UNCOMP_OK) return st;
    hipError_t e = launch_paged_evict(c, budget, pos, w, row_bytes_of(cache), p, ctx->ws, evicted,
                                      Env{static_cast<hipStream_t>(stream), &ctx->prof, ctx->force_alu});
    if (e != hipSuccess) return hip_fail(ctx, e, "paged_evict: launch");
    return UNCOMP_OK;
}

}  // extern "C"

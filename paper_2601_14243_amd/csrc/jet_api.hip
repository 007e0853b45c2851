// C ABI of libjet: host-side argument checks, then one kernel launch on the
// caller's stream.  Nothing here allocates, synchronises or keeps a pointer.
#include "jet_attn.h"
#include "jet_internal.h"

namespace {

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline jet_status after_launch(hipError_t e) { return e == hipSuccess ? JET_OK : JET_ERR_LAUNCH; }

// The launchers report hipGetLastError() after their launch; an error left pending by the caller's
// earlier HIP calls must not be mistaken for this call's, so it is discarded before launching.
inline void discard_stale_error() { (void)hipGetLastError(); }

constexpr int64_t kMaxTileRows = 65535LL * 128;   // the tile quantizers index 128-row tiles with gridDim.y

// shared by the three GEMM entry points: operands (a,sa)[I,R], (b,sb)[J,R], out [I,J]
jet_status gemm_entry(const uint8_t* a, const float* sa, const uint8_t* b, const float* sb, int sb_mode,
                      void* out, int64_t I, int64_t J, int64_t R, bool i_mult_128, void* stream) {
    if (!a || !sa || !b || !sb || !out) return JET_ERR_NULL;
    if (I < 1 || J < 1 || R < 1) return JET_ERR_SHAPE;
    if (J % 128 || R % 128 || (i_mult_128 && I % 128)) return JET_ERR_SHAPE;
    /* kernels form 32-bit byte offsets (row in tile) x R with a 24-bit multiply: reduction length below 2^24 */
    if (I > INT32_MAX / 2 || J > INT32_MAX / 2 || R >= (1 << 24)) return JET_ERR_SHAPE;
    if (misaligned(a) || misaligned(sa) || misaligned(b) || misaligned(sb) || misaligned(out))
        return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_gemm(a, sa, b, sb, sb_mode, out, I, J, R, static_cast<hipStream_t>(stream)));
}

constexpr int64_t kMaxLd = 1 << 24;               // the attention kernels form 32-bit byte offsets of up to 128 rows

bool heads_fit(int64_t n_q, int64_t n_kv, int64_t dim) {
    return n_q >= 1 && n_kv >= 1 && n_q <= 65535 && n_q % n_kv == 0 && n_q / n_kv <= 512 && (dim == 64 || dim == 128);
}
bool row_fits(int64_t ld, int64_t heads, int64_t dim) { return ld >= heads * dim && ld % 8 == 0 && ld <= kMaxLd; }
constexpr int64_t kMaxTokens = 1 << 30;            // of a row of pages: positions a chunk past its end are formed in 32 bits
constexpr int64_t kMaxGroups = 1 << 23;           // workgroups of a launch, which has 32 bits of threads
bool tokens_fit(int64_t T, int64_t heads) { return T >= 1 && T <= (1 << 29) && T * heads <= (1 << 29); }
// x / n = (x * magic) >> 20 for x < n + 128, n <= 512: x times the excess of magic (below n / 2^20) stays under 1 / n
uint32_t magic_of(int64_t n) { return (uint32_t)(((1 << 20) + n - 1) / n); }

jet_status check_cache(const jet_kv_cache* c) {
    if (!c->k || !c->v) return JET_ERR_NULL;
    if ((c->k_scale == nullptr) != (c->v_scale == nullptr)) return JET_ERR_ARG;
    if (c->n_pages < 1 || c->n_pages > INT32_MAX || c->n_kv < 1 || c->n_kv > 65535 || (c->dim != 64 && c->dim != 128)) return JET_ERR_SHAPE;
    if (c->page < 16 || c->page % 16 || c->page > 65536) return JET_ERR_SHAPE;
    if (misaligned(c->k) || misaligned(c->v) || misaligned(c->k_scale) || misaligned(c->v_scale)) return JET_ERR_ALIGN;
    return JET_OK;
}

// shared by the two passes over packed sequences
jet_status attention_args(jet::AttentionArgs& a, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                          const int32_t* cu_q, const int32_t* cu_k, int64_t n_seqs, int64_t Tq, int64_t Tk, int64_t n_q,
                          int64_t n_kv, int64_t dim, float scale) {
    if (!q || !k || !v || !cu_q || !cu_k) return JET_ERR_NULL;
    if (!(scale > 0.0f) || scale > 3.0e38f) return JET_ERR_ARG;
    if (!heads_fit(n_q, n_kv, dim) || !tokens_fit(Tq, n_q) || !tokens_fit(Tk, n_kv)) return JET_ERR_SHAPE;
    if (n_seqs < 1 || n_seqs > (1 << 20)) return JET_ERR_SHAPE;
    // the grid: a workgroup for every tile of rows and key/value head
    if ((Tq * (n_q / n_kv) / 64 + n_seqs + 2) * n_kv > kMaxGroups) return JET_ERR_SHAPE;
    if (!row_fits(ldq, n_q, dim) || !row_fits(ldk, n_kv, dim) || !row_fits(ldv, n_kv, dim)) return JET_ERR_SHAPE;
    if (misaligned(q) || misaligned(k) || misaligned(v)) return JET_ERR_ALIGN;
    a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.ldq = ldq;
    a.ldk = ldk;
    a.ldv = ldv;
    a.sq = {cu_q, (int)n_seqs, (int)Tq};
    a.sk = {cu_k, (int)n_seqs, (int)Tk};
    a.n_q = (int)n_q;
    a.n_kv = (int)n_kv;
    a.group = (int)(n_q / n_kv);
    a.group_magic = magic_of(a.group);
    a.scale = scale;
    return JET_OK;
}

// shared by the norm and rotation of heads and its gradient
jet_status qk_args(jet::QkArgs& a, int64_t T, int64_t n_q, int64_t n_kv, int64_t dim, const float* table, int64_t table_rows,
                   const int32_t* positions, const void* gamma_q, const void* gamma_k, float eps) {
    if (!table || !positions) return JET_ERR_NULL;
    if ((gamma_q == nullptr) != (gamma_k == nullptr)) return JET_ERR_ARG;
    if (!(eps >= 0.0f) || eps > 3.0e38f) return JET_ERR_ARG;
    if (n_q < 1 || n_kv < 1 || n_q > 65535 || n_kv > 65535 || (dim != 64 && dim != 128) || table_rows < 1 || table_rows > INT32_MAX)
        return JET_ERR_SHAPE;
    if (!tokens_fit(T, n_q + 2 * n_kv)) return JET_ERR_SHAPE;
    if (misaligned(table) || misaligned(gamma_q) || misaligned(gamma_k)) return JET_ERR_ALIGN;
    a = {};
    a.T = T;
    a.n_q = (int)n_q;
    a.n_kv = (int)n_kv;
    a.table = table;
    a.table_rows = (int)table_rows;
    a.positions = positions;
    a.gamma_q = static_cast<const uint16_t*>(gamma_q);
    a.gamma_k = static_cast<const uint16_t*>(gamma_k);
    a.eps = eps;
    return JET_OK;
}

}  // namespace

extern "C" {

jet_status jet_quant_act(const void* x, const float* x_scales, jet_src src, int64_t M, int64_t K,
                         uint8_t* q_row, float* s_row, uint8_t* q_colT, float* s_colT, void* stream) {
    if (!x) return JET_ERR_NULL;
    if (src != JET_SRC_BF16 && src != JET_SRC_FP8_ROW) return JET_ERR_ARG;
    if (src == JET_SRC_FP8_ROW && !x_scales) return JET_ERR_ARG;
    const bool any_row = q_row || s_row, any_col = q_colT || s_colT;
    if (!any_row && !any_col) return JET_ERR_ARG;
    if (any_row && (!q_row || !s_row)) return JET_ERR_NULL;
    if (any_col && (!q_colT || !s_colT)) return JET_ERR_NULL;
    if (M < 1 || K < 1) return JET_ERR_SHAPE;
    if (K % 128) return JET_ERR_SHAPE;              /* row groups, FP8-source scales, 128-wide tiles */
    if (any_col && M % 128) return JET_ERR_SHAPE;
    if (M > INT32_MAX / 2 || K > INT32_MAX / 2) return JET_ERR_SHAPE;
    if (any_col && M > kMaxTileRows) return JET_ERR_SHAPE;
    if (misaligned(x) || (src == JET_SRC_FP8_ROW && misaligned(x_scales)) ||
        (any_row && (misaligned(q_row) || misaligned(s_row))) ||
        (any_col && (misaligned(q_colT) || misaligned(s_colT))))
        return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_quant_act(x, x_scales, src, M, K, q_row, s_row, q_colT, s_colT,
                                              static_cast<hipStream_t>(stream)));
}

jet_status jet_quant_weight(const void* w, int64_t N, int64_t K, uint8_t* q, float* s, uint8_t* qT,
                            float* sT, void* stream) {
    if (!w || !q || !s) return JET_ERR_NULL;
    if ((qT == nullptr) != (sT == nullptr)) return JET_ERR_ARG;
    if (N < 1 || K < 1 || N % 128 || K % 128) return JET_ERR_SHAPE;
    if (N > kMaxTileRows || K > INT32_MAX / 2) return JET_ERR_SHAPE;
    if (misaligned(w) || misaligned(q) || misaligned(s) || (qT && (misaligned(qT) || misaligned(sT))))
        return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_quant_weight(w, N, K, q, s, qT, sT, static_cast<hipStream_t>(stream)));
}

jet_status jet_fp8_linear_fwd(const uint8_t* qx, const float* sx, const uint8_t* qw, const float* sw,
                              void* y, int64_t M, int64_t N, int64_t K, void* stream) {
    return gemm_entry(qx, sx, qw, sw, jet::kSbBlock, y, M, N, K, false, stream);
}

jet_status jet_fp8_linear_dgrad(const uint8_t* qdy, const float* sdy, const uint8_t* qwT,
                                const float* swT, void* dx, int64_t M, int64_t N, int64_t K, void* stream) {
    return gemm_entry(qdy, sdy, qwT, swT, jet::kSbBlock, dx, M, K, N, false, stream);
}

jet_status jet_fp8_linear_wgrad(const uint8_t* qdyT, const float* sdyT, const uint8_t* qxT,
                                const float* sxT, void* dw, int64_t M, int64_t N, int64_t K, void* stream) {
    return gemm_entry(qdyT, sdyT, qxT, sxT, jet::kSbRow, dw, N, K, M, true, stream);
}

jet_status jet_rmsnorm_quant(const void* x, const void* gamma, float eps, int64_t M, int64_t K,
                             uint8_t* q_row, float* s_row, void* stream) {
    if (!x || !gamma || !q_row || !s_row) return JET_ERR_NULL;
    if (!(eps >= 0.0f) || eps > 3.0e38f) return JET_ERR_ARG;   /* negative, NaN or infinite */
    if (M < 1 || K < 1 || K % 128 || K > 32768 || M > INT32_MAX / 2) return JET_ERR_SHAPE;
    if (misaligned(x) || misaligned(gamma) || misaligned(q_row) || misaligned(s_row)) return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_rmsnorm_quant(x, gamma, eps, M, K, q_row, s_row, static_cast<hipStream_t>(stream)));
}

jet_status jet_silu_mul_quant(const void* gate, const void* up, int64_t ld, int64_t M, int64_t K,
                              uint8_t* q_row, float* s_row, void* stream) {
    if (!gate || !up || !q_row || !s_row) return JET_ERR_NULL;
    if (M < 1 || K < 1 || K % 128 || ld < K || ld % 8) return JET_ERR_SHAPE;
    if (M > INT32_MAX / 2 || K > INT32_MAX / 2 || ld > INT32_MAX / 2) return JET_ERR_SHAPE;
    if (misaligned(gate) || misaligned(up) || misaligned(q_row) || misaligned(s_row)) return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_silu_mul_quant(gate, up, ld, M, K, q_row, s_row, static_cast<hipStream_t>(stream)));
}

jet_status jet_silu_mul_bwd(const void* gate, const void* up, int64_t ld, const void* dh, int64_t M, int64_t K,
                            void* dgate, void* dup, int64_t ld_out, void* stream) {
    if (!gate || !up || !dh || !dgate || !dup) return JET_ERR_NULL;
    if (M < 1 || K < 1 || K % 128 || ld < K || ld % 8 || ld_out < K || ld_out % 8) return JET_ERR_SHAPE;
    if (M > INT32_MAX / 2 || K > INT32_MAX / 2 || ld > INT32_MAX / 2 || ld_out > INT32_MAX / 2) return JET_ERR_SHAPE;
    if (misaligned(gate) || misaligned(up) || misaligned(dh) || misaligned(dgate) || misaligned(dup)) return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_silu_mul_bwd(gate, up, ld, dh, M, K, dgate, dup, ld_out, static_cast<hipStream_t>(stream)));
}

jet_status jet_silu_mul_bwd_quant(const void* gate, const void* up, int64_t ld, const void* dh, int64_t M, int64_t K, void* dgu,
                                  uint8_t* q_row, float* s_row, uint8_t* q_colT, float* s_colT, void* stream) {
    if (!gate || !up || !dh || !dgu || !q_row || !s_row || !q_colT || !s_colT) return JET_ERR_NULL;
    if (M < 1 || K < 1 || M % 128 || K % 128 || ld < K || ld % 8) return JET_ERR_SHAPE;
    if (M > kMaxTileRows || K > INT32_MAX / 4 || ld > INT32_MAX / 2) return JET_ERR_SHAPE;
    if (misaligned(gate) || misaligned(up) || misaligned(dh) || misaligned(dgu) || misaligned(q_row) || misaligned(s_row) ||
        misaligned(q_colT) || misaligned(s_colT))
        return JET_ERR_ALIGN;
    discard_stale_error();
    return after_launch(jet::launch_silu_mul_bwd_quant(gate, up, ld, dh, M, K, dgu, q_row, s_row, q_colT, s_colT,
                                                       static_cast<hipStream_t>(stream)));
}

jet_status jet_qk_norm_rope(const void* qkv, int64_t ld, int64_t T, int64_t n_q, int64_t n_kv, int64_t dim, const float* table,
                            int64_t table_rows, const int32_t* positions, const void* gamma_q, const void* gamma_k, float eps,
                            void* q, void* k, const jet_kv_cache* cache, const int64_t* slots, void* stream) {
    if (!qkv || !q || !k) return JET_ERR_NULL;
    if ((cache == nullptr) != (slots == nullptr)) return JET_ERR_ARG;
    jet::QkArgs a;
    jet_status st = qk_args(a, T, n_q, n_kv, dim, table, table_rows, positions, gamma_q, gamma_k, eps);
    if (st != JET_OK) return st;
    if (!row_fits(ld, n_q + 2 * n_kv, dim)) return JET_ERR_SHAPE;
    if (misaligned(qkv) || misaligned(q) || misaligned(k)) return JET_ERR_ALIGN;
    a.qkv = static_cast<const uint16_t*>(qkv);
    a.ld = ld;
    a.q = static_cast<uint16_t*>(q);
    a.k = static_cast<uint16_t*>(k);
    if (cache) {
        st = check_cache(cache);
        if (st != JET_OK) return st;
        if (cache->n_kv != n_kv || cache->dim != dim) return JET_ERR_SHAPE;
        a.slots = slots;
        a.cache_k = cache->k;
        a.cache_v = cache->v;
        a.k_scale = cache->k_scale;
        a.v_scale = cache->v_scale;
        a.n_pages = cache->n_pages;
        a.page = (int)cache->page;
    }
    discard_stale_error();
    return after_launch(jet::launch_qk_norm_rope(a, (int)dim, static_cast<hipStream_t>(stream)));
}

int64_t jet_qk_norm_rope_bwd_workspace(int64_t T, int64_t n_q, int64_t n_kv, int64_t dim) {
    if (T < 1 || n_q < 1 || n_kv < 1 || (dim != 64 && dim != 128)) return 0;
    return jet::qk_bwd_workspace(T, n_q, n_kv, dim);
}

jet_status jet_qk_norm_rope_bwd(const void* dq, const void* dk, const void* qkv, int64_t ld, int64_t T, int64_t n_q, int64_t n_kv,
                                int64_t dim, const float* table, int64_t table_rows, const int32_t* positions, const void* gamma_q,
                                const void* gamma_k, float eps, void* dx, int64_t ld_dx, float* dgamma_q, float* dgamma_k,
                                void* workspace, void* stream) {
    if (!dq || !dk || !dx) return JET_ERR_NULL;
    const bool norm = gamma_q && gamma_k;
    if (norm && (!qkv || !dgamma_q || !dgamma_k || !workspace)) return JET_ERR_NULL;
    if (!norm && (dgamma_q || dgamma_k)) return JET_ERR_ARG;
    jet::QkArgs a;
    const jet_status st = qk_args(a, T, n_q, n_kv, dim, table, table_rows, positions, gamma_q, gamma_k, eps);
    if (st != JET_OK) return st;
    if ((norm && !row_fits(ld, n_q + 2 * n_kv, dim)) || !row_fits(ld_dx, n_q + n_kv, dim)) return JET_ERR_SHAPE;
    if (misaligned(dq) || misaligned(dk) || misaligned(qkv) || misaligned(dx) || misaligned(dgamma_q) || misaligned(dgamma_k) ||
        misaligned(workspace))
        return JET_ERR_ALIGN;
    a.qkv = static_cast<const uint16_t*>(qkv);
    a.ld = ld;
    a.dq = static_cast<const uint16_t*>(dq);
    a.dk = static_cast<const uint16_t*>(dk);
    a.dx = static_cast<uint16_t*>(dx);
    a.ld_dx = ld_dx;
    discard_stale_error();
    return after_launch(jet::launch_qk_norm_rope_bwd(a, (int)dim, dgamma_q, dgamma_k, workspace, static_cast<hipStream_t>(stream)));
}

jet_status jet_attention_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* cu_q,
                             const int32_t* cu_k, int64_t n_seqs, int64_t Tq, int64_t Tk, int64_t n_q, int64_t n_kv, int64_t dim,
                             float scale, int causal, void* o, float* lse, void* stream) {
    if (!o || !lse) return JET_ERR_NULL;
    jet::AttentionArgs a;
    const jet_status st = attention_args(a, q, ldq, k, ldk, v, ldv, cu_q, cu_k, n_seqs, Tq, Tk, n_q, n_kv, dim, scale);
    if (st != JET_OK) return st;
    if (misaligned(o) || misaligned(lse)) return JET_ERR_ALIGN;
    a.o = static_cast<uint16_t*>(o);
    a.lse = lse;
    discard_stale_error();
    return after_launch(jet::launch_attention_fwd(a, (int)dim, causal != 0, static_cast<hipStream_t>(stream)));
}

int64_t jet_attention_bwd_workspace(int64_t n_seqs, int64_t Tq, int64_t Tk, int64_t n_q, int64_t n_kv, int64_t dim) {
    if (n_seqs < 1 || !heads_fit(n_q, n_kv, dim) || !tokens_fit(Tq, n_q) || !tokens_fit(Tk, n_kv)) return 0;
    return jet::attention_bwd_workspace(n_seqs, Tq, Tk, n_q, n_kv, dim);
}

jet_status jet_attention_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* o,
                             const float* lse, const void* dout, const int32_t* cu_q, const int32_t* cu_k, int64_t n_seqs,
                             int64_t Tq, int64_t Tk, int64_t n_q, int64_t n_kv, int64_t dim, float scale, int causal, void* dq,
                             int64_t ld_dq, void* dk, int64_t ld_dk, void* dv, int64_t ld_dv, void* workspace, void* stream) {
    if (!o || !lse || !dout || !dq || !dk || !dv || !workspace) return JET_ERR_NULL;
    jet::AttentionArgs a;
    const jet_status st = attention_args(a, q, ldq, k, ldk, v, ldv, cu_q, cu_k, n_seqs, Tq, Tk, n_q, n_kv, dim, scale);
    if (st != JET_OK) return st;
    if ((Tk / 16 + 8 * (n_seqs + 2)) * n_kv > kMaxGroups) return JET_ERR_SHAPE;        // up to eight workgroups for a tile of keys
    if (!row_fits(ld_dq, n_q, dim) || !row_fits(ld_dk, n_kv, dim) || !row_fits(ld_dv, n_kv, dim)) return JET_ERR_SHAPE;
    if (misaligned(o) || misaligned(lse) || misaligned(dout) || misaligned(dq) || misaligned(dk) || misaligned(dv) || misaligned(workspace))
        return JET_ERR_ALIGN;
    a.o = static_cast<uint16_t*>(const_cast<void*>(o));
    a.lse = const_cast<float*>(lse);
    a.dout = static_cast<const uint16_t*>(dout);
    a.dq = static_cast<uint16_t*>(dq);
    a.dk = static_cast<uint16_t*>(dk);
    a.dv = static_cast<uint16_t*>(dv);
    a.ld_dq = ld_dq;
    a.ld_dk = ld_dk;
    a.ld_dv = ld_dv;
    discard_stale_error();
    return after_launch(jet::launch_attention_bwd(a, (int)dim, causal != 0, workspace, static_cast<hipStream_t>(stream)));
}

int64_t jet_attention_decode_workspace(const jet_kv_cache* cache, int64_t B, int64_t n_q, int64_t max_pages) {
    if (!cache || check_cache(cache) != JET_OK || !heads_fit(n_q, cache->n_kv, cache->dim) || !tokens_fit(B, n_q)) return 0;
    if (max_pages < 1 || max_pages > kMaxTokens / cache->page) return 0;
    return jet::attention_decode_workspace(B, n_q, cache->n_kv, cache->dim, cache->k_scale != nullptr, cache->page * max_pages);
}

jet_status jet_attention_decode(const void* q, int64_t ldq, int64_t n_q, const jet_kv_cache* cache, const int32_t* pages, int64_t max_pages,
                                const int32_t* lengths, int64_t B, float scale, void* o, void* workspace, void* stream) {
    if (!q || !cache || !pages || !lengths || !o) return JET_ERR_NULL;
    const jet_status st = check_cache(cache);
    if (st != JET_OK) return st;
    if (!(scale > 0.0f) || scale > 3.0e38f) return JET_ERR_ARG;
    if (!heads_fit(n_q, cache->n_kv, cache->dim) || !tokens_fit(B, n_q) || !row_fits(ldq, n_q, cache->dim)) return JET_ERR_SHAPE;
    if (max_pages < 1 || max_pages > kMaxTokens / cache->page) return JET_ERR_SHAPE;
    const bool fp8 = cache->k_scale != nullptr;
    if (jet::attention_decode_groups(B, n_q, cache->n_kv, cache->dim, fp8, cache->page * max_pages) > kMaxGroups) return JET_ERR_SHAPE;
    if (misaligned(q) || misaligned(o) || misaligned(workspace)) return JET_ERR_ALIGN;
    if (!workspace && jet::attention_decode_workspace(B, n_q, cache->n_kv, cache->dim, fp8, cache->page * max_pages)) return JET_ERR_NULL;
    jet::DecodeArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.ldq = ldq;
    a.k = static_cast<const char*>(cache->k);
    a.v = static_cast<const char*>(cache->v);
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    a.n_pages = cache->n_pages;
    a.page = (int)cache->page;
    a.pages = pages;
    a.max_pages = (int)max_pages;
    a.lengths = lengths;
    a.B = (int)B;
    a.n_q = (int)n_q;
    a.n_kv = (int)cache->n_kv;
    a.group = (int)(n_q / cache->n_kv);
    a.scale = scale;
    a.o = static_cast<uint16_t*>(o);
    discard_stale_error();
    return after_launch(jet::launch_attention_decode(a, (int)cache->dim, fp8, workspace, static_cast<hipStream_t>(stream)));
}

const char* jet_status_str(jet_status st) {
    switch (st) {
        case JET_OK: return "ok";
        case JET_ERR_NULL: return "required pointer is NULL";
        case JET_ERR_SHAPE: return "size < 1 or not a multiple of 128 where required";
        case JET_ERR_ALIGN: return "pointer not 16-byte aligned";
        case JET_ERR_ARG: return "bad enum value or inconsistent optional arguments";
        case JET_ERR_LAUNCH: return "HIP launch failed";
    }
    return "unknown status";
}

int jet_version(void) { return 103; }

}  // extern "C"

// Attention of packed sequences, forward:  o_i = sum_j p_ij v_j,  p_ij = e^(s_ij - lse_i),  s_ij = scale q_i k_j,
// lse_i = ln sum_j e^s_ij over the keys j that row i sees.
#include "jet_attn.h"
#include "jet_internal.h"

namespace jet {

// A workgroup has 128 rows of one sequence and one key/value head: the query heads that share it are rows of their own, token by
// token (row = token * group + head), so that a short sequence fills a tile and the keys are read once for the whole group.  A wave
// has 32 rows, as the columns of the transposed products: S^T = K Q^T (a lane holds half the scores of ONE row, so the
// softmax needs one exchange with lane ^ 32), then O^T = V^T P^T.  Scores in units of log2: 2^(s scale log2 e - m).
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256, 2) attention_fwd_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BN = 64, kTile = BN * T::kRowBytes, kCopies = BN / T::kRowsPerCopy / 4;
    __shared__ __attribute__((aligned(128))) char lds[4 * kTile];   // K, V; K, V
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int kvh = blockIdx.x % a.n_kv, tile = gridDim.x / a.n_kv - 1 - blockIdx.x / a.n_kv;

    int first;
    const int s = sequence_of(a.sq, tile, 128, a.group, l, &first);
    const int q0 = a.sq.bound(s), n = a.sq.bound(s + 1) - q0, rows = n * a.group, row0 = (tile - first) * 128;
    if (n <= 0 || row0 < 0 || row0 >= rows) return;
    const bool outside = s == 0 || s == a.sq.n + 1;
    const int k0 = outside ? 0 : a.sk.bound(s), m = outside ? 0 : max(0, a.sk.bound(s + 1) - k0);
    const int off = m - n;                                            // the last row of a sequence sees its last key

    const int tok0 = row0 / a.group, rem0 = row0 - tok0 * a.group;
    const int row = min(w * 32 + (l & 31), rows - 1 - row0);          // rows past the end repeat the last one
    const bool valid = row == w * 32 + (l & 31);
    const int x = rem0 + row, dt = (int)(x * a.group_magic >> 20), head = kvh * a.group + x - dt * a.group;
    const int token = tok0 + dt;
    const int lim = CAUSAL ? min(m - 1, token + off) : m - 1;         // the last key that the row sees
    const int lim_first = __builtin_amdgcn_readlane(lim, 0), lim_last = __builtin_amdgcn_readlane(lim, 31);
    const int last_token = (min(row0 + 127, rows - 1)) / a.group;
    const int kv_end = __builtin_amdgcn_readfirstlane(CAUSAL ? max(0, min(m, last_token + off + 1)) : m);

    bf16x8 qf[T::kK];
    const uint16_t* qp = a.q + (long)(q0 + token) * a.ldq + head * DIM + 8 * h;
#pragma unroll
    for (int i = 0; i < T::kK; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(qp + 16 * i);

    const uint32_t lds0 = lds_address(lds);
    auto copy = [&](int key0, int buf) {
        const int nr = min(BN, kv_end - key0);
        const i32x4 kb = buffer_of(a.k + (long)(k0 + key0) * a.ldk + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldk + DIM) * 2);
        const i32x4 vb = buffer_of(a.v + (long)(k0 + key0) * a.ldv + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldv + DIM) * 2);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t r = (w * kCopies + c) * T::kRowsPerCopy + l / T::kChunks;
            const uint32_t chunk = ((l % T::kChunks) ^ swizzle(r)) * 16;
            const uint32_t at = lds0 + 2 * buf * kTile + (w * kCopies + c) * 1024;
            copy16(at, kb, r * (uint32_t)a.ldk * 2 + chunk);
            copy16(at + kTile, vb, r * (uint32_t)a.ldv * 2 + chunk);
        }
    };

    f32x16 o[T::kC];
#pragma unroll
    for (int c = 0; c < T::kC; ++c) o[c] = zero16();
    float m2 = -INFINITY, ref = 0.0f, sum = 0.0f;                     // largest score so far, the one subtracted, sum of p
    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);

    if (kv_end > 0) copy(0, 0);
    for (int key0 = 0, buf = 0; key0 < kv_end; key0 += BN, buf ^= 1) {
        wait_copies<0>();
        block_sync();
        if (key0 + BN < kv_end) copy(key0 + BN, buf ^ 1);
        if (key0 > lim_last) continue;
        const char* kt = lds + 2 * buf * kTile;
        const char* vt = kt + kTile;
        f32x16 sc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            sc[b] = zero16();
#pragma unroll
            for (int i = 0; i < T::kK; ++i) sc[b] = mfma32(T::row_frag(kt, rb, b, i), qf[i], sc[b]);
        }
        if (key0 + BN - 1 > lim_first) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3) > lim) sc[b][i] = -INFINITY;
        }
        float top = sc[0][0];
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(fmaxf(top, sc[0][i]), sc[1][i]);
        top = half_max(top) * c2;
        // A new reference only where a score is 2^8 over the old one: p then stays below 2^8, which costs nothing in a
        // floating-point sum, and most tiles rescale nothing.
        if (__any(top > m2 + 8.0f)) {
            const float old = m2;                                     // -inf in front of the first: nothing to rescale
            m2 = fmaxf(m2, top);
            const float next = m2 == -INFINITY ? 0.0f : m2;
            const float f = exp2_hw(old - next);
            ref = next;
            sum *= f;
#pragma unroll
            for (int c = 0; c < T::kC; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[c][i] *= f;
        }
        float part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[b][i] = exp2_hw(__builtin_fmaf(sc[b][i], c2, -ref));
                part[i & 3] += sc[b][i];
            }
        sum += (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bf16x8 p = to_operand(sc[k >> 1], k & 1);   // p rounded to bf16: 2^-9 of each term, of either sign
#pragma unroll
            for (int c = 0; c < T::kC; ++c) o[c] = mfma32(T::col_frag(vt, cb, k, c), p, o[c]);
        }
    }
    sum = half_sum(sum);
    store_row<DIM>(a.o + ((long)(q0 + token) * a.n_q + head) * DIM, o, sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f, h, valid);
    if (valid && h == 0)
        a.lse[(long)head * a.sq.rows + q0 + token] = sum == 0.0f ? -INFINITY : (ref + log2_hw(sum)) * kLn2;
}

hipError_t launch_attention_fwd(const AttentionArgs& a, int dim, bool causal, hipStream_t st) {
    const dim3 grid((unsigned)(tiles_of((long)a.sq.rows * a.group, 128, a.sq.n) * a.n_kv));
    const auto kernel = dim == 128 ? (causal ? attention_fwd_kernel<128, true> : attention_fwd_kernel<128, false>)
                                   : (causal ? attention_fwd_kernel<64, true> : attention_fwd_kernel<64, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace jet

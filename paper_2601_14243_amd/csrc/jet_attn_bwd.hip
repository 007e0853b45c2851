// Attention of packed sequences, backward.  With p_ij = e^(scale q_i k_j - lse_i) recomputed from the saved logarithms,
//   dp_ij = do_i v_j,   delta_i = sum_j p_ij dp_ij = do_i o_i,   ds_ij = p_ij (dp_ij - delta_i),
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i,
// the sums of dk and dv over the rows of all query heads that share the head.  Two kernels, one for sums over keys and one for
// sums over rows, seven products in place of the five that one kernel with atomic sums of dq would take: the order of every
// sum is fixed, so that the same inputs give the same bytes.  (Atomic sums of dq would move rows * keys / 128 * 512 bytes for each head, 4.3 GB
// at 8192 tokens and 32 heads: at the rate of a copy about what the two products take.  That is an estimate, no such kernel was built.)
// Both are bound by power, as the forward pass.  One sequence of 8192 tokens, 32 query and 8 key heads of 128, deviation 1.5: dq 0.82 to 0.88
// ms (0.82 TFLOP, 0.94 to 1.0 PFLOP/s, matrix cores busy 59 % of the cycles; 0.70 ms and 68 % without the correction of delta below), dk
// and dv 1.01 to 1.06 ms (1.10 TFLOP, 1.05 PFLOP/s, 66 %), their join 28 us.
#include <algorithm>
#include <type_traits>

#include "jet_attn.h"
#include "jet_internal.h"

namespace jet {

// A row's query and output gradient, delta = do o and lse in units of log2 (+inf for a row that sees no key, so that 2^(s - lse) is 0).
template <int DIM>
__device__ __forceinline__ void load_row(const AttentionArgs& a, const QueryRow& r, int l, bf16x8 (&qf)[DIM / 16], bf16x8 (&df)[DIM / 16],
                                         float& delta, float& lse2) {
    const int h = l >> 5;
    const uint16_t* qp = a.q + (long)(r.q0 + r.token) * a.ldq + r.head * DIM + 8 * h;
    const long dense = ((long)(r.q0 + r.token) * a.n_q + r.head) * DIM;
    delta = 0.0f;
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) {
        qf[i] = *reinterpret_cast<const bf16x8*>(qp + 16 * i);
        df[i] = *reinterpret_cast<const bf16x8*>(a.dout + dense + 8 * h + 16 * i);
        const bf16x8 of = *reinterpret_cast<const bf16x8*>(a.o + dense + 8 * h + 16 * i);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)df[i][j], (float)of[j], delta);
    }
    delta = half_sum(delta);
    const float lse = a.lse[(long)r.head * a.sq.rows + r.q0 + r.token];
    lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
}
// The statistics also go to the second kernel, in the order of the rows, delta with its sign turned.  Where they go is formed here, from
// what is uniform: a lane's own address would be kept over the loop in front.
__device__ __forceinline__ void leave_row(const AttentionArgs& a, const QueryRow& r, int kvh, int wave_row, int l, float delta, float lse2) {
    uint32_t at = wave_row + l;
    asm volatile("" : "+v"(at));
    const long first = ((long)kvh * a.sq.rows + r.q0) * a.group + r.row0;
    if (l < 32 && (int)at < r.rows - r.row0) {
        a.row_lse[first + at] = lse2;
        a.row_delta[first + at] = -delta;
    }
}

// The o of the forward pass is rounded to bf16, and with it delta = do o.  Where a row's probability lies on few keys, dp - delta is a small
// difference of large numbers and that rounding is most of its error, so delta is corrected, in one of two ways.
// Rows of tiles that see up to kExact keys form delta as sum_j p_ij dp_ij, in a pass over the keys of its own: dq and dk of sequences of 2
// tokens were off by 5.2e-3 in the 2-norm, now 2.4e-3, which is what rounding ds and the results comes to.  1 us of a short call (37 tokens,
// 32 heads of 128: 17.6 -> 18.8 us).
// Beyond, that pass would be two products more.  With delta' = do o and ds' = p (dp - delta'), as the probabilities sum to 1,
// e = sum_j ds'_ij = delta_i - delta'_i: the pass that forms dq has the correction at its end, and the second kernel gets the corrected
// delta.  dq itself lacks e sum_j p_ij k_j.  That is let be where |e| is up to half a step of bf16 of sum_j |ds'_ij|, which is
// what rounding ds to bf16 may come to; a wave with a row beyond goes over its keys again.
// One sequence, 8 heads of 128, queries and keys of standard deviation 1.5 / 2.5 / 4, dq in the 2-norm against 64 bits, 10^-3: 1024 tokens
// 2.59 / 3.96 / 5.23 -> 2.51 / 2.38 / 2.34, 4096 tokens 2.57 / 4.35 / 6.02 -> 2.52 / 2.40 / 2.40; single rows were off by several times
// their gradient.  All gradients, 32 and 8 heads, deviation 1 / 1.5 / 2.5, us: 8192 tokens 1697 / 1724 / 1751 -> 1739 / 1827 / 2530 (the
// sums alone 2.5 %), 1000 tokens, where all tiles run at a time, 80 / 78 / 77 -> 83 / 107 / 108.
// With a quarter of a step as the limit dq at 1.5 would be off by 2.41 and 2.44 in place of 2.51 and 2.52, and 8192 tokens take 1957 in place of 1864
// (one box).
constexpr int kExact = 256;
constexpr float kHalfStep = 0x1p-8f;

// a lane's half of that sum over a block of 32 keys
template <int DIM>
__device__ __forceinline__ float delta_of(const char* kt, const char* vt, uint32_t rb, const bf16x8 (&qf)[DIM / 16], const bf16x8 (&df)[DIM / 16],
                                          float c2, float lse2, int left) {
    using T = Tile<DIM>;
    f32x16 sc = zero16(), dp = zero16();
#pragma unroll
    for (int i = 0; i < T::kK; ++i) sc = mfma32(T::row_frag(kt, rb, 0, i), qf[i], sc);
#pragma unroll
    for (int i = 0; i < T::kK; ++i) dp = mfma32(T::row_frag(vt, rb, 0, i), df[i], dp);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        sum += 8 * (i >> 2) + (i & 3) > left ? 0.0f : exp2_hw(__builtin_fmaf(sc[i], c2, -lse2)) * dp[i];
    return sum;
}

// A block of 32 keys (keys, then values, at kt) by itself: ds of this lane's row, which goes to dq and to the sums.  A row that sees one key
// has p = 1 whatever its score: no gradient, not the rounding of dp - delta.
template <int DIM>
__device__ __forceinline__ void dq_block(const char* kt, int key0, uint32_t rb, uint32_t cb, const bf16x8 (&qf)[DIM / 16],
                                         const bf16x8 (&df)[DIM / 16], float c2, float lse2, float delta, int lim, int lim_first, int h,
                                         f32x16 (&dq)[DIM / 32], float& sum_ds, float& sum_abs) {
    using T = Tile<DIM>;
    constexpr int BN = 32, kTile = BN * T::kRowBytes;
    f32x16 sc = zero16(), dp = zero16();
#pragma unroll
    for (int i = 0; i < T::kK; ++i) sc = mfma32(T::row_frag(kt, rb, 0, i), qf[i], sc);
#pragma unroll
    for (int i = 0; i < T::kK; ++i) dp = mfma32(T::row_frag(kt + kTile, rb, 0, i), df[i], dp);
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = exp2_hw(__builtin_fmaf(sc[i], c2, -lse2)) * (dp[i] - delta);
    if (key0 + BN - 1 > lim_first) {
        const int left = lim == 0 ? -1 : lim - key0 - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (8 * (i >> 2) + (i & 3) > left) sc[i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        sum_ds += sc[i];
        sum_abs += fabsf(sc[i]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const bf16x8 p = to_operand(sc, k);
#pragma unroll
        for (int c = 0; c < T::kC; ++c) dq[c] = mfma32(T::col_frag(kt, cb, k, c), p, dq[c]);
    }
}

// dq; rows and tiles as in the forward pass.  It also leaves the rows' statistics for the second kernel.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256, 2) attention_dq_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BN = 32, kTile = BN * T::kRowBytes, kCopies = BN / T::kRowsPerCopy / 4;
    __shared__ __attribute__((aligned(256))) char lds[8 * kTile];   // K, V; four times
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int kvh = blockIdx.x % a.n_kv, tile = gridDim.x / a.n_kv - 1 - blockIdx.x / a.n_kv;

    QueryRow r;
    if (!query_row<CAUSAL>(a, tile, 128, w * 32, kvh, l, r)) return;
    const int q0 = r.q0, k0 = r.k0, token = r.token, head = r.head, lim = r.lim, lim_first = r.lim_first, lim_last = r.lim_last, kv_end = r.kv_end;

    bf16x8 qf[T::kK], df[T::kK];
    float delta, lse2;
    load_row<DIM>(a, r, l, qf, df, delta, lse2);
    arrived(qf);
    arrived(df);

    const uint32_t lds0 = lds_address(lds);
    auto copy = [&](int key0, int slot) {
        const int nr = min(BN, kv_end - key0);
        const i32x4 kb = buffer_of(a.k + (long)(k0 + key0) * a.ldk + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldk + DIM) * 2);
        const i32x4 vb = buffer_of(a.v + (long)(k0 + key0) * a.ldv + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldv + DIM) * 2);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t key = (w * kCopies + c) * T::kRowsPerCopy + l / T::kChunks;
            const uint32_t chunk = ((l % T::kChunks) ^ T::swizzle(key)) * 16;
            const uint32_t at = lds0 + 2 * slot * kTile + (w * kCopies + c) * 1024;
            copy16(at, kb, key * (uint32_t)a.ldk * 2 + chunk);
            copy16(at + kTile, vb, key * (uint32_t)a.ldv * 2 + chunk);
        }
    };

    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);
    const int blocks = (kv_end + BN - 1) / BN, mine = lim_last < 0 ? 0 : lim_last / BN + 1;
    if (kv_end <= kExact) {
        float sum = 0.0f;
        for (int t0 = 0; t0 < blocks; t0 += 4) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t0 + t < blocks) copy((t0 + t) * BN, t);
            wait_copies<0>();
            block_sync();
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t0 + t < mine)
                    sum += delta_of<DIM>(lds + 2 * t * kTile, lds + (2 * t + 1) * kTile, rb, qf, df, c2, lse2, lim - (t0 + t) * BN - 4 * h);
            block_sync();
        }
        delta = half_sum(sum);
    }

    f32x16 dq[T::kC], sa, sb, dp;
#pragma unroll
    for (int c = 0; c < T::kC; ++c) dq[c] = zero16();
    float sum_ds = 0.0f, sum_abs = 0.0f;                     // this lane's half of a row
    constexpr int kSlots = T::kK, kPer = 16 / (kSlots - 2) + (16 % (kSlots - 2) != 0), LA = 3;   // kK = 2 kC

    // p of a block beside dP; one MFMA a slot, with the LDS reads of LA slots later and a share of the other work.  (A dP that starts from
    // - delta, as in the second kernel, would save a subtraction for each score, but its 16 registers would be spilled.)
    auto second = [&](const char* vt, f32x16& sc) {
        bf16x8 vf[kSlots];
#pragma unroll
        for (int i = 0; i < LA; ++i) vf[i] = T::row_frag(vt, rb, 0, i);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + LA < kSlots) vf[i + LA] = T::row_frag(vt, rb, 0, i + LA);
            dp = mfma32(vf[i], df[i], i == 0 ? zero16() : dp);
            if (i >= 2)
#pragma unroll
                for (int e = (i - 2) * kPer; e < min(16, (i - 1) * kPer); ++e) sc[e] = exp2_hw(__builtin_fmaf(sc[e], c2, -lse2));
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // One block of 32 keys: S of the next one (NEXT) beside ds of this one, dQ += K^T dS, then the next one's dP beside its p
    auto step = [&](auto has_next, auto which, int key0, f32x16& sc, f32x16& nx) {
        constexpr bool NEXT = decltype(has_next)::value;
        const int slot = which;                              // a constant in the loop
        const char* kt = lds + 2 * slot * kTile;
        const char* kn = lds + 2 * ((slot + 1) & 3) * kTile;
        bf16x8 kf[kSlots], cf[kSlots], pw[2];
        float block_ds = 0.0f, block_abs = 0.0f;
        nx = zero16();
        if constexpr (NEXT)
#pragma unroll
            for (int i = 0; i < LA; ++i) kf[i] = T::row_frag(kn, rb, 0, i);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if constexpr (NEXT) {
                if (i + LA < kSlots) kf[i + LA] = T::row_frag(kn, rb, 0, i + LA);
                nx = mfma32(kf[i], qf[i], nx);
            }
            if (i + LA >= kSlots) cf[i + LA - kSlots] = T::col_frag(kt, cb, (i + LA - kSlots) / T::kC, (i + LA - kSlots) % T::kC);
            if (i >= 1)
#pragma unroll
                for (int e = (i - 1) * kPer; e < min(16, i * kPer); ++e) {
                    sc[e] *= dp[e] - delta;
                    block_ds += sc[e];
                    block_abs += fabsf(sc[e]);
                    asm volatile("" : "+v"(block_ds), "+v"(block_abs));   // one chain each, in this order: else they cost 20 registers
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (key0 + BN - 1 > lim_first) {
            // a row that sees one key has p = 1 whatever its score: no gradient, not the rounding of dp - delta
            int left = lim == 0 ? -1 : lim - key0 - 4 * h;
            asm volatile("" : "+v"(left));
            block_ds = block_abs = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (8 * (i >> 2) + (i & 3) > left) sc[i] = 0.0f;
                block_ds += sc[i];
                block_abs += fabsf(sc[i]);
            }
        }
        sum_ds += block_ds;
        sum_abs += block_abs;
        pw[0] = to_operand(sc, 0);                            // ds rounded to bf16: 2^-8 of each term at most, of either sign
        pw[1] = to_operand(sc, 1);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + LA < kSlots) cf[i + LA] = T::col_frag(kt, cb, (i + LA) / T::kC, (i + LA) % T::kC);
            dq[i % T::kC] = mfma32(cf[i], pw[i / T::kC], dq[i % T::kC]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (NEXT) second(kn + kTile, nx);
    };

    // four buffers: in step t block t + 1 is there, t + 2 under way, and t + 3 follows into the buffer of t - 1
    auto turn = [&](int t) {
        if (t + 2 < blocks) wait_copies<2 * kCopies>();
        else wait_copies<0>();
        block_sync();
        if (t + 3 < blocks) copy((t + 3) * BN, (t + 3) & 3);
    };
#pragma unroll
    for (int t = 0; t < 3; ++t)
        if (t < blocks) copy(t * BN, t);
    if (blocks > 0) {
        if (blocks > 2) wait_copies<4 * kCopies>();
        else wait_copies<0>();
        block_sync();
    }
    if (mine > 0) {
        sa = zero16();
#pragma unroll
        for (int i = 0; i < kSlots; ++i) sa = mfma32(T::row_frag(lds, rb, 0, i), qf[i], sa);
        second(lds + kTile, sa);
    }
    constexpr std::true_type next;
    constexpr std::false_type last;
#define JET_SLOT(I) std::integral_constant<int, I>{}
    int t = 0;
    for (; t + 4 < mine; t += 4) {                           // the buffers are constants of the addresses
        turn(t);
        step(next, JET_SLOT(0), t * BN, sa, sb);
        turn(t + 1);
        step(next, JET_SLOT(1), (t + 1) * BN, sb, sa);
        turn(t + 2);
        step(next, JET_SLOT(2), (t + 2) * BN, sa, sb);
        turn(t + 3);
        step(next, JET_SLOT(3), (t + 3) * BN, sb, sa);
    }
    for (; t + 1 < mine; ++t) {
        turn(t);
        step(next, t & 3, t * BN, sa, sb);
        sa = sb;
    }
    if (mine > 0) {
        turn(t);
        step(last, t & 3, t * BN, sa, sb);
        ++t;
    }
    for (; t < blocks; ++t) turn(t);
#undef JET_SLOT
    if (kv_end > kExact) {
        __shared__ int off[4];
        sum_ds = half_sum(sum_ds);
        delta += sum_ds;
        const bool mine_off = __any(fabsf(sum_ds) > kHalfStep * half_sum(sum_abs));
        if (l == 0) off[w] = mine_off;
        block_sync();
        if (__builtin_amdgcn_readfirstlane(off[0] | off[1] | off[2] | off[3])) {
            if (mine_off)
#pragma unroll
                for (int c = 0; c < T::kC; ++c) dq[c] = zero16();
#pragma unroll
            for (t = 0; t < 3; ++t)
                if (t < blocks) copy(t * BN, t);
            for (t = 0; t < blocks; ++t) {                   // the waves that do not need it only copy
                turn(t);
                if (mine_off && t < mine)
                    dq_block<DIM>(lds + 2 * (t & 3) * kTile, t * BN, rb, cb, qf, df, c2, lse2, delta, lim, lim_first, h, dq, sum_ds, sum_abs);
            }
        }
    }
    leave_row(a, r, kvh, w * 32, l, delta, lse2);
    store_row<DIM>(a.dq + (long)(q0 + token) * a.ld_dq + head * DIM, dq, a.scale, h, r.valid);
}

// The same for few tiles: 32 rows, every wave with every fourth block of 32 keys in buffers of its own.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256) attention_dq_few_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BN = 32, kTile = BN * T::kRowBytes, kCopies = BN / T::kRowsPerCopy, kWave = 4 * kTile;
    static_assert(kWave >= 32 * (DIM + 4) * 4, "the buffers hold the sums");
    __shared__ __attribute__((aligned(256))) char lds[4 * kWave];      // K, V; K, V of each wave
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int kvh = blockIdx.x % a.n_kv, tile = gridDim.x / a.n_kv - 1 - blockIdx.x / a.n_kv;
    QueryRow r;
    if (!query_row<CAUSAL>(a, tile, 32, 0, kvh, l, r)) return;
    bf16x8 qf[T::kK], df[T::kK];
    float delta, lse2;
    load_row<DIM>(a, r, l, qf, df, delta, lse2);
    arrived(qf);
    arrived(df);

    char* mine = lds + w * kWave;
    const uint32_t at0 = lds_address(mine);
    auto copy = [&](int key0, int buf) {
        const int nr = min(BN, r.kv_end - key0);
        const i32x4 kb = buffer_of(a.k + (long)(r.k0 + key0) * a.ldk + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldk + DIM) * 2);
        const i32x4 vb = buffer_of(a.v + (long)(r.k0 + key0) * a.ldv + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldv + DIM) * 2);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t key = c * T::kRowsPerCopy + l / T::kChunks, chunk = ((l % T::kChunks) ^ T::swizzle(key)) * 16;
            copy16(at0 + 2 * buf * kTile + c * 1024, kb, key * (uint32_t)a.ldk * 2 + chunk);
            copy16(at0 + (2 * buf + 1) * kTile + c * 1024, vb, key * (uint32_t)a.ldv * 2 + chunk);
        }
    };
    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);
    const bool held = r.kv_end <= kExact;                             // at most two blocks of each wave, which stay in its two buffers
    if (held) {
        __shared__ float halves[4][64];
        static_assert(kExact <= 2 * 4 * BN, "buffers");
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if ((w + 4 * t) * BN < r.kv_end) copy((w + 4 * t) * BN, t);
        wait_copies<0>();
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if ((w + 4 * t) * BN < r.kv_end)
                sum += delta_of<DIM>(mine + 2 * t * kTile, mine + (2 * t + 1) * kTile, rb, qf, df, c2, lse2, r.lim - (w + 4 * t) * BN - 4 * h);
        halves[w][l] = sum;
        __syncthreads();
        delta = half_sum((halves[0][l] + halves[1][l]) + (halves[2][l] + halves[3][l]));
    }
    f32x16 dq[T::kC];
    float sum_ds, sum_abs;                                            // this lane's half of a row, this wave's blocks
    auto all_blocks = [&] {
        sum_ds = sum_abs = 0.0f;
#pragma unroll
        for (int c = 0; c < T::kC; ++c) dq[c] = zero16();
        if (!held && w * BN < r.kv_end) copy(w * BN, 0);
        for (int key0 = w * BN, buf = 0; key0 < r.kv_end; key0 += 4 * BN, buf ^= 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");      // the reads of the block before are done, its buffer is free
            if (!held && key0 + 4 * BN < r.kv_end) {
                copy(key0 + 4 * BN, buf ^ 1);
                wait_copies<2 * kCopies>();
            } else {
                wait_copies<0>();
            }
            dq_block<DIM>(mine + 2 * buf * kTile, key0, rb, cb, qf, df, c2, lse2, delta, r.lim, r.lim_first, h, dq, sum_ds, sum_abs);
        }
    };
    all_blocks();
    if (!held) {
        __shared__ float all_ds[4][64], all_abs[4][64];
        all_ds[w][l] = sum_ds;
        all_abs[w][l] = sum_abs;
        __syncthreads();
        sum_ds = half_sum((all_ds[0][l] + all_ds[1][l]) + (all_ds[2][l] + all_ds[3][l]));
        sum_abs = half_sum((all_abs[0][l] + all_abs[1][l]) + (all_abs[2][l] + all_abs[3][l]));
        delta += sum_ds;
        if (__any(fabsf(sum_ds) > kHalfStep * sum_abs)) all_blocks(); // the same in all waves, which have the same rows
    }
    if (w == 0) leave_row(a, r, kvh, 0, l, delta, lse2);
    float* sums = reinterpret_cast<float*>(lds);
    __syncthreads();
    leave_sums<DIM>(sums, dq, w, l);
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * (DIM / 8); i += 256) {         // 8 channels of a row at a time
        const int row = i / (DIM / 8), ch = i % (DIM / 8) * 8;
        const int token = __shfl(r.token, row), head = __shfl(r.head, row), valid = __shfl((int)r.valid, row);
        float v[8] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += sums[(k * 32 + row) * (DIM + 4) + ch + e];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        if (valid)
            *reinterpret_cast<uint4*>(a.dq + (long)(r.q0 + token) * a.ld_dq + head * DIM + ch) =
                uint4{bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3]), bf16_pack2(v[4], v[5]), bf16_pack2(v[6], v[7])};
    }
}

__device__ __forceinline__ int pieces_of(const AttentionArgs& a, int rows) {
    return __builtin_amdgcn_readfirstlane(max(1, min(a.parts, (rows + a.part_rows - 1) / a.part_rows)));
}

// dk and dv of 128 keys of one head, a wave has 32 of them as the columns of its products; it goes over the rows that see them, 32 at
// a time: S = Q K^T and dP = dO V^T from the rows' tiles, then dV^T += dO^T P and dK^T += Q^T dS from the same tiles read
// by columns.  The keys' fragments stay in registers; the values' are read from LDS again and again, which leaves the other
// operands without spills at two workgroups a CU (2300 -> 1150 us for 8192 tokens, with the slots below).
// The rows of a tile are dealt to at most a.parts workgroups, to no more than one for each a.part_rows of them; the sums of several
// go to a.partial and are joined by a last launch.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256, 2) attention_dkdv_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BM = 32, kTile = BM * T::kRowBytes, kCopies = BM / T::kRowsPerCopy / 4, kStage = 2 * kTile + 512;
    constexpr int kKeys = 128 * T::kRowBytes;
    __shared__ __attribute__((aligned(256))) char lds[kKeys + 2 * kStage];   // V; Q, dO, lse, delta; twice
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    // the parts of a tile lie far apart in the grid: side by side, those that end at once would all be dealt to the same few CUs
    const int tile = blockIdx.x / a.n_kv, kvh = blockIdx.x - tile * a.n_kv, part = blockIdx.y;

    const Place place = place_of(a.sk, a.sq, tile, 128, 1, l);
    const int k0 = place.begin, m = place.count, q0 = place.other_begin, n = place.other_count;
    const int rows = n * a.group, key0 = (tile - place.first_tile) * 128;
    if (key0 < 0 || key0 >= m) return;
    const int off = m - n;

    const int key = key0 + w * 32 + (l & 31);
    int kk = min(key, m - 1);
    // the first row that sees the key; the first one that sees more than one key (ds of the others is 0)
    const int f_min = CAUSAL ? min(max(0, key - off) * a.group, rows) : 0;
    const int f_two = m == 1 ? rows : CAUSAL ? min(max(0, 1 - off) * a.group, rows) : 0;
    const int f_full = max(f_two, __builtin_amdgcn_readlane(f_min, 31)), f_none = __builtin_amdgcn_readlane(f_min, 0);
    const int f_first = __builtin_amdgcn_readfirstlane(CAUSAL ? min(max(0, key0 - off) * a.group, rows) : 0);
    const int pieces = pieces_of(a, rows - f_first);
    if (part >= pieces) return;
    // A piece has every pieces-th step, and goes from the last rows backwards: so the workgroups of an XCD, which have the same heads,
    // read the same rows at a time.
    const int all_steps = (rows - f_first + BM - 1) / BM, steps = (all_steps - part + pieces - 1) / pieces, stride = pieces * BM;
    const int f_last = f_first + (all_steps - 1 - part) * BM;

    const uint32_t lds0 = lds_address(lds);
    bf16x8 kf[T::kK];
    {
        const i32x4 vb = buffer_of(a.v + (long)(k0 + key0) * a.ldv + kvh * DIM, (uint32_t)((min(128, m - key0) - 1) * (int)a.ldv + DIM) * 2);
#pragma unroll
        for (int c = 0; c < 4 * kCopies; ++c) {
            const uint32_t r = (w * 4 * kCopies + c) * T::kRowsPerCopy + l / T::kChunks;
            copy16(lds0 + (w * 4 * kCopies + c) * 1024, vb, r * (uint32_t)a.ldv * 2 + ((l % T::kChunks) ^ T::swizzle(r)) * 16);
        }
#pragma unroll
        for (int i = 0; i < T::kK; ++i) kf[i] = *reinterpret_cast<const bf16x8*>(a.k + (long)(k0 + kk) * a.ldk + kvh * DIM + 8 * h + 16 * i);
    }
    // Where a lane's rows of a step lie behind the step's first token.  A step begins with a token's first head wherever the group divides
    // 32 (so do f_first and the steps): then this holds for all of them, else it is formed for each.
    uint32_t q_off[kCopies], do_off[kCopies];
    auto offsets = [&](int rem) {
        uint32_t ln = l;                                     // keeps what follows from being held over the loop
        asm volatile("" : "+v"(ln));
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t r = (w * kCopies + c) * T::kRowsPerCopy + ln / T::kChunks;
            const uint32_t x = rem + r, t = x * a.group_magic >> 20;
            const uint32_t in_row = (x - t * a.group) * T::kRowBytes + ((ln % T::kChunks) ^ T::swizzle(r)) * 16;
            q_off[c] = t * (uint32_t)a.ldq * 2 + in_row;
            do_off[c] = t * (uint32_t)a.n_q * T::kRowBytes + in_row;
        }
    };
    const bool aligned = BM % a.group == 0;
    if (aligned) offsets(0);
    auto copy = [&](int f0, int buf) {
        const int t0 = f0 / a.group, nt = min(n - t0, BM + 1);
        if (!aligned) offsets(f0 - t0 * a.group);
        const i32x4 qb = buffer_of(a.q + (long)(q0 + t0) * a.ldq + kvh * a.group * DIM, (uint32_t)((nt - 1) * (int)a.ldq + a.group * DIM) * 2);
        const i32x4 db = buffer_of(a.dout + ((long)(q0 + t0) * a.n_q + kvh * a.group) * DIM, (uint32_t)((nt - 1) * a.n_q + a.group) * DIM * 2);
        const uint32_t at0 = lds0 + kKeys + buf * kStage;
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            copy16(at0 + (w * kCopies + c) * 1024, qb, q_off[c]);
            copy16(at0 + kTile + (w * kCopies + c) * 1024, db, do_off[c]);
        }
        if (w < 2) {
            uint32_t ln = l;
            asm volatile("" : "+v"(ln));
            const float* p = (w ? a.row_delta : a.row_lse) + ((long)kvh * a.sq.rows + q0) * a.group + f0;
            copy4(at0 + 2 * kTile + w * 256, buffer_of(p, (uint32_t)min(BM, rows - f0) * 4), ln * 4);
        }
    };

    f32x16 dk[T::kC], dv[T::kC];
#pragma unroll
    for (int c = 0; c < T::kC; ++c) dk[c] = dv[c] = zero16();
    const float c2 = a.scale * kLog2e;
    const uint32_t rb0 = T::row_base(l), cb0 = T::col_base(l);

    if (steps > 0) copy(f_last, 0);
    arrived(kf);
    auto step = [&](int at, auto which) {
        constexpr int buf = decltype(which)::value;
        wait_copies<0>();
        block_sync();
        const int f0 = f_last - at * stride;
        if (at + 1 < steps) copy(f0 - stride, buf ^ 1);
        if (f0 + BM - 1 < f_none) return;
        const char* qt = lds + kKeys + buf * kStage;
        const char* dt = qt + kTile;
        const float* lt = reinterpret_cast<const float*>(qt + 2 * kTile) + 4 * h;
        // addresses are formed where they are used: kept over the loop, their 20 registers would be spilled
        uint32_t rb = rb0, cb = cb0;
        asm volatile("" : "+v"(rb), "+v"(cb));
        // The step in slots of one MFMA each, every slot with the LDS reads of two slots later and a share of the element-wise work
        // of the product before: the barriers keep the compiler from gathering the reads, which would need 64 registers more.
        bf16x8 qa[T::kK], da[T::kK], va[T::kK], dc[2 * T::kC], qc[2 * T::kC], pw[2];
        f32x16 sc = zero16(), dp;
        constexpr int kSlots = T::kK, kPer = 16 / (kSlots - 2) + (16 % (kSlots - 2) != 0);   // = 2 T::kC, too
        qa[0] = T::row_frag(qt, rb, 0, 0);
        qa[1] = T::row_frag(qt, rb, 0, 1);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + 2 < kSlots) qa[i + 2] = T::row_frag(qt, rb, 0, i + 2);
            else {
                da[i + 2 - kSlots] = T::row_frag(dt, rb, 0, i + 2 - kSlots);
                va[i + 2 - kSlots] = T::row_frag(lds, rb, w, i + 2 - kSlots);
            }
            sc = mfma32(qa[i], kf[i], sc);
            __builtin_amdgcn_sched_barrier(0);
        }
        float4 stat = *reinterpret_cast<const float4*>(lt);
#pragma unroll
        for (int g = 0; g < 4; ++g) {                        // dP - delta: the product starts from - delta
            const float4 d = *reinterpret_cast<const float4*>(lt + 64 + 8 * g);
            dp[4 * g] = d.x;
            dp[4 * g + 1] = d.y;
            dp[4 * g + 2] = d.z;
            dp[4 * g + 3] = d.w;
        }
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + 2 < kSlots) {
                da[i + 2] = T::row_frag(dt, rb, 0, i + 2);
                va[i + 2] = T::row_frag(lds, rb, w, i + 2);
            } else {
                dc[i + 2 - kSlots] = T::col_frag(dt, cb, 0, i + 2 - kSlots);
            }
            dp = mfma32(da[i], va[i], dp);
            if (i >= 2)
#pragma unroll
                for (int e = (i - 2) * kPer; e < min(16, (i - 1) * kPer); ++e) {
                    sc[e] = exp2_hw(__builtin_fmaf(sc[e], c2, -(&stat.x)[e & 3]));
                    if ((e & 3) == 3 && e < 15) stat = *reinterpret_cast<const float4*>(lt + 2 * (e + 1));
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (f0 < f_full) {
            int left = f_min - f0 - 4 * h;
            asm volatile("" : "+v"(left));
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) < left) sc[i] = 0.0f;
        }
        pw[0] = to_operand(sc, 0);
        pw[1] = to_operand(sc, 1);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + 2 < kSlots) dc[i + 2] = T::col_frag(dt, cb, (i + 2) / T::kC, (i + 2) % T::kC);
            else qc[i + 2 - kSlots] = T::col_frag(qt, cb, 0, i + 2 - kSlots);
            dv[i % T::kC] = mfma32(dc[i], pw[i / T::kC], dv[i % T::kC]);
            if (i >= 2)
#pragma unroll
                for (int e = (i - 2) * kPer; e < min(16, (i - 1) * kPer); ++e) sc[e] *= dp[e];
            __builtin_amdgcn_sched_barrier(0);
        }
        if (f0 < f_full) {
            int left = max(f_min, f_two) - f0 - 4 * h;
            asm volatile("" : "+v"(left));
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) < left) sc[i] = 0.0f;
        }
        pw[0] = to_operand(sc, 0);
        pw[1] = to_operand(sc, 1);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + 2 < kSlots) qc[i + 2] = T::col_frag(qt, cb, (i + 2) / T::kC, (i + 2) % T::kC);
            dk[i % T::kC] = mfma32(qc[i], pw[i / T::kC], dk[i % T::kC]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int at = 0; at < steps; at += 2) {                  // two steps, so that the buffers are constants of the addresses
        step(at, std::integral_constant<int, 0>{});
        if (at + 1 < steps) step(at + 1, std::integral_constant<int, 1>{});
    }
    wait_copies<0>();                                        // the values', where there was no row
    asm volatile("" : "+v"(kk));                             // the results' addresses are formed here, not in front of the loop
    const bool valid = key0 + w * 32 + (l & 31) < m;
    if (pieces > 1) {
        float* out = a.partial + (((long)part * a.sk.rows + k0 + kk) * a.n_kv + kvh) * 2 * DIM + 4 * h;
        if (valid)
#pragma unroll
            for (int c = 0; c < T::kC; ++c)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    *reinterpret_cast<float4*>(out + 32 * c + 8 * g) = float4{dk[c][4 * g], dk[c][4 * g + 1], dk[c][4 * g + 2], dk[c][4 * g + 3]};
                    *reinterpret_cast<float4*>(out + DIM + 32 * c + 8 * g) = float4{dv[c][4 * g], dv[c][4 * g + 1], dv[c][4 * g + 2], dv[c][4 * g + 3]};
                }
        return;
    }
    store_row<DIM>(a.dk + (long)(k0 + kk) * a.ld_dk + kvh * DIM, dk, a.scale, h, valid);
    store_row<DIM>(a.dv + (long)(k0 + kk) * a.ld_dv + kvh * DIM, dv, 1.0f, h, valid);
}

// The same for few tiles: 32 keys, every wave with every fourth step of 32 rows in buffers of its own.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256) attention_dkdv_few_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BM = 32, kTile = BM * T::kRowBytes, kCopies = BM / T::kRowsPerCopy, kStage = 2 * kTile + 512, kWave = 2 * kStage;
    static_assert(kWave >= 32 * (DIM + 4) * 4, "the buffers hold the sums");
    __shared__ __attribute__((aligned(256))) char lds[4 * kWave];      // Q, dO, lse, delta of each wave; twice
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int tile = blockIdx.x / a.n_kv, kvh = blockIdx.x - tile * a.n_kv, part = blockIdx.y;

    const Place place = place_of(a.sk, a.sq, tile, 32, 1, l);
    const int k0 = place.begin, m = place.count, q0 = place.other_begin, n = place.other_count;
    const int rows = n * a.group, key0 = (tile - place.first_tile) * 32;
    if (key0 < 0 || key0 >= m) return;
    const int off = m - n;
    const int key = key0 + (l & 31), kk = min(key, m - 1);
    auto first_row = [&](int k) { return CAUSAL ? min(max(0, k - off) * a.group, rows) : 0; };   // that sees key k
    const int f_min = first_row(key), f_two = m == 1 ? rows : CAUSAL ? first_row(1) : 0;
    const int f_full = max(f_two, __builtin_amdgcn_readlane(f_min, 31)), f_first = __builtin_amdgcn_readfirstlane(first_row(key0));
    const int pieces = pieces_of(a, rows - first_row(key0 & ~127));    // as the join has it, by tiles of 128
    if (part >= pieces) return;
    const int share = ((rows - f_first + pieces - 1) / pieces + BM - 1) / BM * BM;
    const int f_begin = min(rows, f_first + part * share), f_end = min(rows, f_begin + share);

    bf16x8 kf[T::kK], vf[T::kK];
#pragma unroll
    for (int i = 0; i < T::kK; ++i) {
        kf[i] = *reinterpret_cast<const bf16x8*>(a.k + (long)(k0 + kk) * a.ldk + kvh * DIM + 8 * h + 16 * i);
        vf[i] = *reinterpret_cast<const bf16x8*>(a.v + (long)(k0 + kk) * a.ldv + kvh * DIM + 8 * h + 16 * i);
    }
    char* mine = lds + w * kWave;
    const uint32_t at0 = lds_address(mine);
    auto copy = [&](int f0, int buf) {
        const int t0 = f0 / a.group, rem = f0 - t0 * a.group, nt = min(n - t0, BM + 1);
        const i32x4 qb = buffer_of(a.q + (long)(q0 + t0) * a.ldq + kvh * a.group * DIM, (uint32_t)((nt - 1) * (int)a.ldq + a.group * DIM) * 2);
        const i32x4 db = buffer_of(a.dout + ((long)(q0 + t0) * a.n_q + kvh * a.group) * DIM, (uint32_t)((nt - 1) * a.n_q + a.group) * DIM * 2);
        const uint32_t at = at0 + buf * kStage;
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t r = c * T::kRowsPerCopy + l / T::kChunks, x = rem + r, t = x * a.group_magic >> 20;
            const uint32_t in_row = (x - t * a.group) * T::kRowBytes + ((l % T::kChunks) ^ T::swizzle(r)) * 16;
            copy16(at + c * 1024, qb, t * (uint32_t)a.ldq * 2 + in_row);
            copy16(at + kTile + c * 1024, db, t * (uint32_t)a.n_q * T::kRowBytes + in_row);
        }
        const long stat = ((long)kvh * a.sq.rows + q0) * a.group + f0;
        const uint32_t bytes = (uint32_t)min(BM, rows - f0) * 4;
        copy4(at + 2 * kTile, buffer_of(a.row_lse + stat, bytes), l * 4);
        copy4(at + 2 * kTile + 256, buffer_of(a.row_delta + stat, bytes), l * 4);
    };
    f32x16 dk[T::kC], dv[T::kC];
#pragma unroll
    for (int c = 0; c < T::kC; ++c) dk[c] = dv[c] = zero16();
    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);
    arrived(kf);
    arrived(vf);
    if (f_begin + w * BM < f_end) copy(f_begin + w * BM, 0);
    for (int f0 = f_begin + w * BM, buf = 0; f0 < f_end; f0 += 4 * BM, buf ^= 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");          // the reads of the step before are done, its buffer is free
        if (f0 + 4 * BM < f_end) {
            copy(f0 + 4 * BM, buf ^ 1);
            wait_copies<2 * kCopies + 2>();
        } else {
            wait_copies<0>();
        }
        const char* qt = mine + buf * kStage;
        const char* dt = qt + kTile;
        const float* lt = reinterpret_cast<const float*>(qt + 2 * kTile) + 4 * h;
        f32x16 sc = zero16(), dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) dp[i] = lt[64 + 8 * (i >> 2) + (i & 3)];
#pragma unroll
        for (int i = 0; i < T::kK; ++i) sc = mfma32(T::row_frag(qt, rb, 0, i), kf[i], sc);
#pragma unroll
        for (int i = 0; i < T::kK; ++i) dp = mfma32(T::row_frag(dt, rb, 0, i), vf[i], dp);
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = exp2_hw(__builtin_fmaf(sc[i], c2, -lt[8 * (i >> 2) + (i & 3)]));
        const bool masked = f0 < f_full;
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) < f_min - f0 - 4 * h) sc[i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bf16x8 p = to_operand(sc, k);
#pragma unroll
            for (int c = 0; c < T::kC; ++c) dv[c] = mfma32(T::col_frag(dt, cb, k, c), p, dv[c]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] *= dp[i];
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) < max(f_min, f_two) - f0 - 4 * h) sc[i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bf16x8 p = to_operand(sc, k);
#pragma unroll
            for (int c = 0; c < T::kC; ++c) dk[c] = mfma32(T::col_frag(qt, cb, k, c), p, dk[c]);
        }
    }
    float* sums = reinterpret_cast<float*>(lds);
    auto join = [&](const f32x16(&d)[T::kC], uint16_t* out, long ld, float f, int of_partial) {
        __syncthreads();
        leave_sums<DIM>(sums, d, w, l);
        __syncthreads();
        for (int i = threadIdx.x; i < 32 * (DIM / 8); i += 256) {     // 8 channels of a key at a time
            const int row = i / (DIM / 8), ch = i % (DIM / 8) * 8;
            float v[8] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += sums[(k * 32 + row) * (DIM + 4) + ch + e];
            if (key0 + row >= m) continue;
            if (pieces > 1) {
                float* p = a.partial + (((long)part * a.sk.rows + k0 + key0 + row) * a.n_kv + kvh) * 2 * DIM + of_partial + ch;
                *reinterpret_cast<float4*>(p) = float4{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<float4*>(p + 4) = float4{v[4], v[5], v[6], v[7]};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= f;
                *reinterpret_cast<uint4*>(out + (long)(k0 + key0 + row) * ld + kvh * DIM + ch) =
                    uint4{bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3]), bf16_pack2(v[4], v[5]), bf16_pack2(v[6], v[7])};
            }
        }
    };
    join(dk, a.dk, a.ld_dk, a.scale, 0);
    join(dv, a.dv, a.ld_dv, 1.0f, DIM);
}

// dk and dv of 16 keys (blockIdx.y) of a tile and head whose rows several workgroups had, at most 8, from their sums in a fixed order
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256) attention_dkdv_join_kernel(AttentionArgs a) {
    const int tile = blockIdx.x / a.n_kv, kvh = blockIdx.x - tile * a.n_kv;
    const Place place = place_of(a.sk, a.sq, tile, 128, 1, threadIdx.x & 63);
    const int k0 = place.begin, m = place.count, n = place.other_count, rows = n * a.group, key0 = (tile - place.first_tile) * 128;
    if (key0 < 0 || key0 >= m) return;
    const int pieces = pieces_of(a, rows - (CAUSAL ? min(max(0, key0 - (m - n)) * a.group, rows) : 0));
    if (pieces == 1) return;
    const long stride = (long)a.sk.rows * a.n_kv * 2 * DIM;
    const int row0 = key0 + 16 * blockIdx.y;
#pragma unroll
    for (int i = threadIdx.x; i < 16 * (DIM / 2); i += 256) {            // 4 values of dk, dv at a time
        const int row = row0 + i / (DIM / 2), ch = i % (DIM / 2) * 4;
        if (row >= m) break;
        const float* from = a.partial + ((long)(k0 + row) * a.n_kv + kvh) * 2 * DIM + ch;
        float4 x[8], v = {0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < 8; ++p)
            if (p < pieces) x[p] = *reinterpret_cast<const float4*>(from + p * stride);
#pragma unroll
        for (int p = 0; p < 8; ++p)
            if (p < pieces) {
                v.x += x[p].x;
                v.y += x[p].y;
                v.z += x[p].z;
                v.w += x[p].w;
            }
        const float f = ch < DIM ? a.scale : 1.0f;
        uint16_t* out = ch < DIM ? a.dk + (long)(k0 + row) * a.ld_dk + kvh * DIM + ch : a.dv + (long)(k0 + row) * a.ld_dv + kvh * DIM + ch - DIM;
        *reinterpret_cast<uint2*>(out) = uint2{bf16_pack2(v.x * f, v.y * f), bf16_pack2(v.z * f, v.w * f)};
    }
}

long attention_bwd_workspace(long n_seqs, long Tq, long Tk, long n_q, long n_kv, long dim) {
    auto parts_of = [&](bool causal) { return dkdv_split(n_seqs, Tq, Tk, n_q / n_kv, n_kv, (int)dim, causal).parts; };
    const long parts = std::max(parts_of(true), parts_of(false));
    return (2 * ((Tq * n_q + 3) / 4 * 4) + (parts > 1 ? parts * Tk * n_kv * 2 * dim : 0)) * (long)sizeof(float);
}

hipError_t launch_attention_bwd(AttentionArgs a, int dim, bool causal, void* workspace, hipStream_t st) {
    const long stats = ((long)a.sq.rows * a.n_q + 3) / 4 * 4;
    a.row_lse = static_cast<float*>(workspace);
    a.row_delta = a.row_lse + stats;
    a.partial = a.row_delta + stats;
    const Split split = dkdv_split(a.sq.n, a.sq.rows, a.sk.rows, a.group, a.n_kv, dim, causal);
    a.parts = split.parts;
    a.part_rows = split.rows;
#define JET_BWD(KERNEL) (dim == 128 ? (causal ? KERNEL<128, true> : KERNEL<128, false>) : (causal ? KERNEL<64, true> : KERNEL<64, false>))
    const long rows = (long)a.sq.rows * a.group;
    const bool few_rows = few_row_tiles(a.sq.n, a.sq.rows, a.sk.rows, a.group, a.n_kv, dim);
    const dim3 row_tiles((unsigned)(tiles_of(rows, few_rows ? 32 : 128, a.sq.n) * a.n_kv));
    hipLaunchKernelGGL((few_rows ? JET_BWD(attention_dq_few_kernel) : JET_BWD(attention_dq_kernel)), row_tiles, dim3(256), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 key_tiles((unsigned)(tiles_of(a.sk.rows, split.few ? 32 : 128, a.sk.n) * a.n_kv), (unsigned)a.parts);
    hipLaunchKernelGGL((split.few ? JET_BWD(attention_dkdv_few_kernel) : JET_BWD(attention_dkdv_kernel)), key_tiles, dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    hipLaunchKernelGGL(JET_BWD(attention_dkdv_join_kernel), dim3((unsigned)(tiles_of(a.sk.rows, 128, a.sk.n) * a.n_kv), 8), dim3(256), 0, st, a);
#undef JET_BWD
    return hipGetLastError();
}

}  // namespace jet

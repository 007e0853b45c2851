// Attention of packed sequences, forward:  o_i = sum_j p_ij v_j,  p_ij = e^(s_ij - lse_i),  s_ij = scale q_i k_j,
// lse_i = ln sum_j e^s_ij over the keys j that row i sees.
#include <type_traits>

#include "jet_attn.h"
#include "jet_internal.h"

namespace jet {

// A workgroup has 128 rows of one sequence and one key/value head: the query heads that share it are rows of their own, token by
// token (row = token * group + head), so that a short sequence fills a tile and the keys are read once for the whole group.  A wave
// has 32 rows, as the columns of the transposed products: S^T = K Q^T (a lane holds half the scores of ONE row, so the
// softmax needs one exchange with lane ^ 32), then O^T = V^T P^T.  Scores in units of log2: 2^(s scale log2 e - m).
// What bounds it is power.  One sequence of 16384 tokens, 32 query and 8 key heads of 128 (2.2 TFLOP): 1.90 to 2.0 ms, 1.1 to 1.16
// PFLOP/s, the matrix cores busy 68 % of the cycles at about 1.7 GHz; on zeros in place of normal values 1.49 ms, as a library product
// of 16384 x 16384 x 8192 goes from 1.54 to 2.07 PFLOP/s.  Less work beside the MFMAs is what pays: addresses held in registers and two steps a
// turn (211 -> 150 VALU instructions a tile) gave 6 %, half of the LDS reads left out (a timing copy) 3 %.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256, 2) attention_fwd_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BN = 64, kTile = BN * T::kRowBytes, kCopies = BN / T::kRowsPerCopy / 4;
    __shared__ __attribute__((aligned(128))) char lds[4 * kTile];   // K, K, V, V
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int kvh = blockIdx.x % a.n_kv, tile = gridDim.x / a.n_kv - 1 - blockIdx.x / a.n_kv;

    QueryRow r;
    if (!query_row<CAUSAL>(a, tile, 128, w * 32, kvh, l, r)) return;
    const int q0 = r.q0, k0 = r.k0, token = r.token, head = r.head, lim = r.lim, lim_first = r.lim_first, lim_last = r.lim_last, kv_end = r.kv_end;

    bf16x8 qf[T::kK];
    const uint16_t* qp = a.q + (long)(q0 + token) * a.ldq + head * DIM + 8 * h;
#pragma unroll
    for (int i = 0; i < T::kK; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(qp + 16 * i);

    const uint32_t lds0 = lds_address(lds);
    auto copy = [&](const uint16_t* from, long ld, int key0, uint32_t at) {
        const i32x4 b = buffer_of(from + (long)(k0 + key0) * ld + kvh * DIM, (uint32_t)((min(BN, kv_end - key0) - 1) * (int)ld + DIM) * 2);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t key = (w * kCopies + c) * T::kRowsPerCopy + l / T::kChunks;
            copy16(lds0 + at + (w * kCopies + c) * 1024, b, key * (uint32_t)ld * 2 + ((l % T::kChunks) ^ T::swizzle(key)) * 16);
        }
    };

    f32x16 o[T::kC], sc[2], s2[2];
#pragma unroll
    for (int c = 0; c < T::kC; ++c) o[c] = zero16();
    float m2 = -INFINITY, ref = 0.0f, sum = 0.0f, top = -INFINITY;   // largest score so far, the one subtracted, sum of p
    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);
    const int tiles = (kv_end + BN - 1) / BN, mine = lim_last < 0 ? 0 : lim_last / BN + 1;

    auto mask = [&](f32x16 (&x)[2], int key0) {
        if (key0 + BN - 1 > lim_first) {
            int left = lim - key0 - 4 * h;
            asm volatile("" : "+v"(left));
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * b + 8 * (i >> 2) + (i & 3) > left) x[b][i] = -INFINITY;
        }
    };
    // One tile: S of the next one (NEXT) beside the exponentials of this one, then O += P V beside the maximum of the next
    // one, in slots of one MFMA with the LDS reads of two slots later and a share of the element-wise work.
    auto step = [&](auto has_next, int key0, int buf, f32x16 (&sc)[2], f32x16 (&nx)[2]) {
        constexpr bool NEXT = decltype(has_next)::value;
        const char* kt = lds + (buf ^ 1) * kTile;
        const char* vt = lds + (2 + buf) * kTile;
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
        constexpr int kA = 2 * T::kK, kB = 4 * T::kC, kE = 32 / kA;
        nx[0] = nx[1] = zero16();
        bf16x8 kf[kA], vf[kB], pw[4];
        float part[2] = {0, 0};
        constexpr int LA = 4;
        if constexpr (NEXT)
#pragma unroll
            for (int i = 0; i < LA; ++i) kf[i] = T::row_frag(kt, rb, i / T::kK, i % T::kK);
#pragma unroll
        for (int i = 0; i < kA; ++i) {
            if constexpr (NEXT) {
                if (i + LA < kA) kf[i + LA] = T::row_frag(kt, rb, (i + LA) / T::kK, (i + LA) % T::kK);
                nx[i / T::kK] = mfma32(kf[i], qf[i % T::kK], nx[i / T::kK]);
            }
            if (i + LA >= kA) vf[i + LA - kA] = T::col_frag(vt, cb, (i + LA - kA) / T::kC, (i + LA - kA) % T::kC);
#pragma unroll
            for (int e = i * kE; e < (i + 1) * kE; ++e) {
                const float p = exp2_hw(__builtin_fmaf(sc[e >> 4][e & 15], c2, -ref));
                sc[e >> 4][e & 15] = p;
                part[e & 1] += p;
                if ((e & 7) == 7) pw[e >> 3] = to_operand(sc[e >> 4], (e >> 3) & 1);   // p in bf16: 2^-8 of each term at most, of either sign
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum += part[0] + part[1];
        if constexpr (NEXT) mask(nx, key0 + BN);
        top = -INFINITY;
        constexpr int kM = 32 / kB;
#pragma unroll
        for (int i = 0; i < kB; ++i) {
            if (i + LA < kB) vf[i + LA] = T::col_frag(vt, cb, (i + LA) / T::kC, (i + LA) % T::kC);
            o[i % T::kC] = mfma32(vf[i], pw[i / T::kC], o[i % T::kC]);
            if constexpr (NEXT)
#pragma unroll
                for (int e = i * kM; e < (i + 1) * kM; e += 2) top = fmaxf(fmaxf(top, nx[e >> 4][e & 15]), nx[e >> 4][(e & 15) + 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // K lies one tile ahead of V: in step j both of K(j + 1) and V(j) are there, K(j + 2) and V(j + 1) are under way
    if (tiles > 0) {
        copy(a.k, a.ldk, 0, 0);
        copy(a.v, a.ldv, 0, 2 * kTile);
        if (tiles > 1) {
            copy(a.k, a.ldk, BN, kTile);
            wait_copies<2 * kCopies>();
        } else {
            wait_copies<kCopies>();
        }
        block_sync();
    }
    arrived(qf);
    if (mine > 0) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            sc[b] = zero16();
#pragma unroll
            for (int i = 0; i < T::kK; ++i) sc[b] = mfma32(T::row_frag(lds, rb, b, i), qf[i], sc[b]);
        }
        mask(sc, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(fmaxf(top, sc[0][i]), sc[1][i]);
    }
    auto turn = [&](int j) {
        wait_copies<0>();
        block_sync();
        if (j + 2 < tiles) copy(a.k, a.ldk, (j + 2) * BN, (j & 1) * kTile);
        if (j + 1 < tiles) copy(a.v, a.ldv, (j + 1) * BN, (2 + (~j & 1)) * kTile);
    };
    int j = 0;
    for (; j + 2 < mine; j += 2) {                                   // two steps a turn of the loop: the scores change places for nothing
        turn(j);
        step(std::true_type{}, j * BN, 0, sc, s2);
        turn(j + 1);
        step(std::true_type{}, (j + 1) * BN, 1, s2, sc);
    }
    if (j + 1 < mine) {
        turn(j);
        step(std::true_type{}, j * BN, 0, sc, s2);
        sc[0] = s2[0];
        sc[1] = s2[1];
        ++j;
    }
    if (mine > 0) {
        turn(j);
        step(std::false_type{}, j * BN, j & 1, sc, s2);
        ++j;
    }
    for (; j < tiles; ++j) turn(j);
    sum = half_sum(sum);
    store_row<DIM>(a.o + ((long)(q0 + token) * a.n_q + head) * DIM, o, sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f, h, r.valid);
    if (r.valid && h == 0)
        a.lse[(long)head * a.sq.rows + q0 + token] = sum == 0.0f ? -INFINITY : (ref + log2_hw(sum)) * kLn2;
}

// The same for few tiles: 32 rows, every wave with every fourth block of 32 keys in buffers of its own, so that no wave waits for
// another until their sums are joined.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256) attention_fwd_few_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BN = 32, kTile = BN * T::kRowBytes, kCopies = BN / T::kRowsPerCopy, kWave = 4 * kTile;
    static_assert(kWave >= 32 * (DIM + 4) * 4, "the buffers hold the sums");
    __shared__ __attribute__((aligned(256))) char lds[4 * kWave];      // K, V; K, V of each wave
    __shared__ float stats[2][4][32];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int kvh = blockIdx.x % a.n_kv, tile = gridDim.x / a.n_kv - 1 - blockIdx.x / a.n_kv;
    QueryRow r;
    if (!query_row<CAUSAL>(a, tile, 32, 0, kvh, l, r)) return;

    bf16x8 qf[T::kK];
    const uint16_t* qp = a.q + (long)(r.q0 + r.token) * a.ldq + r.head * DIM + 8 * h;
#pragma unroll
    for (int i = 0; i < T::kK; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(qp + 16 * i);
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

    f32x16 o[T::kC];
#pragma unroll
    for (int c = 0; c < T::kC; ++c) o[c] = zero16();
    float m2 = -INFINITY, ref = 0.0f, sum = 0.0f;
    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);
    arrived(qf);
    if (w * BN < r.kv_end) copy(w * BN, 0);
    for (int key0 = w * BN, buf = 0; key0 < r.kv_end; key0 += 4 * BN, buf ^= 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");          // the reads of the block before are done, its buffer is free
        if (key0 + 4 * BN < r.kv_end) {
            copy(key0 + 4 * BN, buf ^ 1);
            wait_copies<2 * kCopies>();
        } else {
            wait_copies<0>();
        }
        const char* kt = mine + 2 * buf * kTile;
        f32x16 sc = zero16();
#pragma unroll
        for (int i = 0; i < T::kK; ++i) sc = mfma32(T::row_frag(kt, rb, 0, i), qf[i], sc);
        if (key0 + BN - 1 > r.lim_first) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (key0 + 8 * (i >> 2) + 4 * h + (i & 3) > r.lim) sc[i] = -INFINITY;
        }
        float top = sc[0];
#pragma unroll
        for (int i = 0; i < 16; i += 2) top = fmaxf(fmaxf(top, sc[i]), sc[i + 1]);
        top = half_max(top) * c2;
        if (__any(top > m2 + 8.0f)) {
            const float old = m2;
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
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            sc[i] = exp2_hw(__builtin_fmaf(sc[i], c2, -ref));
            sum += sc[i];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bf16x8 p = to_operand(sc, k);
#pragma unroll
            for (int c = 0; c < T::kC; ++c) o[c] = mfma32(T::col_frag(kt + kTile, cb, k, c), p, o[c]);
        }
    }
    sum = half_sum(sum);
    float* sums = reinterpret_cast<float*>(lds);
    __syncthreads();
    leave_sums<DIM>(sums, o, w, l);
    if (h == 0) {
        stats[0][w][l] = m2 == -INFINITY && sum == 0.0f ? -INFINITY : ref;
        stats[1][w][l] = sum;
    }
    __syncthreads();
    // every thread has 8 channels of a row at a time; it reads where its row goes from the lanes that have it
    for (int i = threadIdx.x; i < 32 * (DIM / 8); i += 256) {
        const int row = i / (DIM / 8), ch = i % (DIM / 8) * 8;
        const int token = __shfl(r.token, row), head = __shfl(r.head, row), valid = __shfl((int)r.valid, row);
        float top = stats[0][0][row];
#pragma unroll
        for (int k = 1; k < 4; ++k) top = fmaxf(top, stats[0][k][row]);
        if (top == -INFINITY) top = 0.0f;
        float total = 0.0f, v[8] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = exp2_hw(stats[0][k][row] - top);
            total = __builtin_fmaf(f, stats[1][k][row], total);
            const float* p = sums + (k * 32 + row) * (DIM + 4) + ch;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(f, p[e], v[e]);
        }
        if (!valid) continue;
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        *reinterpret_cast<uint4*>(a.o + ((long)(r.q0 + token) * a.n_q + head) * DIM + ch) =
            uint4{bf16_pack2(v[0] * inv, v[1] * inv), bf16_pack2(v[2] * inv, v[3] * inv), bf16_pack2(v[4] * inv, v[5] * inv), bf16_pack2(v[6] * inv, v[7] * inv)};
        if (ch == 0) a.lse[(long)head * a.sq.rows + r.q0 + token] = total == 0.0f ? -INFINITY : (top + log2_hw(total)) * kLn2;
    }
}

hipError_t launch_attention_fwd(const AttentionArgs& a, int dim, bool causal, hipStream_t st) {
    const long rows = (long)a.sq.rows * a.group;
    const bool few = few_row_tiles(a.sq.n, a.sq.rows, a.sk.rows, a.group, a.n_kv, dim);
    const dim3 grid((unsigned)(tiles_of(rows, few ? 32 : 128, a.sq.n) * a.n_kv));
#define JET_FWD(KERNEL) (dim == 128 ? (causal ? KERNEL<128, true> : KERNEL<128, false>) : (causal ? KERNEL<64, true> : KERNEL<64, false>))
    hipLaunchKernelGGL((few ? JET_FWD(attention_fwd_few_kernel) : JET_FWD(attention_fwd_kernel)), grid, dim3(256), 0, st, a);
#undef JET_FWD
    return hipGetLastError();
}

}  // namespace jet

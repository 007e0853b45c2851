// Attention of packed sequences, backward.  With p_ij = e^(scale q_i k_j - lse_i) recomputed from the saved logarithms,
//   dp_ij = do_i v_j,   delta_i = sum_j p_ij dp_ij = do_i o_i,   ds_ij = p_ij (dp_ij - delta_i),
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i,
// the sums of dk and dv over the rows of all query heads that share the head.  Two kernels, one for sums over keys and one for
// sums over rows, seven products in place of the five that one kernel with atomic sums of dq would take: the order of every
// sum is fixed, so that the same inputs give the same bytes.
#include <algorithm>
#include <type_traits>

#include "jet_attn.h"
#include "jet_internal.h"

namespace jet {

// dq; rows and tiles as in the forward pass.  It also leaves for the second kernel, in the order of the rows, lse in units of log2
// (+inf for a row that sees no key, so that 2^(s - lse) is 0) and - delta.
template <int DIM, bool CAUSAL>
__global__ void __launch_bounds__(256, 2) attention_dq_kernel(AttentionArgs a) {
    using T = Tile<DIM>;
    constexpr int BN = 32, kTile = BN * T::kRowBytes, kCopies = BN / T::kRowsPerCopy / 4;
    __shared__ __attribute__((aligned(256))) char lds[8 * kTile];   // K, V; four times
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = l >> 5;
    const int kvh = blockIdx.x % a.n_kv, tile = gridDim.x / a.n_kv - 1 - blockIdx.x / a.n_kv;

    const Place place = place_of(a.sq, a.sk, tile, 128, a.group, l);
    const int q0 = place.begin, n = place.count, k0 = place.other_begin, m = place.other_count;
    const int rows = n * a.group, row0 = (tile - place.first_tile) * 128;
    if (row0 < 0 || row0 >= rows) return;
    const int off = m - n;

    const int tok0 = row0 / a.group, rem0 = row0 - tok0 * a.group;
    const int row = min(w * 32 + (l & 31), rows - 1 - row0);
    const bool valid = row == w * 32 + (l & 31);
    const int x = rem0 + row, dt = (int)(x * a.group_magic >> 20), head = kvh * a.group + x - dt * a.group;
    const int token = tok0 + dt;
    const int lim = CAUSAL ? min(m - 1, token + off) : m - 1;
    const int lim_first = __builtin_amdgcn_readlane(lim, 0), lim_last = __builtin_amdgcn_readlane(lim, 31);
    const int last_token = (min(row0 + 127, rows - 1)) / a.group;
    const int kv_end = __builtin_amdgcn_readfirstlane(CAUSAL ? max(0, min(m, last_token + off + 1)) : m);

    bf16x8 qf[T::kK], df[T::kK];
    const uint16_t* qp = a.q + (long)(q0 + token) * a.ldq + head * DIM + 8 * h;
    const long dense = ((long)(q0 + token) * a.n_q + head) * DIM;
    float delta = 0.0f;
#pragma unroll
    for (int i = 0; i < T::kK; ++i) {
        qf[i] = *reinterpret_cast<const bf16x8*>(qp + 16 * i);
        df[i] = *reinterpret_cast<const bf16x8*>(a.dout + dense + 8 * h + 16 * i);
        const bf16x8 of = *reinterpret_cast<const bf16x8*>(a.o + dense + 8 * h + 16 * i);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)df[i][j], (float)of[j], delta);
    }
    delta = half_sum(delta);
    const float lse = a.lse[(long)head * a.sq.rows + q0 + token];
    const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
    if (valid && h == 0) {
        const long at = ((long)kvh * a.sq.rows + q0) * a.group + row0 + row;
        a.row_lse[at] = lse2;
        a.row_delta[at] = -delta;
    }

    const uint32_t lds0 = lds_address(lds);
    auto copy = [&](int key0, int slot) {
        const int nr = min(BN, kv_end - key0);
        const i32x4 kb = buffer_of(a.k + (long)(k0 + key0) * a.ldk + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldk + DIM) * 2);
        const i32x4 vb = buffer_of(a.v + (long)(k0 + key0) * a.ldv + kvh * DIM, (uint32_t)((nr - 1) * (int)a.ldv + DIM) * 2);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
            const uint32_t r = (w * kCopies + c) * T::kRowsPerCopy + l / T::kChunks;
            const uint32_t chunk = ((l % T::kChunks) ^ T::swizzle(r)) * 16;
            const uint32_t at = lds0 + 2 * slot * kTile + (w * kCopies + c) * 1024;
            copy16(at, kb, r * (uint32_t)a.ldk * 2 + chunk);
            copy16(at + kTile, vb, r * (uint32_t)a.ldv * 2 + chunk);
        }
    };

    f32x16 dq[T::kC], sa, sb, dp, less_delta;
#pragma unroll
    for (int i = 0; i < 16; ++i) less_delta[i] = -delta;
#pragma unroll
    for (int c = 0; c < T::kC; ++c) dq[c] = zero16();
    const float c2 = a.scale * kLog2e;
    const uint32_t rb = T::row_base(l), cb = T::col_base(l);
    const int blocks = (kv_end + BN - 1) / BN, mine = lim_last < 0 ? 0 : lim_last / BN + 1;
    constexpr int kSlots = T::kK, kPer = 16 / (kSlots - 2) + (16 % (kSlots - 2) != 0), LA = 3;   // kK = 2 kC

    // p of a block beside dP - delta, a product that starts from - delta; one MFMA a slot, with the LDS reads of LA slots later and a share of the other work
    auto second = [&](const char* vt, f32x16& sc) {
        bf16x8 vf[kSlots];
#pragma unroll
        for (int i = 0; i < LA; ++i) vf[i] = T::row_frag(vt, rb, 0, i);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            if (i + LA < kSlots) vf[i + LA] = T::row_frag(vt, rb, 0, i + LA);
            dp = mfma32(vf[i], df[i], i == 0 ? less_delta : dp);
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
                for (int e = (i - 1) * kPer; e < min(16, i * kPer); ++e) sc[e] *= dp[e];
            __builtin_amdgcn_sched_barrier(0);
        }
        if (key0 + BN - 1 > lim_first) {
            // a row that sees one key has p = 1 whatever its score: no gradient, not the rounding of dp - delta
            int left = lim == 0 ? -1 : lim - key0 - 4 * h;
            asm volatile("" : "+v"(left));
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) > left) sc[i] = 0.0f;
        }
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
    arrived(qf);
    arrived(df);
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
    store_row<DIM>(a.dq + (long)(q0 + token) * a.ld_dq + head * DIM, dq, a.scale, h, valid);
}

__device__ __forceinline__ int pieces_of(const AttentionArgs& a, int rows) {
    return __builtin_amdgcn_readfirstlane(max(1, min(a.parts, (rows + a.part_rows - 1) / a.part_rows)));
}

// dk and dv of 128 keys of one head, a wave has 32 of them as the columns of its products; it goes over the rows that see them, 32 at
// a time: S = Q K^T and dP = dO V^T from the rows' tiles, then dV^T += dO^T P and dK^T += Q^T dS from the same tiles read
// by columns.  The keys' fragments stay in registers; the values' are read from LDS again and again, which leaves the other
// operands without spills at two workgroups a CU.
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
    const int share = ((rows - f_first + pieces - 1) / pieces + BM - 1) / BM * BM;        // of a piece, in whole steps
    const int f_begin = min(rows, f_first + part * share), f_end = min(rows, f_begin + share);

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
    // 32 (so do f_begin and the steps): then this holds for all of them, else it is formed for each.
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

    if (f_begin < f_end) copy(f_begin, 0);
    arrived(kf);
    auto step = [&](int f0, auto which) {
        constexpr int buf = decltype(which)::value;
        wait_copies<0>();
        block_sync();
        if (f0 + BM < f_end) copy(f0 + BM, buf ^ 1);
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
    for (int f0 = f_begin; f0 < f_end; f0 += 2 * BM) {       // two steps, so that the buffers are constants of the addresses
        step(f0, std::integral_constant<int, 0>{});
        if (f0 + BM < f_end) step(f0 + BM, std::integral_constant<int, 1>{});
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

// How the rows of a tile of keys are dealt to workgroups, of which 512 run at a time.  One sequence: its first tiles have twice the
// average work, so from 1024 workgroups on they even out by themselves, and each tile is split alike to get there, in pieces of
// 512 rows (16 steps) at least.  Several sequences come in any order, a long one perhaps at the end: no workgroup has more than two
// thirds of what each of the 512 places would get if the sequences were equally long, or 1024 rows where that is more.
struct Split {
    int parts, rows;
};
static Split dkdv_split(long n_seqs, long Tq, long Tk, long group, long n_kv, bool causal) {
    const long tiles = (Tk + 127) / 128, groups = tiles * n_kv;
    const long place = groups * (Tq / n_seqs * group) / (causal ? 2 : 1) / 512;
    const long rows = n_seqs == 1 ? 512 : std::min<long>(1 << 30, std::max<long>(1024, place * 2 / 3 / 32 * 32));
    const long most = n_seqs == 1 ? std::min<long>(8, 1024 / groups) : 8;
    return {(int)std::max<long>(1, std::min(most, (Tq * group + rows - 1) / rows)), (int)rows};
}

long attention_bwd_workspace(long n_seqs, long Tq, long Tk, long n_q, long n_kv, long dim) {
    const long parts = std::max(dkdv_split(n_seqs, Tq, Tk, n_q / n_kv, n_kv, true).parts, dkdv_split(n_seqs, Tq, Tk, n_q / n_kv, n_kv, false).parts);
    return (2 * ((Tq * n_q + 3) / 4 * 4) + (parts > 1 ? parts * Tk * n_kv * 2 * dim : 0)) * (long)sizeof(float);
}

hipError_t launch_attention_bwd(AttentionArgs a, int dim, bool causal, void* workspace, hipStream_t st) {
    const long stats = ((long)a.sq.rows * a.n_q + 3) / 4 * 4;
    a.row_lse = static_cast<float*>(workspace);
    a.row_delta = a.row_lse + stats;
    a.partial = a.row_delta + stats;
    const Split split = dkdv_split(a.sq.n, a.sq.rows, a.sk.rows, a.group, a.n_kv, causal);
    a.parts = split.parts;
    a.part_rows = split.rows;
    const long tiles = tiles_of(a.sk.rows, 128, a.sk.n) * a.n_kv;
#define JET_BWD(KERNEL) (dim == 128 ? (causal ? KERNEL<128, true> : KERNEL<128, false>) : (causal ? KERNEL<64, true> : KERNEL<64, false>))
    hipLaunchKernelGGL(JET_BWD(attention_dq_kernel), dim3((unsigned)(tiles_of((long)a.sq.rows * a.group, 128, a.sq.n) * a.n_kv)), dim3(256), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(JET_BWD(attention_dkdv_kernel), dim3((unsigned)tiles, (unsigned)a.parts), dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    hipLaunchKernelGGL(JET_BWD(attention_dkdv_join_kernel), dim3((unsigned)tiles, 8), dim3(256), 0, st, a);
#undef JET_BWD
    return hipGetLastError();
}

}  // namespace jet

// Attention of one query token per sequence over a paged cache, in bf16 or in E4M3 with a scale for each token and head.
//
// A workgroup has one sequence, one key/value head (16 of the query heads that share it) and a chunk of the keys; its waves
// take blocks of 32 keys in turn, each through LDS buffers of its own, so that nothing but the end of the chunk waits for
// another wave.  The chunks' results (sum of 2^(s - m) v, sum of 2^(s - m), m) are joined by a second launch; a sequence that
// fits one chunk is done in the first.
//
// Fragments of v_mfma_f32_16x16x32_bf16, lane l, g = l >> 4: A[m = l & 15][k = 8 g + j], B[k = 8 g + j][n = l & 15],
// D[m = 4 g + i][n = l & 15].  S^T = K Q^T for keys 0..15 and 16..31 of a block leaves a lane with keys 4 g + i and 16 + 4 g + i,
// which O^T = V^T P^T takes as its k: the values are read by columns in that order.
//
// What bounds it is the stream of keys and values, copied past the caches (with the ordinary policy 178 us in place of 160 for 64 sequences
// of 500 to 8192 tokens): 875 MB in 140 us, 6.2 TB/s; E4M3, 128 sequences up to 16384 tokens, 1447 MB in 248 us, 5.8 TB/s, of which the scales'
// copies take 4 %.  Reading 2 GiB with a library sum goes at 6.08 TB/s.
#include <algorithm>

#include "jet_attn.h"
#include "jet_internal.h"

namespace jet {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quarter_max(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarter_sum(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
// 8 E4M3 codes to bf16, which holds every one of their values
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    const u32x4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
    return __builtin_bit_cast(bf16x8, w);
}

constexpr float kDone = -1.0f;      // in place of a sum of exponentials: the sequence had one chunk and is written

template <int DIM, bool FP8, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, FP8 || DIM == 64 ? 2 : 1) attention_decode_kernel(DecodeArgs a) {
    constexpr int RB = FP8 ? DIM : 2 * DIM;                  // bytes of a row
    constexpr int kChunks = RB / 16, kRowsPerCopy = 64 / kChunks, kCopies = 16 / kRowsPerCopy;   // of half a block
    constexpr int kBlock = 32 * RB, kStage = 2 * kBlock + (FP8 ? 256 : 0), kS = DIM / 32;
    constexpr int kWave = 2 * kStage;
    __shared__ __attribute__((aligned(128))) char lds[WAVES * kWave];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = l >> 4, c = l & 15;
    const int pairs = a.B * a.n_kv * a.q_blocks;
    const int part = blockIdx.x / pairs, pair = blockIdx.x - part * pairs;
    const int qb = pair % a.q_blocks, kvh = pair / a.q_blocks % a.n_kv, b = pair / a.q_blocks / a.n_kv;
    const int asked = a.lengths[b], capacity = a.max_pages * a.page;
    const int len = max(0, min(asked, capacity));
    const int c0 = part * a.chunk, c1 = min(len, c0 + a.chunk);
    const int heads = min(16, a.group - 16 * qb), head0 = kvh * a.group + 16 * qb;
    if (c0 >= len && part > 0) {                             // for the join, which does not read the lengths
        if ((int)threadIdx.x < heads) reinterpret_cast<float2*>(a.part_ml)[((long)b * a.n_q + head0 + threadIdx.x) * a.parts + part] = float2{-INFINITY, 0.0f};
        return;
    }

    // Lane i: where sub-block i of 16 keys of this wave lies, in rows of the cache, and how many of its rows are keys.
    const int my_key = c0 + (w + WAVES * (l >> 1)) * 32 + (l & 1) * 16;
    int page_id = 0, n_rows = max(0, min(16, c1 - my_key));
    bool bad = asked > capacity;                             // keys that no page holds
    if (my_key < capacity) page_id = a.pages[(long)b * a.max_pages + my_key / a.page];
    if (n_rows > 0 && (uint32_t)page_id >= (uint32_t)a.n_pages) {
        bad = true;
        n_rows = 0;
    }
    const uint64_t my_row = n_rows ? ((uint64_t)page_id * a.n_kv + kvh) * a.page + my_key % a.page : 0;
    bad = __any(bad);

    // queries as the B operand; where a row is in E4M3 a 16-byte read holds the k of two steps, 64 s + 16 g + 8 e + j
    bf16x8 qf[kS];
    const uint16_t* qp = a.q + (long)b * a.ldq + (long)(head0 + min(c, heads - 1)) * DIM;
#pragma unroll
    for (int s = 0; s < kS; ++s)
        qf[s] = *reinterpret_cast<const bf16x8*>(qp + (FP8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g));

    const uint32_t lds_w = lds_address(lds) + w * kWave;
    const char* mine = lds + w * kWave;
    // orders in which 16 keys at one chunk, and for the values 8 rows at two chunks (bf16) or 8 + 8 rows at one (E4M3), cover
    // 256 bytes of LDS once
    auto k_swizzle = [](uint32_t r) { return RB == 256 ? r & 15 : RB == 128 ? (r >> 1) & 7 : (r >> 2) & 3; };
    auto v_swizzle = [](uint32_t r) {
        return !FP8 ? (RB == 256 ? (r & 7) << 1 : ((r >> 1) & 3) << 1)
                    : (RB == 128 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : ((r >> 2) & 1) | ((r >> 4) & 1) << 1);
    };
    const int n_blocks = c1 > c0 + 32 * w ? (c1 - c0 - 32 * w + 32 * WAVES - 1) / (32 * WAVES) : 0;   // of this wave
    auto copy = [&](int j, int buf) {
        const uint32_t at = lds_w + buf * kStage;
        uint64_t rows[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            rows[t] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)my_row, 2 * j + t) |
                      (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(my_row >> 32), 2 * j + t) << 32;
            const uint32_t bytes = __builtin_amdgcn_readlane(n_rows, 2 * j + t) * RB;
            const i32x4 kb = buffer_of(a.k + rows[t] * RB, bytes), vb = buffer_of(a.v + rows[t] * RB, bytes);
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const uint32_t r = i * kRowsPerCopy + l / kChunks, rt = 16 * t + r;
                copy16_nt(at + (t * kCopies + i) * 1024, kb, r * RB + ((l % kChunks) ^ k_swizzle(rt)) * 16);
                copy16_nt(at + kBlock + (t * kCopies + i) * 1024, vb, r * RB + ((l % kChunks) ^ v_swizzle(rt)) * 16);
            }
        }
        if constexpr (FP8) {       // lanes 0..31: scales of the keys, 32..63: of the values
            const float* p = ((l & 32) ? a.v_scale : a.k_scale) + ((l & 16) ? rows[1] : rows[0]) + (l & 15);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off nt" : : "s"(at + 2 * kBlock), "v"(p) : "memory");
        }
    };
    constexpr int kInFlight = 4 * kCopies + (FP8 ? 1 : 0);

    f32x4 o[DIM / 16];
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m2 = -INFINITY, ref = 0.0f, sum = 0.0f;
    const float c2 = a.scale * kLog2e;

    if (n_blocks > 0) copy(0, 0);
    for (int j = 0, buf = 0; j < n_blocks; ++j, buf ^= 1) {
        // the reads of block j - 1 are done, its buffer is free
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        if (j + 1 < n_blocks) {
            copy(j + 1, buf ^ 1);
            wait_copies<kInFlight>();
        } else {
            wait_copies<0>();
        }
        const char* kt = mine + buf * kStage;
        const char* vt = kt + kBlock;
        const float* st = reinterpret_cast<const float*>(kt + 2 * kBlock);
        f32x4 sc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int r = 16 * t + c;
            if constexpr (!FP8) {
#pragma unroll
                for (int s = 0; s < kS; ++s)
                    sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        *reinterpret_cast<const bf16x8*>(kt + r * RB + (((4 * s + g) ^ k_swizzle(r)) << 4)), qf[s], sc[t], 0, 0, 0);
            } else {
#pragma unroll
                for (int s = 0; s < kS / 2; ++s) {
                    const uint4 x = *reinterpret_cast<const uint4*>(kt + r * RB + (((4 * s + g) ^ k_swizzle(r)) << 4));
                    sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(x.x, x.y), qf[2 * s], sc[t], 0, 0, 0);
                    sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(x.z, x.w), qf[2 * s + 1], sc[t], 0, 0, 0);
                }
                const f32x4 f = *reinterpret_cast<const f32x4*>(st + 16 * t + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[t][i] *= f[i];
            }
        }
        const int key0 = c0 + (w + WAVES * j) * 32 + 4 * g;
        const bool last = key0 - 4 * g + 32 > c1;
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (last && key0 + 16 * t + i >= c1) sc[t][i] = -INFINITY;
                top = fmaxf(top, sc[t][i]);
            }
        top = quarter_max(top) * c2;
        if (__any(top > m2 + 8.0f)) {
            const float old = m2;                                     // -inf in front of the first: nothing to rescale
            m2 = fmaxf(m2, top);
            const float next = m2 == -INFINITY ? 0.0f : m2;
            const float f = exp2_hw(old - next);
            ref = next;
            sum *= f;
#pragma unroll
            for (int i = 0; i < DIM / 16; ++i) o[i] *= f;
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = exp2_hw(__builtin_fmaf(sc[i >> 2][i & 3], c2, -ref));
            sum += p[i];
        }
        if constexpr (FP8) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const f32x4 f = *reinterpret_cast<const f32x4*>(st + 32 + 16 * t + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) p[4 * t + i] = last && key0 + 16 * t + i >= c1 ? 0.0f : p[4 * t + i] * f[i];
            }
        }
        const u32x4 pw = {bf16_pack2(p[0], p[1]), bf16_pack2(p[2], p[3]), bf16_pack2(p[4], p[5]), bf16_pack2(p[6], p[7])};
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
        for (int i = 0; i < DIM / 16; ++i) {
            bf16x8 vf;
            if constexpr (!FP8) {
                const int r = 4 * g + (c >> 2);
                const char* at = vt + r * RB + (((2 * i + ((c >> 1) & 1)) ^ v_swizzle(r)) << 4) + (c & 1) * 8;
                union {
                    s16x4 q[2];
                    bf16x8 f;
                } u;
                u.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(JET_LDS(s16x4, at));
                u.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(JET_LDS(s16x4, at + 16 * RB));
                vf = u.f;
            } else {
                typedef int i32x2 __attribute__((ext_vector_type(2)));
                const int e = c >> 1, r = 4 * g + (e & 3) + 16 * (e >> 2);
                const char* at = vt + r * RB + ((i ^ v_swizzle(r)) << 4) + (c & 1) * 8;
                const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(JET_LDS(i32x2, at));
                vf = widen((uint32_t)x[0], (uint32_t)x[1]);
            }
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[i], 0, 0, 0);
        }
    }

    // the waves' results, through LDS
    sum = quarter_sum(sum);
    float* all = reinterpret_cast<float*>(lds);              // [WAVES][16][DIM], then [WAVES][16] references and sums
    float* ml = all + WAVES * 16 * DIM;
    static_assert(kWave >= (16 * DIM + 2 * 16) * 4, "the buffers hold the results");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) *reinterpret_cast<f32x4*>(all + (w * 16 + c) * DIM + 16 * i + 4 * g) = o[i];
    if (g == 0) {
        ml[w * 16 + c] = m2 == -INFINITY && sum == 0.0f ? -INFINITY : ref;
        ml[(WAVES + w) * 16 + c] = sum;
    }
    __shared__ int any_bad;
    if (threadIdx.x == 0) any_bad = 0;
    __syncthreads();
    if (bad && l == 0) any_bad = 1;
    __syncthreads();
    const bool whole = len <= a.chunk;
    for (int at = threadIdx.x; at < heads * (DIM / 4); at += 64 * WAVES) {
        const int q = at / (DIM / 4), ch = at % (DIM / 4) * 4;
        float largest = ml[q];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) largest = fmaxf(largest, ml[16 * i + q]);
        const float m = largest == -INFINITY ? 0.0f : largest;
        float total = 0.0f;
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float f = exp2_hw(ml[16 * i + q] - m);
            total = __builtin_fmaf(f, ml[16 * (WAVES + i) + q], total);
            const f32x4 x = *reinterpret_cast<const f32x4*>(all + (i * 16 + q) * DIM + ch);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(f, x[e], v[e]);
        }
        if (any_bad) {                                       // a page outside the cache: no answer, and not a wrong one
            total = NAN;
            v = f32x4{NAN, NAN, NAN, NAN};
        }
        const long row = (long)b * a.n_q + head0 + q;
        if (whole) {
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            *reinterpret_cast<uint2*>(a.o + row * DIM + ch) = uint2{bf16_pack2(v[0] * inv, v[1] * inv), bf16_pack2(v[2] * inv, v[3] * inv)};
            if (ch == 0 && a.parts > 1) reinterpret_cast<float2*>(a.part_ml)[row * a.parts] = float2{0.0f, kDone};
        } else {
            *reinterpret_cast<f32x4*>(a.part_o + (row * a.parts + part) * DIM + ch) = v;
            // A sum that is no number has the reference +inf: its factor in the join, 2^(inf - inf), is none either, however large
            // the scores of other chunks are.
            if (ch == 0) *reinterpret_cast<float2*>(a.part_ml + (row * a.parts + part) * 2) = float2{total == total ? largest : INFINITY, total};
        }
    }
}

// Joins the chunks of a sequence that has several: a wave for each query head, DIM / 64 channels a lane.  Of a few chunks of a
// few rows the sums are read without waiting for the word which of them there are (3.1 -> 2.7 us for one sequence); of many rows that reads
// too much that is not there.
template <int DIM>
__global__ void __launch_bounds__(256) attention_join_kernel(DecodeArgs a) {
    constexpr int N = DIM / 64, FEW = 16;
    typedef float Sums __attribute__((ext_vector_type(N)));
    const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int l = threadIdx.x & 63;
    if (row >= (long)a.B * a.n_q) return;
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + row * a.parts;
    const Sums* part = reinterpret_cast<const Sums*>(a.part_o + row * a.parts * DIM) + l;
    float m = -INFINITY, total = 0.0f;
    Sums v = 0.0f;
    if (a.parts <= FEW && a.B * a.n_q <= 1024) {
        const float2 mine = ml[min(l, a.parts - 1)];
        Sums x[FEW];
#pragma unroll
        for (int i = 0; i < FEW; ++i)
            if (i < a.parts) x[i] = part[i * 64];
        if (__builtin_amdgcn_readlane(__float_as_int(mine.y), 0) == __float_as_int(kDone)) return;
        m = l < a.parts ? mine.x : -INFINITY;
#pragma unroll
        for (int d = 1; d < FEW; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
        m = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(m)));
        if (m == -INFINITY) m = 0.0f;
        const float f = exp2_hw(mine.x - m);
#pragma unroll
        for (int i = 0; i < FEW; ++i)
            if (i < a.parts) {
                const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i));
                if (fi == 0.0f) continue;                    // a chunk behind the length, whose sums were not written
                total = __builtin_fmaf(fi, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine.y), i)), total);
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = __builtin_fmaf(fi, x[i][e], v[e]);
            }
    } else {
        if (ml[0].y == kDone) return;
        for (int i = l; i < a.parts; i += 64) m = fmaxf(m, ml[i].x);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
        if (m == -INFINITY) m = 0.0f;
        for (int i0 = 0; i0 < a.parts; i0 += 64) {           // 64 chunks' words in the lanes, then 8 of their sums at a time
            const float2 mine = i0 + l < a.parts ? ml[i0 + l] : float2{-INFINITY, 0.0f};
            const float f = exp2_hw(mine.x - m);
            const uint64_t any = __ballot(f != 0.0f);
            const int n = any ? 64 - __builtin_clzll(any) : 0;
            for (int b = 0; b < n; b += 8) {
                Sums x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = part[(long)min(i0 + b + i, a.parts - 1) * 64];
#pragma unroll
                for (int i = 0; i < 8; ++i) {                // past the lengths f is 0 and nothing was written
                    const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), b + i));
                    total = __builtin_fmaf(fi, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine.y), b + i)), total);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] = __builtin_fmaf(fi, fi == 0.0f ? 0.0f : x[i][e], v[e]);
                }
            }
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t* out = a.o + row * DIM + N * l;
    if constexpr (N == 2) *reinterpret_cast<uint32_t*>(out) = bf16_pack2(v[0] * inv, v[1] * inv);
    else *out = (uint16_t)bf16_pack2(v[0] * inv, 0.0f);
}

long attention_decode_workspace(long B, long n_q, long n_kv, long dim, bool fp8, long capacity) {
    const long parts = attention_decode_groups(B, n_q, n_kv, dim, fp8, capacity) / (B * n_kv * ((n_q / n_kv + 15) / 16));
    return parts <= 1 ? 0 : B * n_q * parts * (dim + 2) * (long)sizeof(float);
}

hipError_t launch_attention_decode(DecodeArgs a, int dim, bool fp8, void* workspace, hipStream_t st) {
    const long capacity = (long)a.max_pages * a.page;
    a.q_blocks = (a.group + 15) / 16;
    const long pairs = (long)a.B * a.n_kv * a.q_blocks;
    a.chunk = decode_chunk(pairs, capacity, decode_waves(dim, fp8));
    a.parts = (int)((capacity + a.chunk - 1) / a.chunk);
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o + (a.parts > 1 ? (long)a.B * a.n_q * a.parts * dim : 0);
#define JET_DECODE(DIM, FP8) attention_decode_kernel<DIM, FP8, decode_waves(DIM, FP8)>
    const auto kernel = dim == 128 ? (fp8 ? JET_DECODE(128, true) : JET_DECODE(128, false))
                                   : (fp8 ? JET_DECODE(64, true) : JET_DECODE(64, false));
#undef JET_DECODE
    hipLaunchKernelGGL(kernel, dim3((unsigned)(pairs * a.parts)), dim3(64 * decode_waves(dim, fp8)), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    const auto join = dim == 128 ? attention_join_kernel<128> : attention_join_kernel<64>;
    hipLaunchKernelGGL(join, dim3((unsigned)(((long)a.B * a.n_q + 3) / 4)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace jet

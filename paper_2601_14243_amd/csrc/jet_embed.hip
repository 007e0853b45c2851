// Embedding: rows of the table for the tokens of a call, and the table's gradient.
#include <utility>

#include "jet_internal.h"
#include "jet_numerics.h"
#include "jet_step.h"

namespace jet {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kNoRow = 0xfffffffeu;             // a token whose id the table does not hold; behind all rows in their order, and
                                                     // in front of what fills the last block

__device__ __forceinline__ uint32_t row_of(const void* ids, bool wide, long t, long first, long rows) {
    const int64_t id = wide ? reinterpret_cast<const int64_t*>(ids)[t] : (int64_t)reinterpret_cast<const int32_t*>(ids)[t];
    const uint64_t r = (uint64_t)id - (uint64_t)first;
    return r < (uint64_t)rows ? (uint32_t)r : kNoRow;
}

// ------------------------------------------------------------------------
// y[t] = bf16(scale w[row of t]), zeros without a row.  tx threads (a power of two) go along a row, 8 columns each, with the loads of
// four such pieces under way.  Bound by memory: 16384 tokens x 5120 from f32 61 us (308 MB with each row of the table once, 5.0 TB/s; rows
// that many tokens have come from the caches, which the output leaves to them where it is large).
// ------------------------------------------------------------------------
template <bool kF32, bool kNt>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(EmbedArgs a, int tx_log2) {
    const int tx = 1 << tx_log2, l = threadIdx.x & (tx - 1);
    const long t = (long)blockIdx.x * (256 >> tx_log2) + (threadIdx.x >> tx_log2);
    if (t >= a.T) return;
    const uint32_t r = row_of(a.ids, a.wide, t, a.first, a.rows);
    uint16_t* const y = a.y + t * a.H;
    constexpr int kAtOnce = 4;
    for (int k0 = l * 8; k0 < a.H; k0 += tx * 8 * kAtOnce) {
        u32x4 u[kAtOnce][kF32 ? 2 : 1];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int k = k0 + i * tx * 8;
#pragma unroll
            for (int j = 0; j < (kF32 ? 2 : 1); ++j) {
                u[i][j] = u32x4{0, 0, 0, 0};
                if (r != kNoRow && k < a.H) u[i][j] = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.w) + ((long)r * a.H + k) * (kF32 ? 4 : 2))[j];
            }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int k = k0 + i * tx * 8;
            if (k >= a.H) break;
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float lo = kF32 ? __uint_as_float(u[i][kF32 ? j >> 1 : 0][2 * (j & 1)]) : bf16_lo(u[i][0][j]);
                const float hi = kF32 ? __uint_as_float(u[i][kF32 ? j >> 1 : 0][2 * (j & 1) + 1]) : bf16_hi(u[i][0][j]);
                o[j] = bf16_pack2(lo * a.scale, hi * a.scale);
            }
            const uint4 v = {o[0], o[1], o[2], o[3]};
            if (kNt) store16_nt(y + k, v);
            else *reinterpret_cast<uint4*>(y + k) = v;
        }
    }
}

// ------------------------------------------------------------------------
// The gradient: dw[r] = scale sum of dy[t] over the tokens t of row r, in the order of the tokens.
//   1. the tokens are put in the order of (row, token): up to kPlaceTokens of them by counting for each those in front of it, more by
//      sorting every 1024 of them and a binary search of each in the other sorted blocks (very many: of groups of blocks, which are then merged
//      in the same way); the other workgroups of these launches fill dw with zeros;
//   2. a wave adds up 512 columns of L tokens that follow each other in that order, and stores the sum of each row of the table
//      that has all its tokens there; of the others it keeps partial sums;
//   3. where a row's tokens go on in the next wave's, the partial sums are added up.
// No atomic sums: the order of a sum depends on the sizes and ids of the call alone.
// Bound by the writes: 131072 x 4096 in f32 from 16384 tokens, 391 us: zeros 305 (2.15 GB at 7 TB/s, one workgroup for every 4 KB; 2048
// persistent ones 425), search 5, sums 58 (134 MB read, 119 written: 4.4 TB/s; the slices of a row in workgroups far apart
// 92), joins 6, four launches.  Zeros only where no token is, in the launch of the sums: 472 us in all, as reads and writes here and there slow the
// fill.  Few tokens have a workgroup for each row in place of 2 and 3.
// ------------------------------------------------------------------------
// 16-byte pieces, in the order in which workgroups begin: those of a launch write near each other
__device__ __forceinline__ void fill_zeros(uint4* __restrict__ to, long n, long group, long groups) {
    for (long i = group * 256 + threadIdx.x; i < n; i += groups * 256) to[i] = uint4{0, 0, 0, 0};
}

// Up to kPlaceTokens tokens: a workgroup counts for 64 of them the tokens in front of each, a wave a quarter of all.  512 tokens 4.6 us, 1024
// 6.4; sorting them 8.3.
__global__ __launch_bounds__(256) void embedding_place_kernel(const void* ids, bool wide, int T, long first, long rows, int blocks, uint32_t* __restrict__ row_out,
                                                              uint32_t* __restrict__ token_out, uint4* __restrict__ fill, long fill16) {
    __shared__ u32x4 lds4[kPlaceTokens / 4];
    __shared__ int found[4][64];
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    if ((int)blockIdx.x >= blocks) return fill_zeros(fill, fill16, (int)blockIdx.x - blocks, (int)gridDim.x - blocks);
    uint32_t* const lds = reinterpret_cast<uint32_t*>(lds4);
    const int words = blocks;                            // of 64 tokens
    for (int i = t; i < words * 64; i += 256) lds[i] = i < T ? row_of(ids, wide, i, first, rows) : ~0u;
    __syncthreads();
    const int mine = blockIdx.x, token = mine * 64 + l;
    const uint32_t row = lds[token];
    int count = 0;
    for (int q = w; q < words; q += 4) {
        const u32x4* p = lds4 + q * 16;
        const bool own = q == mine;
        const uint32_t under = row + (q < mine ? 1u : 0u);               // of tokens in front of these those of the same row come first
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            const u32x4 other = p[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) count += other[j] < (own ? row + (4 * i + j < l ? 1u : 0u) : under) ? 1 : 0;
        }
    }
    found[w][l] = count;
    __syncthreads();
    if (w != 0 || token >= T) return;
    const int place = found[0][l] + found[1][l] + found[2][l] + found[3][l];
    row_out[place] = row;
    token_out[place] = (uint32_t)token;
}

__device__ __forceinline__ uint32_t xor_lane(uint32_t v, int mask) { return __shfl_xor(v, mask); }
__device__ __forceinline__ uint64_t xor_lane(uint64_t v, int mask) {
    const uint32_t lo = __shfl_xor((uint32_t)v, mask), hi = __shfl_xor((uint32_t)(v >> 32), mask);
    return (uint64_t)hi << 32 | lo;
}

// A key is a row and a token's place in the block, 10 bits: 32 bits for tables of up to kNarrowRows rows, else 64.  The keys of tokens
// without a row and of what fills the block have the largest rows there are.  A chain of exchanges across lanes, 8.5 us, which the zeros hide; with
// keys of 64 bits 9.4.
template <class Key>
__global__ __launch_bounds__(256) void embedding_sort_kernel(const void* ids, bool wide, long T, long first, long rows, int blocks, uint32_t* __restrict__ row_out,
                                                             uint32_t* __restrict__ token_out, uint4* __restrict__ fill, long fill16) {
    constexpr int kPlace = 10;
    static_assert(kSortBlock == 1 << kPlace, "");
    constexpr Key kNone = (Key)~(Key)0 >> kPlace;        // row of a key, of no token; kNone - 1: of a token without a row
    __shared__ Key lds[kSortBlock];
    const int t = threadIdx.x;
    if ((int)blockIdx.x >= blocks) return fill_zeros(fill, fill16, (int)blockIdx.x - blocks, (int)gridDim.x - blocks);
    // bitonic network over element e = 4 thread + i: distances 1 and 2 in a thread, 4 to 128 across lanes, 256 and 512 across waves
    const long base = (long)blockIdx.x * kSortBlock;
    Key v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long at = base + 4 * t + i;
        const uint32_t r = at < T ? row_of(ids, wide, at, first, rows) : kNoRow;
        v[i] = (at >= T ? kNone : r == kNoRow ? kNone - 1 : (Key)r) << kPlace | (Key)(4 * t + i);
    }
    auto order = [](Key& lo, Key& hi, bool up) {
        const bool swap = (lo > hi) == up;
        const Key a = swap ? hi : lo, b = swap ? lo : hi;
        lo = a;
        hi = b;
    };
    for (int k = 2; k <= kSortBlock; k *= 2) {
        for (int j = k / 2; j > 2; j /= 2) {
            Key other[4];
            if (j >= 256) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) lds[i * 256 + t] = v[i];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) other[i] = lds[i * 256 + (t ^ (j / 4))];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) other[i] = xor_lane(v[i], j / 4);
            }
            const bool up = ((4 * t) & k) == 0, lower = ((4 * t) & j) == 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool take = (other[i] < v[i]) == (up == lower);
                v[i] = take ? other[i] : v[i];
            }
        }
        if (k >= 4) {
            const bool up = ((4 * t) & k) == 0;
            order(v[0], v[2], up);
            order(v[1], v[3], up);
            order(v[0], v[1], up);
            order(v[2], v[3], up);
        } else {
            order(v[0], v[1], true);
            order(v[2], v[3], false);
        }
    }
    // (the arrays have whole blocks)
    uint32_t r[4], token[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Key row = v[i] >> kPlace;
        r[i] = row >= kNone - 1 ? kNoRow + (uint32_t)(row - (kNone - 1)) : (uint32_t)row;
        token[i] = (uint32_t)base + (uint32_t)(v[i] & (kSortBlock - 1));
    }
    *reinterpret_cast<uint4*>(row_out + base + 4 * t) = uint4{r[0], r[1], r[2], r[3]};
    *reinterpret_cast<uint4*>(token_out + base + 4 * t) = uint4{token[0], token[1], token[2], token[3]};
}

// A workgroup finds the places of 64 tokens: each of its four waves searches all of them in every fourth block, kAtOnce (8) blocks in LDS at a
// time, the next ones on their way.  16384 tokens 4.8 us, 32768 7.0 (with a branch for every comparison, and the rows on their way in scratch
// memory, 13 and 25).  Others fill what zeros are left; kAtOnce is 4 then, so that LDS holds twice as many of them (3 us less, of 55).
template <int kAtOnce>
__global__ __launch_bounds__(256) void embedding_rank_kernel(const uint32_t* __restrict__ row_in, const uint32_t* __restrict__ token_in, long T, int all, int at_once,
                                                             uint32_t* __restrict__ row_out, uint32_t* __restrict__ token_out, int groups, uint4* __restrict__ fill,
                                                             long fill16) {
    constexpr int kEach = kAtOnce / 4;
    __shared__ u32x4 lds4[kAtOnce * kSortBlock / 4];
    __shared__ int found[4][64];
    if ((int)blockIdx.x >= groups) return fill_zeros(fill, fill16, (int)blockIdx.x - groups, (int)gridDim.x - groups);
    // of at_once blocks that become one run: this one's place among them, and how many there are
    const int block = blockIdx.x / (kSortBlock / 64), first = block / at_once * at_once, mine = block - first, blocks = min(at_once, all - first);
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    const uint32_t* const lds = reinterpret_cast<const uint32_t*>(lds4) + w * kSortBlock;
    const long at = (long)blockIdx.x * 64 + l;
    const uint32_t row = row_in[at];
    const u32x4* const from = reinterpret_cast<const u32x4*>(row_in + first * kSortBlock) + t;
    u32x4 q[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) q[i] = from[(long)min(i, blocks - 1) * (kSortBlock / 4)];
    int count = 0;
    for (int b0 = 0; b0 < blocks; b0 += kAtOnce) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) lds4[i * 256 + t] = q[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) q[i] = from[(long)min(b0 + kAtOnce + i, blocks - 1) * (kSortBlock / 4)];
        // tokens of block b in front of this one: those of rows below `under`, which is the next row where the block comes first
        int pos[kEach] = {};
        uint32_t under[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) under[i] = row + (b0 + 4 * i + w < mine ? 1u : 0u);
#pragma unroll
        for (int step = kSortBlock / 2; step > 0; step /= 2) {
            uint32_t other[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) other[i] = lds[4 * i * kSortBlock + pos[i] + step - 1];
#pragma unroll
            for (int i = 0; i < kEach; ++i) pos[i] += other[i] < under[i] ? step : 0;
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int b = b0 + 4 * i + w;
            pos[i] += lds[4 * i * kSortBlock + pos[i]] < under[i] ? 1 : 0;
            if (b < blocks && b != mine) count += pos[i];            // uniform
        }
    }
    found[w][l] = count;
    __syncthreads();
    if (w != 0 || at >= T) return;
    const long place = at - (long)mine * kSortBlock + found[0][l] + found[1][l] + found[2][l] + found[3][l];
    row_out[place] = row;
    token_out[place] = token_in[at];
}

// Each kMergeRuns runs of `run` tokens, a power of two (the last one as long as it is), become one: a thread searches the place of its token in all
// others of them.  Neighbours search for neighbouring rows, in the same cache lines.
__global__ __launch_bounds__(256) void embedding_merge_kernel(const uint32_t* __restrict__ row_in, const uint32_t* __restrict__ token_in, long T, long run,
                                                              uint32_t* __restrict__ row_out, uint32_t* __restrict__ token_out) {
    constexpr int kAtOnce = 4;
    const long at = (long)blockIdx.x * 256 + threadIdx.x;
    if (at >= T) return;
    const uint32_t row = row_in[at];
    const long mine = at / run, first = mine / kMergeRuns * kMergeRuns;
    long count = at - mine * run;
    for (long j0 = first; j0 < first + kMergeRuns && j0 * run < T; j0 += kAtOnce) {
        uint32_t pos[kAtOnce], under[kAtOnce], n[kAtOnce];
        const uint32_t* from[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const long j = j0 + i;
            n[i] = j == mine ? 0 : (uint32_t)max(0L, min(run, T - j * run));
            from[i] = row_in + (n[i] ? j * run : 0);     // (none of it: the first one is read, and does not count)
            under[i] = row + (j < mine ? 1u : 0u);
            pos[i] = 0;
        }
        auto below = [&](int i, uint32_t p) {
            const uint32_t other = from[i][p < n[i] ? p : 0];
            return p < n[i] && other < under[i];
        };
        for (uint32_t step = (uint32_t)run / 2; step > 0; step /= 2) {
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) pos[i] += below(i, pos[i] + step - 1) ? step : 0;
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) count += pos[i] + (below(i, pos[i]) ? 1 : 0);
    }
    const long place = first * run + count;
    row_out[place] = row;
    token_out[place] = token_in[at];
}

struct Sum8 {
    float v[8];
};
__device__ __forceinline__ void add_row(Sum8& s, uint4 u) {
    s.v[0] += bf16_lo(u.x), s.v[1] += bf16_hi(u.x), s.v[2] += bf16_lo(u.y), s.v[3] += bf16_hi(u.y);
    s.v[4] += bf16_lo(u.z), s.v[5] += bf16_hi(u.z), s.v[6] += bf16_lo(u.w), s.v[7] += bf16_hi(u.w);
}
template <bool kF32, bool kAdd>
__device__ __forceinline__ void store_sum(void* dw, long at, const Sum8& s, float scale) {
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = s.v[i] * scale;
    if (kF32) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(dw) + at);
        if (kAdd) {
            const float4 a = p[0], b = p[1];
            o[0] += a.x, o[1] += a.y, o[2] += a.z, o[3] += a.w, o[4] += b.x, o[5] += b.y, o[6] += b.z, o[7] += b.w;
        }
        p[0] = float4{o[0], o[1], o[2], o[3]};
        p[1] = float4{o[4], o[5], o[6], o[7]};
    } else {
        uint4* p = reinterpret_cast<uint4*>(static_cast<uint16_t*>(dw) + at);
        if (kAdd) {
            const uint4 u = *p;
            o[0] += bf16_lo(u.x), o[1] += bf16_hi(u.x), o[2] += bf16_lo(u.y), o[3] += bf16_hi(u.y);
            o[4] += bf16_lo(u.z), o[5] += bf16_hi(u.z), o[6] += bf16_lo(u.w), o[7] += bf16_hi(u.w);
        }
        *p = uint4{bf16_pack2(o[0], o[1]), bf16_pack2(o[2], o[3]), bf16_pack2(o[4], o[5]), bf16_pack2(o[6], o[7])};
    }
}

// Few tokens: the wave of a token finds those of the same row; that of the first of them adds them up, with 16 rows on their way.  One launch
// and no scratch memory: 64 tokens 3.8 us in place of 18 with the order found first, 256 of them on one id 19.5 to 26 in place of 18.
template <bool kF32, bool kAdd>
__global__ __launch_bounds__(256) void embedding_bwd_direct_kernel(EmbedArgs a) {
    constexpr int kWords = kEmbedDirect / 64, kAtOnce = 16;
    const int l = threadIdx.x & 63, t = blockIdx.x, T = (int)a.T, col = (blockIdx.y * 4 + (threadIdx.x >> 6)) * 512 + l * 8;
    const uint32_t mine = row_of(a.ids, a.wide, t, a.first, a.rows);
    if (mine == kNoRow) return;
    uint64_t same[kWords];
#pragma unroll
    for (int q = 0; q < kWords; ++q) same[q] = __ballot(q * 64 + l < T && row_of(a.ids, a.wide, min(q * 64 + l, T - 1), a.first, a.rows) == mine);
    bool earlier = false;
#pragma unroll
    for (int q = 0; q < kWords; ++q) {
        const int from = t - q * 64;
        earlier |= from > 0 && (same[q] & (from >= 64 ? ~0ull : (1ull << from) - 1)) != 0;
    }
    if (earlier || col >= a.H) return;
    Sum8 s = {};
#pragma unroll
    for (int q = 0; q < kWords; ++q) {
        while (same[q]) {
            int at[kAtOnce];
            uint4 u[kAtOnce];
            at[0] = q * 64 + __ffsll((unsigned long long)same[q]) - 1;
            same[q] &= same[q] - 1;
#pragma unroll
            for (int i = 1; i < kAtOnce; ++i) {          // past the last one: the first one again
                at[i] = same[q] ? q * 64 + __ffsll((unsigned long long)same[q]) - 1 : at[0];
                same[q] &= same[q] - 1;
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) u[i] = load16_nt(a.dy + (long)at[i] * a.H + col);
            add_row(s, u[0]);
#pragma unroll
            for (int i = 1; i < kAtOnce; ++i)
                if (at[i] != at[0]) add_row(s, u[i]);
        }
    }
    store_sum<kF32, kAdd>(a.dw, (long)mine * a.H + col, s, a.scale);
}

// Up to kPlaceTokens tokens of a few columns, in their order: the workgroup of the first token of a row adds up 512 columns of all of them, each wave 8
// of every 64; those of the other tokens end at once.  One launch for two (1001 x 1024 to f32 24 us in place of 26), until there are too many
// workgroups that only end.
template <bool kF32, bool kAdd>
__global__ __launch_bounds__(512) void embedding_run_kernel(EmbedArgs a, const uint32_t* __restrict__ rows, const uint32_t* __restrict__ tokens) {
    constexpr int kWaves = 8, kAtOnce = 8;
    __shared__ float part[kWaves - 1][8][64];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = blockIdx.x, T = (int)a.T, col = (int)blockIdx.y * 512 + l * 8;
    const uint16_t* const from = a.dy + min(col, a.H - 8);
    uint32_t at_row = rows[min(p + l, T - 1)], token = tokens[min(p + l, T - 1)];
    const uint32_t before = rows[max(p - 1, 0)], row = __builtin_amdgcn_readfirstlane(at_row);
    if (row == kNoRow || (p > 0 && before == row)) return;
    Sum8 s = {};
    bool several = false;
    for (int base = p; base < T; base += 64) {
        const int ahead = min(base + 64 + l, T - 1);
        const uint32_t next_row = rows[ahead], next_token = tokens[ahead];
        const uint64_t other = __ballot(base + l >= T || at_row != row);
        const int n = other ? __ffsll((unsigned long long)other) - 1 : 64;
        several |= n > kAtOnce || base > p;
        if (w * kAtOnce < n) {
            uint4 u[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) u[i] = load16_nt(from + (long)(uint32_t)__builtin_amdgcn_readlane((int)token, min(w * kAtOnce + i, n - 1)) * a.H);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (w * kAtOnce + i < n) add_row(s, u[i]);
        }
        if (n < 64) break;
        at_row = next_row;
        token = next_token;
    }
    if (several) {
        if (w > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) part[w - 1][i][l] = s.v[i];
        }
        __syncthreads();
        if (w > 0) return;
#pragma unroll
        for (int j = 0; j < kWaves - 1; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s.v[i] += part[j][i][l];
    }
    if (w > 0 || col >= a.H) return;
    store_sum<kF32, kAdd>(a.dw, (long)row * a.H + col, s, a.scale);
}

template <bool kF32, bool kAdd>
__global__ __launch_bounds__(256) void embedding_sum_kernel(EmbedArgs a, int L, long blocks, const uint32_t* __restrict__ rows, const uint32_t* __restrict__ tokens,
                                                            float* __restrict__ partial) {
    // the slices of 512 columns of a block are neighbours
    const int l = threadIdx.x & 63, slices = (a.H + 511) >> 9;
    const long unit = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = unit / slices;
    const int col = (int)(unit - b * slices) * 512 + l * 8;
    if (b >= blocks) return;
    const long p0 = b * L;
    const int n = (int)min((long)L, a.T - p0);
    // lane i: row and token of place p0 + i, lane L (n) the row behind the last
    const uint32_t my_row = l <= n && p0 + l < a.T ? rows[p0 + l] : kNoRow, my_token = l < n ? tokens[p0 + l] : 0;
    const uint32_t before = p0 > 0 ? rows[p0 - 1] : kNoRow;
    const bool have = col < a.H;
    auto row_at = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)my_row, i); };
    uint32_t cur = row_at(0);
    if (cur == kNoRow) return;                           // nor has any token behind it a row
    bool began_here = before != cur;
    Sum8 s = {};
    auto flush = [&](bool goes_on) {
        if (!have || cur == kNoRow) return;
        if (began_here && !goes_on) {
            store_sum<kF32, kAdd>(a.dw, (long)cur * a.H + col, s, a.scale);
        } else {
            float4* p = reinterpret_cast<float4*>(partial + (b * 2 + (began_here ? 1 : 0)) * a.H + col);
            p[0] = float4{s.v[0], s.v[1], s.v[2], s.v[3]};
            p[1] = float4{s.v[4], s.v[5], s.v[6], s.v[7]};
        }
    };
    // No branch around a load, so that the next ones are on their way: tokens without a row (at the end of the last block that has one) are read
    // like others, and their sum is not stored.  With branches, one round after the other, an eighth of 32768 tokens x 5120 took 14.4 us in
    // place of 13.6, all of 16384 x 4096 to f32 61 in place of 57.
    constexpr int kAtOnce = 8;
    const uint16_t* const from = a.dy + min(col, a.H - 8);
    auto load = [&](uint4 (&u)[kAtOnce], int i0) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) u[i] = load16_nt(from + (long)(uint32_t)__builtin_amdgcn_readlane((int)my_token, min(i0 + i, n - 1)) * a.H);
    };
    auto add = [&](const uint4 (&u)[kAtOnce], int i0) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (i0 + i >= n) break;
            const uint32_t row = row_at(i0 + i);
            if (row != cur) {
                flush(false);
                cur = row;
                began_here = true;
                s = Sum8{};
            }
            add_row(s, u[i]);
        }
    };
    uint4 u[kAtOnce], v[kAtOnce];
    load(u, 0);
    for (int i0 = 0; i0 < n; i0 += 2 * kAtOnce) {        // the next ones on their way
        if (i0 + kAtOnce < n) load(v, i0 + kAtOnce);
        add(u, i0);
        if (i0 + 2 * kAtOnce < n) load(u, i0 + 2 * kAtOnce);
        add(v, i0 + kAtOnce);
    }
    flush(row_at(n) == cur);
}

template <bool kF32, bool kAdd>
__device__ __forceinline__ void store_joined(const EmbedArgs& a, uint32_t row, int col, float4 s) {
    const long at = (long)row * a.H + col;
    float4 o = {s.x * a.scale, s.y * a.scale, s.z * a.scale, s.w * a.scale};
    if (kF32) {
        float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.dw) + at);
        if (kAdd) o.x += to->x, o.y += to->y, o.z += to->z, o.w += to->w;
        *to = o;
    } else {
        uint2* to = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.dw) + at);
        if (kAdd) o.x += bf16_lo(to->x), o.y += bf16_hi(to->x), o.z += bf16_lo(to->y), o.w += bf16_hi(to->y);
        *to = uint2{bf16_pack2(o.x, o.y), bf16_pack2(o.z, o.w)};
    }
}
__device__ __forceinline__ void add4(float4& s, float4 v) { s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w; }

constexpr int kJoinCols = 2048;                          // of a workgroup: most of them find nothing to add (1024: 0.7 us more for 32768 tokens x 5120)
// Blocks from c on that begin with `row`, c being one of them or the one in front
__device__ __forceinline__ long blocks_of(const uint32_t* __restrict__ rows, uint32_t row, long c, int L, long blocks) {
    const int l = threadIdx.x & 63;
    for (long n = 0;; n += 64) {
        const long at = c + n + l;
        const uint64_t other = __ballot(at >= blocks || rows[min(at, blocks - 1) * L] != row);
        if (other) return n + __ffsll((unsigned long long)other) - 1;
    }
}

// The workgroups of the first `grid` numbers add up a row that goes on in up to kLongRun blocks behind the one where it begins: each thread twice 4
// columns, all partial sums one after the other.  A longer one belongs to the first multiple of kLongRun among the blocks that it goes
// on in, which has workgroups of 64 columns and 16 runs of partial sums each.  All tokens on one id, as padding has it, added to f32, all
// launches, us, without / with them: 16384 x 1024 184 / 43, 32768 x 1024 192 / 51, 32768 x 4096 141 / 78.
template <bool kF32, bool kAdd>
__global__ __launch_bounds__(256) void embedding_join_kernel(EmbedArgs a, int L, long blocks, const uint32_t* __restrict__ rows, const float* __restrict__ partial,
                                                             int grid, int wide_cols, int narrow_cols) {
    const int l = threadIdx.x & 63;
    if ((int)blockIdx.x < grid) {
        const long b = blockIdx.x / wide_cols, next = (b + 1) * L;       // b is not the last block
        const uint32_t row = rows[next], last = rows[next - 1], first = rows[b * L], before = rows[b ? b * L - 1 : 0];
        if (row == kNoRow || last != row || (first == row && b > 0 && before == row)) return;      // begins behind this block, or in front of it
        const long n = blocks_of(rows, row, b + 1, L, blocks);
        if (n > kLongRun) return;
        const int c0 = (int)(blockIdx.x - b * wide_cols) * kJoinCols + threadIdx.x * 4;
        for (int col = c0; col < min(c0 + kJoinCols, a.H); col += 1024) {
            const float* p = partial + b * 2 * a.H + col;
            float4 s = *reinterpret_cast<const float4*>(p + a.H);
            constexpr int kAtOnce = 8;
            for (long i = 1; i <= n; i += kAtOnce) {
                float4 v[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) v[j] = i + j <= n ? *reinterpret_cast<const float4*>(p + (i + j) * 2 * a.H) : float4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) add4(s, v[j]);
            }
            store_joined<kF32, kAdd>(a, row, col, s);
        }
        return;
    }
    __shared__ float4 part[16][16];
    const int i = blockIdx.x - grid;
    const long c = (long)(i / narrow_cols + 1) * kLongRun;               // a block; does a row that began earlier go on in it?
    const uint32_t row = rows[c * L];
    if (row == kNoRow || rows[c * L - 1] != row) return;
    // of the kLongRun blocks in front of it, those that the row goes on in (as far as there is no gap)
    const long e = c - 1 - l;
    const uint64_t not_on = __ballot(l >= kLongRun || e < 1 || rows[max(e, 0L) * L] != row || rows[max(e * L, 1L) - 1] != row);
    const int back = __ffsll((unsigned long long)not_on) - 1;
    if (back >= kLongRun) return;                                        // that of the multiple before has it
    const long b = c - 1 - back, n = back + blocks_of(rows, row, c, L, blocks);
    if (n <= kLongRun) return;
    const int part_id = threadIdx.x >> 4, l16 = threadIdx.x & 15, col = (i % narrow_cols) * 64 + l16 * 4;
    float4 s = {0, 0, 0, 0};
    if (col < a.H) {
        const float* p = partial + b * 2 * a.H + col;
        const long from = (n + 1) * part_id / 16, to = (n + 1) * (part_id + 1) / 16;
        constexpr int kAtOnce = 8;
        for (long j0 = from; j0 < to; j0 += kAtOnce) {
            float4 v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                v[j] = j0 + j < to ? *reinterpret_cast<const float4*>(p + (j0 + j) * 2 * a.H + (j0 + j == 0 ? a.H : 0)) : float4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) add4(s, v[j]);
        }
    }
    part[part_id][l16] = s;
    __syncthreads();
    if (part_id != 0 || col >= a.H) return;
#pragma unroll
    for (int j = 1; j < 16; ++j) add4(s, part[j][l16]);
    store_joined<kF32, kAdd>(a, row, col, s);
}

template <bool kF32, bool kAdd>
hipError_t launch_sums(const EmbedArgs& a, char* ws, hipStream_t st) {
    if (a.T <= kEmbedDirect) {
        hipLaunchKernelGGL((embedding_bwd_direct_kernel<kF32, kAdd>), dim3((unsigned)a.T, (unsigned)((a.H + 2047) / 2048)), dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const EmbedSpace sp = embed_space(a.T, a.H);
    const long each = sp.tmp / 2;
    const uint32_t *rows = reinterpret_cast<uint32_t*>(ws), *tokens = reinterpret_cast<uint32_t*>(ws + each);
    if (embed_by_runs(a.T, a.H)) {
        hipLaunchKernelGGL((embedding_run_kernel<kF32, kAdd>), dim3((unsigned)a.T, (unsigned)((a.H + 511) / 512)), dim3(512), 0, st, a, rows, tokens);
        return hipGetLastError();
    }
    float* partial = reinterpret_cast<float*>(ws + sp.partial);
    const int L = embed_block(a.T, a.H);
    const long blocks = (a.T + L - 1) / L;
    hipLaunchKernelGGL((embedding_sum_kernel<kF32, kAdd>), dim3((unsigned)((blocks * ((a.H + 511) / 512) + 3) / 4)), dim3(256), 0, st, a, L, blocks,
                       rows, tokens, partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    const int wide_cols = (a.H + kJoinCols - 1) / kJoinCols, narrow_cols = (a.H + 63) / 64;
    const long grid = (blocks - 1) * wide_cols, longs = (blocks - 1) / kLongRun * narrow_cols;
    hipLaunchKernelGGL((embedding_join_kernel<kF32, kAdd>), dim3((unsigned)(grid + longs)), dim3(256), 0, st, a, L, blocks, rows, partial, (int)grid, wide_cols,
                       narrow_cols);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_fwd(const EmbedArgs& a, hipStream_t st) {
    int log2 = 0;
    while (log2 < 8 && (8 << log2) < a.H) ++log2;
    const long per = 256 >> log2;
    const bool nt = writes_past_the_caches(2 * a.T * a.H);
    const auto kernel = a.f32 ? (nt ? embedding_fwd_kernel<true, true> : embedding_fwd_kernel<true, false>)
                              : (nt ? embedding_fwd_kernel<false, true> : embedding_fwd_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.T + per - 1) / per)), dim3(256), 0, st, a, log2);
    return hipGetLastError();
}

hipError_t launch_embedding_bwd(const EmbedArgs& a, void* workspace, hipStream_t st) {
    char* ws = static_cast<char*>(workspace);
    const bool direct = a.T <= kEmbedDirect, places = !direct && a.T <= kPlaceTokens;
    const long each = places ? 64 : kSortBlock, blocks = direct ? 0 : (a.T + each - 1) / each, fill16 = a.add ? 0 : a.rows * a.H * (a.f32 ? 4 : 2) / 16;
    const long later = direct || places ? 0 : embed_zeros_later(fill16 * 16) / 16, now = fill16 - later;
    const long fillers = std::min<long>((now + 255) / 256, 1L << 23);
    if (blocks + fillers > 0) {
        const EmbedSpace sp = embed_space(a.T, a.H);
        const long array = sp.tmp / 2;
        auto rows = [&](long at) { return reinterpret_cast<uint32_t*>(ws + at); };
        auto tokens = [&](long at) { return reinterpret_cast<uint32_t*>(ws + at + array); };
        const dim3 grid((unsigned)(blocks + fillers));
        uint4* const fill = static_cast<uint4*>(a.dw);
        // the last of the launches that put them in order leaves them at 0
        const int merges = direct || places ? 0 : embed_merges(a.T);
        long at = direct || places || merges % 2 ? 0 : sp.tmp;
        if (direct || places) {
            hipLaunchKernelGGL(embedding_place_kernel, grid, dim3(256), 0, st, a.ids, a.wide, (int)a.T, a.first, a.rows, (int)blocks, rows(at), tokens(at), fill, now);
        } else {
            const auto sort = a.rows <= kNarrowRows ? embedding_sort_kernel<uint32_t> : embedding_sort_kernel<uint64_t>;
            hipLaunchKernelGGL(sort, grid, dim3(256), 0, st, a.ids, a.wide, a.T, a.first, a.rows, (int)blocks, rows(at), tokens(at), fill, now);
        }
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (!direct && !places) {
            long run = merges ? kRankBlocks * kSortBlock : a.T, to = sp.tmp - at;
            const long groups = (a.T + 63) / 64, behind = (later + 255) / 256;
            const auto rank = later ? embedding_rank_kernel<4> : embedding_rank_kernel<8>;
            hipLaunchKernelGGL(rank, dim3((unsigned)(groups + behind)), dim3(256), 0, st, rows(at), tokens(at), a.T, (int)blocks, merges ? (int)kRankBlocks : (int)blocks,
                               rows(to), tokens(to), (int)groups, fill + now, later);
            e = hipGetLastError();
            for (int i = 0; i < merges && e == hipSuccess; ++i, run *= kMergeRuns) {
                std::swap(at, to);
                hipLaunchKernelGGL(embedding_merge_kernel, dim3((unsigned)((a.T + 255) / 256)), dim3(256), 0, st, rows(at), tokens(at), a.T, run, rows(to), tokens(to));
                e = hipGetLastError();
            }
            if (e != hipSuccess) return e;
        }
    }
    if (a.f32) return a.add ? launch_sums<true, true>(a, ws, st) : launch_sums<true, false>(a, ws, st);
    return a.add ? launch_sums<false, true>(a, ws, st) : launch_sums<false, false>(a, ws, st);
}

}  // namespace jet

// Embedding: rows of the table for the tokens of a call, and the table's gradient.
#include "jet_internal.h"
#include "jet_numerics.h"
#include "jet_step.h"

namespace jet {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kNoRow = 0xfffffffeu;             // a token whose id the table does not hold; behind all rows in their order, and
                                                     // in front of what fills the last block

__device__ __forceinline__ uint32_t row_of(const void* ids, bool wide, long t, long first, long rows) {
    const long r = (wide ? reinterpret_cast<const int64_t*>(ids)[t] : (int64_t)reinterpret_cast<const int32_t*>(ids)[t]) - first;
    return r >= 0 && r < rows ? (uint32_t)r : kNoRow;
}

// ------------------------------------------------------------------------
// y[t] = bf16(scale w[row of t]), zeros without a row.  tx threads (a power of two) go along a row, 8 columns each, with the loads of
// four such pieces under way.
// ------------------------------------------------------------------------
template <bool kF32>
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
            store16_nt(y + k, uint4{o[0], o[1], o[2], o[3]});
        }
    }
}

// ------------------------------------------------------------------------
// The gradient: dw[r] = scale sum of dy[t] over the tokens t of row r, in the order of the tokens.
//   1. every 1024 tokens are sorted by (row, token); the other workgroups of the launch fill dw with zeros;
//   2. with more than 1024 tokens, each finds its place in the order of all of them by binary search in the other sorted blocks;
//   3. a wave adds up the rows of L tokens that follow each other in that order, and stores the sum of each row of the table
//      that has all its tokens there; of the others it keeps partial sums;
//   4. where a row's tokens go on in the next wave's, the partial sums are added up.
// No atomic sums: the order depends on the sizes and ids of the call alone.
// ------------------------------------------------------------------------
__device__ __forceinline__ uint64_t xor_lane(uint64_t v, int mask) {
    const uint32_t lo = __shfl_xor((uint32_t)v, mask), hi = __shfl_xor((uint32_t)(v >> 32), mask);
    return (uint64_t)hi << 32 | lo;
}

__global__ __launch_bounds__(256) void embedding_sort_kernel(const void* ids, bool wide, long T, long first, long rows, int blocks, uint32_t* __restrict__ row_out,
                                                             uint32_t* __restrict__ token_out, uint4* __restrict__ fill, long fill16) {
    __shared__ uint64_t lds[kSortBlock];
    const int t = threadIdx.x;
    if ((int)blockIdx.x >= blocks) {
        const long step = (long)(gridDim.x - blocks) * 256;
        for (long i = (long)(blockIdx.x - blocks) * 256 + t; i < fill16; i += step) fill[i] = uint4{0, 0, 0, 0};
        return;
    }
    // bitonic network over element e = 4 thread + i: distances 1 and 2 in a thread, 4 to 128 across lanes, 256 and 512 across waves
    const long base = (long)blockIdx.x * kSortBlock;
    uint64_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long at = base + 4 * t + i;
        v[i] = at < T ? (uint64_t)row_of(ids, wide, at, first, rows) << 32 | (uint32_t)at : ~0ull;
    }
    auto order = [](uint64_t& lo, uint64_t& hi, bool up) {
        const bool swap = (lo > hi) == up;
        const uint64_t a = swap ? hi : lo, b = swap ? lo : hi;
        lo = a;
        hi = b;
    };
    for (int k = 2; k <= kSortBlock; k *= 2) {
        for (int j = k / 2; j > 2; j /= 2) {
            uint64_t other[4];
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
    *reinterpret_cast<uint4*>(row_out + base + 4 * t) = uint4{(uint32_t)(v[0] >> 32), (uint32_t)(v[1] >> 32), (uint32_t)(v[2] >> 32), (uint32_t)(v[3] >> 32)};
    *reinterpret_cast<uint4*>(token_out + base + 4 * t) = uint4{(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]};
}

// A workgroup finds the places of 64 tokens: each of its four waves searches all of them in every fourth block.
__global__ __launch_bounds__(256) void embedding_rank_kernel(const uint32_t* __restrict__ row_in, const uint32_t* __restrict__ token_in, long T, int blocks,
                                                             uint32_t* __restrict__ row_out, uint32_t* __restrict__ token_out) {
    constexpr int kAtOnce = 8, kEach = kAtOnce / 4;
    __shared__ u32x4 lds4[kAtOnce * kSortBlock / 4];
    __shared__ int found[4][64];
    const int t = threadIdx.x, l = t & 63, w = t >> 6, mine = blockIdx.x / (kSortBlock / 64);
    const uint32_t* const lds = reinterpret_cast<const uint32_t*>(lds4) + w * kSortBlock;
    const long at = (long)blockIdx.x * 64 + l;
    const uint32_t row = row_in[at];
    const u32x4* const from = reinterpret_cast<const u32x4*>(row_in) + t;
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

// Up to 64 tokens: the wave of a token finds those of the same row; that of the first of them adds them up.
template <bool kF32, bool kAdd>
__global__ __launch_bounds__(256) void embedding_bwd_direct_kernel(EmbedArgs a) {
    const int l = threadIdx.x & 63, t = blockIdx.x, col = (blockIdx.y * 4 + (threadIdx.x >> 6)) * 512 + l * 8;
    const uint32_t row = l < a.T ? row_of(a.ids, a.wide, l, a.first, a.rows) : kNoRow;
    const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)row, t);
    if (mine == kNoRow) return;
    uint64_t same = __ballot(row == mine);
    if (__ffsll((unsigned long long)same) - 1 != t || col >= a.H) return;
    Sum8 s = {};
    while (same) {
        const int at = __ffsll((unsigned long long)same) - 1;
        same &= same - 1;
        add_row(s, *reinterpret_cast<const uint4*>(a.dy + (long)at * a.H + col));
    }
    store_sum<kF32, kAdd>(a.dw, (long)mine * a.H + col, s, a.scale);
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
    constexpr int kAtOnce = 8;
    for (int i0 = 0; i0 < n; i0 += kAtOnce) {
        uint4 u[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int at = min(i0 + i, n - 1);
            u[i] = uint4{0, 0, 0, 0};
            if (have && row_at(at) != kNoRow)
                u[i] = load16_nt(a.dy + (long)(uint32_t)__builtin_amdgcn_readlane((int)my_token, at) * a.H + col);
        }
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
    }
    flush(row_at(n) == cur);
}

template <bool kF32, bool kAdd>
__global__ __launch_bounds__(256) void embedding_join_kernel(EmbedArgs a, int L, long blocks, const uint32_t* __restrict__ rows, const float* __restrict__ partial) {
    const int l = threadIdx.x & 63;
    const long b = blockIdx.x, next = (b + 1) * L;       // b is not the last block
    const uint32_t row = rows[next], last = rows[next - 1], first = rows[b * L], before = rows[b ? b * L - 1 : 0];
    if (row == kNoRow || last != row || (first == row && b > 0 && before == row)) return;      // begins behind this block, or in front of it
    long n = 0;                                          // blocks behind b that begin with this row
    for (;;) {
        const long c = b + 1 + n + l;
        const uint64_t other = __ballot(c >= blocks || rows[c * L] != row);
        if (other) {
            n += __ffsll((unsigned long long)other) - 1;
            break;
        }
        n += 64;
    }
    const int col = (blockIdx.y * 256 + threadIdx.x) * 4;
    if (col >= a.H) return;
    const float* p = partial + b * 2 * a.H + col;
    float4 s = *reinterpret_cast<const float4*>(p + a.H);
    constexpr int kAtOnce = 8;
    for (long i = 1; i <= n; i += kAtOnce) {
        float4 v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) v[j] = i + j <= n ? *reinterpret_cast<const float4*>(p + (i + j) * 2 * a.H) : float4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) s.x += v[j].x, s.y += v[j].y, s.z += v[j].z, s.w += v[j].w;
    }
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

template <bool kF32, bool kAdd>
hipError_t launch_sums(const EmbedArgs& a, char* ws, hipStream_t st) {
    if (a.T <= kEmbedDirect) {
        hipLaunchKernelGGL((embedding_bwd_direct_kernel<kF32, kAdd>), dim3((unsigned)a.T, (unsigned)((a.H + 2047) / 2048)), dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const EmbedSpace sp = embed_space(a.T, a.H);
    const long each = sp.tmp / 2;
    const uint32_t *rows = reinterpret_cast<uint32_t*>(ws), *tokens = reinterpret_cast<uint32_t*>(ws + each);
    float* partial = reinterpret_cast<float*>(ws + sp.partial);
    const int L = embed_block(a.T, a.H);
    const long blocks = (a.T + L - 1) / L;
    hipLaunchKernelGGL((embedding_sum_kernel<kF32, kAdd>), dim3((unsigned)((blocks * ((a.H + 511) / 512) + 3) / 4)), dim3(256), 0, st, a, L, blocks,
                       rows, tokens, partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    hipLaunchKernelGGL((embedding_join_kernel<kF32, kAdd>), dim3((unsigned)(blocks - 1), (unsigned)((a.H + 1023) / 1024)), dim3(256), 0, st, a, L, blocks, rows,
                       partial);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_fwd(const EmbedArgs& a, hipStream_t st) {
    int log2 = 0;
    while (log2 < 8 && (8 << log2) < a.H) ++log2;
    const long per = 256 >> log2;
    hipLaunchKernelGGL(a.f32 ? embedding_fwd_kernel<true> : embedding_fwd_kernel<false>, dim3((unsigned)((a.T + per - 1) / per)), dim3(256), 0, st, a, log2);
    return hipGetLastError();
}

hipError_t launch_embedding_bwd(const EmbedArgs& a, void* workspace, hipStream_t st) {
    char* ws = static_cast<char*>(workspace);
    const bool sorts = a.T > kEmbedDirect;
    const long blocks = sorts ? (a.T + kSortBlock - 1) / kSortBlock : 0, fill16 = a.add ? 0 : a.rows * a.H * (a.f32 ? 4 : 2) / 16;
    const long fillers = std::min<long>((fill16 + 255) / 256, 1L << 23);
    if (blocks + fillers > 0) {
        const EmbedSpace sp = embed_space(a.T, a.H);
        const long each = sp.tmp / 2, at = blocks > 1 ? sp.tmp : 0;
        uint32_t *rows = reinterpret_cast<uint32_t*>(ws + at), *tokens = reinterpret_cast<uint32_t*>(ws + at + each);
        hipLaunchKernelGGL(embedding_sort_kernel, dim3((unsigned)(blocks + fillers)), dim3(256), 0, st, a.ids, a.wide, a.T, a.first, a.rows, (int)blocks, rows,
                           tokens, static_cast<uint4*>(a.dw), fill16);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (blocks > 1) {
            hipLaunchKernelGGL(embedding_rank_kernel, dim3((unsigned)((a.T + 63) / 64)), dim3(256), 0, st, rows, tokens, a.T, (int)blocks,
                               reinterpret_cast<uint32_t*>(ws), reinterpret_cast<uint32_t*>(ws + each));
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    if (a.f32) return a.add ? launch_sums<true, true>(a, ws, st) : launch_sums<true, false>(a, ws, st);
    return a.add ? launch_sums<false, true>(a, ws, st) : launch_sums<false, false>(a, ws, st);
}

}  // namespace jet

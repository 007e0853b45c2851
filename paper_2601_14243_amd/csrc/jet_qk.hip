// Norm of every query and key head, and the rotation of its channel pairs (i, i + dim / 2) by the token's position, from the output
// of the q/k/v projection; in serving the rotated keys and the values also go to their slots of a paged cache.
//   n = x / sqrt(mean x^2 + eps) gamma,   y_i = n_i cos - n_{i + dim/2} sin,   y_{i + dim/2} = n_{i + dim/2} cos + n_i sin.
// Streams: a head is read and written once, everything in between stays in binary32 registers and is rounded once.  A lane
// has 8 channels of each half, so that a pair never leaves it, and dim / 16 lanes have a head; the angles of a token are read once
// for the heads that a lane has in turn.  16384 tokens, 32 query and 8 key heads of 128: 65.5 us for 338 MB with the angles, 5.2 TB/s;
// the gradient with 40 and 8 heads 122 us for 606 MB, 5.0 TB/s; a copy of 2 GiB goes at 4.8.  With the keys and values into a cache 85 us (436
// MB) where it is bf16, 82 (404 MB) in E4M3; one token 6.0 either way, 5.9 without.
#include <algorithm>

#include "jet_attn.h"
#include "jet_internal.h"

namespace jet {

namespace {

// sum over a team of dim / 16 lanes
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int TEAM>
__device__ __forceinline__ float team_sum(float v) {
    v = dpp_add<0xB1>(v);                        // quad_perm [1,0,3,2]
    v = dpp_add<0x4E>(v);                        // quad_perm [2,3,0,1]
    if constexpr (TEAM == 8) v = dpp_add<0x141>(v);   // row_half_mirror
    return v;
}
template <int TEAM>
__device__ __forceinline__ float team_max(float v) {
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    if constexpr (TEAM == 8) v = dpp_max<0x141>(v);
    return v;
}
__device__ __forceinline__ void unpack8(uint4 w, float* f) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo(u[i]);
        f[2 * i + 1] = bf16_hi(u[i]);
    }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
    return uint4{bf16_pack2(f[0], f[1]), bf16_pack2(f[2], f[3]), bf16_pack2(f[4], f[5]), bf16_pack2(f[6], f[7])};
}
__device__ __forceinline__ void load8(const float* p, float* f) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// cosines and sines of a token's 8 angles of this lane; NaN where the position has no row in the table
template <int DIM>
__device__ __forceinline__ void angles(const QkArgs& a, long token, int c, float (&cs)[8], float (&sn)[8]) {
    const int pos = a.positions[token];
    const bool ok = (uint32_t)pos < (uint32_t)a.table_rows;
    const float* p = a.table + (long)(ok ? pos : 0) * DIM + 8 * c;
    load8(p, cs);
    load8(p + DIM / 2, sn);
    if (!ok) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = sn[i] = NAN;
    }
}

// One head to its row of a cache: bf16, or E4M3 codes with their scale amax / 448, by the row quantizer's arithmetic on the bf16 values
template <int DIM>
__device__ __forceinline__ void to_cache(void* cache, float* scales, long row, int c, uint4 lo, uint4 hi) {
    if (!scales) {
        uint16_t* p = static_cast<uint16_t*>(cache) + row * DIM + 8 * c;
        *reinterpret_cast<uint4*>(p) = lo;
        *reinterpret_cast<uint4*>(p + DIM / 2) = hi;
        return;
    }
    float v[16];
    unpack8(lo, v);
    unpack8(hi, v + 8);
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[i]));
    const GroupScale gs = make_scale(team_max<DIM / 16>(top));
    uint32_t code[4];
    encode<kBf16Values, 16>(v, gs, code);
    uint8_t* p = static_cast<uint8_t*>(cache) + row * DIM + 8 * c;
    *reinterpret_cast<uint2*>(p) = uint2{code[0], code[1]};
    *reinterpret_cast<uint2*>(p + DIM / 2) = uint2{code[2], code[3]};
    if (c == 0) scales[row] = gs.S;
}

}  // namespace

// HB heads of one token and kind (query, key, value) for a team of DIM / 16 lanes.
template <int DIM, int HB, bool NORM>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkArgs a) {
    constexpr int TEAM = DIM / 16;
    const long unit = ((long)blockIdx.x * 256 + threadIdx.x) / TEAM;
    const int c = threadIdx.x % TEAM;
    const int nb_q = (a.n_q + HB - 1) / HB, nb_k = (a.n_kv + HB - 1) / HB, nb = nb_q + nb_k + (a.slots ? nb_k : 0);
    const long token = unit / nb;
    if (token >= a.T) return;
    int block = (int)(unit - token * nb);
    const int kind = block < nb_q ? 0 : block < nb_q + nb_k ? 1 : 2;
    block -= kind == 0 ? 0 : kind == 1 ? nb_q : nb_q + nb_k;
    const int of = kind == 0 ? a.n_q : a.n_kv, head0 = block * HB, heads = min(HB, of - head0);
    const int first = kind == 0 ? 0 : kind == 1 ? a.n_q : a.n_q + a.n_kv;

    const uint16_t* p = a.qkv + token * a.ld + (long)(first + head0) * DIM + 8 * c;
    uint4 lo[HB], hi[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i)
        if (i < heads) {
            lo[i] = *reinterpret_cast<const uint4*>(p + i * DIM);
            hi[i] = *reinterpret_cast<const uint4*>(p + i * DIM + DIM / 2);
        }
    long slot = -1;
    if (kind > 0 && a.slots) slot = a.slots[token];
    const bool cached = (uint64_t)slot < (uint64_t)(a.n_pages * a.page);      // no other slot is one: the token is not kept
    const long cache_row = cached ? (slot / a.page * a.n_kv + head0) * a.page + slot % a.page : 0;
    if (kind == 2) {
#pragma unroll
        for (int i = 0; i < HB; ++i)
            if (i < heads && cached) to_cache<DIM>(a.cache_v, a.v_scale, cache_row + (long)i * a.page, c, lo[i], hi[i]);
        return;
    }
    float cs[8], sn[8], gm[16];
    angles<DIM>(a, token, c, cs, sn);
    if constexpr (NORM) {
        const uint16_t* gp = (kind == 0 ? a.gamma_q : a.gamma_k) + 8 * c;
        unpack8(*reinterpret_cast<const uint4*>(gp), gm);
        unpack8(*reinterpret_cast<const uint4*>(gp + DIM / 2), gm + 8);
    }
    uint16_t* out = (kind == 0 ? a.q + (token * a.n_q + head0) * DIM : a.k + (token * a.n_kv + head0) * DIM) + 8 * c;
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i >= heads) break;
        float x[16], y[16];
        unpack8(lo[i], x);
        unpack8(hi[i], x + 8);
        if constexpr (NORM) {
            float sq = 0.0f;
#pragma unroll
            for (int j = 0; j < 16; ++j) sq = __builtin_fmaf(x[j], x[j], sq);
            const float r = 1.0f / sqrtf(team_sum<TEAM>(sq) * (1.0f / DIM) + a.eps);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = x[j] * r * gm[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = x[j] * cs[j] - x[j + 8] * sn[j];
            y[j + 8] = x[j + 8] * cs[j] + x[j] * sn[j];
        }
        const uint4 ylo = pack8(y), yhi = pack8(y + 8);
        *reinterpret_cast<uint4*>(out + i * DIM) = ylo;
        *reinterpret_cast<uint4*>(out + i * DIM + DIM / 2) = yhi;
        if (kind == 1 && cached) to_cache<DIM>(a.cache_k, a.k_scale, cache_row + (long)i * a.page, c, ylo, yhi);
    }
}

// The gradient: g = the rotation's transpose of dy; dgamma = sum over tokens and heads of g n, n = x r; with u = g gamma,
// dx = r (u - n mean(u n)).  The first a.groups_q workgroups have the query heads, the others the key heads; each leaves its sums of
// dgamma in `partial`, a second launch adds them in a fixed order.
template <int DIM, int HB, bool NORM>
__global__ void __launch_bounds__(256) qk_norm_rope_bwd_kernel(QkArgs a) {
    constexpr int TEAM = DIM / 16, TEAMS = 256 / TEAM;
    const int c = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const bool is_k = (int)blockIdx.x >= a.groups_q;
    const int group = blockIdx.x - (is_k ? a.groups_q : 0), groups = is_k ? gridDim.x - a.groups_q : a.groups_q;
    const int of = is_k ? a.n_kv : a.n_q, nb = (of + HB - 1) / HB;
    const uint16_t* dyp = is_k ? a.dk : a.dq;
    float gm[16], acc[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] = 0.0f;
    if constexpr (NORM) {
        const uint16_t* gp = (is_k ? a.gamma_k : a.gamma_q) + 8 * c;
        unpack8(*reinterpret_cast<const uint4*>(gp), gm);
        unpack8(*reinterpret_cast<const uint4*>(gp + DIM / 2), gm + 8);
    }
    const long units = a.T * nb;
    for (long unit = (long)group * TEAMS + team; unit < units; unit += (long)groups * TEAMS) {
        const long token = unit / nb;
        const int head0 = (int)(unit - token * nb) * HB, heads = min(HB, of - head0);
        const long col = (long)((is_k ? a.n_q : 0) + head0) * DIM + 8 * c;
        uint4 d[HB][2], xw[HB][2];
#pragma unroll
        for (int i = 0; i < HB; ++i)
            if (i < heads) {
                const uint16_t* dp = dyp + (token * of + head0 + i) * DIM + 8 * c;
                d[i][0] = *reinterpret_cast<const uint4*>(dp);
                d[i][1] = *reinterpret_cast<const uint4*>(dp + DIM / 2);
                if constexpr (NORM) {
                    const uint16_t* xp = a.qkv + token * a.ld + col + i * DIM;
                    xw[i][0] = *reinterpret_cast<const uint4*>(xp);
                    xw[i][1] = *reinterpret_cast<const uint4*>(xp + DIM / 2);
                }
            }
        float cs[8], sn[8];
        angles<DIM>(a, token, c, cs, sn);
        uint16_t* out = a.dx + token * a.ld_dx + col;
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            if (i >= heads) break;
            float y[16], u[16];
            unpack8(d[i][0], y);
            unpack8(d[i][1], y + 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                u[j] = y[j] * cs[j] + y[j + 8] * sn[j];
                u[j + 8] = y[j + 8] * cs[j] - y[j] * sn[j];
            }
            if constexpr (NORM) {
                float x[16], sq = 0.0f, dot = 0.0f;
                unpack8(xw[i][0], x);
                unpack8(xw[i][1], x + 8);
#pragma unroll
                for (int j = 0; j < 16; ++j) sq = __builtin_fmaf(x[j], x[j], sq);
                const float r = 1.0f / sqrtf(team_sum<TEAM>(sq) * (1.0f / DIM) + a.eps);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    x[j] *= r;
                    acc[j] = __builtin_fmaf(u[j], x[j], acc[j]);
                    u[j] *= gm[j];
                    dot = __builtin_fmaf(u[j], x[j], dot);
                }
                dot = team_sum<TEAM>(dot) * (1.0f / DIM);
#pragma unroll
                for (int j = 0; j < 16; ++j) u[j] = __builtin_fmaf(-x[j], dot, u[j]) * r;
            }
            *reinterpret_cast<uint4*>(out + i * DIM) = pack8(u);
            *reinterpret_cast<uint4*>(out + i * DIM + DIM / 2) = pack8(u + 8);
        }
    }
    if constexpr (NORM) {                                    // a channel's sums: 256 / DIM threads over the teams, then they
        constexpr int SHARE = 256 / DIM;
        __shared__ float sums[TEAMS][DIM], last[SHARE][DIM];
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            *reinterpret_cast<float4*>(&sums[team][(j >> 3) * (DIM / 2) + 8 * c + (j & 7)]) = float4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
        __syncthreads();
        const int ch = threadIdx.x % DIM, share = threadIdx.x / DIM;
        float s = 0.0f;
#pragma unroll
        for (int t = share; t < TEAMS; t += SHARE) s += sums[t][ch];
        last[share][ch] = s;
        __syncthreads();
        if (share == 0) {
#pragma unroll
            for (int t = 1; t < SHARE; ++t) s += last[t][ch];
            a.partial[(long)blockIdx.x * DIM + ch] = s;
        }
    }
}

// dgamma[channel] = sum over the workgroups' sums, of the query heads (blockIdx.y = 0) or the key heads; 16 channels and 64 of
// the workgroups at a time
__global__ void __launch_bounds__(1024) qk_dgamma_kernel(const float* partial, int groups_q, int groups, int dim, float* dgamma_q, float* dgamma_k) {
    __shared__ float sums[64][17];
    const int ch = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
    const int first = blockIdx.y ? groups_q : 0, n = blockIdx.y ? groups : groups_q;
    float s = 0.0f;
#pragma unroll 8
    for (int i = first + r; i < n; i += 64) s += partial[(long)i * dim + ch];
    sums[r][threadIdx.x & 15] = s;
    __syncthreads();
    if (r < 8) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += sums[r + 8 * i][threadIdx.x & 15];
        sums[r][threadIdx.x & 15] = s;
    }
    __syncthreads();
    if (r == 0) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += sums[i][threadIdx.x & 15];
        (blockIdx.y ? dgamma_k : dgamma_q)[ch] = s;
    }
}

long qk_bwd_workspace(long T, long n_q, long n_kv, long dim) {
    const QkBwdGroups g = qk_bwd_groups(T, n_q, n_kv, dim);
    return (g.q + g.k) * dim * (long)sizeof(float);
}

hipError_t launch_qk_norm_rope(const QkArgs& a, int dim, hipStream_t st) {
    const bool few = qk_few_heads(a.T, a.n_q, a.n_kv, dim, a.slots), norm = a.gamma_q != nullptr;
    const auto kernel = dim == 128 ? (few ? (norm ? qk_norm_rope_kernel<128, 1, true> : qk_norm_rope_kernel<128, 1, false>)
                                          : (norm ? qk_norm_rope_kernel<128, 4, true> : qk_norm_rope_kernel<128, 4, false>))
                                   : (few ? (norm ? qk_norm_rope_kernel<64, 1, true> : qk_norm_rope_kernel<64, 1, false>)
                                          : (norm ? qk_norm_rope_kernel<64, 4, true> : qk_norm_rope_kernel<64, 4, false>));
    hipLaunchKernelGGL(kernel, dim3((unsigned)qk_workgroups(a.T, a.n_q, a.n_kv, dim, a.slots, few ? 1 : 4)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_qk_norm_rope_bwd(QkArgs a, int dim, float* dgamma_q, float* dgamma_k, void* workspace, hipStream_t st) {
    const bool norm = a.gamma_q != nullptr;
    const QkBwdGroups g = qk_bwd_groups(a.T, a.n_q, a.n_kv, dim);
    a.groups_q = (int)g.q;
    a.partial = static_cast<float*>(workspace);
    const auto kernel = dim == 128 ? (g.few ? (norm ? qk_norm_rope_bwd_kernel<128, 1, true> : qk_norm_rope_bwd_kernel<128, 1, false>)
                                            : (norm ? qk_norm_rope_bwd_kernel<128, 4, true> : qk_norm_rope_bwd_kernel<128, 4, false>))
                                   : (g.few ? (norm ? qk_norm_rope_bwd_kernel<64, 1, true> : qk_norm_rope_bwd_kernel<64, 1, false>)
                                            : (norm ? qk_norm_rope_bwd_kernel<64, 4, true> : qk_norm_rope_bwd_kernel<64, 4, false>));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(g.q + g.k)), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !norm) return e;
    hipLaunchKernelGGL(qk_dgamma_kernel, dim3((unsigned)(dim / 16), 2), dim3(1024), 0, st, a.partial, (int)g.q, (int)(g.q + g.k), dim, dgamma_q,
                       dgamma_k);
    return hipGetLastError();
}

}  // namespace jet

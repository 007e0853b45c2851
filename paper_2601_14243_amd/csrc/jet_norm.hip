// Layer norm and its gradient, and that of the RMS norm.
#include "jet_internal.h"
#include "jet_numerics.h"
#include "jet_reduce.h"
#include "jet_step.h"

namespace jet {

namespace {

struct Vec8 {
    float v[8];
};
__device__ __forceinline__ Vec8 unpack(uint4 u) {
    return Vec8{{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y), bf16_lo(u.z), bf16_hi(u.z), bf16_lo(u.w), bf16_hi(u.w)}};
}
__device__ __forceinline__ uint4 pack(const Vec8& a) {
    return uint4{bf16_pack2(a.v[0], a.v[1]), bf16_pack2(a.v[2], a.v[3]), bf16_pack2(a.v[4], a.v[5]), bf16_pack2(a.v[6], a.v[7])};
}
__device__ __forceinline__ uint4 load16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void store16(uint16_t* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }

// Sums of a row over its team of W waves; `scratch` is not in use by an earlier sum of this workgroup
template <int W, int N>
__device__ __forceinline__ void team_sums(double (&s)[N], double (*scratch)[N], int team, int wave_in_team) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    if (W == 1) return;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) scratch[team * W + wave_in_team][i] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) t += scratch[team * W + w][i];
        s[i] = t;
    }
}

// Mean as two binary32 numbers, and 1 / sqrt(var + eps), from the binary64 sums of a row's values and squares.  A square of a bf16
// value has 16 significant bits: the sums are exact where the values' exponents differ by less than about 10, and
// K S2 - S1^2 loses no more than 2^-53 of S1^2.
struct Moments {
    float hi, lo, r;
};
__device__ __forceinline__ Moments moments(double s1, double s2, int K, float eps) {
    const double mean = s1 / K, var = fmax((s2 * K - s1 * s1) / ((double)K * K), 0.0);
    const float hi = (float)mean;
    return {hi, (float)(mean - (double)hi), 1.0f / sqrtf((float)(var + (double)eps))};
}

template <int W, int P, bool kQuant, bool kRes>
__global__ __launch_bounds__(W < 4 ? 256 : 64 * W) void layernorm_kernel(NormArgs a) {
    constexpr int kTeams = W < 4 ? 4 / W : 1;
    __shared__ double scratch[kTeams * W][2];
    const int w = threadIdx.x >> 6, team = w / W, wt = w % W, tl = (wt << 6) + (threadIdx.x & 63);
    const long m = (long)blockIdx.x * kTeams + team;
    const bool row = m < a.M;
    uint4 x[P], gm[P], bt[P];
    double s[2] = {0.0, 0.0};
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int k = (c * 64 * W + tl) * 8;
        x[c] = gm[c] = bt[c] = uint4{0, 0, 0, 0};
        if (!row || k >= a.K) continue;
        x[c] = load16(a.x + m * a.K + k);
        if (kRes) {
            const Vec8 u = unpack(x[c]), r = unpack(load16(a.res + m * a.K + k));
            Vec8 t;
#pragma unroll
            for (int i = 0; i < 8; ++i) t.v[i] = u.v[i] + r.v[i];
            x[c] = pack(t);
            store16(a.sum + m * a.K + k, x[c]);
        }
        gm[c] = load16(a.gamma + k);
        if (a.beta) bt[c] = load16(a.beta + k);
    }
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const Vec8 u = unpack(x[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double v = (double)u.v[i];
            s[0] += v;
            s[1] = fma(v, v, s[1]);
        }
    }
    team_sums<W, 2>(s, scratch, team, wt);
    if (!row) return;
    const Moments mo = moments(s[0], s[1], a.K, a.eps);
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int k = (c * 64 * W + tl) * 8;
        if (k >= a.K) continue;                          // whole teams of 16 lanes where the output is quantized
        const Vec8 u = unpack(x[c]), g = unpack(gm[c]), b = unpack(bt[c]);
        Vec8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y.v[i] = __builtin_fmaf(((u.v[i] - mo.hi) - mo.lo) * mo.r, g.v[i], b.v[i]);
        const uint4 h = pack(y);
        if (!kQuant) {
            store16(a.y + m * a.K + k, h);
            continue;
        }
        y = unpack(h);
        float am = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) am = fmaxf(am, fabsf(y.v[i]));
        const GroupScale gs = make_scale(team16_max(am));
        uint32_t o[2];
        encode<kBf16Values>(y.v, gs, o);
        *reinterpret_cast<uint2*>(a.q + m * a.K + k) = uint2{o[0], o[1]};
        if ((tl & 15) == 0) a.s[m * (a.K >> 7) + (k >> 7)] = gs.S;
    }
}

// dx = r (g - mean(g) - n mean(g n)) + res with g = dy gamma and n = (x - mean) r (RMS: n = x r, without mean(g)); the sums of dy n and
// dy over the rows of a workgroup go to its place in `partial`, [workgroup][dgamma, dbeta][K].
template <int W, int P, bool kLayer, bool kRes>
__global__ __launch_bounds__(W < 4 ? 256 : 64 * W) void norm_bwd_kernel(NormArgs a) {
    constexpr int kTeams = W < 4 ? 4 / W : 1, kSums = kLayer ? 4 : 2;
    __shared__ double scratch[2][kTeams * W][kSums];
    const int w = threadIdx.x >> 6, team = w / W, wt = w % W, tl = (wt << 6) + (threadIdx.x & 63);
    float dg[P][8], db[P][8];
    uint4 gm[P];
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int k = (c * 64 * W + tl) * 8;
        gm[c] = k < a.K ? load16(a.gamma + k) : uint4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = db[c][i] = 0.0f;
    }
    auto load = [&](long m, uint4 (&x)[P], uint4 (&dy)[P], uint4 (&rs)[P]) {
#pragma unroll
        for (int c = 0; c < P; ++c) {
            const int k = (c * 64 * W + tl) * 8;
            x[c] = dy[c] = rs[c] = uint4{0, 0, 0, 0};
            if (m >= a.M || k >= a.K) continue;
            x[c] = load16(a.x + m * a.K + k);
            dy[c] = load16(a.dy + m * a.K + k);
            if (kRes) rs[c] = load16(a.res + m * a.K + k);
        }
    };
    const long step = (long)gridDim.x * kTeams;
    uint4 x[P], dy[P], rs[P];
    load((long)blockIdx.x * kTeams + team, x, dy, rs);
    int turn = 0;
    for (long m0 = (long)blockIdx.x * kTeams; m0 < a.M; m0 += step, turn ^= 1) {
        const long m = m0 + team;
        uint4 xn[P], dyn[P], rsn[P];
        load(m + step, xn, dyn, rsn);
        double s[kSums] = {};
#pragma unroll
        for (int c = 0; c < P; ++c) {
            const Vec8 u = unpack(x[c]), d = unpack(dy[c]), g = unpack(gm[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double v = (double)u.v[i], t = (double)(d.v[i] * g.v[i]);
                s[0] = fma(v, v, s[0]);
                s[1] = fma(v, t, s[1]);
                if (kLayer) {
                    s[2] += v;
                    s[kSums - 1] += t;
                }
            }
        }
        team_sums<W, kSums>(s, scratch[turn], team, wt);
        float hi = 0.0f, lo = 0.0f, r, c1, c2 = 0.0f;
        if (kLayer) {
            const Moments mo = moments(s[2], s[0], a.K, a.eps);
            hi = mo.hi, lo = mo.lo, r = mo.r;
            c2 = (float)(s[kSums - 1] / a.K);
            c1 = (float)((s[1] - s[2] / a.K * s[kSums - 1]) / a.K) * r;
        } else {
            r = 1.0f / sqrtf((float)(s[0] / a.K + (double)a.eps));
            c1 = (float)(s[1] / a.K) * r;
        }
        if (m < a.M) {
#pragma unroll
            for (int c = 0; c < P; ++c) {
                const int k = (c * 64 * W + tl) * 8;
                if (k >= a.K) continue;
                const Vec8 u = unpack(x[c]), d = unpack(dy[c]), g = unpack(gm[c]), e = unpack(rs[c]);
                Vec8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float n = (kLayer ? (u.v[i] - hi) - lo : u.v[i]) * r;
                    const float t = __builtin_fmaf(-n, c1, kLayer ? __builtin_fmaf(d.v[i], g.v[i], -c2) : d.v[i] * g.v[i]);
                    o.v[i] = kRes ? __builtin_fmaf(t, r, e.v[i]) : t * r;
                    dg[c][i] = __builtin_fmaf(d.v[i], n, dg[c][i]);
                    if (kLayer) db[c][i] += d.v[i];
                }
                store16(a.dx + m * a.K + k, pack(o));
            }
        }
#pragma unroll
        for (int c = 0; c < P; ++c) x[c] = xn[c], dy[c] = dyn[c], rs[c] = rsn[c];
    }
    // the teams of a workgroup one after the other
    constexpr int kMine = kLayer ? 2 : 1;
    float* const to = a.partial + (long)blockIdx.x * kMine * a.K;
    __shared__ float both[kTeams > 1 ? P * 64 * W * 16 : 1];
    for (int t = kTeams - 1; t > 0; --t) {
        if (team == t) {
#pragma unroll
            for (int c = 0; c < P; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    both[((c * 2) * 8 + i) * 64 * W + tl] = dg[c][i];
                    both[((c * 2 + 1) * 8 + i) * 64 * W + tl] = db[c][i];
                }
        }
        __syncthreads();
        if (team == t - 1) {
#pragma unroll
            for (int c = 0; c < P; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dg[c][i] += both[((c * 2) * 8 + i) * 64 * W + tl];
                    db[c][i] += both[((c * 2 + 1) * 8 + i) * 64 * W + tl];
                }
        }
        __syncthreads();
    }
    if (team == 0) {
#pragma unroll
        for (int c = 0; c < P; ++c) {
            const int k = (c * 64 * W + tl) * 8;
            if (k >= a.K) continue;
            float4* p = reinterpret_cast<float4*>(to + k);
            p[0] = float4{dg[c][0], dg[c][1], dg[c][2], dg[c][3]};
            p[1] = float4{dg[c][4], dg[c][5], dg[c][6], dg[c][7]};
            if (!kLayer) continue;
            p = reinterpret_cast<float4*>(to + a.K + k);
            p[0] = float4{db[c][0], db[c][1], db[c][2], db[c][3]};
            p[1] = float4{db[c][4], db[c][5], db[c][6], db[c][7]};
        }
    }
}

// Sums of the workgroups -> dgamma [K], dbeta [K]: 16 lanes take 64 columns, 64 of those teams every 64th workgroup each.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float* __restrict__ partial, int groups, int cols, int K, float* __restrict__ dgamma,
                                                         float* __restrict__ dbeta) {
    __shared__ double part[64][65];
    const int part_id = threadIdx.x >> 4, l = threadIdx.x & 15, col = blockIdx.x * 64 + l * 4;
    double s[4] = {0, 0, 0, 0};
    if (col < cols) {
        for (int g = part_id; g < groups; g += 64) {
            const float4 v = *reinterpret_cast<const float4*>(partial + (long)g * cols + col);
            s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[part_id][l * 4 + i] = s[i];
    __syncthreads();
    if (threadIdx.x < 64) {
        const int c = blockIdx.x * 64 + threadIdx.x;
        if (c >= cols) return;
        double t = 0.0;
        for (int p = 0; p < 64; ++p) t += part[p][threadIdx.x];
        if (c < K) dgamma[c] = (float)t;
        else dbeta[c - K] = (float)t;
    }
}

template <int W, int P>
hipError_t launch_fwd(const NormArgs& a, hipStream_t st) {
    constexpr int kTeams = W < 4 ? 4 / W : 1;
    const auto kernel = a.q ? (a.res ? layernorm_kernel<W, P, true, true> : layernorm_kernel<W, P, true, false>)
                            : (a.res ? layernorm_kernel<W, P, false, true> : layernorm_kernel<W, P, false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.M + kTeams - 1) / kTeams)), dim3(W < 4 ? 256 : 64 * W), 0, st, a);
    return hipGetLastError();
}

template <int W, int P>
hipError_t launch_bwd(const NormArgs& a, int groups, hipStream_t st) {
    const auto kernel = a.layer ? (a.res ? norm_bwd_kernel<W, P, true, true> : norm_bwd_kernel<W, P, true, false>)
                                : (a.res ? norm_bwd_kernel<W, P, false, true> : norm_bwd_kernel<W, P, false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(W < 4 ? 256 : 64 * W), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm_fwd(const NormArgs& a, hipStream_t st) {
    const NormTeam t = norm_team(a.K, norm_few_rows(a.M));
#define JET_TEAM(W, P) \
    if (t.waves == W && t.pieces == P) return launch_fwd<W, P>(a, st)
    JET_TEAM(4, 1); JET_TEAM(8, 1); JET_TEAM(16, 1);
    JET_TEAM(1, 1); JET_TEAM(1, 2); JET_TEAM(1, 4); JET_TEAM(4, 2); JET_TEAM(4, 4); JET_TEAM(8, 4); JET_TEAM(16, 4);
#undef JET_TEAM
    return hipErrorInvalidValue;
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t st) {
    const NormTeam t = norm_bwd_team(a.K);
    const int groups = (int)norm_bwd_groups(a.M, a.K), cols = a.layer ? 2 * a.K : a.K;
    hipError_t e = hipErrorInvalidValue;
#define JET_TEAM(W, P) \
    if (t.waves == W && t.pieces == P) e = launch_bwd<W, P>(a, groups, st)
    JET_TEAM(1, 1); JET_TEAM(1, 2); JET_TEAM(4, 1); JET_TEAM(4, 2); JET_TEAM(8, 2); JET_TEAM(16, 2); JET_TEAM(16, 4);
#undef JET_TEAM
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(norm_sums_kernel, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, st, a.partial, groups, cols, a.K, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace jet

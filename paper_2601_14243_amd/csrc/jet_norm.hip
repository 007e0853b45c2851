// Layer norm and its gradient, and that of the RMS norm.  All three are bound by memory: at 16384 x 4096, each call to one of two buffers in
// turn, layer norm with a residual 89 us (537 MB, 6.0 TB/s), without 47 (5.7), in E4M3 54, the gradients with one beside the norm 104 with the
// second launch (5.2), the RMS norm's at 16384 x 5120 121 (5.5); a 128 MB copy goes at 5.3.
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
// The compiler knows no more of the values than that they are here: it unpacks them again where they are used again, instead of
// keeping twice as many registers
__device__ __forceinline__ void stay_packed(uint4& u) { asm("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w)); }
__device__ __forceinline__ void store16(uint16_t* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }

// Sums over the waves of a row's team: one, or (kWaves) all of the workgroup, whose `scratch` is not in use by an earlier sum
template <bool kWaves, int N>
__device__ __forceinline__ void wave_sums(float (&s)[N], float4* scratch) {
    static_assert(N <= 4, "");
    if (!kWaves) return;
    const int w = threadIdx.x >> 6, waves = blockDim.x >> 6, l = threadIdx.x & 15;
    if ((threadIdx.x & 63) == 0) scratch[w] = float4{s[0], N > 1 ? s[N > 1 ? 1 : 0] : 0, N > 2 ? s[N > 2 ? 2 : 0] : 0, N > 3 ? s[N > 3 ? 3 : 0] : 0};
    __syncthreads();
    const float4 v = l < waves ? scratch[l] : float4{0, 0, 0, 0};        // 16 waves at most, one a lane
    const float t[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = row_sum(t[i]);
}
template <bool kWaves, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float4* scratch) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    wave_sums<kWaves>(s, scratch);
}
__device__ __forceinline__ float sum8(const Vec8& u) {
    return ((u.v[0] + u.v[1]) + (u.v[2] + u.v[3])) + ((u.v[4] + u.v[5]) + (u.v[6] + u.v[7]));
}

// Sums are binary32.  The mean is corrected by the mean of the differences from it, in every sum that it enters: with x = m + d,
// e = mean(d): mean(x) = m + e, var = mean(d^2) - e^2, sum g (x - mean) = sum g d - e sum g.  Mean squares are added as (d / K) d, as a
// sum of squares might leave the range.

// A row has a wave (four rows a workgroup) or (kWaves) a workgroup; a wave P times 64 pieces of 8 columns, each lane one of every 64.  The sums
// of 64 pieces are added across lanes, those sums in pairs of neighbours, of pairs, and so on, in a wave and across waves: whatever P
// is, and so whatever company a row has, it gets the same bytes.
template <int P, int N>
__device__ __forceinline__ void pairs(float (&s)[N][P], float (&out)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int c = 0; c < P; ++c) s[n][c] = wave_sum(s[n][c]);
        out[n] = s[n][0];
        if (P > 1) out[n] += s[n][P > 1 ? 1 : 0];
        if (P > 2) out[n] += s[n][P > 2 ? 2 : 0] + s[n][P > 3 ? 3 : 0];
    }
}
template <bool kWaves, int P, bool kQuant, bool kRes>
__global__ __launch_bounds__(kWaves ? 1024 : 256) void layernorm_kernel(NormArgs a) {
    constexpr bool kLate = P == 4;                       // the weights, where they are used: 64 registers in place of 96, and so two workgroups a CU
    __shared__ float4 scratch[2][16];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6, k0 = ((kWaves ? w * P * 64 : 0) + l) * 8;
    const long m = kWaves ? (long)blockIdx.x : (long)blockIdx.x * 4 + w;
    if (m >= a.M) return;                                // whole waves; only with a wave for a row
    const float inv = 1.0f / a.K;
    uint4 x[P], gm[P], bt[P];
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int k = k0 + c * 512;
        x[c] = gm[c] = bt[c] = uint4{0, 0, 0, 0};
        if (k >= a.K) continue;
        x[c] = load16_nt(a.x + m * a.K + k);
        if (kRes) {
            const Vec8 u = unpack(x[c]), r = unpack(load16_nt(a.res + m * a.K + k));
            Vec8 t;
#pragma unroll
            for (int i = 0; i < 8; ++i) t.v[i] = u.v[i] + r.v[i];
            x[c] = pack(t);
            store16_nt(a.sum + m * a.K + k, x[c]);       // not needed before the next block's end
        }
        if (!kLate) {
            gm[c] = load16(a.gamma + k);
            if (a.beta) bt[c] = load16(a.beta + k);
        }
    }
    float part[1][P], mean[1];
#pragma unroll
    for (int c = 0; c < P; ++c) part[0][c] = sum8(unpack(x[c]));
    pairs(part, mean);
    wave_sums<kWaves, 1>(mean, scratch[0]);
    const float m0 = mean[0] * inv;
    float both[2][P], s[2];                              // of the squares' share and of the differences
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const Vec8 u = unpack(x[c]);
        const float at = k0 + c * 512 < a.K ? m0 : 0.0f; // zeros behind the row stay zeros
        both[0][c] = both[1][c] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = u.v[i] - at;
            both[0][c] = __builtin_fmaf(d * inv, d, both[0][c]);
            both[1][c] += d;
        }
    }
    pairs(both, s);
    wave_sums<kWaves>(s, scratch[1]);
    const float e = s[1] * inv, r = 1.0f / sqrtf(fmaxf(__builtin_fmaf(-e, e, s[0]), 0.0f) + a.eps), er = -e * r;
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int k = k0 + c * 512;
        if (k >= a.K) continue;                          // whole teams of 16 lanes where the output is quantized
        if (kLate) {
            gm[c] = load16(a.gamma + k);
            if (a.beta) bt[c] = load16(a.beta + k);
        }
        stay_packed(x[c]);
        const Vec8 u = unpack(x[c]), g = unpack(gm[c]), b = unpack(bt[c]);
        Vec8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y.v[i] = __builtin_fmaf(__builtin_fmaf(u.v[i] - m0, r, er), g.v[i], b.v[i]);
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
        if ((l & 15) == 0) a.s[m * (a.K >> 7) + (k >> 7)] = gs.S;
    }
}

// A row of K bf16 values as a buffer: what lies behind it reads as zero and is not written, with no branch around the access, so that
// the compiler can count what is under way and no load has to wait for a store in front of it.  No row: nothing of it.
typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kPastCaches = 2;                           // nt: lines that are not needed again
struct Row {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ Row(const uint16_t* p, long m, long M, int K)
        : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(m < M ? p + m * K : p), 0, m < M ? K * 2 : 0, 0x00020000)) {}
    __device__ __forceinline__ uint4 load(int k) const {
        return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, k * 2, 0, kPastCaches));
    }
    template <int kPolicy>
    __device__ __forceinline__ void store(int k, uint4 v) const {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, v), r, k * 2, 0, kPolicy);
    }
};

// dx = r (g - mean(g) - n mean(g n)) + res with g = dy gamma and n = (x - mean) r (RMS: n = x r, without mean(g)); the sums of dy n and
// dy over the rows of a workgroup go to its place in `partial`, [workgroup][dgamma, dbeta][K].
//
// A row has a wave (K <= 1024, four rows a workgroup) or a workgroup, a lane P times 8 columns; the loads of the next D - 1 rows are
// under way while one is worked on (D = 2, 3, 4: 105.8, 104.6, 106.7 us at 16384 x 4096, the RMS norm's at 16384 x 5120 125, 122,
// 124).  1001 x 2048, 8.5 us and 3.3 for the second launch, is a chain of launch, loads, two barriers a row and the write-back
// of the sums; several rows of a workgroup at once, whose sums meet in LDS, gave 0.2 us.  Beyond 16384 columns the layer norm's form has some 80
// values more than 128 registers hold, the RMS norm's with a gradient beside it 20, which go through scratch memory: 2048 x 32768 218 us, the RMS
// norm's without 88.
template <bool kWaves, int P, bool kLayer, bool kRes, bool kNt>
__global__ __launch_bounds__(kWaves ? 1024 : 256) void norm_bwd_kernel(NormArgs a) {
    constexpr bool kLate = P == 4;                       // the weights and res where they are used: 128 registers do not hold them as well
    constexpr int kTeams = kWaves ? 1 : 4, D = P == 1 ? kNormAhead : P == 2 && !kWaves ? 2 : 1;
    __shared__ float4 scratch[kWaves ? 3 : 1][16];
    const int team = kWaves ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tl = kWaves ? threadIdx.x : threadIdx.x & 63,
              lanes = kWaves ? blockDim.x : 64;
    float dg[P][8], db[P][8];
    uint4 gm[P];
    struct Values {
        uint4 x[P], dy[P], rs[P];
    };
    auto load = [&](long m, Values& v) {
        const Row x(a.x, m, a.M, a.K), dy(a.dy, m, a.M, a.K), rs(kRes ? a.res : a.x, m, a.M, a.K);
#pragma unroll
        for (int c = 0; c < P; ++c) {
            const int k = (c * lanes + tl) * 8;
            v.x[c] = x.load(k);
            v.dy[c] = dy.load(k);
            v.rs[c] = kRes && !kLate ? rs.load(k) : uint4{0, 0, 0, 0};
        }
    };
    const long step = (long)gridDim.x * kTeams;
    const float inv = 1.0f / a.K;
    long m0 = (long)blockIdx.x * kTeams;
    Values ring[D];
#pragma unroll
    for (int j = 0; j < D; ++j) load(m0 + team + j * step, ring[j]);
    const Row gamma(a.gamma, 0, 1, a.K);
#pragma unroll
    for (int c = 0; c < P; ++c) {
        if (!kLate) gm[c] = gamma.load((c * lanes + tl) * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = db[c][i] = 0.0f;
    }
    int turn = 0;
    auto row = [&](long m, Values& v) {
        float mean = 0.0f, r, c1, c2 = 0.0f, er = 0.0f;
        if (kLayer) {
            float s[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < P; ++c) s[0] += sum8(unpack(v.x[c]));
            row_sums<kWaves, 1>(s, scratch[kWaves ? 2 : 0]);
            mean = s[0] * inv;
        }
        float s[kLayer ? 4 : 2] = {};
#pragma unroll
        for (int c = 0; c < P; ++c) {
            if (P > 2) stay_packed(v.x[c]);
            if (kLate) gm[c] = load16(a.gamma + min((c * lanes + tl) * 8, a.K - 8));     // (dy is zero behind the row)
            const Vec8 u = unpack(v.x[c]), d = unpack(v.dy[c]), g = unpack(gm[c]);
            const float at = (c * lanes + tl) * 8 < a.K ? mean : 0.0f;       // zeros behind the row stay zeros
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = kLayer ? u.v[i] - at : u.v[i], t = d.v[i] * g.v[i];
                s[0] = __builtin_fmaf(x * inv, x, s[0]);
                s[1] = __builtin_fmaf(x, t, s[1]);
                if (kLayer) {
                    s[kLayer ? 2 : 0] += x;
                    s[kLayer ? 3 : 0] += t;
                }
            }
        }
        row_sums<kWaves>(s, scratch[turn]);
        turn ^= 1;
        if (kLayer) {
            const float e = s[kLayer ? 2 : 0] * inv, sg = s[kLayer ? 3 : 0];
            r = 1.0f / sqrtf(fmaxf(__builtin_fmaf(-e, e, s[0]), 0.0f) + a.eps);
            if (m >= a.M) r = 0.0f;                      // no row: no infinity, of which the sums would keep a NaN
            c2 = sg * inv;
            c1 = __builtin_fmaf(-e, sg, s[1]) * inv * r;
            er = -e * r;
        } else {
            r = 1.0f / sqrtf(s[0] + a.eps);
            if (m >= a.M) r = 0.0f;
            c1 = s[1] * inv * r;
        }
        const Row dx(a.dx, m, a.M, a.K), late(kRes && kLate ? a.res : a.x, m, a.M, a.K);
#pragma unroll
        for (int c = 0; c < P; ++c) {
            if (P > 2) stay_packed(v.x[c]), stay_packed(v.dy[c]);
            if (kLate) {
                gm[c] = load16(a.gamma + min((c * lanes + tl) * 8, a.K - 8));
                if (kRes) v.rs[c] = late.load((c * lanes + tl) * 8);
            }
            const Vec8 u = unpack(v.x[c]), d = unpack(v.dy[c]), g = unpack(gm[c]), e = unpack(v.rs[c]);
            Vec8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float n = kLayer ? __builtin_fmaf(u.v[i] - mean, r, er) : u.v[i] * r;
                const float t = __builtin_fmaf(-n, c1, kLayer ? __builtin_fmaf(d.v[i], g.v[i], -c2) : d.v[i] * g.v[i]);
                o.v[i] = kRes ? __builtin_fmaf(t, r, e.v[i]) : t * r;
                dg[c][i] = __builtin_fmaf(d.v[i], n, dg[c][i]);              // (no row: dy is zero)
                if (kLayer) db[c][i] += d.v[i];
            }
            dx.store<kNt ? kPastCaches : 0>((c * lanes + tl) * 8, pack(o));
        }
    };
    while (m0 < a.M) {                                   // the same for all waves: they meet in the sums
#pragma unroll
        for (int j = 0; j < D; ++j) {
            if (j > 0 && m0 >= a.M) break;
            row(m0 + team, ring[j]);
            load(m0 + team + D * step, ring[j]);
            m0 += step;
        }
    }
    // the teams of a workgroup one after the other
    constexpr int kMine = kLayer ? 2 : 1;
    if (!kWaves) {
        __shared__ float both[kWaves ? 1 : P * 16 * 64];
        for (int t = kTeams - 1; t > 0; --t) {
            if (team == t) {
#pragma unroll
                for (int c = 0; c < P; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        both[((c * 2) * 8 + i) * 64 + tl] = dg[c][i];
                        if (kLayer) both[((c * 2 + 1) * 8 + i) * 64 + tl] = db[c][i];
                    }
            }
            __syncthreads();
            if (team == t - 1) {
#pragma unroll
                for (int c = 0; c < P; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dg[c][i] += both[((c * 2) * 8 + i) * 64 + tl];
                        if (kLayer) db[c][i] += both[((c * 2 + 1) * 8 + i) * 64 + tl];
                    }
            }
            __syncthreads();
        }
    }
    if (team != 0) return;
    float* const to = a.partial + (long)blockIdx.x * kMine * a.K;
#pragma unroll
    for (int c = 0; c < P; ++c) {
        const int k = (c * lanes + tl) * 8;
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

// Sums of the workgroups -> dgamma [K], dbeta [K]: 16 lanes take 64 columns, 64 of those teams every 64th workgroup each.  A launch and a
// read: 3.3 us for 251 workgroups of 2048 columns, 5.4 for 512 of 4096 (17 MB).
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float* __restrict__ partial, int groups, int cols, int K, float* __restrict__ dgamma,
                                                         float* __restrict__ dbeta) {
    __shared__ double part[64][65];
    const int part_id = threadIdx.x >> 4, l = threadIdx.x & 15, col = blockIdx.x * 64 + l * 4;
    double s[4] = {0, 0, 0, 0};
    if (col < cols) {
        constexpr int kAtOnce = 8;
        for (int g0 = part_id; g0 < groups; g0 += 64 * kAtOnce) {
            float4 v[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                v[i] = g0 + 64 * i < groups ? *reinterpret_cast<const float4*>(partial + (long)(g0 + 64 * i) * cols + col) : float4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) s[0] += v[i].x, s[1] += v[i].y, s[2] += v[i].z, s[3] += v[i].w;
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

template <bool kWaves, int P>
hipError_t launch_fwd(const NormArgs& a, int threads, hipStream_t st) {
    const auto kernel = a.q ? (a.res ? layernorm_kernel<kWaves, P, true, true> : layernorm_kernel<kWaves, P, true, false>)
                            : (a.res ? layernorm_kernel<kWaves, P, false, true> : layernorm_kernel<kWaves, P, false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(kWaves ? a.M : (a.M + 3) / 4)), dim3((unsigned)threads), 0, st, a);
    return hipGetLastError();
}

template <bool kWaves, int P>
hipError_t launch_bwd(const NormArgs& a, int groups, int threads, hipStream_t st) {
    const bool nt = writes_past_the_caches(2 * a.M * a.K);
#define JET_BWD(LAYER, RES) (nt ? norm_bwd_kernel<kWaves, P, LAYER, RES, true> : norm_bwd_kernel<kWaves, P, LAYER, RES, false>)
    const auto kernel = a.layer ? (a.res ? JET_BWD(true, true) : JET_BWD(true, false)) : (a.res ? JET_BWD(false, true) : JET_BWD(false, false));
#undef JET_BWD
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3((unsigned)threads), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm_fwd(const NormArgs& a, hipStream_t st) {
    const NormTeam t = norm_team(a.M, a.K, a.res && !a.q);
    const int threads = t.waves == 1 ? 256 : 64 * t.waves;
    if (t.waves == 1) return t.pieces == 1 ? launch_fwd<false, 1>(a, threads, st) : launch_fwd<false, 2>(a, threads, st);
    if (t.pieces == 1) return launch_fwd<true, 1>(a, threads, st);
    return t.pieces == 2 ? launch_fwd<true, 2>(a, threads, st) : launch_fwd<true, 4>(a, threads, st);
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t st) {
    const NormTeam t = norm_bwd_team(a.K);
    const int groups = (int)norm_bwd_groups(a.M, a.K), cols = a.layer ? 2 * a.K : a.K, threads = t.waves == 1 ? 256 : 64 * t.waves;
    hipError_t e = hipErrorInvalidValue;
    if (t.waves == 1) e = t.pieces == 1 ? launch_bwd<false, 1>(a, groups, threads, st) : launch_bwd<false, 2>(a, groups, threads, st);
    else if (t.pieces == 1) e = launch_bwd<true, 1>(a, groups, threads, st);
    else if (t.pieces == 2) e = launch_bwd<true, 2>(a, groups, threads, st);
    else e = launch_bwd<true, 4>(a, groups, threads, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(norm_sums_kernel, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, st, a.partial, groups, cols, a.K, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace jet

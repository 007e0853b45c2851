// The norm over many tensors, and their scaling down to a given norm.
//
// The addresses and sizes of up to kClipBatch tensors are the arguments of a launch, so that nothing has to be copied to the device or kept
// for a call; longer lists take several launches.  The elements of a batch are numbered in chunks of kClipChunk, no
// chunk in two tensors; a workgroup takes every gridDim-th one.  Squares and their sums are binary64: neither a square nor a sum
// leaves the range, and the norm is right to binary32.
//
// Bound by memory: 1.95 GB in bf16, scaled to new tensors, 926 us: squares 302 (6.5 TB/s; through the caches 361), norm 4, scaling 678
// (5.75 TB/s; in 2048 persistent workgroups, forward and through the caches 732).  45 MB that are within the limit: squares 10.8, norm 2.9.
#include <cmath>

#include "jet_internal.h"
#include "jet_numerics.h"
#include "jet_reduce.h"
#include "jet_step_plan.h"

namespace jet {

namespace {

struct Batch {
    uint64_t src[kClipBatch];       // address; bit 0: binary32, else bf16
    uint64_t dst[kClipBatch];
    uint32_t end[kClipBatch];       // chunks up to this tensor's last
    uint32_t last[kClipBatch];      // elements of its last chunk
    int n;
};
static_assert(sizeof(Batch) < 4000, "arguments of a launch");

// Chunk c of the batch: tensor, first element, elements
struct Chunk {
    int tensor;
    long at;
    int count;
};
__device__ __forceinline__ Chunk chunk_of(const Batch& b, uint32_t c) {
    int lo = 0, hi = b.n - 1;       // the first tensor whose end is behind c
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (b.end[mid] > c) hi = mid;
        else lo = mid + 1;
    }
    const uint32_t first = lo ? b.end[lo - 1] : 0;
    return {lo, (long)(c - first) * kClipChunk, c + 1 == b.end[lo] ? (int)b.last[lo] : (int)kClipChunk};
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double part[4];
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ __forceinline__ uint4 load16(const void* p, bool past) { return past ? load16_nt(p) : *static_cast<const uint4*>(p); }

__device__ __forceinline__ void square(double& s, float v) { s = fma((double)v, (double)v, s); }
__device__ __forceinline__ void square8(double& s, uint4 u) {
    square(s, bf16_lo(u.x)), square(s, bf16_hi(u.x)), square(s, bf16_lo(u.y)), square(s, bf16_hi(u.y));
    square(s, bf16_lo(u.z)), square(s, bf16_hi(u.z)), square(s, bf16_lo(u.w)), square(s, bf16_hi(u.w));
}

// Chunks from `keep` on are read through the memory-side cache, those before past it
__global__ __launch_bounds__(256) void square_sum_kernel(const Batch b, uint32_t chunks, uint32_t keep, double* __restrict__ partial) {
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = chunk_of(b, c);
        const uint64_t src = b.src[k.tensor];
        if (src & 1) {
            const float* p = reinterpret_cast<const float*>(src & ~1ull) + k.at;
            const int whole = k.count & ~3;
            if (k.count == kClipChunk) {
                float4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float4, load16(reinterpret_cast<const float4*>(p) + i * 256 + threadIdx.x, c < keep));
#pragma unroll
                for (int i = 0; i < 8; ++i) square(s, v[i].x), square(s, v[i].y), square(s, v[i].z), square(s, v[i].w);
                continue;
            }
            for (int i = threadIdx.x * 4; i < whole; i += 1024) {
                const float4 v = *reinterpret_cast<const float4*>(p + i);
                square(s, v.x), square(s, v.y), square(s, v.z), square(s, v.w);
            }
            if ((int)threadIdx.x < k.count - whole) square(s, p[whole + threadIdx.x]);
        } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(src) + k.at;
            const int whole = k.count & ~7;
            if (k.count == kClipChunk) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = load16(reinterpret_cast<const uint4*>(p) + i * 256 + threadIdx.x, c < keep);
#pragma unroll
                for (int i = 0; i < 4; ++i) square8(s, v[i]);
                continue;
            }
            for (int i = threadIdx.x * 8; i < whole; i += 2048) square8(s, *reinterpret_cast<const uint4*>(p + i));
            if ((int)threadIdx.x < k.count - whole) square(s, __uint_as_float((uint32_t)p[whole + threadIdx.x] << 16));
        }
    }
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_of(const double* __restrict__ partial, int n) {
    if (n == 1) return partial[0];
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
    return block_sum(s);
}

// the norm, and the sum of squares where it is asked for
__global__ __launch_bounds__(256) void norm_kernel(const double* __restrict__ partial, int n, float* __restrict__ norm, double* __restrict__ sum) {
    const double s = sum_of(partial, n);
    if (threadIdx.x != 0) return;
    if (norm) *norm = (float)sqrt(s);
    if (sum) *sum = s;
}

__device__ __forceinline__ uint32_t scaled2(uint32_t u, float f) { return bf16_pack2(bf16_lo(u) * f, bf16_hi(u) * f); }

// given: the norm, else the n partial sums of squares, from which it is formed
__global__ __launch_bounds__(256) void clip_kernel(const Batch b, uint32_t chunks, const double* __restrict__ partial, int n, const float* __restrict__ given,
                                                   float max_norm, float* __restrict__ norm, bool in_place) {
    const double total = given ? (double)*given : sqrt(sum_of(partial, n));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    // a norm that is not finite leaves the values as they are
    const bool clips = total > (double)max_norm && (float)total <= 3.4028235e38f;
    if (!clips && in_place) return;
    const float f = clips ? (float)((double)max_norm / total) : 1.0f;
    for (uint32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const Chunk k = chunk_of(b, chunks - 1 - i);
        const uint64_t src = b.src[k.tensor], dst = b.dst[k.tensor];
        if (src & 1) {
            const float* p = reinterpret_cast<const float*>(src & ~1ull) + k.at;
            float* o = reinterpret_cast<float*>(dst) + k.at;
            const int whole = k.count & ~3;
#pragma unroll 8
            for (int i = threadIdx.x * 4; i < whole; i += 1024) {
                const float4 v = __builtin_bit_cast(float4, load16_nt(p + i));
                store16_nt(o + i, __builtin_bit_cast(uint4, float4{v.x * f, v.y * f, v.z * f, v.w * f}));
            }
            if ((int)threadIdx.x < k.count - whole) o[whole + threadIdx.x] = p[whole + threadIdx.x] * f;
        } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(src) + k.at;
            uint16_t* o = reinterpret_cast<uint16_t*>(dst) + k.at;
            const int whole = k.count & ~7;
#pragma unroll 4
            for (int i = threadIdx.x * 8; i < whole; i += 2048) {
                const uint4 v = load16_nt(p + i);
                store16_nt(o + i, uint4{scaled2(v.x, f), scaled2(v.y, f), scaled2(v.z, f), scaled2(v.w, f)});
            }
            if ((int)threadIdx.x < k.count - whole)
                o[whole + threadIdx.x] = (uint16_t)scaled2((uint32_t)p[whole + threadIdx.x], f);
        }
    }
}

// The batch that begins with tensor i; its chunks; i moves behind it
uint32_t fill_batch(Batch& b, const jet_tensor* src, const jet_tensor* dst, long n, long& i) {
    uint32_t chunks = 0;
    for (b.n = 0; b.n < kClipBatch && i < n; ++i) {
        const long count = src[i].n, c = (count + kClipChunk - 1) / kClipChunk;
        if (count == 0) continue;
        if (b.n && chunks + c > INT32_MAX) break;
        b.src[b.n] = reinterpret_cast<uint64_t>(src[i].data) | (src[i].type == JET_F32 ? 1 : 0);
        b.dst[b.n] = reinterpret_cast<uint64_t>((dst ? dst : src)[i].data);
        chunks += (uint32_t)c;
        b.end[b.n] = chunks;
        b.last[b.n] = (uint32_t)(count - (c - 1) * kClipChunk);
        ++b.n;
    }
    return chunks;
}

}  // namespace

hipError_t launch_clip(const jet_tensor* src, const jet_tensor* dst, long n, bool scales, float max_norm, const float* given, float* norm, double* partial,
                       hipStream_t st) {
    Batch b;
    int sums = 0;
    long left = 0;                                       // bytes from tensor i on
    for (long i = 0; i < n; ++i) left += src[i].n * (src[i].type == JET_F32 ? 4 : 2);
    const bool large = left > kClipFuse;
    if (!given) {
        for (long i = 0; i < n;) {
            long bytes = 0;
            const long from = i;
            const uint32_t chunks = fill_batch(b, src, nullptr, n, i);
            if (!chunks) continue;
            for (long j = from; j < i; ++j) bytes += src[j].n * (src[j].type == JET_F32 ? 4 : 2);
            // the batch's chunks in front of the last kClipKeep bytes of all tensors, as if all chunks were alike
            const uint32_t keep = left <= kClipKeep ? 0 : left - bytes >= kClipKeep ? chunks : (uint32_t)((double)chunks * (left - kClipKeep) / bytes);
            left -= bytes;
            const unsigned groups = (unsigned)clip_groups(chunks);
            hipLaunchKernelGGL(square_sum_kernel, dim3(groups), dim3(256), 0, st, b, chunks, scales ? keep : chunks, partial + sums);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            sums += (int)groups;
        }
    }
    if (!scales || (large && !given)) {
        double* const sum = scales ? partial + sums : nullptr;
        hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(256), 0, st, partial, sums, norm, sum);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || !scales) return e;
        partial = sum;
        sums = 1;
        norm = nullptr;
    }
    // backwards: what the first pass read last may still be in the memory-side cache
    bool first = true;
    for (long end = n; end > 0 || first;) {
        long i = std::max<long>(0, end - kClipBatch);
        const long from = i;
        uint32_t chunks = fill_batch(b, src, dst, end, i);
        if (i < end) {                                   // too many chunks for a launch: one tensor at a time
            i = end - 1;
            chunks = fill_batch(b, src, dst, end, i);
            end = end - 1;
        } else {
            end = from;
        }
        if (!chunks && !(first && end == 0)) continue;   // nothing at all: the norm is still written
        const long groups = large ? std::min<long>(chunks, dst ? 1 << 23 : kClipInPlace) : clip_groups(chunks);
        hipLaunchKernelGGL(clip_kernel, dim3((unsigned)std::max<long>(1, groups)), dim3(256), 0, st, b, chunks, partial, sums, given, max_norm,
                           first ? norm : nullptr, dst == nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        first = false;
    }
    return hipSuccess;
}

}  // namespace jet

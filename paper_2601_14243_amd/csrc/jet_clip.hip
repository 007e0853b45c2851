// The norm over many tensors, and their scaling down to a given norm.
//
// The addresses and sizes of up to kClipBatch tensors are the arguments of a launch, so that nothing has to be copied to the device or kept
// for a call; longer lists take several launches.  The elements of a batch are numbered in chunks of kClipChunk, no
// chunk in two tensors; a workgroup takes every gridDim-th one.  Squares and their sums are binary64: neither a square nor a sum
// leaves the range, and the norm is right to binary32.
//
// Bound by memory: 1.95 GB in bf16, scaled to new tensors, 912 us: squares 275 (7.1 TB/s; through the caches 361), norm 4, scaling 630
// (6.2 TB/s; in 2048 persistent workgroups, forward and through the caches 732).  45 MB that are within the limit: squares 9.5, norm 3.
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

// Chunk c of the batch: tensor, first element, elements.  Each lane asks about a tensor of every 64 whether it ends in front of c: one round of
// loads and one that depends on it, where a binary search is a chain of eight (the whole of 1.95 GB 927 us, 45 MB 1 us more).
struct Chunk {
    int tensor;
    long at;
    int count;
};
__device__ __forceinline__ Chunk chunk_of(const Batch& b, uint32_t c) {
    static_assert(kClipBatch <= 3 * 64, "");
    const int l = threadIdx.x & 63, n = b.n;
    int tensor = __popcll(__ballot(l < n && b.end[min(l, n - 1)] <= c));
    if (n > 64) tensor += __popcll(__ballot(l + 64 < n && b.end[min(l + 64, n - 1)] <= c));
    if (n > 128) tensor += __popcll(__ballot(l + 128 < n && b.end[min(l + 128, n - 1)] <= c));
    const uint32_t first = tensor ? b.end[tensor - 1] : 0;
    return {tensor, (long)(c - first) * kClipChunk, c + 1 == b.end[tensor] ? (int)b.last[tensor] : (int)kClipChunk};
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double part[4];
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// Global memory: an address out of a table would else be taken for one of any kind, whose accesses wait for LDS as well
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) u32x4 Piece;
typedef __attribute__((address_space(1))) float GlobalF32;
typedef __attribute__((address_space(1))) uint16_t GlobalBf16;
// The pieces of this thread of a whole chunk, past the caches or through them.  (As plain loads the two would be taken for one.)
template <int N, bool kPast>
__device__ __forceinline__ void load_all(uint4 (&v)[N], uint64_t p) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(p), 0, N * 4096, 0x00020000);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, threadIdx.x * 16, i * 4096, kPast ? 2 : 0));
}

__device__ __forceinline__ void square(double& s, float v) { s = fma((double)v, (double)v, s); }
__device__ __forceinline__ void square8(double& s, uint4 u) {
    square(s, bf16_lo(u.x)), square(s, bf16_hi(u.x)), square(s, bf16_lo(u.y)), square(s, bf16_hi(u.y));
    square(s, bf16_lo(u.z)), square(s, bf16_hi(u.z)), square(s, bf16_lo(u.w)), square(s, bf16_hi(u.w));
}

__device__ __forceinline__ void square4(double& s, uint4 u) {
    square(s, __uint_as_float(u.x)), square(s, __uint_as_float(u.y)), square(s, __uint_as_float(u.z)), square(s, __uint_as_float(u.w));
}

template <bool kF32>
__device__ __forceinline__ void square_piece(double& s, uint4 u) {
    if (kF32) square4(s, u);
    else square8(s, u);
}
// A chunk's squares.  Past the caches one piece after the other: with 2048 workgroups that is 8 MB under way, and more of them at once is slower
// (both passes over 1.95 GB, 1 / 2 / 4 at once: 913 920 928 us).  From the caches all at once.
template <bool kF32>
__device__ __forceinline__ void square_chunk(double& s, uint64_t p, int count, bool past) {
    constexpr int kEach = kF32 ? 4 : 8, N = kClipChunk / 256 / kEach;
    if (count == kClipChunk) {
        if (past) {
#pragma unroll 1
            for (int i = 0; i < N; ++i) {
                uint4 v[1];
                load_all<1, true>(v, p + i * 4096);
                square_piece<kF32>(s, v[0]);
            }
        } else {
            uint4 v[N];
            load_all<N, false>(v, p);
#pragma unroll
            for (int i = 0; i < N; ++i) square_piece<kF32>(s, v[i]);
        }
        return;
    }
    const int whole = count / kEach, rest = count % kEach, at = whole * kEach + threadIdx.x;
    for (int i = threadIdx.x; i < whole; i += 256) square_piece<kF32>(s, __builtin_bit_cast(uint4, reinterpret_cast<const Piece*>(p)[i]));
    if ((int)threadIdx.x >= rest) return;
    square(s, kF32 ? reinterpret_cast<const GlobalF32*>(p)[at] : __uint_as_float((uint32_t)reinterpret_cast<const GlobalBf16*>(p)[at] << 16));
}

// Chunks from `keep` on are read through the memory-side cache, those before past it
__global__ __launch_bounds__(256) void square_sum_kernel(const Batch b, uint32_t chunks, uint32_t keep, double* __restrict__ partial) {
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = chunk_of(b, c);
        const uint64_t src = b.src[k.tensor];
        if (src & 1) square_chunk<true>(s, (src & ~1ull) + k.at * 4, k.count, c < keep);
        else square_chunk<false>(s, src + k.at * 2, k.count, c < keep);
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

__device__ __forceinline__ uint32_t times(uint32_t u, float f) { return __float_as_uint(__uint_as_float(u) * f); }
template <bool kF32>
__device__ __forceinline__ u32x4 scaled16(uint4 v, float f) {
    return kF32 ? u32x4{times(v.x, f), times(v.y, f), times(v.z, f), times(v.w, f)} : u32x4{scaled2(v.x, f), scaled2(v.y, f), scaled2(v.z, f), scaled2(v.w, f)};
}
template <bool kF32>
__device__ __forceinline__ void scale_chunk(uint64_t from, uint64_t to, int count, float f) {
    constexpr int kEach = kF32 ? 4 : 8, N = kClipChunk / 256 / kEach;
    const Piece* p = reinterpret_cast<const Piece*>(from);
    Piece* o = reinterpret_cast<Piece*>(to);
    if (count == kClipChunk) {                           // all loads first: in place, the compiler takes none past a store
        uint4 v[N];
        load_all<N, true>(v, from);
#pragma unroll
        for (int i = 0; i < N; ++i) __builtin_nontemporal_store(scaled16<kF32>(v[i], f), o + i * 256 + threadIdx.x);
        return;
    }
    const int whole = count / kEach, rest = count % kEach, at = whole * kEach + threadIdx.x;
    for (int i = threadIdx.x; i < whole; i += 256) {
        const uint4 v = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p + i));
        __builtin_nontemporal_store(scaled16<kF32>(v, f), o + i);
    }
    if ((int)threadIdx.x >= rest) return;
    if (kF32) reinterpret_cast<GlobalF32*>(to)[at] = reinterpret_cast<const GlobalF32*>(from)[at] * f;
    else reinterpret_cast<GlobalBf16*>(to)[at] = (uint16_t)scaled2((uint32_t)reinterpret_cast<const GlobalBf16*>(from)[at], f);
}

// The same for a factor below the normal numbers of binary32, which would have few bits or none there (max_norm 1e-6 for a norm of 3e38: 16 % off):
// products in binary64
template <bool kF32>
__device__ __forceinline__ void scale_chunk_tiny(uint64_t from, uint64_t to, int count, double f) {
#pragma unroll 1
    for (int i = threadIdx.x; i < count; i += 256) {
        if (kF32) reinterpret_cast<GlobalF32*>(to)[i] = (float)(reinterpret_cast<const GlobalF32*>(from)[i] * f);
        else reinterpret_cast<GlobalBf16*>(to)[i] = (uint16_t)bf16_pack2((float)(bf16_lo(reinterpret_cast<const GlobalBf16*>(from)[i]) * f), 0.0f);
    }
}

// given: the norm, else the n partial sums of squares, from which it is formed
__global__ __launch_bounds__(256) void clip_kernel(const Batch b, uint32_t chunks, const double* __restrict__ partial, int n, const float* __restrict__ given,
                                                   float max_norm, float* __restrict__ norm, bool in_place) {
    const double total = given ? (double)*given : sqrt(sum_of(partial, n));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    // a norm that is not finite leaves the values as they are
    const bool clips = total > (double)max_norm && (float)total <= 3.4028235e38f;
    if (!clips && in_place) return;
    const double ratio = clips ? (double)max_norm / total : 1.0;
    const float f = (float)ratio;
    const bool tiny = ratio < 0x1p-126 && ratio > 0.0;   // uniform
    for (uint32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const Chunk k = chunk_of(b, chunks - 1 - i);
        const uint64_t src = b.src[k.tensor], dst = b.dst[k.tensor];
        if (tiny) {
            if (src & 1) scale_chunk_tiny<true>((src & ~1ull) + k.at * 4, dst + k.at * 4, k.count, ratio);
            else scale_chunk_tiny<false>(src + k.at * 2, dst + k.at * 2, k.count, ratio);
            continue;
        }
        if (src & 1) scale_chunk<true>((src & ~1ull) + k.at * 4, dst + k.at * 4, k.count, f);
        else scale_chunk<false>(src + k.at * 2, dst + k.at * 2, k.count, f);
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
    const long bytes = left;
    const bool large = bytes > kClipFuse;
    if (!given) {
        for (long i = 0; i < n;) {
            long mine = 0;
            const long from = i;
            const uint32_t chunks = fill_batch(b, src, nullptr, n, i);
            if (!chunks) continue;
            for (long j = from; j < i; ++j) mine += src[j].n * (src[j].type == JET_F32 ? 4 : 2);
            // the batch's chunks in front of the last kClipKeep bytes of all tensors, as if all chunks were alike
            const uint32_t keep = left <= kClipKeep ? 0 : left - mine >= kClipKeep ? chunks : (uint32_t)((double)chunks * (left - kClipKeep) / mine);
            left -= mine;
            const unsigned groups = (unsigned)clip_groups(chunks);
            hipLaunchKernelGGL(square_sum_kernel, dim3(groups), dim3(256), 0, st, b, chunks, scales ? keep : chunks, partial + sums);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            sums += (int)groups;
        }
    }
    if (!scales || (!given && clip_norm_alone(bytes, sums))) {
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

// What the attention kernels share: matrix instructions, tiles in LDS, and which rows of which sequence a workgroup has.
//
// Tiles.  A tile holds rows of DIM bf16 values (keys, values, queries or output gradients), copied from global memory
// straight into LDS, 16 bytes a lane.  LDS gives 256 bytes a cycle where 16 lanes of 16 bytes (32 of 8) meet all 64 banks, so
// the 16-byte chunk c of row r lies at chunk c ^ swizzle(r) of its row, which serves both readers: 16 consecutive rows at one
// chunk (row_frag), and 4 consecutive rows at 4 chunks that differ in their lowest two bits (col_frag), cover 256 bytes once.
// Measured per CU: 568 and 518 B/ns, the same as for consecutive addresses; with an order that is only free of conflicts over 128
// bytes 299 and 293 (forward pass of 16384 tokens: 930 million busy cycles of all CUs in place of 882).
//
// Fragments of v_mfma_f32_32x32x16_bf16, lane l, h = l >> 5: A[m = l & 31][k = 8 h + j], B[k = 8 h + j][n = l & 31],
// D[m = 8 (i >> 2) + 4 h + (i & 3)][n = l & 31].  A product's D holds, for 16 values of m, exactly 8 of a lane's: m = 4 h + j
// and 8 + 4 h + j, j < 4.  The next product, which sums over m, takes them as they are as its B operand, and its A operand is
// read with the same order of k (col_frag): no value crosses lanes in between.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "jet_attn_plan.h"
#include "jet_numerics.h"

namespace jet {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

#define JET_LDS(T, p) ((__attribute__((address_space(3))) T*)(p))

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)JET_LDS(const void, p); }

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }   // 2^x, 1 ulp; 0 below -149
__device__ __forceinline__ float log2_hw(float x) { return __builtin_amdgcn_logf(x); }

// the other half's value: lane l gets that of lane l ^ 32
__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A buffer descriptor of `bytes` bytes from p on: what a load or a copy asks beyond them reads as zero.
__device__ __forceinline__ i32x4 buffer_of(const void* p, uint32_t bytes) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    i32x4 r = {(int)__builtin_amdgcn_readfirstlane((uint32_t)v), (int)(__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) & 0xffff),
               (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000};
    return r;
}
// Lane l's 16 (4) bytes at offset voff of the buffer go to LDS address lds + 16 l (4 l); asynchronous, awaited with
// wait_copies and a barrier.
__device__ __forceinline__ void copy16(uint32_t lds, i32x4 buffer, uint32_t voff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(voff), "s"(buffer) : "memory");
}
// the same for lines that are not needed again
__device__ __forceinline__ void copy16_nt(uint32_t lds, i32x4 buffer, uint32_t voff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" : : "s"(lds), "v"(voff), "s"(buffer) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t lds, i32x4 buffer, uint32_t voff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds), "v"(voff), "s"(buffer) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
    static_assert(N < 64, "six bits");
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
// every wave's LDS reads and writes in front of it are done behind it
__device__ __forceinline__ void block_sync() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

template <int DIM>
struct Tile {
    static constexpr int kRowBytes = 2 * DIM;
    static constexpr int kChunks = kRowBytes / 16;          // of a row
    static constexpr int kRowsPerCopy = 64 / kChunks;       // a wave's copy of 1 KB
    static constexpr int kK = DIM / 16;                     // k steps of a product over the channels
    static constexpr int kC = DIM / 32;                     // blocks of 32 channels

    // two bits of the row choose among the four 64-byte parts of 256 bytes (with 128-byte rows one of them does so by itself)
    static __device__ __forceinline__ uint32_t swizzle(uint32_t r) {
        return DIM == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
    }

    // where lane l reads the rows of A or B fragments whose k is the channel; block of 32 rows b, k step s: row_frag
    static __device__ __forceinline__ uint32_t row_base(int l) {
        return (l & 31) * kRowBytes + (((l >> 5) ^ swizzle(l & 15)) << 4);
    }
    static __device__ __forceinline__ bf16x8 row_frag(const char* tile, uint32_t base, int b, int s) {
        return *reinterpret_cast<const bf16x8*>(tile + (base ^ (s << 5)) + b * 32 * kRowBytes);
    }
    // where lane l reads the A fragments whose m is the channel and whose k runs over rows, in the order that the top of this
    // file names; rows 16 s .. 16 s + 15, channels 32 c .. 32 c + 31: col_frag.  ds_read_b64_tr_b16 gives lane t of 16 the
    // value t of four rows, whose 32 bytes lanes 4 r .. 4 r + 3 address.
    static __device__ __forceinline__ uint32_t col_base(int l) {
        const int h = l >> 5, r = (l & 15) >> 2, chunk = 2 * ((l >> 4) & 1) + ((l >> 1) & 1);
        return (4 * h + r) * kRowBytes + ((chunk ^ swizzle(4 * h + r)) << 4) + (l & 1) * 8;
    }
    static __device__ __forceinline__ bf16x8 col_frag(const char* tile, uint32_t base, int s, int c) {
        const char* p = tile + s * 16 * kRowBytes;
        union {
            s16x4 q[2];
            bf16x8 f;
        } u;
        u.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(JET_LDS(s16x4, p + (base ^ (c << 6))));
        // row + 8: another (row >> 2) & 3
        u.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(JET_LDS(s16x4, p + (base ^ (c << 6 | 32)) + 8 * kRowBytes));
        return u.f;
    }
};

// Fragments that were loaded from global memory are here.  Without it the compiler waits for them where they are first used, in the
// loop: at every turn, and for the copies under way as well.
template <int N>
__device__ __forceinline__ void arrived(bf16x8 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Values 8 s .. 8 s + 7 of a product's D, rounded to bf16 (nearest even), as the B operand of the next one.
__device__ __forceinline__ bf16x8 to_operand(const f32x16& d, int s) {
    const u32x4 w = {bf16_pack2(d[8 * s], d[8 * s + 1]), bf16_pack2(d[8 * s + 2], d[8 * s + 3]),
                     bf16_pack2(d[8 * s + 4], d[8 * s + 5]), bf16_pack2(d[8 * s + 6], d[8 * s + 7])};
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// One lane's D of a transposed product (channels 32 c + m of row n = l & 31) as bf16 to row `out`; half h of a row's lanes has
// 4 of every 8 channels, an exchange gives each 8 consecutive ones (16 bytes).
template <int DIM>
__device__ __forceinline__ void store_row(uint16_t* out, const f32x16 (&d)[DIM / 32], float f, int h, bool valid) {
#pragma unroll
    for (int c = 0; c < DIM / 32; ++c)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t a0 = bf16_pack2(d[c][8 * s] * f, d[c][8 * s + 1] * f), a1 = bf16_pack2(d[c][8 * s + 2] * f, d[c][8 * s + 3] * f);
            const uint32_t b0 = bf16_pack2(d[c][8 * s + 4] * f, d[c][8 * s + 5] * f), b1 = bf16_pack2(d[c][8 * s + 6] * f, d[c][8 * s + 7] * f);
            const auto x = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);   // channels 8 h' .. + 1 and + 4 .. 5
            const auto y = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            if (valid) *reinterpret_cast<uint4*>(out + 32 * c + 16 * s + 8 * h) = uint4{x[0], y[0], x[1], y[1]};
        }
}

// -------------------------------------------------------------- sequences --
//
// Rows of packed sequences are dealt to workgroups in tiles of R without a table of lengths on the host: with boundaries
// b_0 <= b_1 <= ..., sequence s has the tiles from floor(b_s / R) + s on, which leaves each enough of them, since
// floor(a / R) + ceil(n / R) <= floor((a + n) / R) + 1; a workgroup without rows ends at once.  In front of the first sequence
// and behind the last one stand two more, for rows that belong to none: they have no keys.  Boundaries are read as the caller's
// device has them and cut to [0, rows], so that no boundaries, however wrong, lead out of the arrays.
struct Sequences {
    const int32_t* cu;    // [n + 1]
    int n;
    int rows;             // rows of the array
    __device__ __forceinline__ int bound(int i) const {      // of the n + 2 sequences, i = 0 .. n + 2
        if (i == 0) return 0;
        if (i == n + 2) return rows;
        const int v = cu[i - 1];
        return v < 0 ? 0 : v > rows ? rows : v;
    }
};
// Where a workgroup's tile lies: its sequence's rows [begin, begin + count) in the array that is dealt out, and in the other one (none for
// the two sequences at the ends), and the first of the sequence's tiles
struct Place {
    int first_tile, begin, count, other_begin, other_count;
};
// of tile `tile` of R units, a row of `by` being `per` units; uniform over the wave.  Up to 61 sequences lie in the lanes of one
// read of each array; with more the wave counts its way through and reads its bounds again.
__device__ __forceinline__ Place place_of(const Sequences& by, const Sequences& other, int tile, int R, int per, int lane) {
    const int n = by.n;
    auto tiles_before = [&](int bound, int i) { return (int)((uint32_t)(bound * per) / (uint32_t)R) + i; };
    Place p;
    int s, end, other_end;
    if (n + 3 <= 64) {
        const int i = min(lane, n + 2), b = by.bound(i), o = other.bound(i);
        s = __popcll(__ballot(lane < n + 2 && tiles_before(b, i) <= tile));
        s = s > 0 ? s - 1 : 0;
        p.begin = __builtin_amdgcn_readlane(b, s);
        end = __builtin_amdgcn_readlane(b, s + 1);
        p.other_begin = __builtin_amdgcn_readlane(o, s);
        other_end = __builtin_amdgcn_readlane(o, s + 1);
    } else {
        s = 0;
        for (int i0 = 0; i0 < n + 2; i0 += 64) {
            const int i = i0 + lane;
            s += __popcll(__ballot(i < n + 2 && tiles_before(by.bound(i), i) <= tile));
        }
        s = __builtin_amdgcn_readfirstlane(s > 0 ? s - 1 : 0);
        p.begin = __builtin_amdgcn_readfirstlane(by.bound(s));
        end = __builtin_amdgcn_readfirstlane(by.bound(s + 1));
        p.other_begin = __builtin_amdgcn_readfirstlane(other.bound(s));
        other_end = __builtin_amdgcn_readfirstlane(other.bound(s + 1));
    }
    const bool outside = s == 0 || s == n + 1;
    p.first_tile = __builtin_amdgcn_readfirstlane(tiles_before(p.begin, s));
    p.count = max(0, end - p.begin);
    p.other_count = outside ? 0 : max(0, other_end - p.other_begin);
    return p;
}
// Arguments of the kernels over packed sequences.  Row strides ld* are in elements; o, dout are dense [rows, n_q, dim], lse is
// [n_q, rows], row_lse and row_delta [n_kv, rows * group].
struct AttentionArgs {
    const uint16_t *q, *k, *v;
    long ldq, ldk, ldv;
    Sequences sq, sk;
    int n_q, n_kv, group;         // group = n_q / n_kv
    uint32_t group_magic;         // x / group = (x * magic) >> 20 for x < group + 128
    float scale;
    uint16_t* o;
    float* lse;
    const uint16_t* dout;
    float *row_lse, *row_delta;
    float* partial;               // [parts, Tk, n_kv, 2, dim]
    int parts, part_rows;
    uint16_t *dq, *dk, *dv;
    long ld_dq, ld_dk, ld_dv;
};

// Arguments of attention over a paged cache: k, v [n_pages, n_kv, page, dim] of bf16 or E4M3 codes, scales [n_pages, n_kv, page].
struct DecodeArgs {
    const uint16_t* q;
    long ldq;
    const char *k, *v;
    const float *k_scale, *v_scale;
    long n_pages;
    int page;
    const int32_t* pages;         // [B, max_pages]
    int max_pages;
    const int32_t* lengths;       // [B]
    int B, n_q, n_kv, group;
    float scale;
    uint16_t* o;                  // [B, n_q, dim]
    int q_blocks, chunk, parts;   // 16 query heads a block; keys of a workgroup; most chunks of a sequence
    float *part_o, *part_ml;      // [B, n_q, parts, dim], [B, n_q, parts, 2]
};

// Arguments of the norm and rotation of heads: qkv [T, ld], q and dq [T, n_q, dim], k and dk [T, n_kv, dim], dx [T, ld_dx]
struct QkArgs {
    const uint16_t* qkv;
    long ld, T;
    int n_q, n_kv;
    const float* table;           // [table_rows, dim]: cosines of a position, then its sines
    int table_rows;
    const int32_t* positions;     // [T]
    const uint16_t *gamma_q, *gamma_k;   // both or neither
    float eps;
    uint16_t *q, *k;
    const int64_t* slots;         // [T], or none
    void *cache_k, *cache_v;      // [n_pages, n_kv, page, dim]
    float *k_scale, *v_scale;
    long n_pages;
    int page;
    const uint16_t *dq, *dk;
    uint16_t* dx;
    long ld_dx;
    int groups_q;                 // workgroups of the gradient that have query heads
    float* partial;               // [workgroups, dim]
};

// A lane's row (l & 31 of the wave's 32) in the kernels over query rows, and what it sees.  Rows past a sequence's end repeat its last
// one and are not valid.
struct QueryRow {
    int q0, k0;                   // first rows of the sequence
    int row0, rows;               // the tile's first row, the sequence's rows (token * group + head of the group)
    int row, token, head;         // in the sequence, in the sequence, of all heads
    bool valid;
    int lim;                      // the last key that the row sees, -1: none
    int lim_first, lim_last;      // of the wave's first and last row
    int kv_end;                   // keys that any row of the tile sees
};
// false: the tile of R rows has none.  The wave's rows begin at `wave_row` of the tile.
template <bool CAUSAL>
__device__ __forceinline__ bool query_row(const AttentionArgs& a, int tile, int R, int wave_row, int kvh, int l, QueryRow& r) {
    const Place place = place_of(a.sq, a.sk, tile, R, a.group, l);
    const int n = place.count, m = place.other_count, rows = n * a.group, row0 = (tile - place.first_tile) * R;
    if (row0 < 0 || row0 >= rows) return false;
    const int off = m - n;                                            // the last row of a sequence sees its last key
    const int tok0 = row0 / a.group, rem0 = row0 - tok0 * a.group;
    const int asked = wave_row + (l & 31), in_tile = min(asked, rows - 1 - row0);
    const int x = rem0 + in_tile, dt = (int)(x * a.group_magic >> 20);
    r.q0 = place.begin;
    r.k0 = place.other_begin;
    r.row0 = row0;
    r.rows = rows;
    r.row = row0 + in_tile;
    r.token = tok0 + dt;
    r.head = kvh * a.group + x - dt * a.group;
    r.valid = in_tile == asked;
    r.lim = CAUSAL ? min(m - 1, r.token + off) : m - 1;
    r.lim_first = __builtin_amdgcn_readlane(r.lim, 0);
    r.lim_last = __builtin_amdgcn_readlane(r.lim, 31);
    const int last_token = min(row0 + R - 1, rows - 1) / a.group;
    r.kv_end = __builtin_amdgcn_readfirstlane(CAUSAL ? max(0, min(m, last_token + off + 1)) : m);
    return true;
}

// Sums that the four waves of such a workgroup have of the same rows (D of transposed products, channels by rows) are left in LDS, a
// row of DIM + 4 values each, so that the rows of a column of lanes do not meet in a bank.
template <int DIM>
__device__ __forceinline__ void leave_sums(float* sums, const f32x16 (&d)[DIM / 32], int w, int l) {
    float* p = sums + (w * 32 + (l & 31)) * (DIM + 4) + 4 * (l >> 5);
#pragma unroll
    for (int c = 0; c < DIM / 32; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<float4*>(p + 32 * c + 8 * g) = float4{d[c][4 * g], d[c][4 * g + 1], d[c][4 * g + 2], d[c][4 * g + 3]};
}

}  // namespace jet

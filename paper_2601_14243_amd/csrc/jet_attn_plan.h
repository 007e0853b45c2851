// Which kernel, tile and split the attention operators take: rules on the sizes of a call, host code without HIP, so that the tests can ask
// them too.
#pragma once
#include <algorithm>

namespace jet {

inline long tiles_of(long units, int R, long n_seqs) { return units / R + n_seqs + 2; }

// Few tiles of 128 rows would leave CUs without work and each wave with all the keys that its rows see, one block after the other.  Then a
// workgroup has 32 rows, and its four waves every fourth block of 32 keys each, joined at the end: a path of little more than a
// third, but four times as many workgroups, of which one a CU runs at a time (128 KB of buffers; two with 64 channels, and two of
// those of 128 rows).  The rule sets rounds of the one against rounds of the other, a workgroup's start and end being worth as much
// as 230 (350) keys.  us for one sequence of n rows, forward, tiles of 128 / of 32: 32 query and 8 key heads of 128, n = 256: 9.9 / 7.7, 512:
// 14.2 / 14.5, 1000: 23.5 / 33.3; 12 and 2, n = 1000: 22.0 / 15.7, 4000: 75 / 108; 8 and 8 of 64, n = 1000: 16.3 / 9.3, 4000: 49.9 / 39.7,
// 8000: 100 / 121; 8 sequences of 40 rows, 32 and 8 heads of 128: 6.6 / 10.4.
inline bool few_row_tiles(long n_seqs, long Tq, long Tk, long group, long n_kv, int dim) {
    const double rows = (double)Tq * group, keys = (double)Tk / n_seqs, start = dim == 128 ? 230 : 350;
    const double small = (rows / 32 + n_seqs) * n_kv / (dim == 128 ? 256 : 512), large = (rows / 128 + n_seqs) * n_kv / 512;
    return keys > 32 && (small > 1 ? small : 1) * (start + 0.36 * keys) < (large > 1 ? large : 1) * (start + keys);
}

// How the rows of a tile of keys are dealt to workgroups, of which 512 run at a time (256 of those of 32 keys where a head has 128
// channels).
// Few tiles, with rows for each wave and not much more than a few rounds of work: 32 keys a workgroup, in as many pieces of 512 rows
// (four steps of each wave) as run at a time.  All gradients, tiles of 128 / of 32 keys, us: one sequence of 64 rows, 32 query and 8 key
// heads of 128 21.2 / 17.4; 8 of 20 rows 14.1 / 15.2; 12 and 2 heads, one of 1000 rows (96 k rows over all tiles) 73 / 57, of 4000
// (1.5 M) 254 / 279; 6 heads and 1 of 64, 4000 rows (768 k) 154 / 104.
// One sequence: its first tiles have twice the average work, so from 1024 workgroups on they even out by themselves, and each
// tile is split alike to get there.  Several sequences come in any order, a long one perhaps at the end: no workgroup has more
// than two thirds of what each of the 512 places would get if the sequences were equally long, or 1024 rows where that is more.
struct Split {
    bool few;
    int parts, rows;              // workgroups of a tile at most; rows of one at least, where there are several
};
inline Split dkdv_split(long n_seqs, long Tq, long Tk, long group, long n_kv, int dim, bool causal) {
    const long groups = (Tk + 127) / 128 * n_kv, rows_each = Tq * group / n_seqs, place = groups * rows_each / (causal ? 2 : 1) / 512;
    const bool few = rows_each >= 192 && groups + (n_seqs - 1) * n_kv <= (dim == 128 ? 128 : 256) && groups * rows_each <= (dim == 128 ? 1 << 18 : 1 << 20);
    const long rows = few || n_seqs == 1 ? 512 : std::min<long>(1 << 30, std::max<long>(1024, place * 2 / 3 / 32 * 32));
    const long most = few ? (dim == 128 ? 512 : 1024) / ((Tk + 31) / 32 * n_kv) : n_seqs == 1 ? 1024 / groups : 8;
    return {few, (int)std::max<long>(1, std::min({8L, most, (Tq * group + rows - 1) / rows})), (int)rows};
}

// Waves of a workgroup.  Rows of 256 bytes: two waves have 64 KB of buffers, so that a CU has two workgroups and streams for one while
// the other starts or ends; four waves and one workgroup took 159.6 us in place of 144.7 for 64 sequences of 500 to 8192 tokens, 8 heads.
// Smaller rows have two workgroups of four waves.
constexpr int decode_waves(int dim, bool fp8) { return dim == 128 && !fp8 ? 2 : 4; }

// Keys a workgroup takes, a multiple of 64 and at most 4096 (32 blocks of a wave, whose pages its 64 lanes hold).  Up to four blocks for
// each wave make one chunk, and up to eight where there are workgroups for all CUs, since a second launch costs more.  Else as few as
// let all workgroups run at a time, for the shortest path; from 256 on that many rounds of workgroups cost more than they give, and
// the count grows with the work, up to 2048.  The rule goes by the width of the page table, as the lengths are on the device: one sequence of
// 700 tokens, 8 heads of 128, takes 8.2 us with a table of 704 positions and 10.4 with one of 32768 (E4M3 8.6 and 9.3), 64
// sequences of 500 to 8192 tokens 206 and 199.
inline int decode_chunk(long pairs, long capacity, int waves) {
    if (capacity <= (pairs < 256 ? 128 : 256) * waves) return 256 * waves;
    const long once = (pairs * capacity / 512 + 63) / 64 * 64;
    if (once <= 256) return (int)std::max<long>(once, 64);
    return (int)std::min<long>(2048, std::max<long>(256, (pairs * capacity / 4096 + 127) / 128 * 128));
}

inline long attention_decode_groups(long B, long n_q, long n_kv, long dim, bool fp8, long capacity) {
    const long pairs = B * n_kv * ((n_q / n_kv + 15) / 16), chunk = decode_chunk(pairs, capacity, decode_waves((int)dim, fp8));
    return pairs * ((capacity + chunk - 1) / chunk);
}

// Norm and rotation of heads: four heads a team where that still makes a workgroup for every CU, else one, for the shortest path
inline long qk_workgroups(long T, long n_q, long n_kv, int dim, bool cached, int heads) {
    const long nb = (n_q + heads - 1) / heads + (n_kv + heads - 1) / heads * (cached ? 2 : 1);
    return (T * nb * (dim / 16) + 255) / 256;
}
inline bool qk_few_heads(long T, long n_q, long n_kv, int dim, bool cached) { return qk_workgroups(T, n_q, n_kv, dim, cached, 4) < 512; }

// Workgroups of the gradient: four heads a team where that fills 256 CUs with 16 waves each, those dealt to query and key heads
// as the heads are; else one head a team and a workgroup for every unit there is.
struct QkBwdGroups {
    bool few;
    long q, k;
};
inline QkBwdGroups qk_bwd_groups(long T, long n_q, long n_kv, long dim) {
    const long teams = 4096 / dim, heads = n_q + n_kv;
    const bool few = T * heads < 1024 * teams;
    auto need = [&](long n) { return (T * (few ? n : (n + 3) / 4) + teams - 1) / teams; };
    return {few, std::min(need(n_q), std::max<long>(1, 1024 * n_q / heads)), std::min(need(n_kv), std::max<long>(1, 1024 * n_kv / heads))};
}

}  // namespace jet

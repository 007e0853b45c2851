// Which kernels the embedding, layer norm and clipping operators run on: rules on the sizes of a call, host code without HIP, so that the
// tests can ask them too.
#pragma once
#include <algorithm>

namespace jet {

// Whether an output of so many bytes is written past the 256 MB memory-side cache, as lines that are not needed again.  Alone, each call to
// one of two buffers in turn, and with jet_quant_act behind it, us, through / past: gradients of layer norm 16384x4096 108 / 106 and 140.6 /
// 141.2, of the RMS norm 16384x5120 135 / 126 and 169.5 / 171.5; 4096x4096 36.2 / 39.1 and 45.1 / 46.2.  Embedding of 16384 tokens x 5120 65
// / 62.
constexpr bool writes_past_the_caches(long bytes) { return bytes >= 1L << 27; }

// ---- gradient of the embedding ----
constexpr long kSortBlock = 1024;        // tokens that a workgroup sorts
constexpr long kNarrowRows = (1L << 22) - 2;   // rows of a table whose keys have 32 bits: row and place in the block
constexpr long kEmbedDirect = 256;       // up to so many tokens a wave finds those of its own id by itself
constexpr long kPlaceTokens = 1024;      // up to so many their order is found by counting
// Up to kRankTokens tokens the place of each is searched in all sorted blocks at once, the work of which grows with the square; more, in kRankBlocks at a
// time, whose runs are then merged, kMergeRuns of them in a launch.  The whole gradient, 512 columns, at once / merged, us: 40000 tokens 47.8 / 51.9,
// 65536 58.9 / 60.1, 100000 93.8 / 80.8, 262144 290 / 146; of 256 columns, 2^22 tokens, 49100 / 1800.
constexpr long kRankTokens = 1L << 16;
constexpr long kRankBlocks = 32;
constexpr long kMergeRuns = 16;
constexpr int kLongRun = 16;             // blocks behind its first one in which a row's tokens go on, from where they are many

// Whether a workgroup adds up all tokens of a row, and not a wave so many of them, whatever their rows.  us, tokens on few rows and many, zeros
// with them / added to what is there, by waves and a join | so: 257x1024 18.2/12.7 | 14.2/7.7, 1001x1024 26.1/16.6 | 23.5/12.0, 512x4096 89.4/14.0 | 89.1/11.3,
// 1024x4096 20.0/18.9 | 21.0/17.1 and of 1024 rows 21.6/18.0 | 27.5/21.9, 600x16384 21.7/18.1 | 33.2/25.8; 1024x1024 all on one row 16.1 | 28.7.
constexpr bool embed_by_runs(long T, long H) { return T > kEmbedDirect && T <= kPlaceTokens && T * ((H + 511) / 512) <= 4096; }

// Tokens, in the order of their ids, that a wave adds up: 32, or fewer where there are not eight waves for each CU.  Added to f32, us, by
// tokens of a wave (8, 16, 32): 1024 x 1024 17.2 19.1 24.0, 4096 x 4096 38.9 35.9 37.7, 16384 x 1024 38.5 37.8 39.8, all on one id 42.7 33.1
// 30.1; 32768 x 4096 141 131 130.
inline int embed_block(long T, long H) {
    const long waves = T * ((H + 511) / 512);
    int L = 32;
    while (L > 8 && waves / L < 2048) L /= 2;
    return L;
}
// Launches behind the search that make one run of several
inline int embed_merges(long T) {
    int n = 0;
    for (long run = kSortBlock * kRankBlocks; T > kRankTokens && run < T; run *= kMergeRuns) ++n;
    return n;
}
// Bytes of zeros that are not written beside the sort, which 64 MB hide, but beside the search, which another 64 MB hide.  us, all at first / so:
// 32768 tokens, 168 MB 55.0 / 50.0; 65536, 168 MB 76.9 / 71.8; 16384, 2.1 GB 393.5 / 390.5; 1 GB 218.6 / 217.
constexpr long embed_zeros_later(long bytes) { return bytes <= 64L << 20 ? 0 : std::min(bytes - (64L << 20), 64L << 20); }
struct EmbedSpace {
    long tmp, partial, bytes;            // rows and tokens in order from 0 on; offsets of the blockwise sorted ones and of the partial sums
};
inline EmbedSpace embed_space(long T, long H) {
    EmbedSpace s = {0, 0, 0};
    if (T <= kEmbedDirect) return s;
    const long L = embed_block(T, H), blocks = (T + L - 1) / L, array = (T + kSortBlock - 1) / kSortBlock * kSortBlock * 4;
    s.tmp = 2 * array;
    s.partial = s.tmp + (T > kPlaceTokens ? 2 * array : 0);
    s.bytes = s.partial + (embed_by_runs(T, H) ? 0 : blocks * 2 * H * 4);
    return s;
}

// ---- layer norm ----
// Waves of a row's team and 8-column pieces of a lane: a wave, which needs no barrier, or as many waves as give each lane 8 (16, 32) columns.
struct NormTeam {
    int waves, pieces;
};
inline NormTeam norm_bwd_team(long K) {
    if (K <= 1024) return {1, K <= 512 ? 1 : 2};
    const int pieces = K <= 8192 ? 1 : K <= 16384 ? 2 : 4;
    return {(int)((K + 512 * pieces - 1) / (512 * pieces)), pieces};
}
// Forward: few rows, 8 columns a lane; many, 16, unless sum and y are both written, which takes longer than anything else.  us, 8 / 16 columns, each
// call to one of two buffers in turn: 1024 rows of 4096 5.9 / 5.7, 16384x2048 26.0 / 23.6, 16384x4096 53.0 / 46.7, in E4M3 62 / 54, with a
// residual 78.5 / 74.9, in bf16 with a residual 89 / 93; 16384x8192 109 / 95.  Rows of 1024, two waves / one, us captured: 1 row 2.1 / 2.5, 256
// 2.6 / 3.2, 1024 3.6 / 3.6, 16384 28.1 / 25.1.
inline NormTeam norm_team(long M, long K, bool both) {
    if (K <= 512) return {1, 1};
    if (K <= 1024) return M <= 1024 ? NormTeam{2, 1} : NormTeam{1, 2};
    if (K <= 8192 && M > 1024 && !both) return {(int)((K + 1023) / 1024), 2};
    return norm_bwd_team(K);
}
constexpr int kNormAhead = 3;             // rows whose loads are under way
// Workgroups of the backward pass, each with sums of its own: 128, and from there on one for every four rows of each team, since every
// workgroup writes 8 K bytes and the second launch reads them; at most two for a CU, or one where it does not hold the waves of two: it holds 20 with 8
// columns a lane (up to 89 registers), 16 with more (up to 128).  us with two / one where a row has 9 or 10 waves of 16 columns a lane, without a gradient
// beside the norm: 1100x8200 44 / 35, 4096x8200 78 / 70, 8192x10240 136 / 128, RMS 33 / 26, 57 / 53, 107 / 103; of 32: 1100x16392 119 / 95, 4096x20480
// 273 / 258, RMS 58 / 45, 126 / 117.  Both launches, us, by workgroups (64, 128, 256, 512, 1024): 256x4096 12.1 11.0 12.4, 512x4096 18.3 13.7 14.2 19.6, 1001x2048
// 23.3 14.9 12.4 13.9 20.7, 4096x4096 109 60 38 36 40, 4096x8192 170 93 60 68 87, 16384x4096 with a gradient beside the norm (256, 512,
// 1024) 119 104 108.
inline long norm_bwd_groups(long M, long K) {
    const NormTeam t = norm_bwd_team(K);
    const long rows = t.waves == 1 ? 4 : 1;              // at a time
    return std::min({(M + rows - 1) / rows, std::max(128L, (M + 4 * rows - 1) / (4 * rows)), t.waves > (t.pieces > 1 ? 8 : 10) ? 256L : 512L});
}

// ---- norm over all gradients ----
constexpr int kClipBatch = 144;          // tensors of a launch, whose addresses are its arguments
constexpr long kClipChunk = 8192;        // elements that a workgroup takes at a time
constexpr long kClipGroups = 2048;       // workgroups of a launch at most, each with a sum of its own
// Workgroups for so many chunks: as few as have the longest as little to do
constexpr long clip_groups(long chunks) {
    const long rounds = (chunks + kClipGroups - 1) / kClipGroups;
    return rounds ? (chunks + rounds - 1) / rounds : 1;
}
// From so many bytes on the norm has a launch of its own (5 us) and, out of place, every chunk a workgroup of its own: workgroups that end where
// others begin keep the writes near each other.  In place those would only read the norm and end where nothing is clipped, which
// takes a tenth of the time: kClipInPlace then.  us, small / large form, out of place: 128 MB 67.8 / 68.7, 256 MB 132 / 129, 1 GB 539 / 508, 2 GB
// 1093 / 1024.  In place, by workgroups (2048, 16384, one for each chunk): 2 GB not clipped 315 317 343, clipped 792 763 757.
constexpr long kClipFuse = 192L << 20;
constexpr long kClipInPlace = 16384;
// The norm also has a launch of its own where there are more partial sums than one launch makes, which every workgroup of every launch of the second pass
// would add up again.  us, one call in a graph (10 of them its start), in place and within the limit, without / with it: 290 tensors of 100000 elements 37.7 / 32.6, 600 of them
// 85 / 55, 10000 of 1000 586 / 305, 65536 of 1000 14400 / 2300; to new tensors 64 / 60, 139 / 110, 756 / 465.
constexpr bool clip_norm_alone(long bytes, long sums) { return bytes > kClipFuse || sums > kClipGroups; }
// Bytes that the first pass reads through the memory-side cache, the last ones; the second pass goes backwards and finds them there.  us, by MB: 1 GB
// (0, 128, 192, 224, 256) 520 512 509 505 505, 2 GB 1039 1030 1022 1021 1020.
constexpr long kClipKeep = 224L << 20;
// Launches over n tensors at most: a batch ends at kClipBatch tensors or 2^31 chunks, which 15 tensors of 2^40 elements do not reach
constexpr long clip_launches(long n) { return n / 15 + 2; }

}  // namespace jet

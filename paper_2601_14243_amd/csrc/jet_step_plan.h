// Which kernels the embedding, layer norm and clipping operators run on: rules on the sizes of a call, host code without HIP, so that the
// tests can ask them too.
#pragma once
#include <algorithm>

namespace jet {

// ---- gradient of the embedding ----
constexpr long kSortBlock = 1024;        // tokens that a workgroup sorts
constexpr long kEmbedDirect = 64;        // up to so many tokens a wave finds those of its own id by itself

// Tokens, in the order of their ids, that a wave adds up
inline int embed_block(long T, long H) {
    const long waves = T * ((H + 511) / 512);
    int L = 32;
    while (L > 8 && waves / L < 4096) L /= 2;
    return L;
}
struct EmbedSpace {
    long sorted, tmp, partial, bytes;    // offsets of the sorted (id, token) arrays, of the blockwise sorted ones, of the partial sums
};
inline EmbedSpace embed_space(long T, long H) {
    auto up = [](long n) { return (n + 255) / 256 * 256; };
    EmbedSpace s = {0, 0, 0, 0};
    if (T <= kEmbedDirect) return s;
    const long L = embed_block(T, H), blocks = (T + L - 1) / L;
    s.tmp = 2 * up(4 * T);
    s.partial = s.tmp + (T > kSortBlock ? 2 * up(4 * T) : 0);
    s.bytes = s.partial + blocks * 2 * H * 4;
    return s;
}

// ---- layer norm ----
// Waves of a row's team and 8-column pieces of a lane
struct NormTeam {
    int waves, pieces;
};
inline NormTeam norm_team(long K, bool few) {
    if (few) {
        if (K <= 2048) return {4, 1};
        if (K <= 4096) return {8, 1};
        if (K <= 8192) return {16, 1};
    }
    if (K <= 512) return {1, 1};
    if (K <= 1024) return {1, 2};
    if (K <= 2048) return {1, 4};
    if (K <= 4096) return {4, 2};
    if (K <= 8192) return {4, 4};
    if (K <= 16384) return {8, 4};
    return {16, 4};
}
inline bool norm_few_rows(long M) { return M <= 512; }
inline NormTeam norm_bwd_team(long K) {
    if (K <= 512) return {1, 1};
    if (K <= 1024) return {1, 2};
    if (K <= 2048) return {4, 1};
    if (K <= 4096) return {4, 2};
    if (K <= 8192) return {8, 2};
    if (K <= 16384) return {16, 2};
    return {16, 4};
}
inline int norm_rows_at_once(NormTeam t) { return t.waves < 4 ? 4 / t.waves : 1; }
// Workgroups of the backward pass, each with sums of its own
inline long norm_bwd_groups(long M, long K) {
    const NormTeam t = norm_bwd_team(K);
    const long r = norm_rows_at_once(t);
    return std::min<long>((M + r - 1) / r, t.waves <= 4 ? 512 : t.waves == 8 ? 512 : 256);
}

// ---- norm over all gradients ----
constexpr int kClipBatch = 144;          // tensors of a launch, whose addresses are its arguments
constexpr long kClipChunk = 8192;        // elements that a workgroup takes at a time
constexpr long kClipGroups = 2048;       // workgroups of a launch at most
// Launches over n tensors at most: a batch ends at kClipBatch tensors or 2^31 chunks, which 15 tensors of 2^40 elements do not reach
constexpr long clip_launches(long n) { return n / 15 + 1; }

}  // namespace jet

// Attention without a [J][K] tensor (attn_fwd, attn_bwd): what the kernels,
// instantiated per storage type, and the host code that launches them share.
#pragma once

#include <algorithm>

#include "internal.hpp"

namespace dm {

// Element (b, head, token, d) of a tensor sits at ptr + b*sb + head*sh + token*st + d.
struct StreamRows {
    char* ptr;
    int64_t sb, sh, st;
};

struct StreamArgs {
    StreamRows q, k, v, o;       // o: forward's output (backward: read)
    StreamRows dout, dq, dk, dv; // backward (dout as o, dq as q, dk as k, dv as v)
    int B, J, K, H, G, P;
    int pack;                    // query heads of one key/value head side by side in a row tile
    float scaler, cap;           // scores: scaler q.k, then cap tanh(. / cap) where cap > 0
    int causal;
    const int32_t *q_len, *k_len, *doc, *prefix;
    const float* slopes;
    float* lse;      // [B][H][J]: log2 of the row's sum of 2^scores (+inf: no key is seen)
    char* lo;        // [B][J][H][P]: out - round(out), 16-bit types (forward: nullptr = not wanted)
    int4* ranges;    // [B][ceil(K / 64)]: smallest and largest document id of 64 keys, and whether some have none
    int splits;      // forward: parts the keys are split into
    float* part_o;   // splits > 1: [splits][B][H][J][P], unscaled
    float2* part_ml; // splits > 1: [splits][B][H][J]: running maximum and sum
    float* dsum;     // backward: [B][H][J] row terms dout . out
    float* dmax;     // backward, fp16: [B][H][dmax_n] largest |dout| of row groups
    int dmax_n;
    float* vmax;     // backward, fp16: [B][G][vmax_n] largest |v| of vmax_rows keys
    int vmax_n, vmax_rows;
    int hparts;      // backward: parts the query heads of a key/value head are split into
    float* part_k;   // hparts > 1: [hparts][B][G][K][dk, dv]
};

constexpr int STREAM_RANGE = 64;   // keys of one entry of `ranges`
constexpr int STREAM_DROWS = 256;  // rows of one entry of `dmax`
// keys of one entry of `vmax`: so many that a wave reads all of a head's in four loads
inline int stream_vmax_rows(int K) { return 256 * std::max(1, (K + 65535) / 65536); }

// Row tiles and head sizes of the kernels (one function each for the host's
// grid and the kernels' own constants).
inline int stream_head_pad(int P) { return P <= 32 ? 32 : P <= 64 ? 64 : P <= 96 ? 96 : 128; }
// queries of a block: 4 waves side by side, or all on the same 32 rows, each on keys of its own
constexpr int STREAM_BM = 128, STREAM_BM_FEW = 32;
constexpr int STREAM_BN = 64, STREAM_BN_FEW = 128;  // keys of a step
// Head sizes above 64: blocks of the backward's two kernels up to which one
// launch does both.  (There the dK / dV kernel's registers leave one wave a
// SIMD, with which dQ takes 800 us where its own kernel takes 565, for 8192
// causal queries in 16 heads of 128; 300 queries in 16 heads take 45 us in
// one launch and 60 in two.  Up to 64 one launch is never slower.)
constexpr int STREAM_BOTH = 512;
constexpr bool stream_apart(int head, int64_t blocks) { return head > 64 && blocks > STREAM_BOTH; }
constexpr int STREAM_KEYS = 128;                    // keys of a block of the dK / dV kernel

template <typename T> void stream_fwd(const StreamArgs& a, bool few, hipStream_t st);
template <typename T> void stream_bwd(const StreamArgs& a, hipStream_t st);

}  // namespace dm

// Host side of attention without a [J][K] tensor: descriptor checks,
// workspace layout and the choice of the forward's form.
#include <math.h>

#include <algorithm>

#include "checks.hpp"
#include "stream.hpp"

namespace dm {
namespace {

constexpr size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t esize(int dtype) { return dtype == DM_F32 ? 4 : 2; }

// Query heads that share a key/value head lie side by side in a row tile
// where the queries alone would leave it part empty.
int packed_heads(const dm_attn_desc& d) { return d.J < STREAM_BM ? d.H / d.G : 1; }

// Few rows of a key/value head (single tokens), or a small product in all:
// the waves of a block share 32 rows and walk keys of their own.  (In the
// second case tiles of 128 rows would leave most CUs idle; but every block
// then reads all keys for itself.  Forward of 12 heads of 64, 2 sequences of
// 256: 7.0 us for 8.9; of 8 heads, one sequence of 1000: 19.2 for 16.6.)
bool few_rows(const dm_attn_desc& d) {
    const int64_t rows = (int64_t)d.J * packed_heads(d);
    const int64_t blocks = (rows + STREAM_BM - 1) / STREAM_BM * d.B * (d.H / packed_heads(d));
    return rows <= 2 * STREAM_BM_FEW || blocks * d.K <= 64 * 512;
}

// Parts the keys are split into where the rows alone give few blocks.
// Few rows: a block for each of the 256 CUs while a part has two steps to
// walk, and four (sequences differ in length) while it has eight; a block
// costs about what five steps do.  (16 sequences of 4096 keys in 8 heads of
// 64: 4 parts of 8 steps 30 us, 8 of 4 35, 16 of 2 44; 64 of up to 8192 in 4
// heads of 128: 2 parts 144, 4 132, 8 147.)
// Otherwise: two blocks for each CU while a part has four steps.
int key_splits(const dm_attn_desc& d) {
    const bool few = few_rows(d);
    const int64_t bm = few ? STREAM_BM_FEW : STREAM_BM, bn = few ? STREAM_BN_FEW : STREAM_BN;
    const int64_t pack = packed_heads(d);
    const int64_t blocks = ((int64_t)d.J * pack + bm - 1) / bm * d.B * (d.H / pack);
    const int64_t steps = (d.K + bn - 1) / bn;
    if (blocks == 0) return 1;
    auto parts = [&](int64_t target, int64_t least) {
        return blocks >= target ? 1 : std::max<int64_t>(1, std::min((target + blocks - 1) / blocks, steps / least));
    };
    const int64_t s = few ? std::max(parts(256, 2), parts(1024, 8)) : blocks >= 384 ? 1 : parts(512, 4);
    return (int)std::min<int64_t>(s, 64);
}

// Parts the query heads of a key/value head are split into in the dK / dV
// kernel, whose blocks otherwise walk all of them: four blocks for each CU
// (causal ones differ in length), against the parts' sums in memory.
int head_parts(const dm_attn_desc& d) {
    const int grp = d.H / d.G;
    const int64_t blocks = ((int64_t)d.K + STREAM_KEYS - 1) / STREAM_KEYS * d.B * d.G;
    if (blocks == 0 || grp == 1) return 1;
    const int64_t want = (1024 + blocks - 1) / blocks;
    return (int)(want < grp ? want : grp);
}

// A grid holds less than 2^32 threads along x (more wrap, without an error).
constexpr int64_t GRID_THREADS = ((int64_t)1 << 32) - 1;

int64_t forward_blocks(const dm_attn_desc& d) {
    const int64_t bm = few_rows(d) ? STREAM_BM_FEW : STREAM_BM, pack = packed_heads(d);
    return ((int64_t)d.J * pack + bm - 1) / bm * d.B * (d.H / pack) * key_splits(d);
}
int64_t key_blocks(const dm_attn_desc& d) {
    return ((int64_t)d.K + STREAM_KEYS - 1) / STREAM_KEYS * d.B * d.G * head_parts(d);
}
int64_t row_blocks(const dm_attn_desc& d) { return ((int64_t)d.J + STREAM_BM - 1) / STREAM_BM * d.B * d.H; }

// Threads of the forward's launches: row tiles, ranges of documents.  (The
// parts are joined only where there are few rows.)
bool forward_fits(const dm_attn_desc& d) {
    const int64_t ranges = d.doc ? ((int64_t)d.K + STREAM_RANGE - 1) / STREAM_RANGE * d.B : 0;
    return forward_blocks(d) * 256 <= GRID_THREADS && ranges * 64 <= GRID_THREADS;
}
// Of the backward's: key tiles (wide heads: 512 threads each) and row tiles,
// in one launch or two; the row terms' blocks are fewer than the row tiles.
bool backward_fits(const dm_attn_desc& d) {
    return (key_blocks(d) * (d.P > 64 ? 2 : 1) + row_blocks(d)) * 256 <= GRID_THREADS;
}

struct Sizes {
    size_t lo, saved;                     // saved: lse, then lo
    size_t ranges, part_o, part_ml, fwd;  // forward workspace: ends of its parts
    size_t dsum, dmax, vmax, bwd;         // backward workspace (ranges first)
    int splits, dmax_n, vmax_n, hparts;
};

Sizes sizes_of(const dm_attn_desc& d) {
    Sizes s{};
    const size_t rows = (size_t)d.B * d.H * d.J;
    s.lo = align256(rows * 4);
    s.saved = s.lo + (d.dtype == DM_F32 ? 0 : align256(rows * d.P * esize(d.dtype)));
    s.ranges = d.doc ? align256((size_t)d.B * ((d.K + STREAM_RANGE - 1) / STREAM_RANGE) * sizeof(int4)) : 0;
    s.splits = key_splits(d);
    const size_t parts = s.splits > 1 ? (size_t)s.splits * rows : 0;
    s.part_o = s.ranges + align256(parts * d.P * 4);
    s.part_ml = s.part_o + align256(parts * 8);
    s.fwd = s.part_ml;
    s.dmax_n = (d.J + STREAM_DROWS - 1) / STREAM_DROWS;
    s.dsum = s.ranges + align256(rows * 4);
    s.dmax = s.dsum + (d.dtype == DM_F16 ? align256((size_t)d.B * d.H * s.dmax_n * 4) : 0);
    s.vmax_n = (d.K + stream_vmax_rows(d.K) - 1) / stream_vmax_rows(d.K);
    s.vmax = s.dmax + (d.dtype == DM_F16 ? align256((size_t)d.B * d.G * s.vmax_n * 4) : 0);
    s.hparts = head_parts(d);
    s.bwd = s.vmax + (s.hparts > 1 ? align256((size_t)s.hparts * d.B * d.G * d.K * 2 * d.P * 4) : 0);
    return s;
}

int check_stride(const dm_attn_stride& s, int tokens, int P, const char* n) {
    if (s.b < 0 || s.h < 0 || s.t < 0) return set_error(DM_ERR_UNSUPPORTED, "%s: negative stride", n);
    if (s.b % 8 || s.h % 8 || s.t % 8)
        return set_error(DM_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements", n);
    // (a step's rows are addressed by 32-bit offsets from its first)
    if (tokens > 1 && (s.t < P || s.t > (1 << 22)))
        return set_error(DM_ERR_UNSUPPORTED, "%s: token stride %lld outside [P, 2^22]", n, (long long)s.t);
    return DM_OK;
}

// a tensor that is written: no element twice, as far as strides tell (sorted
// by size, each steps over what the smaller ones span)
int check_written(const dm_attn_stride& s, int64_t nb, int64_t nh, int64_t nt, int64_t P, const char* n) {
    int64_t st[3] = {s.b, s.h, s.t}, len[3] = {nb, nh, nt};
    if (nb == 0 || nh == 0 || nt == 0) return DM_OK;
    for (int i = 0; i < 2; ++i)
        for (int k = 0; k < 2 - i; ++k)
            if (st[k] > st[k + 1]) {
                const int64_t a = st[k], c = len[k];
                st[k] = st[k + 1]; len[k] = len[k + 1];
                st[k + 1] = a; len[k + 1] = c;
            }
    int64_t span = P;
    for (int i = 0; i < 3; ++i) {
        if (len[i] <= 1) continue;
        if (st[i] < span) return set_error(DM_ERR_UNSUPPORTED, "%s: strides let elements overlap", n);
        span = st[i] * (len[i] - 1) + span;
    }
    return DM_OK;
}

int check_desc(const dm_attn_desc* d) {
    if (!d) return set_error(DM_ERR_ARG, "descriptor is NULL");
    DM_TRY(check_dtype(d->dtype));
    if (d->B < 0 || d->J < 0 || d->K < 0) return set_error(DM_ERR_ARG, "negative size");
    if (d->H <= 0 || d->G <= 0 || d->H % d->G)
        return set_error(DM_ERR_ARG, "H=%d heads are no multiple of G=%d key/value heads", d->H, d->G);
    if (d->P <= 0 || d->P % 8 || d->P > 128)
        return set_error(DM_ERR_UNSUPPORTED, "head size P=%d is not a multiple of 8 up to 128", d->P);
    // (products of three sizes are formed once those of two are known to be small)
    if (d->J > (1 << 30) || d->K > (1 << 30) || (int64_t)d->B * d->H > INT32_MAX / 64 ||
        (int64_t)d->H * d->J > INT32_MAX || (int64_t)d->B * d->H * d->J > INT32_MAX ||
        (int64_t)d->B * d->G * d->K > INT32_MAX)
        return set_error(DM_ERR_UNSUPPORTED, "B=%d H=%d G=%d J=%d K=%d: more than 2^31 - 1 rows", d->B, d->H, d->G, d->J,
                         d->K);
    if (!forward_fits(*d))
        return set_error(DM_ERR_UNSUPPORTED, "B=%d H=%d J=%d K=%d: more blocks than a launch holds", d->B, d->H, d->J, d->K);
    if (!isfinite(d->scaler)) return set_error(DM_ERR_ARG, "scaler=%g", d->scaler);
    // (the kernels' tanh is off by about 1e-7 of the cap)
    if (d->cap != 0.f && !(d->cap >= 0x1p-10f && d->cap <= 0x1p10f))
        return set_error(DM_ERR_ARG, "cap=%g is neither 0 nor from 2^-10 to 2^10", d->cap);
    if (d->causal != 0 && d->causal != 1) return set_error(DM_ERR_ARG, "causal=%d", d->causal);
    const void* aux[5] = {d->q_len, d->k_len, d->doc, d->prefix, d->slopes};
    const char* name[5] = {"q_len", "k_len", "doc", "prefix", "slopes"};
    for (int i = 0; i < 5; ++i)
        if ((uintptr_t)aux[i] & 3u) return set_error(DM_ERR_ARG, "%s is not 4-byte aligned", name[i]);
    if (d->prefix && !d->causal) return set_error(DM_ERR_ARG, "prefix without causal: every key is seen already");
    DM_TRY(check_stride(d->q, d->J, d->P, "q"));
    DM_TRY(check_stride(d->k, d->K, d->P, "k"));
    DM_TRY(check_stride(d->v, d->K, d->P, "v"));
    DM_TRY(check_stride(d->out, d->J, d->P, "out"));
    return check_written(d->out, d->B, d->H, d->J, d->P, "out");
}

// (The copies end a step's rows behind the last by the token stride: an axis
// of one token, which never takes a step, gets a row's own size.)
StreamRows rows_of(const void* p, const dm_attn_stride& s, int tokens, int P) {
    return {(char*)p, s.b, s.h, tokens > 1 ? s.t : P};
}

StreamArgs args_of(const dm_attn_desc& d) {
    StreamArgs a{};
    a.B = d.B; a.J = d.J; a.K = d.K; a.H = d.H; a.G = d.G; a.P = d.P;
    a.pack = packed_heads(d);
    a.scaler = d.scaler > 0.f ? d.scaler : 1.f / sqrtf((float)d.P);
    a.cap = d.cap;
    a.causal = d.causal;
    a.q_len = d.q_len; a.k_len = d.k_len; a.doc = d.doc; a.prefix = d.prefix; a.slopes = d.slopes;
    a.splits = 1;
    return a;
}

}  // namespace
}  // namespace dm

using namespace dm;

extern "C" {

int attn_sizes(const dm_attn_desc* d, size_t* saved_bytes, size_t* fwd_ws_bytes, size_t* bwd_ws_bytes) {
    DM_TRY(check_desc(d));
    const Sizes s = sizes_of(*d);
    if (saved_bytes) *saved_bytes = s.saved;
    if (fwd_ws_bytes) *fwd_ws_bytes = s.fwd;
    if (bwd_ws_bytes) *bwd_ws_bytes = s.bwd;
    return DM_OK;
}

int attn_form(const dm_attn_desc* d, int32_t* rows, int32_t* key_parts, int32_t* head_parts_, int32_t* apart) {
    DM_TRY(check_desc(d));
    if (rows) *rows = few_rows(*d) ? STREAM_BM_FEW : STREAM_BM;
    if (key_parts) *key_parts = key_splits(*d);
    if (head_parts_) *head_parts_ = head_parts(*d);
    if (apart) *apart = stream_apart(d->P, key_blocks(*d) + row_blocks(*d)) ? 1 : 0;
    return DM_OK;
}

int attn_fwd(const dm_attn_desc* d, const void* q, const void* k, const void* v, void* out, void* saved, void* ws,
             size_t ws_bytes, void* stream) {
    DM_TRY(check_desc(d));
    if (d->B == 0 || d->J == 0) return DM_OK;
    const Sizes s = sizes_of(*d);
    DM_TRY(check_ptr(q, "q"));
    if (d->K > 0) {
        DM_TRY(check_ptr(k, "k"));
        DM_TRY(check_ptr(v, "v"));
    }
    DM_TRY(check_ptr(out, "out"));
    if (saved) DM_TRY(check_ptr(saved, "saved"));
    if (ws_bytes < s.fwd) return set_error(DM_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, s.fwd);
    if (s.fwd) DM_TRY(check_ptr(ws, "ws"));
    if (d->K > 0) DM_TRY(check_apart(out, "out", {k, v}));
    DM_TRY(check_apart(out, "out", {q, saved}));
    StreamArgs a = args_of(*d);
    a.q = rows_of(q, d->q, d->J, d->P); a.o = rows_of(out, d->out, d->J, d->P);
    a.k = rows_of(k, d->k, d->K, d->P); a.v = rows_of(v, d->v, d->K, d->P);
    if (saved) {
        a.lse = (float*)saved;
        if (d->dtype != DM_F32) a.lo = (char*)saved + s.lo;
    }
    a.ranges = (int4*)ws;
    a.splits = s.splits;
    a.part_o = (float*)((char*)ws + s.ranges);
    a.part_ml = (float2*)((char*)ws + s.part_o);
    const hipStream_t st = S(stream);
    const bool few = few_rows(*d);
    if (d->dtype == DM_F16) stream_fwd<half_t>(a, few, st);
    else if (d->dtype == DM_BF16) stream_fwd<bf16_t>(a, few, st);
    else stream_fwd<float>(a, few, st);
    return check_launch("attn_fwd");
}

int attn_bwd(const dm_attn_desc* d, const void* q, const void* k, const void* v, const void* out, const void* saved,
             const void* dout, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
    DM_TRY(check_desc(d));
    if (!backward_fits(*d))
        return set_error(DM_ERR_UNSUPPORTED, "B=%d H=%d G=%d J=%d K=%d: more blocks than a launch holds", d->B, d->H, d->G,
                         d->J, d->K);
    DM_TRY(check_written(d->q, d->B, d->H, d->J, d->P, "dq"));
    DM_TRY(check_written(d->k, d->B, d->G, d->K, d->P, "dk"));
    DM_TRY(check_written(d->v, d->B, d->G, d->K, d->P, "dv"));
    if (d->B == 0 || (d->J == 0 && d->K == 0)) return DM_OK;
    const Sizes s = sizes_of(*d);
    if (d->J > 0) {
        DM_TRY(check_ptr(q, "q")); DM_TRY(check_ptr(out, "out")); DM_TRY(check_ptr(saved, "saved"));
        DM_TRY(check_ptr(dout, "dout")); DM_TRY(check_ptr(dq, "dq"));
    }
    if (d->K > 0) {
        DM_TRY(check_ptr(k, "k")); DM_TRY(check_ptr(v, "v"));
        DM_TRY(check_ptr(dk, "dk")); DM_TRY(check_ptr(dv, "dv"));
    }
    if (ws_bytes < s.bwd) return set_error(DM_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, s.bwd);
    if (s.bwd) DM_TRY(check_ptr(ws, "ws"));
    // (of axes without elements the pointers say nothing)
    const void* rows = d->J > 0 ? dq : nullptr;
    if (d->J > 0) DM_TRY(check_apart(dq, "dq", {q, out, dout, saved}));
    if (d->K > 0) {
        DM_TRY(check_apart(dk, "dk", {k, v, rows}));
        DM_TRY(check_apart(dv, "dv", {k, v, dk, rows}));
        if (d->J > 0) DM_TRY(check_apart(dk, "dk", {q, out, dout, saved}));
        if (d->J > 0) DM_TRY(check_apart(dv, "dv", {q, out, dout, saved}));
        if (d->J > 0) DM_TRY(check_apart(dq, "dq", {k, v}));
    }
    StreamArgs a = args_of(*d);
    a.q = rows_of(q, d->q, d->J, d->P); a.o = rows_of(out, d->out, d->J, d->P);
    a.k = rows_of(k, d->k, d->K, d->P); a.v = rows_of(v, d->v, d->K, d->P);
    a.dout = rows_of(dout, d->out, d->J, d->P); a.dq = rows_of(dq, d->q, d->J, d->P);
    a.dk = rows_of(dk, d->k, d->K, d->P); a.dv = rows_of(dv, d->v, d->K, d->P);
    a.lse = (float*)saved;
    if (d->dtype != DM_F32) a.lo = (char*)saved + s.lo;
    a.ranges = (int4*)ws;
    a.dsum = (float*)((char*)ws + s.ranges);
    a.dmax = d->dtype == DM_F16 ? (float*)((char*)ws + s.dsum) : nullptr;
    a.dmax_n = s.dmax_n;
    a.vmax = d->dtype == DM_F16 ? (float*)((char*)ws + s.dmax) : nullptr;
    a.vmax_n = s.vmax_n;
    a.vmax_rows = stream_vmax_rows(d->K);
    a.hparts = s.hparts;
    a.part_k = (float*)((char*)ws + s.vmax);
    const hipStream_t st = S(stream);
    if (d->dtype == DM_F16) stream_bwd<half_t>(a, st);
    else if (d->dtype == DM_BF16) stream_bwd<bf16_t>(a, st);
    else stream_bwd<float>(a, st);
    return check_launch("attn_bwd");
}

}  // extern "C"

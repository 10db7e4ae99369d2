// Embedding lookup and its gradient.
#include "checks.hpp"

namespace dm {
namespace {

constexpr int NT = 256;

// y[t] = scale table[ids[t]]: `lanes` lanes a token (a power of two), 16
// bytes of the storage type each at a time.
template <typename T>
__global__ __launch_bounds__(NT) void embed_fwd_k(int64_t tokens, int vocab, int cols, int lanes, const int32_t* ids,
                                                  const T* table, float scale, T* y) {
    const int tpb = NT / lanes, gl = threadIdx.x & (lanes - 1);
    const int64_t t = (int64_t)blockIdx.x * tpb + threadIdx.x / lanes;
    if (t >= tokens) return;
    const int id = ids[t];
    const bool in = id >= 0 && id < vocab;
    for (int c = 8 * gl; c < cols; c += 8 * lanes) {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (in) {
            V8<T>::load(table + (int64_t)id * cols + c, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= scale;
        }
        V8<T>::store(y + t * cols + c, x);
    }
}

// dtable rows of a block: it looks through all ids for those of its rows
// and adds up their tokens' gradients, in the order of the tokens, in LDS.
constexpr int EROWS = 16, ECOLS = 1024;
template <typename T>
__global__ __launch_bounds__(NT) void embed_bwd_k(int64_t tokens, int vocab, int cols, const int32_t* ids, int pad,
                                                  const T* dy, float scale, float* dtable) {
    __shared__ float acc[EROWS * ECOLS];
    __shared__ int hit_t[NT], hit_r[NT];
    __shared__ int wcount[NT / 64];
    const int v0 = (int)blockIdx.x * EROWS, c0 = (int)blockIdx.y * ECOLS, nc = min(ECOLS, cols - c0);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < EROWS * ECOLS; i += NT) acc[i] = 0.f;
    __syncthreads();
    for (int64_t t0 = 0; t0 < tokens; t0 += NT) {
        const int64_t t = t0 + tid;
        const int id = t < tokens ? ids[t] : -1;
        const bool hit = id >= v0 && id < v0 + EROWS && id < vocab && id != pad;
        const uint64_t m = __ballot(hit);
        if (lane == 0) wcount[wave] = __popcll(m);
        __syncthreads();
        int at = 0, n = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            if (w < wave) at += wcount[w];
            n += wcount[w];
        }
        if (hit) {
            at += __popcll(m & ((1ull << lane) - 1));
            hit_t[at] = tid;
            hit_r[at] = id - v0;
        }
        __syncthreads();
        for (int i = 0; i < n; ++i) {
            const T* p = dy + (t0 + hit_t[i]) * cols + c0;
            float* a = acc + hit_r[i] * ECOLS;
            for (int c = tid; c < nc; c += NT) a[c] += to_f(p[c]);
        }
        __syncthreads();
    }
    for (int r = 0; r < EROWS && v0 + r < vocab; ++r)
        for (int c = tid; c < nc; c += NT) dtable[(int64_t)(v0 + r) * cols + c0 + c] = acc[r * ECOLS + c] * scale;
}

int check_embed(int32_t dtype, int64_t tokens, int32_t vocab, int32_t cols, float scale) {
    DM_TRY(check_dtype(dtype));
    DM_TRY(check_rows(tokens, cols, 16384));
    if (tokens > INT32_MAX) return set_error(DM_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
    if (vocab <= 0) return set_error(DM_ERR_ARG, "vocab=%d", vocab);
    if (!(scale - scale == 0.f)) return set_error(DM_ERR_ARG, "scale=%g", scale);
    return DM_OK;
}

template <typename T>
void launch_fwd(int64_t tokens, int vocab, int cols, const int32_t* ids, const void* table, float scale, void* y,
                hipStream_t st) {
    int lanes = 1;
    while (lanes < 64 && lanes * 8 < cols) lanes *= 2;
    const int64_t tpb = NT / lanes;
    embed_fwd_k<T><<<dim3((unsigned)((tokens + tpb - 1) / tpb)), NT, 0, st>>>(tokens, vocab, cols, lanes, ids,
                                                                             (const T*)table, scale, (T*)y);
}
template <typename T>
void launch_bwd(int64_t tokens, int vocab, int cols, const int32_t* ids, int pad, const void* dy, float scale,
                float* dtable, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)vocab + EROWS - 1) / EROWS), (unsigned)((cols + ECOLS - 1) / ECOLS));
    embed_bwd_k<T><<<grid, NT, 0, st>>>(tokens, vocab, cols, ids, pad, (const T*)dy, scale, dtable);
}

}  // namespace
}  // namespace dm

using namespace dm;

extern "C" {

size_t embed_ws_bytes(int64_t tokens, int32_t vocab, int32_t cols) {
    (void)tokens; (void)vocab; (void)cols;
    return 0;
}

int embed_fwd(int32_t dtype, int64_t tokens, int32_t vocab, int32_t cols, const int32_t* ids, const void* table,
              float scale, void* y, void* stream) {
    DM_TRY(check_embed(dtype, tokens, vocab, cols, scale));
    if (tokens == 0) return DM_OK;
    DM_TRY(check_ptr(ids, "ids")); DM_TRY(check_ptr(table, "table")); DM_TRY(check_ptr(y, "y"));
    const hipStream_t st = S(stream);
    if (dtype == DM_F16) launch_fwd<half_t>(tokens, vocab, cols, ids, table, scale, y, st);
    else if (dtype == DM_BF16) launch_fwd<bf16_t>(tokens, vocab, cols, ids, table, scale, y, st);
    else launch_fwd<float>(tokens, vocab, cols, ids, table, scale, y, st);
    return check_launch("embed_fwd");
}

int embed_bwd(int32_t dtype, int64_t tokens, int32_t vocab, int32_t cols, const int32_t* ids, int32_t pad_id,
              const void* dy, float scale, float* dtable, void* ws, size_t ws_bytes, void* stream) {
    DM_TRY(check_embed(dtype, tokens, vocab, cols, scale));
    if (tokens > 0) {
        DM_TRY(check_ptr(ids, "ids"));
        DM_TRY(check_ptr(dy, "dy"));
    }
    DM_TRY(check_ptr(dtable, "dtable"));
    const size_t need = embed_ws_bytes(tokens, vocab, cols);
    if (ws_bytes < need) return set_error(DM_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    if (need) DM_TRY(check_ptr(ws, "ws"));
    const hipStream_t st = S(stream);
    if (dtype == DM_F16) launch_bwd<half_t>(tokens, vocab, cols, ids, pad_id, dy, scale, dtable, st);
    else if (dtype == DM_BF16) launch_bwd<bf16_t>(tokens, vocab, cols, ids, pad_id, dy, scale, dtable, st);
    else launch_bwd<float>(tokens, vocab, cols, ids, pad_id, dy, scale, dtable, st);
    return check_launch("embed_bwd");
}

}  // extern "C"

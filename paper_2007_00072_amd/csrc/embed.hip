// Embedding lookup and its gradient.
#include <algorithm>

#include "checks.hpp"

namespace dm {
namespace {

constexpr int NT = 256;

// A grid holds less than 2^32 threads along x (more wrap, without an error):
// more blocks go in several rows, whose last may have blocks without work.
constexpr int64_t GRID_ROW = (int64_t)1 << 22;
dim3 rows_of_blocks(int64_t n) {
    return dim3((unsigned)std::min(n, GRID_ROW), (unsigned)((n + GRID_ROW - 1) / GRID_ROW));
}
__device__ __forceinline__ int64_t block_of_rows() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// y[t] = scale table[ids[t]]: `lanes` lanes a token (a power of two), 16
// bytes of the storage type each at a time.  Bound by memory: 16384 tokens of
// 1024 in fp16, 34 MB read and 34 written, in 12.7 us.
template <typename T>
__global__ __launch_bounds__(NT) void embed_fwd_k(int64_t tokens, int vocab, int cols, int lanes, const int32_t* ids,
                                                  const T* table, float scale, T* y) {
    const int tpb = NT / lanes, gl = threadIdx.x & (lanes - 1);
    const int64_t t = block_of_rows() * tpb + threadIdx.x / lanes;
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

// ------------------------------------------------------------ gradient
// dtable[v] = scale sum over the tokens of id v: the tokens are sorted by id
// (stable: the order of the sums is given by the ids alone), then every
// wave adds up a piece of the sorted list, writing the rows whose tokens all
// lie there and leaving partial sums of the first and the last otherwise,
// which a last pass joins in order.  dy is read once, evenly, and rows that no
// token has come from the fill that runs beside the sort: the pass is bound by
// writing dtable and reading dy, while no id has a large share of the tokens.
// An id's parts are joined by one wave (for each 256 columns): 16384 tokens of
// 1024 in fp16 take 51 us as words are and 101 with two ids, 131072 with two
// ids 790.
//
// The sort: up to 16384 tokens in lists of 1024, each by one block in LDS
// while the other blocks of the launch fill; a second launch places every
// token by counting, in each list, what comes before it.  (One block for all
// 16384 takes 52 us: the ballots of a radix pass are bound by its CU's
// vector units.)  16384 is what 14 bits of a token's number beside 18 of its id
// and 64 KB of LDS for all lists hold.  More tokens, or ids past 18 bits, by
// passes over blocks of tokens (count, scan, place: three launches for each 8
// bits of the ids, with 4096 tokens or more a block): 16385 tokens of 1024 in
// fp16 101 us, 65536 173, 2^20 1500 (1060 with ids evenly spread).
constexpr int PIECE = 8;           // sorted tokens of a wave, all requested together
constexpr int PIECE_FEW = 4;       // up to RUN_TOKENS tokens: shorter chains
// Up to RUN_TOKENS a wave follows its last id to the end instead of leaving it
// in parts: one launch less.  768 columns in bf16, ids as words are: 256 tokens
// 19 us, 512 21, 1024 29, where 1025 in parts take 30.  A wave adds a long run
// by itself, four tokens at a time: tokens all of one id take 49 us for 128, 145
// for 512 and 270 for 1024, 34 for 1025 in parts.
constexpr int RUN_TOKENS = 1024;
constexpr int SORT_TOKENS = 16384;
constexpr int IDX_BITS = 14;       // of a token's number in the sort of lists, below its id
constexpr int LIST = 1024;         // tokens of a list
constexpr int SORT_NT = 1024, SORT_W = SORT_NT / 64;
constexpr int LIST_NT = 256, LIST_W = LIST_NT / 64;
constexpr int BINS = 256;          // of a pass: 8 bits
constexpr int PASS_NT = 256, PASS_W = PASS_NT / 64;
constexpr int PASS_BLOCKS = 1024;

// An id as a sorting key: ids outside the table and the padding id come last.
__device__ __forceinline__ uint32_t key_of(int id, int vocab, int pad) {
    return id >= 0 && id < vocab && id != pad ? (uint32_t)id : (uint32_t)vocab;
}

// Lanes of the wave with the same digit, among the `in` lanes.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool in) {
    uint64_t m = __ballot(in);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const uint64_t s = __ballot((d >> b) & 1u);
        m &= (d >> b) & 1u ? s : ~s;
    }
    return m;
}

// Exclusive sums of x[0 .. n) in LDS, in place; n a multiple of 4 * NT.
template <int THREADS> __device__ void scan_lds(uint32_t* x, int n, uint32_t* wsum) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t carry = 0;
    for (int i0 = 0; i0 < n; i0 += 4 * THREADS) {
        uint32_t v[4], t = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = x[i0 + 4 * tid + k];
            t += v[k];
        }
        uint32_t inc = t;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t o = __shfl_up(inc, s, 64);
            if (lane >= s) inc += o;
        }
        __syncthreads();
        if (lane == 63) wsum[wave] = inc;
        __syncthreads();
        uint32_t base = carry, all = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) base += wsum[w];
            all += wsum[w];
        }
        base += inc - t;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[i0 + 4 * tid + k] = base;
            base += v[k];
        }
        carry += all;
    }
    __syncthreads();
}

// Blocks `first` .. of a launch write zeros over dtable (n floats, a multiple of 8).
template <int THREADS> __device__ __forceinline__ void fill(float* p, int64_t n, int first) {
    const int64_t step = (int64_t)((int)gridDim.x - first) * THREADS * 4;
    for (int64_t i = ((int64_t)((int)blockIdx.x - first) * THREADS + threadIdx.x) * 4; i < n; i += step)
        *reinterpret_cast<floatx4*>(p + i) = floatx4{0.f, 0.f, 0.f, 0.f};
}

// Blocks 0 .. lists - 1 sort 1024 tokens each, the others fill.  A list
// holds (id, token) packed, so that all differ and their order is the
// stable one.  With one list, the result is the final one.  Bound by the
// fill: 125 MB in 22 us, 94 MB in 14 (the sort of a list takes 12).
__global__ __launch_bounds__(LIST_NT) void sort_fill_k(int tokens, int lists, int vocab, const int32_t* ids, int pad,
                                                      int key_bits, uint32_t* packed, uint32_t* keys, uint32_t* toks,
                                                      float* dtable, int64_t n) {
    __shared__ uint32_t mem[2][LIST], cnt[BINS * LIST_W], wsum[LIST_W];
    if ((int)blockIdx.x >= lists) {
        fill<LIST_NT>(dtable, n, lists);
        return;
    }
    uint32_t *a = mem[0], *b = mem[1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = (int)blockIdx.x * LIST, len = min(LIST, tokens - t0);
    const int i0 = wave * (LIST / LIST_W), i1 = min(len, i0 + LIST / LIST_W);
    for (int t = tid; t < len; t += LIST_NT) a[t] = key_of(ids[t0 + t], vocab, pad) << IDX_BITS | (uint32_t)(t0 + t);
    for (int shift = IDX_BITS; shift < IDX_BITS + key_bits; shift += 8) {
        for (int i = tid; i < BINS * LIST_W; i += LIST_NT) cnt[i] = 0;
        __syncthreads();
        for (int i = i0; i < i1; i += 64) {
            const bool in = i + lane < i1;
            const uint32_t d = in ? a[i + lane] >> shift & (BINS - 1) : 0;
            const uint64_t m = same_digit(d, in);
            if (in && (m & ((1ull << lane) - 1)) == 0) cnt[d * LIST_W + wave] += (uint32_t)__popcll(m);
        }
        __syncthreads();
        scan_lds<LIST_NT>(cnt, BINS * LIST_W, wsum);
        for (int i = i0; i < i1; i += 64) {
            const bool in = i + lane < i1;
            const uint32_t x = in ? a[i + lane] : 0, d = x >> shift & (BINS - 1);
            const uint64_t m = same_digit(d, in), below = m & ((1ull << lane) - 1);
            uint32_t at = 0;
            if (in) {
                at = cnt[d * LIST_W + wave];
                b[at + (uint32_t)__popcll(below)] = x;
            }
            // (the lanes of a wave run together: all have read the counter)
            __builtin_amdgcn_wave_barrier();
            if (in && below == 0) cnt[d * LIST_W + wave] = at + (uint32_t)__popcll(m);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t* t = a;
        a = b;
        b = t;
    }
    for (int t = tid; t < len; t += LIST_NT) {
        if (lists == 1) {
            keys[t] = a[t] >> IDX_BITS;
            toks[t] = a[t] & ((1u << IDX_BITS) - 1);
        } else {
            packed[t0 + t] = a[t];
        }
    }
}

// Every token's place: what comes before it in its own list and in the others.
// 16384 tokens: 5.7 us, the latency of ten steps of four searches at a time.
__global__ __launch_bounds__(LIST_NT) void merge_k(int tokens, const uint32_t* packed, uint32_t* keys, uint32_t* toks) {
    __shared__ __attribute__((aligned(16))) uint32_t x[SORT_TOKENS];
    __shared__ int place[LIST_W][64];
    u32x4 r[SORT_TOKENS / (LIST_NT * 4)];  // all requested together (packed has room to a multiple of 64)
#pragma unroll
    for (int k = 0; k < SORT_TOKENS / (LIST_NT * 4); ++k)
        r[k] = *reinterpret_cast<const u32x4*>(packed + min((k * LIST_NT + (int)threadIdx.x) * 4, (tokens - 1) & ~3));
#pragma unroll
    for (int k = 0; k < SORT_TOKENS / (LIST_NT * 4); ++k)
        *reinterpret_cast<u32x4*>(x + (k * LIST_NT + threadIdx.x) * 4) = r[k];
    __syncthreads();
    // 64 tokens a block; each wave searches a quarter of the lists for them,
    // side by side, so that their steps wait together
    constexpr int U = SORT_TOKENS / LIST / LIST_W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = (int)blockIdx.x * 64 + lane;
    const uint32_t p = x[min(i, tokens - 1)];
    // how many of each list's are below p (in its own list: the token's place there)
    int lo[U] = {0, 0, 0, 0};
#pragma unroll
    for (int step = LIST; step > 0; step >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = lo[u] + step, q = (wave * U + u) * LIST + h - 1;
            if (h <= LIST && q < tokens && x[min(q, SORT_TOKENS - 1)] < p) lo[u] = h;
        }
    place[wave][lane] = lo[0] + lo[1] + lo[2] + lo[3];
    __syncthreads();
    if (wave > 0 || i >= tokens) return;
    const int at = place[0][lane] + place[1][lane] + place[2][lane] + place[3][lane];
    keys[at] = p >> IDX_BITS;
    toks[at] = p & ((1u << IDX_BITS) - 1);
}

// One pass of the sort over blocks of `per` tokens (a multiple of PASS_NT).
struct PassArgs {
    int tokens, per, nblk, shift, vocab, pad;
    const int32_t* ids;               // first pass: the ids; else null
    const uint32_t *k_in, *t_in;
    uint32_t *k_out, *t_out, *table;  // table [BINS][nblk]
    float* dtable;                    // first pass: filled by the blocks behind nblk
    int64_t n;
};
__device__ __forceinline__ uint32_t pass_key(const PassArgs& g, int i) {
    return g.ids ? key_of(g.ids[i], g.vocab, g.pad) : g.k_in[i];
}

// cnt[wave][digit] of this block's tokens
__device__ __forceinline__ void pass_count(const PassArgs& g, uint32_t* cnt, int i0, int i1) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < BINS * PASS_W; i += PASS_NT) cnt[i] = 0;
    __syncthreads();
    for (int i = i0; i < i1; i += 64) {
        const bool in = i + lane < i1;
        const uint32_t d = in ? pass_key(g, i + lane) >> g.shift & (BINS - 1) : 0;
        const uint64_t m = same_digit(d, in);
        if (in && (m & ((1ull << lane) - 1)) == 0) cnt[wave * BINS + d] += (uint32_t)__popcll(m);
    }
    __syncthreads();
}

__global__ __launch_bounds__(PASS_NT) void pass_count_k(PassArgs g) {
    __shared__ uint32_t cnt[BINS * PASS_W];
    if ((int)blockIdx.x >= g.nblk) {
        fill<PASS_NT>(g.dtable, g.n, g.nblk);
        return;
    }
    const int wave = threadIdx.x >> 6, end = min(g.tokens, ((int)blockIdx.x + 1) * g.per);
    const int i0 = (int)blockIdx.x * g.per + wave * (g.per / PASS_W);
    pass_count(g, cnt, i0, min(end, i0 + g.per / PASS_W));
    uint32_t c = 0;
#pragma unroll
    for (int w = 0; w < PASS_W; ++w) c += cnt[w * BINS + threadIdx.x];
    g.table[threadIdx.x * g.nblk + blockIdx.x] = c;
}

// Exclusive sums over the table, by one block.
__global__ __launch_bounds__(SORT_NT) void pass_scan_k(uint32_t* table, int n) {
    __shared__ uint32_t x[4 * SORT_NT], wsum[SORT_W];
    uint32_t carry = 0;
    for (int i0 = 0; i0 < n; i0 += 4 * SORT_NT) {
        uint32_t last = 0;
        for (int k = threadIdx.x; k < 4 * SORT_NT; k += SORT_NT) x[k] = i0 + k < n ? table[i0 + k] : 0;
        __syncthreads();
        last = x[4 * SORT_NT - 1];
        __syncthreads();
        scan_lds<SORT_NT>(x, 4 * SORT_NT, wsum);
        for (int k = threadIdx.x; k < 4 * SORT_NT; k += SORT_NT)
            if (i0 + k < n) table[i0 + k] = x[k] + carry;
        carry += x[4 * SORT_NT - 1] + last;
        __syncthreads();
    }
}

__global__ __launch_bounds__(PASS_NT) void pass_place_k(PassArgs g) {
    __shared__ uint32_t cnt[BINS * PASS_W];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int end = min(g.tokens, ((int)blockIdx.x + 1) * g.per);
    const int i0 = (int)blockIdx.x * g.per + wave * (g.per / PASS_W), i1 = min(end, i0 + g.per / PASS_W);
    pass_count(g, cnt, i0, i1);
    uint32_t at = g.table[tid * g.nblk + blockIdx.x];
#pragma unroll
    for (int w = 0; w < PASS_W; ++w) {
        const uint32_t c = cnt[w * BINS + tid];
        cnt[w * BINS + tid] = at;
        at += c;
    }
    __syncthreads();
    for (int i = i0; i < i1; i += 64) {
        const bool in = i + lane < i1;
        const uint32_t k = in ? pass_key(g, i + lane) : 0, d = k >> g.shift & (BINS - 1);
        const uint64_t m = same_digit(d, in), below = m & ((1ull << lane) - 1);
        uint32_t base = 0;
        if (in) {
            base = cnt[wave * BINS + d];
            const uint32_t to = base + (uint32_t)__popcll(below);
            g.k_out[to] = k;
            g.t_out[to] = g.ids ? (uint32_t)(i + lane) : g.t_in[i + lane];
        }
        __builtin_amdgcn_wave_barrier();
        if (in && below == 0) cnt[wave * BINS + d] = base + (uint32_t)__popcll(m);
        __builtin_amdgcn_wave_barrier();
    }
}

// Where the sums of sorted tokens go.
struct SumArgs {
    int tokens, vocab, cols;
    const uint32_t *keys, *toks;
    const void* dy;
    float scale;
    float* dtable;
    float* part;  // [pieces][2][cols]: first and last id's part; null: ids are followed to their end
};

// 8 elements as they lie in memory
template <typename T> struct Raw8 {
    u32x4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) v[i] = reinterpret_cast<const u32x4*>(p)[i];
    }
    __device__ __forceinline__ void add_to(float acc[8]) const {
        float x[8];
        if constexpr (sizeof(T) == 2) {
            V8<T>::unpack(v[0], x);
        } else {
            const floatx4 a = __builtin_bit_cast(floatx4, v[0]), b = __builtin_bit_cast(floatx4, v[1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += x[i];
    }
};

// A wave takes PC sorted tokens and 512 columns (8 a lane; lanes past the
// last column read the last ones again and store nothing).  Bound by memory:
// 16384 tokens of 1024 in fp16, 34 MB read and up to 125 written, in 18 us.
template <typename T, int PC>
__global__ __launch_bounds__(NT) void sum_k(SumArgs g) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pieces = (g.tokens + PC - 1) / PC, slabs = (g.cols + 511) / 512;
    const int64_t id = block_of_rows() * (NT / 64) + wave;
    if (id >= (int64_t)pieces * slabs) return;
    const int piece = (int)(id / slabs), col = (int)(id - (int64_t)piece * slabs) * 512 + lane * 8;
    const bool in = col < g.cols;
    int i = piece * PC, end = min(g.tokens, i + PC);
    // the piece's keys and its neighbours', requested together
    const uint32_t key0 = g.keys[min(i + lane, g.tokens - 1)];
    const uint32_t before = i > 0 ? g.keys[i - 1] : ~0u;
    const uint32_t first = __builtin_amdgcn_readlane(key0, 0);
    if (first >= (uint32_t)g.vocab) return;  // ids without a gradient are the last
    if (!g.part) {
        // ids that began here, to their end
        const uint32_t k = __builtin_amdgcn_readlane(key0, end - 1 - i);
        i += (int)__popcll(__ballot(i + lane < end && key0 == before));
        if (i == end) return;
        for (;;) {
            const uint64_t m = __ballot(end + lane < g.tokens && g.keys[min(end + lane, g.tokens - 1)] == k);
            end += (int)__popcll(m);
            if (m != ~0ull) break;
        }
    }
    const uint32_t after = end < g.tokens ? g.keys[end] : ~0u;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const T* dy = reinterpret_cast<const T*>(g.dy) + min(col, g.cols - 8);
    for (; i < end; i += PC) {
        const int n = min(PC, end - i), me = i + min(lane, n - 1);
        const uint32_t my_key = g.keys[me], my_tok = g.toks[me];
        const uint32_t ahead = i + n < end ? g.keys[i + n] : after;
        Raw8<T> x[PC];
#pragma unroll
        for (int u = 0; u < PC; ++u)
            x[u].load(dy + (int64_t)__builtin_amdgcn_readlane(my_tok, min(u, n - 1)) * g.cols);
#pragma unroll
        for (int u = 0; u < PC; ++u) {
            if (u >= n) break;
            const uint32_t k = __builtin_amdgcn_readlane(my_key, u);
            if (k >= (uint32_t)g.vocab) return;
            x[u].add_to(acc);
            const uint32_t nk = u + 1 < n ? __builtin_amdgcn_readlane(my_key, u + 1) : ahead;
            const bool done = u + 1 == n && i + n == end;  // of this piece
            if (nk == k && !done) continue;
            // the id ends here, or the piece does
            float* to = g.dtable + (int64_t)k * g.cols;
            bool whole = true;
            if (g.part) {
                if (k == first && before == first) {
                    to = g.part + (int64_t)piece * 2 * g.cols;
                    whole = false;
                } else if (nk == k) {
                    to = g.part + ((int64_t)piece * 2 + 1) * g.cols;
                    whole = false;
                }
            }
            if (in) {
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] *= g.scale;
                }
                V8<float>::store(to + col, acc);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.f;
        }
    }
}

// Joins the parts of the ids that begin in a piece and end in a later one:
// a wave takes 256 columns.  16384 tokens whose most frequent id has a
// fifteenth of them: 11 us, the latency of that id's 140 parts.
__global__ __launch_bounds__(NT) void join_parts_k(SumArgs g) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pieces = (g.tokens + PIECE - 1) / PIECE, slabs = (g.cols + 255) / 256;
    const int64_t id = block_of_rows() * (NT / 64) + wave;
    if (id >= (int64_t)pieces * slabs) return;
    const int piece = (int)(id / slabs);
    const int col = (int)(id - (int64_t)piece * slabs) * 256 + lane * 4;
    const int i = piece * PIECE, last = i + PIECE - 1;
    if (last + 1 >= g.tokens) return;
    const uint32_t k = g.keys[last], next = g.keys[last + 1], first = g.keys[i], before = i > 0 ? g.keys[i - 1] : ~0u;
    if (k >= (uint32_t)g.vocab || next != k) return;
    if (first == k && before == k) return;  // began earlier
    const float* part = g.part + min(col, g.cols - 4);
    floatx4 acc = *reinterpret_cast<const floatx4*>(part + ((int64_t)piece * 2 + 1) * g.cols);
    for (int p0 = piece + 1;; p0 += 64) {
        // pieces that begin with the id: a run of the next ones
        const int64_t at = ((int64_t)p0 + lane) * PIECE;
        const uint64_t m = __ballot(at < g.tokens && g.keys[min(at, (int64_t)g.tokens - 1)] == k);
        const int n = (int)__popcll(m);
        constexpr int U = 32;  // requested together
        for (int s = 0; s < n; s += U) {
            floatx4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                x[u] = *reinterpret_cast<const floatx4*>(part + (int64_t)(p0 + min(s + u, n - 1)) * 2 * g.cols);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s + u < n) acc += x[u];
        }
        if (n < 64) break;
    }
    if (col < g.cols) *reinterpret_cast<floatx4*>(g.dtable + (int64_t)k * g.cols + col) = acc * g.scale;
}

constexpr size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
int key_bits(int vocab) { return 32 - __builtin_clz((unsigned)vocab); }  // of 0 .. vocab
bool sorted_in_lists(int64_t tokens, int vocab) { return tokens <= SORT_TOKENS && key_bits(vocab) <= 32 - IDX_BITS; }

// Workspace: keys and tokens, the lists (or, for passes, a second pair of
// them and the table), the parts.
struct EmbedWs {
    size_t list, table, part, bytes;
    int per, nblk;
};
EmbedWs embed_ws(int64_t tokens, int vocab, int cols) {
    EmbedWs w{};
    w.list = align256((size_t)tokens * 4);
    size_t at = 3 * w.list;
    if (!sorted_in_lists(tokens, vocab)) {
        at = 4 * w.list;
        w.per = 4096;
        while ((tokens + w.per - 1) / w.per > PASS_BLOCKS) w.per *= 2;
        w.nblk = (int)((tokens + w.per - 1) / w.per);
        w.table = at;
        at += align256((size_t)BINS * w.nblk * 4);
    }
    w.part = at;
    if (tokens > RUN_TOKENS) at += align256((size_t)((tokens + PIECE - 1) / PIECE) * 2 * cols * 4);
    w.bytes = at;
    return w;
}

template <typename T>
void launch_sums(const SumArgs& a, hipStream_t st) {
    const int64_t pc = a.part ? PIECE : PIECE_FEW;
    const int64_t waves = (a.tokens + pc - 1) / pc * ((a.cols + 511) / 512);
    const dim3 grid = rows_of_blocks((waves + NT / 64 - 1) / (NT / 64));
    if (a.part) {
        sum_k<T, PIECE><<<grid, NT, 0, st>>>(a);
        const int64_t joins = (a.tokens + pc - 1) / pc * ((a.cols + 255) / 256);
        join_parts_k<<<rows_of_blocks((joins + NT / 64 - 1) / (NT / 64)), NT, 0, st>>>(a);
    } else {
        sum_k<T, PIECE_FEW><<<grid, NT, 0, st>>>(a);
    }
}

int check_embed(int32_t dtype, int64_t tokens, int32_t vocab, int32_t cols, float scale) {
    DM_TRY(check_dtype(dtype));
    DM_TRY(check_rows(tokens, cols, 16384));
    if (tokens > (1 << 30)) return set_error(DM_ERR_UNSUPPORTED, "more than 2^30 tokens");
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
    embed_fwd_k<T><<<rows_of_blocks((tokens + tpb - 1) / tpb), NT, 0, st>>>(tokens, vocab, cols, lanes, ids,
                                                                           (const T*)table, scale, (T*)y);
}
}  // namespace
}  // namespace dm

using namespace dm;

extern "C" {

size_t embed_ws_bytes(int64_t tokens, int32_t vocab, int32_t cols) {
    if (tokens <= 0 || tokens > (1 << 30) || vocab <= 0 || cols <= 0) return 0;
    return embed_ws(tokens, vocab, cols).bytes;
}

int embed_fwd(int32_t dtype, int64_t tokens, int32_t vocab, int32_t cols, const int32_t* ids, const void* table,
              float scale, void* y, void* stream) {
    DM_TRY(check_embed(dtype, tokens, vocab, cols, scale));
    if (tokens == 0) return DM_OK;
    DM_TRY(check_ptr(ids, "ids")); DM_TRY(check_ptr(table, "table")); DM_TRY(check_ptr(y, "y"));
    DM_TRY(check_apart(y, "y", {ids, table}));
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
    if (tokens > 0) DM_TRY(check_apart(dtable, "dtable", {ids, dy}));
    const hipStream_t st = S(stream);
    const int64_t n = (int64_t)vocab * cols;
    // zeros: blocks of 64 KB, up to four for each of the 256 CUs
    const int64_t fills = std::min<int64_t>((n + 16383) / 16384, 1024);
    const EmbedWs w = tokens > 0 ? embed_ws(tokens, vocab, cols) : EmbedWs{};
    uint32_t* keys = (uint32_t*)ws;
    uint32_t* toks = (uint32_t*)((char*)ws + w.list);
    if (tokens == 0 || sorted_in_lists(tokens, vocab)) {
        const int lists = (int)((tokens + LIST - 1) / LIST);
        uint32_t* packed = (uint32_t*)((char*)ws + 2 * w.list);
        sort_fill_k<<<dim3((unsigned)(lists + fills)), LIST_NT, 0, st>>>((int)tokens, lists, vocab, ids, pad_id,
                                                                        key_bits(vocab), packed, keys, toks, dtable, n);
        if (lists > 1)
            merge_k<<<dim3((unsigned)((tokens + 63) / 64)), LIST_NT, 0, st>>>((int)tokens, packed, keys, toks);
    } else {
        PassArgs a{};
        a.tokens = (int)tokens; a.per = w.per; a.nblk = w.nblk; a.vocab = vocab; a.pad = pad_id;
        a.ids = ids; a.table = (uint32_t*)((char*)ws + w.table);
        a.dtable = dtable; a.n = n;
        uint32_t* list[2][2] = {{keys, toks}, {(uint32_t*)((char*)ws + 2 * w.list), (uint32_t*)((char*)ws + 3 * w.list)}};
        int to = 0;
        for (a.shift = 0; a.shift < key_bits(vocab); a.shift += 8) {
            a.k_out = list[to][0];
            a.t_out = list[to][1];
            pass_count_k<<<dim3((unsigned)(w.nblk + (a.ids ? fills : 0))), PASS_NT, 0, st>>>(a);
            pass_scan_k<<<dim3(1), SORT_NT, 0, st>>>(a.table, BINS * w.nblk);
            pass_place_k<<<dim3((unsigned)w.nblk), PASS_NT, 0, st>>>(a);
            a.ids = nullptr;
            a.k_in = keys = list[to][0];
            a.t_in = toks = list[to][1];
            to ^= 1;
        }
    }
    if (tokens > 0) {
        SumArgs a{};
        a.tokens = (int)tokens; a.vocab = vocab; a.cols = cols;
        a.keys = keys; a.toks = toks; a.dy = dy; a.scale = scale; a.dtable = dtable;
        if (tokens > RUN_TOKENS) a.part = (float*)((char*)ws + w.part);
        if (dtype == DM_F16) launch_sums<half_t>(a, st);
        else if (dtype == DM_BF16) launch_sums<bf16_t>(a, st);
        else launch_sums<float>(a, st);
    }
    return check_launch("embed_bwd");
}

}  // extern "C"

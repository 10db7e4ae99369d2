// Kernels of attention without a [J][K] tensor.
//
// One pass over the keys with a running row maximum m and sum l: with scores
// s in units of log2, m' = max(m, max s), p = 2^(s - m'), l' = l 2^(m - m') +
// sum p, o' = o 2^(m - m') + p v; at the end o / l.  The backward recomputes
// p = 2^(s - lse) from the saved lse = m + log2 l, and with the row term
// D = dout . out: ds = p (dout . v - D) (1 - tanh^2 where scores are capped),
// dq = scaler ds k, dk = scaler ds^T q, dv = p^T dout.
//
// All products run on 32x32x16 MFMAs (32x32x2 in float32), transposed so
// that what the softmax needs per row lies in one lane: the first product
// gives a lane one query (its column) and 16 of 32 keys (its accumulators),
// so row maxima and sums are in-lane but for one exchange between the two
// lane halves, and the accumulators, converted in place, are the second
// product's operand: the order of a contraction is free, so its other
// operand is read in the order the accumulators have (a lane half holds keys
// 4 hh + {0..3, 8..11} of 16).  The dK / dV kernel does the same with keys
// and queries exchanged.
#pragma once

#include <math.h>

#include <type_traits>

#include "stream.hpp"

namespace dm {
namespace stream {

constexpr int NT = 256;  // threads of a block: 4 waves
constexpr float LOG2E = 1.4426950408889634f;

// ------------------------------------------------------------- fragments
// 8 contraction elements of one row (or column) of an MFMA operand
template <typename T> struct Frag { u32x4 v[sizeof(T) / 2]; };

template <typename T> __device__ __forceinline__ floatx16 mma(const Frag<T>& a, const Frag<T>& b, floatx16 c);
template <> __device__ __forceinline__ floatx16 mma(const Frag<half_t>& a, const Frag<half_t>& b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a.v[0]), __builtin_bit_cast(half8, b.v[0]),
                                                  c, 0, 0, 0);
}
template <> __device__ __forceinline__ floatx16 mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v[0]),
                                                   __builtin_bit_cast(bf16x8, b.v[0]), c, 0, 0, 0);
}
template <> __device__ __forceinline__ floatx16 mma(const Frag<float>& a, const Frag<float>& b, floatx16 c) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const floatx4 x = __builtin_bit_cast(floatx4, a.v[k]), y = __builtin_bit_cast(floatx4, b.v[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
    }
    return c;
}

template <typename T> __device__ __forceinline__ Frag<T> frag_zero() {
    Frag<T> f;
#pragma unroll
    for (auto& x : f.v) x = u32x4{0, 0, 0, 0};
    return f;
}
template <typename T> __device__ __forceinline__ Frag<T> frag_load(const T* p) {
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) f.v[i] = reinterpret_cast<const u32x4*>(p)[i];
    return f;
}
// accumulators 8 c .. 8 c + 7 as the operand of the next product, rounded to
// the storage type (what the MFMA takes; sums stay in 32 bits)
template <typename T> __device__ __forceinline__ Frag<T> frag_acc(const float* x) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
        f.v[0] = V8<T>::pack(x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, x[i]);
    }
    return f;
}

// ------------------------------------------------------------- LDS tiles
// Rows of PITCH bytes (a power of two, at least the padded head size); the
// 16-byte pieces of row r are permuted by piece ^ f(r), with f such that the
// 16 lanes that read one piece of 16 rows, and the lanes that read 4 pieces
// of 4 rows with the transposing read, each reach all 64 banks once.
template <int PITCH> __device__ __forceinline__ int swz(int r) {
    if constexpr (PITCH == 64) return (r >> 2) & 3;
    if constexpr (PITCH == 128) return ((r & 2) << 1) + ((r >> 2) & 3);
    return 4 * (r & 3) + ((r >> 2) & 3);
}
template <int PITCH> __device__ __forceinline__ int piece_off(int r, int piece) {
    return r * PITCH + ((piece ^ swz<PITCH>(r)) << 4);
}

template <typename T, int DP> struct Tile {
    static constexpr int PITCH = (DP == 96 ? 128 : DP) * (int)sizeof(T);
    static constexpr int PIECES = PITCH / 16;       // of a row
    static constexpr int EPP = 16 / (int)sizeof(T);  // elements of a piece
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4 lds_s4;

    // elements e .. e + 7 of row r
    static __device__ __forceinline__ Frag<T> row(const char* t, int r, int e) {
        Frag<T> f;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i)
            f.v[i] = *reinterpret_cast<const u32x4*>(t + piece_off<PITCH>(r, e / EPP + i));
        return f;
    }
    // column c + lane % 32, rows r + 4 hh + {0..3, 8..11} (hh: lane half)
    static __device__ __forceinline__ Frag<T> col(const char* t, int r, int c, int lane) {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            // 16 lanes of a transposing read take 4 rows of 16 columns
            const int sl = lane & 15, cc = c + 16 * ((lane >> 4) & 1) + 4 * (sl & 3);
            const int rr = r + 4 * (lane >> 5) + (sl >> 2);
            const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s4*)(t + piece_off<PITCH>(rr, cc >> 3) + (cc & 7) * 2));
            const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s4*)(t + piece_off<PITCH>(rr + 8, cc >> 3) + (cc & 7) * 2));
            const u32x2 lo = __builtin_bit_cast(u32x2, a), hi = __builtin_bit_cast(u32x2, b);
            f.v[0] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const int cc = c + (lane & 31), rr = r + 4 * (lane >> 5);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f.v[i >> 2][i & 3] = *reinterpret_cast<const uint32_t*>(
                    t + piece_off<PITCH>(rr + (i & 3) + 8 * (i >> 2), cc >> 2) + (cc & 3) * 4);
        }
        return f;
    }
};

// One step's rows of a tensor, copied from memory straight into a tile:
// buffer_load ... lds writes the 64 lanes' 16 bytes side by side, so lane l of
// copy i takes the row and the piece that lie at that place of the tile.  The
// buffer begins at the step's first row and ends behind its last one that
// holds data: pieces behind the end, and behind the head size, become zeros
// whatever memory holds there.  The copies are issued from inline assembly,
// so that the compiler does not wait for them before the LDS reads of the
// step at hand; copied() does, ahead of the barrier that publishes the tile.
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}
// ONCE: nobody reads these rows again soon, they need not stay in the caches
template <bool ONCE> __device__ __forceinline__ void copy16(uint32_t lds, uint32_t voff, u32x4 rsrc) {
    // (m0 and the descriptor may come from VALU instructions right before:
    // five wait states to their use)
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(voff),
                     "s"(rsrc)
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff),
                     "s"(rsrc)
                     : "memory", "m0");
}
// (The builtin tells the compiler that its own loads have come as well: else
// it waits for one from ahead of a loop, a row's q, in every step of the
// loop, and by then for the copies that were asked for a moment ago.)
__device__ __forceinline__ void copied() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0) alone
}
// all copies but the last N of this wave
template <int N> __device__ __forceinline__ void copied_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// this wave's LDS reads so far
__device__ __forceinline__ void lds_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename T, int DP, int ROWS, int LANES = NT> struct Copies {
    using TL = Tile<T, DP>;
    static constexpr int N = ROWS * TL::PIECES / LANES;
    static_assert(ROWS * TL::PIECES % LANES == 0, "pieces");
    static constexpr uint32_t NONE = 0xfffffff0u;  // behind any end
    uint32_t vo[N];
    uint32_t step;  // bytes between rows
    __device__ __forceinline__ int row(int tid, int i) const { return (i * LANES + tid) / TL::PIECES; }
    __device__ __forceinline__ void init(int tid, int P, int64_t st) {
        step = (uint32_t)(st * (int64_t)sizeof(T));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = row(tid, i), c = (i * LANES + tid) % TL::PIECES ^ swz<TL::PITCH>(r);
            vo[i] = c * TL::EPP < P ? (uint32_t)r * step + (uint32_t)c * 16 : NONE;
        }
    }
    // rows 0 .. left - 1 from `base` into the tile at `lds`; in(r): the row may be read
    template <bool ONCE = false, typename In>
    __device__ __forceinline__ void issue(int tid, const char* base, int left, uint32_t lds, bool all, In in) const {
        const uint32_t n = (uint32_t)min(max(left, 0), ROWS) * step;
        const u32x4 rsrc{uniform((uint32_t)(uintptr_t)base), uniform((uint32_t)((uintptr_t)base >> 32) & 0xffffu),
                         uniform(n), 0x00020000u};
        const uint32_t to = lds + (uint32_t)(tid >> 6) * 1024u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t v = vo[i];
            if (!all && !in(row(tid, i))) v = NONE;
            copy16<ONCE>(uniform(to + (uint32_t)i * (LANES * 16)), v, rsrc);
        }
    }
};

// --------------------------------------------------------------- scores
// 4 elements, rounded
template <typename T> __device__ __forceinline__ void store4(T* p, const float* y) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T4*>(p) = T4{from_f<T>(y[0]), from_f<T>(y[1]), from_f<T>(y[2]), from_f<T>(y[3])};
}
// both lane halves' values: gfx950 swaps the upper half of one register with
// the lower half of another (a lane shuffle through the LDS unit would stand
// in every step's chain of dependent instructions)
struct Halves { float lo, hi; };
__device__ __forceinline__ Halves halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t lo = r[0], hi = r[1];
    return Halves{__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}

// Raw products to scores.  With x the returned value, a score in units of
// log2 is factor x + offset - what the bias takes, and the same for all of a
// row but for x, so that the offset only matters where lse does.
// Capped scores: the 16-bit types take t = tanh z = 1 - 2 u, u = 1 / (e^2z + 1),
// by one exponential and one reciprocal (absolute error about 1e-7, far
// under their resolution) and go on with x = -u: no instruction makes t, and
// 1 - t^2 = 4 (u - u^2) in the backward.  float32 takes the library's tanh.
template <typename T, bool CAP, bool BIAS> struct Scorer {
    static constexpr bool U = CAP && sizeof(T) == 2;
    float zc, scale, offset;  // z (or its exponent's argument) per product; log2 units per x
    __device__ __forceinline__ Scorer(const StreamArgs& g) {
        zc = CAP ? g.scaler / g.cap * (U ? 2.f * LOG2E : 1.f) : 0.f;
        scale = (CAP ? g.cap * (U ? 2.f : 1.f) : g.scaler) * LOG2E;
        offset = U ? g.cap * LOG2E : 0.f;
    }
    __device__ __forceinline__ float value(float raw) const {
        if constexpr (U) return -__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(raw * zc) + 1.f);
        if constexpr (CAP) return tanhf(raw * zc);
        return raw;
    }
    // 1 - t^2, less the factor SLOPE
    static constexpr float SLOPE = U ? 4.f : 1.f;
    __device__ __forceinline__ static float slope(float x) {
        if constexpr (U) return fmaf(-x, x, -x);
        return fmaf(-x, x, 1.f);
    }
};

// Which keys a query sees.  A causal query at position p sees keys 0 .. p,
// and keys below the sequence's prefix: all keys below `hi`, of which its
// own document's.
struct Seq {
    int q_len, k_len, off, prefix;  // off: position of query 0
    __device__ __forceinline__ Seq(const StreamArgs& g, int b) {
        k_len = g.k_len ? min(max(g.k_len[b], 0), g.K) : g.K;
        q_len = g.q_len ? min(max(g.q_len[b], 0), g.J) : g.J;
        off = k_len - q_len;
        prefix = g.causal && g.prefix ? g.prefix[b] : 0;
    }
    __device__ __forceinline__ int hi(const StreamArgs& g, int j) const {
        if (j >= q_len) return 0;
        return g.causal ? min(k_len, max(off + j + 1, prefix)) : k_len;
    }
    // document of query j (-1: none)
    __device__ __forceinline__ int doc_of(const StreamArgs& g, int b, int j) const {
        const int p = off + j;
        return j < q_len && p >= 0 && p < k_len ? g.doc[(int64_t)b * g.K + p] : -1;
    }
};

// documents of 64 keys: x the smallest id, y the largest (without any,
// none matches), z: some of the keys are no document's
__device__ __forceinline__ bool ranges_meet(int4 a, int2 b) { return a.x <= b.y && b.x <= a.y; }
// all of them of one document
__device__ __forceinline__ bool range_is(int4 a, int id) { return a.x == id && a.y == id && a.z == 0; }

// 64 ids to (smallest, largest) of those that are documents
__device__ __forceinline__ int2 wave_range(int id) {
    int lo = id >= 0 ? id : INT32_MAX, hi = id >= 0 ? id : -1;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        lo = min(lo, __shfl_xor(lo, s, 64));
        hi = max(hi, __shfl_xor(hi, s, 64));
    }
    return int2{__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi)};
}

// Smallest and largest document of each 64 keys, and whether some are of
// none: what the walks below need of documents, at a 64th of the reads.
// A launch: 3 to 5 us for 4 x 4096 keys.
template <typename T>
__global__ __launch_bounds__(64) void ranges_k(StreamArgs g) {
    const int nr = (g.K + STREAM_RANGE - 1) / STREAM_RANGE, b = (int)blockIdx.x / nr, e = (int)blockIdx.x - b * nr;
    const int k = e * STREAM_RANGE + (int)threadIdx.x;
    const Seq s(g, b);
    const int id = k < s.k_len ? g.doc[(int64_t)b * g.K + k] : -1;
    const int2 r = wave_range(id);
    const bool holes = __ballot(id < 0) != 0;
    if (threadIdx.x == 0) g.ranges[(int64_t)b * nr + e] = int4{r.x, r.y, holes ? 1 : 0, 0};
}

// Which of 64 steps a block walks, and how: bits for step `base` + i.  The
// entries behind a step's keys (or rows) are read once for the 64.
struct Window {
    int base;
    uint64_t meet;   // some of it may be of the block's documents
    uint64_t holes;  // some of it is of none: copied row by row
    uint64_t whole;  // all of it is of the one document of this wave's rows (keys)
    __device__ __forceinline__ bool is(uint64_t m, int step) const { return (m >> (step - base)) & 1; }
};

// Block number -> (tile, head): the tiles of a head on one XCD (blocks reach
// the 8 XCDs in turn), so that its L2 serves the rows they share; all heads'
// first tiles before the second ones.
__device__ __forceinline__ void place(int lid, int nz, int& tile, int& z) {
    if ((nz & 7) == 0) {
        const int hp = nz >> 3, i = lid >> 3;
        tile = i / hp;
        z = (i - tile * hp) * 8 + (lid & 7);
    } else {
        tile = lid / nz;
        z = lid - tile * nz;
    }
}

// ------------------------------------------------------------- forward
// A block takes 32 WQ query rows; its waves lie WQ along the queries and
// WK = 4 / WQ along the keys of a step (each wave 32 NS of them).
// WQ = 4: the waves share the step's tiles, of which one pair is filled
// while the other is read.  128 rows: with 256 registers a wave holds its 32
// rows' sums and two waves fit a SIMD, of which one multiplies while the
// other takes exponentials.  A third pair of tiles in flight changes nothing
// (126 us with and without, heads of 64); what bounds it are the vector
// instructions of the softmax (59 % of the vector unit's time) and the products'
// latency, with capped scores the vector unit (69 %: an exponential and a
// reciprocal more for each).
// 4 x 4096 tokens in documents of about 700, 16 heads of 64: 126 us, 0.40
// PFLOP/s of the pairs that are seen; 8192 causal tokens, capped, 16 heads of
// 128: 375 us, 0.73; 500 queries behind up to 4096 keys, 16 heads of 96: 39.
// WQ = 1, few rows: reading the keys is what takes time.  Each wave copies
// its own 32 keys of a step and waits for nobody else; tiles are asked for as
// soon as they have been read.  Two blocks fit a CU (64 KB of LDS: two pairs of
// tiles a wave up to heads of 64 in 16 bits and 32 in float32, else one pair),
// so that the one's first and last steps lie beside the other's reads; float32
// heads above 64 take 128 KB, one block a CU.  64 sequences of 1 to 8192 keys,
// about uniform, in 4 key/value heads of 128 in bf16 (538 MB at the mean): 103
// us, 5.2 TB/s; 133 with two pairs of tiles and one block a CU, 165 with tiles
// that the waves share and a barrier in every step.
template <typename T, int DP, bool CAP, bool BIAS, int WQ, int NS>
__global__ __launch_bounds__(NT, sizeof(T) == 2 ? 2 : 1) void fwd_k(StreamArgs g) {
    constexpr int WK = 4 / WQ, BM = 32 * WQ, BN = 32 * WK * NS, ND = DP / 32, NC = DP / 16;
    constexpr bool OWN = WK > 1;  // tiles of a wave's own
    using TL = Tile<T, DP>;
    constexpr int TB = BN * TL::PITCH;  // bytes of a step's keys
    // pairs of tiles: one is filled while the other is read (a wave's own: where two blocks then fit a CU)
    constexpr int NB = !OWN || 4 * TB <= 65536 ? 2 : 1;
    static_assert(OWN || 4 * TB <= 131072, "two pairs of tiles");
    constexpr int ROWS = OWN ? 32 * NS : BN, RB = ROWS * TL::PITCH;  // of a tile
    // joining the waves along the keys: m, l and o of all but the first
    constexpr int JOIN = WK > 1 ? (WK - 1) * 64 * (2 + 16 * ND) * 4 : 0;
    constexpr int TILES = 2 * NB * TB > JOIN ? 2 * NB * TB : JOIN;
    __shared__ __attribute__((aligned(16))) char lds[TILES + (OWN ? 0 : 2 * BN * 4)];
    int* kdoc = reinterpret_cast<int*>(lds + TILES);

    const int hz = g.H / g.pack, rows = g.J * g.pack, nqt = (rows + BM - 1) / BM;
    int tile, z;
    place((int)blockIdx.x, g.B * hz * g.splits, tile, z);
    const int split = z % g.splits;
    z /= g.splits;
    if (g.causal) tile = nqt - 1 - tile;  // rows with the most keys first
    const int b = z / hz, h0 = (z - b * hz) * g.pack, kvh = h0 / (g.H / g.G);
    const int tid = threadIdx.x, lane = tid & 63, c32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wq = wave % WQ, wk = wave / WQ;
    const Seq sq(g, b);

    const int r0 = tile * BM, row = r0 + 32 * wq + c32;  // this lane's query row
    const int j = row / g.pack, h = h0 + row - j * g.pack;
    const bool live = row < rows && j < sq.q_len;
    const int pos = sq.off + j;
    const int mydoc = g.doc && live ? sq.doc_of(g, b, j) : -1;
    const int hi = live && !(g.doc && mydoc < 0) ? sq.hi(g, j) : 0;
    const float slope2 = g.slopes && live ? g.slopes[h] * LOG2E : 0.f;
    const Scorer<T, CAP, BIAS> sc(g);

    Frag<T> qf[NC];
    {
        const T* qp = reinterpret_cast<const T*>(g.q.ptr) + b * g.q.sb + h * g.q.sh + j * g.q.st;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e = 16 * c + 8 * hh;
            qf[c] = hi > 0 && e < g.P ? frag_load<T>(qp + e) : frag_zero<T>();
        }
    }

    // rows of the block that hold queries: the last has the largest hi, the
    // first of a wave the smallest
    const int jlast = min(min(r0 + BM, rows) - 1, sq.q_len * g.pack - 1) / g.pack;
    const int hi_all = r0 < sq.q_len * g.pack ? sq.hi(g, jlast) : 0;
    // (rows without a query need no mask: their sums are dropped at the end)
    const int wrow = r0 + 32 * wq, hi_low = wrow < sq.q_len * g.pack ? sq.hi(g, wrow / g.pack) : INT32_MAX;
    int2 qr{0, 0};
    int onedoc = -1;  // the document of all the wave's rows, if one
    if (g.doc) {
        __shared__ int2 wrange[4];
        const int2 r = wave_range(mydoc);
        if (r.x == r.y && __ballot(mydoc < 0) == 0) onedoc = r.x;
        if (lane == 0) wrange[wave] = r;
        __syncthreads();
        qr = wrange[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) qr = int2{min(qr.x, wrange[w].x), max(qr.y, wrange[w].y)};
    }
    const int steps = (hi_all + BN - 1) / BN, per = (steps + g.splits - 1) / g.splits;
    const int s_end = min(steps, (split + 1) * per);
    const int nr = (g.K + STREAM_RANGE - 1) / STREAM_RANGE;
    Window win{-64, 0, 0, 0};
    auto read = [&](int from) {
        int4 r[BN / STREAM_RANGE];
        bool meet = false, holes = false, whole = onedoc >= 0;
#pragma unroll
        for (int i = 0; i < BN / STREAM_RANGE; ++i) {
            const int e = (from + lane) * (BN / STREAM_RANGE) + i;
            r[i] = e < nr ? g.ranges[(int64_t)b * nr + e] : int4{INT32_MAX, -1, 1, 0};
            meet = meet || ranges_meet(r[i], qr);
            holes = holes || r[i].z != 0;
            whole = whole && range_is(r[i], onedoc);
        }
        win = Window{from, __ballot(meet && from + lane < s_end), __ballot(holes), __ballot(whole)};
    };
    // next step from `from` on whose keys may be of the rows' documents
    auto next = [&](int from) {
        if (!g.doc) return from;
        while (from < s_end) {
            if (from >= win.base + 64) read(from);
            const uint64_t m = win.meet >> (from - win.base);
            if (m) return from + (int)__builtin_ctzll(m);
            from = win.base + 64;
        }
        return s_end;
    };

    const T* kp = reinterpret_cast<const T*>(g.k.ptr) + b * g.k.sb + kvh * g.k.sh;
    const T* vp = reinterpret_cast<const T*>(g.v.ptr) + b * g.v.sb + kvh * g.v.sh;
    const int32_t* docs = g.doc ? g.doc + (int64_t)b * g.K : nullptr;
    // (a wave's own tiles lie together: K and V of one step, then of the other)
    const int who = OWN ? lane : tid, own = OWN ? wave * 2 * NB * RB : 0;
    Copies<T, DP, ROWS, OWN ? 64 : NT> ck, cv;
    ck.init(who, g.P, g.k.st);
    cv.init(who, g.P, g.v.st);
    const uint32_t base = lds_offset(lds) + (uint32_t)own;
    int fdoc = -1;  // documents of the step on its way, in LDS once its turn is near (put)
    auto put = [&](int buf) {
        if (!OWN && docs && tid < BN) kdoc[buf * BN + tid] = fdoc;
    };
    auto fetch = [&](int step, int buf) {
        const int k0 = step * BN + (OWN ? ROWS * wk : 0);
        if (!OWN && docs && tid < BN) fdoc = k0 + tid < sq.k_len ? docs[k0 + tid] : -1;
        const bool all = !docs || !win.is(win.holes, step);
        auto in = [&](int r) { return k0 + r < sq.k_len && docs[k0 + r] >= 0; };
        const uint32_t to = base + (uint32_t)(buf * 2 * RB);
        const char *kb = reinterpret_cast<const char*>(kp + (int64_t)k0 * g.k.st);
        const char *vb = reinterpret_cast<const char*>(vp + (int64_t)k0 * g.v.st);
        if (OWN && nqt == 1) {  // (the only rows that read these keys)
            ck.template issue<OWN>(who, kb, sq.k_len - k0, to, all, in);
            cv.template issue<OWN>(who, vb, sq.k_len - k0, to + RB, all, in);
        } else {
            ck.issue(who, kb, sq.k_len - k0, to, all, in);
            cv.issue(who, vb, sq.k_len - k0, to + RB, all, in);
        }
    };

    floatx16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    // m: in the scores' own units.  What is summed is 2^UP p with p relative to
    // 2^m: 2^10 in fp16, as in the backward, whose normal numbers then hold
    // probabilities down to 2^-24 (many of 2^-22 behind one large one are what
    // a long sequence sums up; they had one or two bits there), and the
    // reference follows closer so that 2^14 is the largest.
    constexpr bool HALF = __is_same(T, half_t);
    constexpr float UP = HALF ? 10.f : 0.f;
    float m = -INFINITY, l = 0.f;
    const float f = BIAS ? 1.f : sc.scale, slack = (HALF ? 4.f : 8.f) / f;

    auto mixed = [&](int step) { return docs && step < s_end && !win.is(win.whole, step); };
    int cur = next(split * per), nxt = s_end;
    bool cur_mixed = mixed(cur), nxt_mixed = false;
    if (cur < s_end) {
        fetch(cur, 0);
        put(0);
        if (OWN && NB == 2) {
            nxt = next(cur + 1);
            nxt_mixed = mixed(nxt);
            if (nxt < s_end) fetch(nxt, 1);
        }
    }
    for (int buf = 0; cur < s_end; buf ^= NB - 1) {
        if (!OWN) {
            copied();
            __syncthreads();
        } else if (NB == 2 && nxt < s_end) {
            copied_but<2 * Copies<T, DP, ROWS, OWN ? 64 : NT>::N>();
        } else {
            copied();
        }
        const int k0 = cur * BN + 32 * NS * wk;  // this wave's keys
        const char *tk = lds + own + buf * 2 * RB, *tv = tk + RB;
        if (!OWN || NB == 1) {
            nxt = next(cur + 1);
            nxt_mixed = mixed(nxt);
            if (!OWN && nxt < s_end) fetch(nxt, buf ^ 1);
        }

        floatx16 a[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) a[n][i] = 0.f;
        // (all of K's fragments are asked for ahead of the first product: left
        // to itself the compiler waits for each right after asking)
        constexpr int AH = sizeof(T) == 2 && !OWN ? (DP <= 96 ? NS * NC : 12) : 0;
        Frag<T> kf[AH ? AH : 1];
#pragma unroll
        for (int i = 0; i < AH; ++i) kf[i] = TL::row(tk, 32 * (i / NC) + c32, 16 * (i % NC) + 8 * hh);
        if constexpr (AH > 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NS * NC; ++i) {
            const int n = i / NC, c = i % NC;
            a[n] = mma<T>(i < AH ? kf[i < AH ? i : 0] : TL::row(tk, 32 * n + c32, 16 * c + 8 * hh), qf[c], a[n]);
        }
        float x[NS][16];
        const float far = BIAS ? (float)(pos - k0 - 4 * hh) : 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[n][i] = sc.value(a[n][i]);
                if constexpr (BIAS)
                    x[n][i] = fmaf(-slope2, fabsf(far - (float)(32 * n + 8 * (i >> 2) + (i & 3))), x[n][i] * sc.scale);
            }
        if (cur_mixed) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int kk = 32 * n + 8 * q + 4 * hh;
                    int id[4];
                    if constexpr (OWN) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) id[i] = docs[min(k0 + kk + i, g.K - 1)];  // (past the end: bounded by hi)
                    } else {
                        const int4 kd = *reinterpret_cast<const int4*>(kdoc + buf * BN + kk);
                        id[0] = kd.x; id[1] = kd.y; id[2] = kd.z; id[3] = kd.w;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (id[i] != mydoc) x[n][4 * q + i] = -INFINITY;
                }
        }
        if (k0 + 32 * NS > hi_low) {
            const int end = hi - k0 - 4 * hh;
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * n + 8 * (i >> 2) + (i & 3) >= end) x[n][i] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, x[n][i]), x[n][i + 1]);
        const Halves both = halves(mx);
        mx = fmaxf(both.lo, both.hi);
        // the row's reference value follows its maximum only once that is 2^8
        // (fp16: 2^4) above it: until then sums and products stay inside their types
        if (__any(mx > m + slack)) {
            const float mn = fmaxf(m, mx);
            const float alpha = mn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * f);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
        }
        const float mf = m == -INFINITY ? 0.f : fmaf(-m, f, UP);
        float p[NS][16];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[n][i] = __builtin_amdgcn_exp2f(fmaf(x[n][i], f, mf));
                l += p[n][i];
            }
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const Frag<T> pf = frag_acc<T>(&p[n][8 * c]);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[d] = mma<T>(TL::col(tv, 32 * n + 16 * c, 32 * d, lane), pf, o[d]);
            }
        int then = nxt;
        bool then_mixed = nxt_mixed;
        if (OWN) {
            lds_read();
            if (NB == 2 && nxt < s_end) {
                then = next(nxt + 1);
                then_mixed = mixed(then);
            }
            if (then < s_end && (NB == 1 || then != nxt)) fetch(then, NB == 2 ? buf : 0);
        } else {
            put(buf ^ 1);
        }
        cur = nxt;
        cur_mixed = nxt_mixed;
        nxt = then;
        nxt_mixed = then_mixed;
    }
    m = sc.offset - fmaf(-m, f, UP);  // from here in units of log2 (what the sums are relative to, as rounded)
    if (hi == 0) {  // a row that sees nothing
        m = -INFINITY;
        l = 0.f;
    }
    const Halves sums = halves(l);
    l = sums.lo + sums.hi;

    if constexpr (WK > 1) {
        // join the waves along the keys, in wave order
        __syncthreads();
        float* jm = reinterpret_cast<float*>(lds);
        if (wk > 0) {
            float* w = jm + (wk - 1) * 64 * (2 + 16 * ND) + lane;
            w[0] = m;
            w[64] = l;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) w[64 * (2 + 16 * d + i)] = o[d][i];
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int w = 0; w < WK - 1; ++w) {
            const float* p = jm + w * 64 * (2 + 16 * ND) + lane;
            const float mn = fmaxf(m, p[0]), ms = mn == -INFINITY ? 0.f : mn;
            const float a = __builtin_amdgcn_exp2f(m - ms), c = __builtin_amdgcn_exp2f(p[0] - ms);
            m = mn;
            l = l * a + p[64] * c;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * a + p[64 * (2 + 16 * d + i)] * c;
        }
    }
    if (row >= rows) return;
    const int64_t zr = ((int64_t)b * g.H + h) * g.J + j;
    if (g.splits > 1) {
        const int64_t at = (int64_t)split * g.B * g.H * g.J + zr;
        if (hh == 0) g.part_ml[at] = float2{m, l};
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int e = 32 * d + 8 * q + 4 * hh;
                if (e < g.P)
                    *reinterpret_cast<floatx4*>(g.part_o + at * g.P + e) =
                        floatx4{o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]};
            }
        return;
    }
    // (a row that sees no key: zeros, and +inf so that 2^(s - lse) is zero)
    const float inv = l > 0.f ? 1.f / l : 0.f;
    if (g.lse && hh == 0) g.lse[zr] = l > 0.f ? m + __builtin_amdgcn_logf(l) : INFINITY;
    T* op = reinterpret_cast<T*>(g.o.ptr) + b * g.o.sb + h * g.o.sh + j * g.o.st;
    T* lp = g.lo ? reinterpret_cast<T*>(g.lo) + (((int64_t)b * g.J + j) * g.H + h) * g.P : nullptr;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = 32 * d + 8 * q + 4 * hh;
            if (e >= g.P) continue;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = o[d][4 * q + i] * inv;
            store4<T>(op + e, y);
            if (lp) {
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] -= to_f(from_f<T>(y[i]));
                store4<T>(lp + e, y);
            }
        }
}

// Joins the parts that fwd_k left, in their order: 16 lanes a row.  Bound by
// reading them: 4 parts of 16000 rows of 96, 25 MB, in 7 us.
template <typename T>
__global__ __launch_bounds__(NT) void join_k(StreamArgs g) {
    const int64_t n = (int64_t)g.B * g.H * g.J, zr = ((int64_t)blockIdx.x * NT + threadIdx.x) >> 4;
    const int gl = threadIdx.x & 15;
    if (zr >= n) return;
    const int j = (int)(zr % g.J), h = (int)(zr / g.J % g.H), b = (int)(zr / g.J / g.H);
    float m = -INFINITY;
    for (int s = 0; s < g.splits; ++s) m = fmaxf(m, g.part_ml[s * n + zr].x);
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    for (int s = 0; s < g.splits; ++s) {
        const float2 p = g.part_ml[s * n + zr];
        l += p.y * __builtin_amdgcn_exp2f(p.x - ms);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    if (g.lse && gl == 0) g.lse[zr] = l > 0.f ? m + __builtin_amdgcn_logf(l) : INFINITY;
    T* op = reinterpret_cast<T*>(g.o.ptr) + b * g.o.sb + h * g.o.sh + j * g.o.st;
    T* lp = g.lo ? reinterpret_cast<T*>(g.lo) + (((int64_t)b * g.J + j) * g.H + h) * g.P : nullptr;
    for (int e = 8 * gl; e < g.P; e += 128) {
        float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < g.splits; ++s) {
            const float w = __builtin_amdgcn_exp2f(g.part_ml[s * n + zr].x - ms) * inv;
            float x[8];
            V8<float>::load(g.part_o + (s * n + zr) * g.P + e, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(w, x[i], y[i]);
        }
        V8<T>::store(op + e, y);
        if (lp) {
            float lo[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) lo[i] = y[i] - to_f(from_f<T>(y[i]));
            V8<T>::store(lp + e, lo);
        }
    }
}

// ------------------------------------------------------------ backward
// Row terms D = dout . out, out as the forward had it before rounding (its
// stored value and the saved rest): LPR lanes a row, 8 elements each, four
// rows of a lane group requested together.  fp16 also: the largest |dout| of
// every 256 rows of a head, and the largest |v| of vmax_rows keys of a
// key/value head (blocks behind the rows'), from which the score gradients get
// a power of two that keeps them inside the type (Gain).
// Bound by reading three tensors: 262144 rows of 64 in bf16, 101 MB, in 20 us.
__device__ __forceinline__ void block_max(float top, float* to) {
    __shared__ float w[NT / 64];
    top = group_max<64>(top);
    if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) *to = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
}
template <typename T, int LPR>
__global__ __launch_bounds__(NT) void rows_k(StreamArgs g) {
    constexpr int RPB = NT / LPR, U = 4;
    const int gl = threadIdx.x % LPR, e = min(8 * gl, g.P - 8);
    const int nch = (g.J + STREAM_DROWS - 1) / STREAM_DROWS, nrows = nch * g.B * g.H;
    float top = 0.f;
    if (__is_same(T, half_t) && (int)blockIdx.x >= nrows) {
        const int i = (int)blockIdx.x - nrows, z = i / g.vmax_n, k0 = (i - z * g.vmax_n) * g.vmax_rows;
        const int b = z / g.G, end = min(k0 + g.vmax_rows, Seq(g, b).k_len);
        const T* vp = reinterpret_cast<const T*>(g.v.ptr) + b * g.v.sb + (z - b * g.G) * g.v.sh + e;
        for (int r0 = k0; r0 < end; r0 += RPB * U) {
            float x[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) V8<T>::load(vp + (int64_t)min(r0 + u * RPB + (int)threadIdx.x / LPR, end - 1) * g.v.st, x[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int key = min(r0 + u * RPB + (int)threadIdx.x / LPR, end - 1);
                if (g.doc && g.doc[(int64_t)b * g.K + key] < 0) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[u][j]));
            }
        }
        block_max(top, g.vmax + i);
        return;
    }
    const int z = (int)blockIdx.x / nch, ch = (int)blockIdx.x - z * nch, b = z / g.H, h = z - b * g.H;
    const Seq s(g, b);
    const T* dp = reinterpret_cast<const T*>(g.dout.ptr) + b * g.dout.sb + h * g.dout.sh + e;
    const T* op = reinterpret_cast<const T*>(g.o.ptr) + b * g.o.sb + h * g.o.sh + e;
    const T* lp = reinterpret_cast<const T*>(g.lo) + ((int64_t)b * g.J * g.H + h) * g.P + e;
    for (int r0 = 0; r0 < STREAM_DROWS; r0 += RPB * U) {
        float a[U][8], y[U][8], lo[U][8];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = ch * STREAM_DROWS + r0 + u * RPB + threadIdx.x / LPR, j = min(row, g.J - 1);
            in[u] = row < s.q_len && 8 * gl < g.P && !(g.doc && s.doc_of(g, b, j) < 0);
            V8<T>::load(dp + (int64_t)j * g.dout.st, a[u]);
            V8<T>::load(op + (int64_t)j * g.o.st, y[u]);
            if constexpr (sizeof(T) == 2) V8<T>::load(lp + (int64_t)j * g.H * g.P, lo[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = ch * STREAM_DROWS + r0 + u * RPB + threadIdx.x / LPR;
            float d = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d = fmaf(a[u][i], sizeof(T) == 2 ? y[u][i] + lo[u][i] : y[u][i], d);
                if (in[u]) top = fmaxf(top, fabsf(a[u][i]));
            }
            d = group_sum<LPR>(in[u] ? d : 0.f);
            if (gl == 0 && row < g.J) g.dsum[(int64_t)z * g.J + row] = d;
        }
    }
    if (g.dmax) block_max(top, g.dmax + (int64_t)z * g.dmax_n + ch);
}

// fp16: probabilities are held as 2^10 p; score gradients as 2^e ds with
// 2^e = 2^14 over the powers of two below max |dout| (of the heads of a
// key/value head) and P max |v|.  ds = p (dout . v - D) is at most P max |dout|
// max |v| / 2 (p (1 - p) is at most 1/4, and dout . v differs between keys by
// up to 2 P |dout| |v|), so what is held stays below 2^15, the type's numbers
// end at 2^16, and it keeps all its bits down to 2^-29 of that bound.
struct Gain {
    float p2;   // added to the exponents of the probabilities
    float pinv; // 1 / 2^p2
    float ds, dsinv;  // (dout . v - D) times ds; 1 / (ds 2^p2)
};
template <typename T>
__device__ __forceinline__ Gain gain(const StreamArgs& g, int b, int kvh) {
    if constexpr (!__is_same(T, half_t)) return Gain{0.f, 1.f, 1.f, 1.f};
    const int n = g.H / g.G * g.dmax_n;
    const float* p = g.dmax + ((int64_t)b * g.H + kvh * (g.H / g.G)) * g.dmax_n;
    float top = 0.f;
    for (int i = threadIdx.x & 63; i < n; i += 64) top = fmaxf(top, p[i]);
    const float* pv = g.vmax + ((int64_t)b * g.G + kvh) * g.vmax_n;
    float v = 0.f;
    for (int i = threadIdx.x & 63; i < g.vmax_n; i += 64) v = fmaxf(v, pv[i]);
    top = group_max<64>(top);
    v = group_max<64>(v) * (float)g.P;
    const bool known = top > 0.f && top < INFINITY && v > 0.f && v < INFINITY;  // (else all gradients of scores are zeros)
    const int e = known ? 14 - ilogbf(top) - ilogbf(v) : 0;
    return Gain{10.f, 1.f / 1024.f, ldexpf(1.f, e - 10), ldexpf(1.f, -e)};
}
// p (dout . v - D), scaled
template <typename T> __device__ __forceinline__ float score_grad(float p, float dpd, const Gain& gn) {
    if constexpr (__is_same(T, half_t)) return p * dpd * gn.ds;
    return p * dpd;
}

// dK and dV of 128 keys (32 a wave) of one key/value head: walks the query
// rows of its query heads (of a part of them where the heads are split),
// 64 a step.
// QH = 1: 4 waves, each with its keys' K and V in registers.
// QH = 2, head sizes above 64: there the sums' registers alone leave one wave
// a SIMD, which waits for LDS half of its time; so 8 waves, of which two
// share 32 keys and take half a step's rows each, K and V in LDS, and the
// pairs' sums meet at the end.
// Four products of the formula's five are here.  Bound by the registers: dK,
// dV and the operands allow two waves a SIMD, whose exponentials, conversions
// and LDS reads hide half of the products.  8192 causal tokens, capped, 16
// heads of 128 over 4 key/value heads: 685 us, 0.80 PFLOP/s, in a row of steps;
// alone on an idle card 785 (QH = 1: 975).
template <typename T, int DP, int QH> struct DkvTiles {
    static constexpr int BQ = 64, TB = BQ * Tile<T, DP>::PITCH;
    static constexpr int KT = QH == 2 ? STREAM_KEYS * Tile<T, DP>::PITCH : 0;  // of K, and of V
    // tiles of q and dout, and the rows' numbers: -lse, -D, bounds, documents
    static constexpr int STEP = 2 * TB + BQ * 16;
    static constexpr int LDS = 2 * KT + 2 * STEP;  // one step's tiles are filled while the other's are read
    static_assert(LDS <= 160 * 1024, "LDS of a CU");
};
template <typename T, int DP, bool CAP, bool BIAS, int QH>
__device__ __forceinline__ void dkv_block(const StreamArgs& g, int block, char* lds) {
    constexpr int BQ = 64, ND = DP / 32, NC = DP / 16, LANES = NT * QH;
    constexpr bool FRAGS = sizeof(T) == 2 && QH == 1;
    using TL = Tile<T, DP>;
    using Tiles = DkvTiles<T, DP, QH>;
    constexpr int TB = Tiles::TB, STEP = Tiles::STEP;
    int tile, z;
    place(block, g.B * g.G * g.hparts, tile, z);
    const int part = z % g.hparts;
    z /= g.hparts;
    const int b = z / g.G, kvh = z - b * g.G, grp = g.H / g.G, k0 = tile * STREAM_KEYS;
    const int tid = threadIdx.x, lane = tid & 63, c32 = lane & 31, hh = lane >> 5;
    const int w8 = __builtin_amdgcn_readfirstlane(tid >> 6), wave = QH == 2 ? w8 & 3 : w8, qh = QH == 2 ? w8 >> 2 : 0;
    const Seq sq(g, b);
    const int32_t* docs = g.doc ? g.doc + (int64_t)b * g.K : nullptr;
    const int key = k0 + 32 * wave + c32;
    const int kd = docs ? (key < sq.k_len ? docs[key] : -1) : 0;
    const bool kin = key < sq.k_len && kd >= 0;
    const Scorer<T, CAP, BIAS> sc(g);
    const Gain gn = gain<T>(g, b, kvh);

    const T* kp = reinterpret_cast<const T*>(g.k.ptr) + b * g.k.sb + kvh * g.k.sh;
    const T* vp = reinterpret_cast<const T*>(g.v.ptr) + b * g.v.sb + kvh * g.v.sh;
    Frag<T> kr_[QH == 1 ? NC : 1], vr_[QH == 1 ? NC : 1];
    if constexpr (QH == 1) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e = 16 * c + 8 * hh;
            kr_[c] = kin && e < g.P ? frag_load<T>(kp + (int64_t)key * g.k.st + e) : frag_zero<T>();
            vr_[c] = kin && e < g.P ? frag_load<T>(vp + (int64_t)key * g.v.st + e) : frag_zero<T>();
        }
    } else {
        Copies<T, DP, STREAM_KEYS, LANES> c;
        auto in = [&](int r) { return k0 + r < sq.k_len && docs[k0 + r] >= 0; };
        c.init(tid, g.P, g.k.st);
        c.issue(tid, reinterpret_cast<const char*>(kp + (int64_t)k0 * g.k.st), sq.k_len - k0, lds_offset(lds), !docs, in);
        c.init(tid, g.P, g.v.st);
        c.issue(tid, reinterpret_cast<const char*>(vp + (int64_t)k0 * g.v.st), sq.k_len - k0, lds_offset(lds) + Tiles::KT,
                !docs, in);
    }
    auto kf = [&](int c) {
        if constexpr (QH == 1) return kr_[c];
        else return TL::row(lds, 32 * wave + c32, 16 * c + 8 * hh);
    };
    auto vf = [&](int c) {
        if constexpr (QH == 1) return vr_[c];
        else return TL::row(lds + Tiles::KT, 32 * wave + c32, 16 * c + 8 * hh);
    };
    char* const steps = lds + 2 * Tiles::KT;
    floatx16 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;

    // query steps that may see one of these keys: rows from the first whose
    // position reaches them, all where the prefix does
    const int first = g.causal && sq.prefix <= k0 ? max(0, k0 - sq.off) / BQ : 0;
    const int nst = k0 < sq.k_len ? (sq.q_len + BQ - 1) / BQ : 0;
    const int nr = (g.K + STREAM_RANGE - 1) / STREAM_RANGE;
    int2 kr{0, 0};
    int onedoc = -1;  // the document of all the wave's keys, if one
    if (docs) {
        kr = int2{INT32_MAX, -1};
#pragma unroll
        for (int i = 0; i < STREAM_KEYS / STREAM_RANGE; ++i) {
            const int e = k0 / STREAM_RANGE + i;
            if (e < nr) {
                const int4 r = g.ranges[(int64_t)b * nr + e];
                kr = int2{min(kr.x, r.x), max(kr.y, r.y)};
                if (i == 32 * wave / STREAM_RANGE && r.x == r.y && r.z == 0) onedoc = r.x;
            }
        }
    }
    // the step's rows lie in at most two entries
    auto entry = [&](int step, int i) {
        const int p = sq.off + step * BQ + i * (BQ - 1), e = max(p, 0) / STREAM_RANGE;
        return p >= 0 && e < nr ? g.ranges[(int64_t)b * nr + e] : int4{INT32_MAX, -1, 1, 0};
    };
    Window win{-64, 0, 0, 0};
    auto next = [&](int from) {
        if (!docs) return from;
        while (from < nst) {
            if (from < win.base || from >= win.base + 64) {
                const int4 r0 = entry(from + lane, 0), r1 = entry(from + lane, 1);
                win = Window{from, __ballot(from + lane < nst && (ranges_meet(r0, kr) || ranges_meet(r1, kr))),
                             __ballot(r0.z != 0 || r1.z != 0),
                             __ballot(onedoc >= 0 && range_is(r0, onedoc) && range_is(r1, onedoc))};
            }
            const uint64_t m = win.meet >> (from - win.base);
            if (m) return from + (int)__builtin_ctzll(m);
            from = win.base + 64;
        }
        return nst;
    };

    Copies<T, DP, BQ, LANES> cq, cd;
    cq.init(tid, g.P, g.q.st);
    cd.init(tid, g.P, g.dout.st);
    const uint32_t base = lds_offset(steps);
    auto rows_of = [&](int buf) { return reinterpret_cast<float*>(steps + buf * STEP + 2 * TB); };
    const int h_end = min(grp, (part + 1) * ((grp + g.hparts - 1) / g.hparts));
    for (int hg = part * ((grp + g.hparts - 1) / g.hparts); hg < h_end; ++hg) {
        const int h = kvh * grp + hg;
        const float slope2 = g.slopes ? g.slopes[h] * LOG2E : 0.f;
        const T* qp = reinterpret_cast<const T*>(g.q.ptr) + b * g.q.sb + h * g.q.sh;
        const T* dp = reinterpret_cast<const T*>(g.dout.ptr) + b * g.dout.sb + h * g.dout.sh;
        const int64_t zr = ((int64_t)b * g.H + h) * g.J;
        float f_lse = 0.f, f_d = 0.f;  // the step on its way: its rows' numbers, in LDS once its turn is near
        int f_hi = 0, f_doc = 0;
        auto put = [&](int buf) {
            if (tid < BQ) {
                float* r = rows_of(buf) + tid;
                r[0] = gn.p2 + sc.offset - f_lse;  // in the score's units without its offset
                r[BQ] = -f_d;
                reinterpret_cast<int*>(r)[2 * BQ] = f_hi;
                reinterpret_cast<int*>(r)[3 * BQ] = f_doc;
            }
        };
        auto fetch = [&](int step, int buf) {
            const int j0 = step * BQ;
            const bool all = !docs || !win.is(win.holes, step);
            auto in = [&](int r) { return sq.doc_of(g, b, j0 + r) >= 0; };
            if (tid < BQ) {
                const int j = j0 + tid;
                const bool row = j < sq.q_len;
                f_lse = row ? g.lse[zr + j] : INFINITY;
                f_d = row ? g.dsum[zr + j] : 0.f;
                f_hi = sq.hi(g, j);
                f_doc = docs ? sq.doc_of(g, b, j) : 0;
            }
            const uint32_t to = base + (uint32_t)(buf * STEP);
            cq.issue(tid, reinterpret_cast<const char*>(qp + (int64_t)j0 * g.q.st), sq.q_len - j0, to, all, in);
            cd.issue(tid, reinterpret_cast<const char*>(dp + (int64_t)j0 * g.dout.st), sq.q_len - j0, to + TB, all, in);
        };
        int s = next(first);
        __syncthreads();  // (the last head's last step has been read)
        if (s < nst) {
            fetch(s, 0);
            put(0);
        }
        for (int buf = 0; s < nst; buf ^= 1) {
            copied();
            __syncthreads();
            const int j0 = s * BQ;
            // (rows behind the last query have zeros and no probabilities)
            const bool some = k0 + 32 * wave + 32 > sq.hi(g, j0) || (docs && !win.is(win.whole, s));
            const char *tq = steps + buf * STEP, *td = tq + TB;
            const float* rows = rows_of(buf);
            s = next(s + 1);
            if (s < nst) fetch(s, buf ^ 1);
#pragma unroll
            for (int n0 = 0; n0 < BQ / 32; n0 += QH) {
                const int n = QH == 2 ? qh : n0;
                floatx16 x, dpd;
                float nl[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const floatx4 a = *reinterpret_cast<const floatx4*>(rows + 32 * n + 8 * q + 4 * hh);
                    const floatx4 d = *reinterpret_cast<const floatx4*>(rows + BQ + 32 * n + 8 * q + 4 * hh);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[4 * q + i] = 0.f;
                        nl[4 * q + i] = a[i];
                        dpd[4 * q + i] = d[i];  // dout . v - D
                    }
                }
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    x = mma<T>(TL::row(tq, 32 * n + c32, 16 * c + 8 * hh), kf(c), x);
                    dpd = mma<T>(TL::row(td, 32 * n + c32, 16 * c + 8 * hh), vf(c), dpd);
                }
                // (the second products' fragments are asked for ahead of the
                // exponentials, which hide the reads)
                Frag<T> df[2][ND], qf[2][ND];
                if constexpr (FRAGS) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            df[c][d] = TL::col(td, 32 * n + 16 * c, 32 * d, lane);
                            qf[c][d] = TL::col(tq, 32 * n + 16 * c, 32 * d, lane);
                        }
                    __builtin_amdgcn_sched_barrier(0x41f);
                }
                float p[16], ds[16];
                const float far = BIAS ? (float)(sq.off + j0 + 32 * n + 4 * hh - key) : 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v = sc.value(x[i]);
                    float e = fmaf(v, sc.scale, nl[i]);
                    if constexpr (BIAS) e = fmaf(-slope2, fabsf(far + (float)(8 * (i >> 2) + (i & 3))), e);
                    p[i] = __builtin_amdgcn_exp2f(e);
                    ds[i] = CAP ? dpd[i] * sc.slope(v) : dpd[i];
                }
                if (some) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int* r = reinterpret_cast<const int*>(rows) + 2 * BQ + 32 * n + 8 * q + 4 * hh;
                        const int4 rh = *reinterpret_cast<const int4*>(r);
                        const int4 rd = *reinterpret_cast<const int4*>(r + BQ);
                        const int hi4[4] = {rh.x, rh.y, rh.z, rh.w}, id4[4] = {rd.x, rd.y, rd.z, rd.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if ((key >= hi4[i]) | (id4[i] != kd) | !kin) p[4 * q + i] = 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] = score_grad<T>(p[i], ds[i], gn);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const Frag<T> pf = frag_acc<T>(p + 8 * c), sf = frag_acc<T>(ds + 8 * c);
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        dv[d] = mma<T>(FRAGS ? df[c][d] : TL::col(td, 32 * n + 16 * c, 32 * d, lane), pf, dv[d]);
                        dk[d] = mma<T>(FRAGS ? qf[c][d] : TL::col(tq, 32 * n + 16 * c, 32 * d, lane), sf, dk[d]);
                    }
                }
            }
            put(buf ^ 1);
        }
    }
    if constexpr (QH == 2) {
        copied();  // (K and V, where no step waited for them)
        __syncthreads();
        float* sum = reinterpret_cast<float*>(lds) + (wave * 32 * ND) * 64 + lane;
        if (qh == 1) {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sum[(32 * d + i) * 64] = dk[d][i];
                    sum[(32 * d + 16 + i) * 64] = dv[d][i];
                }
        }
        __syncthreads();
        if (qh == 1) return;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                dk[d][i] += sum[(32 * d + i) * 64];
                dv[d][i] += sum[(32 * d + 16 + i) * 64];
            }
    }
    if (key >= g.K) return;
    const float fk = g.scaler * sc.SLOPE * gn.dsinv;
    T* dkp = reinterpret_cast<T*>(g.dk.ptr) + b * g.dk.sb + kvh * g.dk.sh + (int64_t)key * g.dk.st;
    T* dvp = reinterpret_cast<T*>(g.dv.ptr) + b * g.dv.sb + kvh * g.dv.sh + (int64_t)key * g.dv.st;
    float* pk = g.part_k + ((((int64_t)part * g.B + b) * g.G + kvh) * g.K + key) * 2 * g.P;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = 32 * d + 8 * q + 4 * hh;
            if (e >= g.P) continue;
            float y[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = dk[d][4 * q + i] * fk;
                w[i] = dv[d][4 * q + i] * gn.pinv;
            }
            if (g.hparts > 1) {
                store4<float>(pk + e, y);
                store4<float>(pk + g.P + e, w);
            } else {
                store4<T>(dkp + e, y);
                store4<T>(dvp + e, w);
            }
        }
}

// Sums of the head parts' dK and dV, in their order: 8 elements a thread.
// Bound by reading them: 4 parts of 32768 rows of 128, 134 MB, in 24 us.
template <typename T>
__global__ __launch_bounds__(NT) void dkv_join_k(StreamArgs g) {
    const int np = 2 * g.P / 8;
    const int64_t rows = (int64_t)g.B * g.G * g.K, at = (int64_t)blockIdx.x * NT + threadIdx.x, row = at / np;
    if (row >= rows) return;
    const int e = (int)(at - row * np) * 8;
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < g.hparts; ++s) {
        float x[8];
        V8<float>::load(g.part_k + (s * rows + row) * 2 * g.P + e, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += x[i];
    }
    const int key = (int)(row % g.K), kvh = (int)(row / g.K % g.G), b = (int)(row / g.K / g.G);
    const StreamRows& to = e < g.P ? g.dk : g.dv;
    V8<T>::store(reinterpret_cast<T*>(to.ptr) + b * to.sb + kvh * to.sh + (int64_t)key * to.st + (e < g.P ? e : e - g.P), y);
}

// dQ of 128 query rows (32 a wave) of one head: walks their keys as the
// forward does.  Three products, of which two form the probabilities' and
// their gradients' sums again: that is the price of writing no J x K tensor
// and adding nothing atomically.  8192 causal tokens, capped, 16 heads of
// 128: 522 us, 0.79 PFLOP/s, in a row of steps.
template <typename T, int DP> struct DqTiles {
    static constexpr int BN = 64, TB = BN * Tile<T, DP>::PITCH;
    static constexpr int LDS = 4 * TB + 2 * BN * 4 + 4 * 8;  // two pairs of tiles, documents of the keys, of the waves' rows
    static_assert(LDS <= 160 * 1024, "LDS of a CU");
};
template <typename T, int DP, bool CAP, bool BIAS>
__device__ __forceinline__ void dq_block(const StreamArgs& g, int block, char* lds) {
    constexpr int BM = 128, BN = 64, NS = 2, ND = DP / 32, NC = DP / 16;
    using TL = Tile<T, DP>;
    using Tiles = DqTiles<T, DP>;
    constexpr int TB = Tiles::TB;
    int* kdoc = reinterpret_cast<int*>(lds + 4 * TB);
    int2* wrange = reinterpret_cast<int2*>(kdoc + 2 * BN);
    const int nqt = (g.J + BM - 1) / BM;
    int tile, z;
    place(block, g.B * g.H, tile, z);
    if (g.causal) tile = nqt - 1 - tile;
    const int b = z / g.H, h = z - b * g.H, kvh = h / (g.H / g.G);
    const int tid = threadIdx.x, lane = tid & 63, c32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Seq sq(g, b);
    const int j0 = tile * BM, j = j0 + 32 * wave + c32, pos = sq.off + j;
    const int32_t* docs = g.doc ? g.doc + (int64_t)b * g.K : nullptr;
    const int mydoc = docs ? sq.doc_of(g, b, j) : 0;
    const bool live = j < sq.q_len && mydoc >= 0;
    const int hi = live ? sq.hi(g, j) : 0;
    const float slope2 = g.slopes ? g.slopes[h] * LOG2E : 0.f;
    const Scorer<T, CAP, BIAS> sc(g);
    const Gain gn = gain<T>(g, b, kvh);
    const int64_t zr = ((int64_t)b * g.H + h) * g.J + j;
    const float nl = live ? gn.p2 + sc.offset - g.lse[zr] : -INFINITY, nd = live ? -g.dsum[zr] : 0.f;

    Frag<T> qf[NC], df[NC];
    {
        const T* qp = reinterpret_cast<const T*>(g.q.ptr) + b * g.q.sb + h * g.q.sh + (int64_t)j * g.q.st;
        const T* dp = reinterpret_cast<const T*>(g.dout.ptr) + b * g.dout.sb + h * g.dout.sh + (int64_t)j * g.dout.st;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e = 16 * c + 8 * hh;
            qf[c] = hi > 0 && e < g.P ? frag_load<T>(qp + e) : frag_zero<T>();
            df[c] = live && e < g.P ? frag_load<T>(dp + e) : frag_zero<T>();
        }
    }
    const int jlast = min(min(j0 + BM, g.J), sq.q_len) - 1, wj = j0 + 32 * wave;
    const int steps = j0 < sq.q_len ? (sq.hi(g, jlast) + BN - 1) / BN : 0;
    // (rows without a query have no probabilities)
    const int hi_low = wj < sq.q_len ? sq.hi(g, wj) : INT32_MAX;
    int2 qr{0, 0};
    int onedoc = -1;
    if (docs) {
        const int2 r = wave_range(mydoc);
        if (r.x == r.y && __ballot(mydoc < 0) == 0) onedoc = r.x;
        if (lane == 0) wrange[wave] = r;
        __syncthreads();
        qr = wrange[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) qr = int2{min(qr.x, wrange[w].x), max(qr.y, wrange[w].y)};
    }
    const int nr = (g.K + STREAM_RANGE - 1) / STREAM_RANGE;
    const int4* ranges = g.ranges + (int64_t)b * nr;
    Window win{-64, 0, 0, 0};
    auto next = [&](int from) {
        if (!docs) return from;
        while (from < steps) {
            if (from >= win.base + 64) {
                const int4 r = from + lane < steps ? ranges[from + lane] : int4{INT32_MAX, -1, 1, 0};
                win = Window{from, __ballot(ranges_meet(r, qr)), __ballot(r.z != 0),
                             __ballot(onedoc >= 0 && range_is(r, onedoc))};
            }
            const uint64_t m = win.meet >> (from - win.base);
            if (m) return from + (int)__builtin_ctzll(m);
            from = win.base + 64;
        }
        return steps;
    };
    const T* kp = reinterpret_cast<const T*>(g.k.ptr) + b * g.k.sb + kvh * g.k.sh;
    const T* vp = reinterpret_cast<const T*>(g.v.ptr) + b * g.v.sb + kvh * g.v.sh;
    Copies<T, DP, BN> ck, cv;
    ck.init(tid, g.P, g.k.st);
    cv.init(tid, g.P, g.v.st);
    const uint32_t base = lds_offset(lds);
    int fdoc = -1;
    auto put = [&](int buf) {
        if (docs && tid < BN) kdoc[buf * BN + tid] = fdoc;
    };
    auto fetch = [&](int step, int buf) {
        const int k0 = step * BN;
        if (docs && tid < BN) fdoc = k0 + tid < sq.k_len ? docs[k0 + tid] : -1;
        const bool all = !docs || !win.is(win.holes, step);
        auto in = [&](int r) { return k0 + r < sq.k_len && docs[k0 + r] >= 0; };
        const uint32_t to = base + (uint32_t)(buf * 2 * TB);
        ck.issue(tid, reinterpret_cast<const char*>(kp + (int64_t)k0 * g.k.st), sq.k_len - k0, to, all, in);
        cv.issue(tid, reinterpret_cast<const char*>(vp + (int64_t)k0 * g.v.st), sq.k_len - k0, to + TB, all, in);
    };
    floatx16 dq[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.f;

    int s = next(0);
    if (s < steps) {
        fetch(s, 0);
        put(0);
    }
    for (int buf = 0; s < steps; buf ^= 1) {
        copied();
        __syncthreads();
        const int k0 = s * BN;
        const char *tk = lds + buf * 2 * TB, *tv = tk + TB;
        const bool mixed = docs && !win.is(win.whole, s);
        s = next(s + 1);
        if (s < steps) fetch(s, buf ^ 1);
#pragma unroll 1
        for (int n = 0; n < NS; ++n) {
            floatx16 x, dpd;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = 0.f;
                dpd[i] = nd;  // dout . v - D
            }
            // (fragments asked for ahead of the first product, as the forward does)
            constexpr int AH = sizeof(T) == 2 ? (DP == 32 ? 4 : DP <= 96 ? 8 : 4) : 0;
            Frag<T> rf[AH ? AH : 1];
#pragma unroll
            for (int i = 0; i < AH; ++i) rf[i] = TL::row(i & 1 ? tv : tk, 32 * n + c32, 16 * (i / 2) + 8 * hh);
            if constexpr (AH > 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const bool got = 2 * c < AH;
                x = mma<T>(got ? rf[got ? 2 * c : 0] : TL::row(tk, 32 * n + c32, 16 * c + 8 * hh), qf[c], x);
                dpd = mma<T>(got ? rf[got ? 2 * c + 1 : 0] : TL::row(tv, 32 * n + c32, 16 * c + 8 * hh), df[c], dpd);
            }
            // (up to 64 the registers hold the second product's fragments too)
            constexpr bool COLS = sizeof(T) == 2 && DP <= 64;
            Frag<T> cf[2][COLS ? ND : 1];
            if constexpr (COLS) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int d = 0; d < ND; ++d) cf[c][d] = TL::col(tk, 32 * n + 16 * c, 32 * d, lane);
                __builtin_amdgcn_sched_barrier(0x41f);
            }
            // 16 keys at a time: the second 16's exponentials run beside the
            // first's products, and fewer values are held at once
            const float far = BIAS ? (float)(pos - k0 - 32 * n - 4 * hh) : 0.f;
            const int end = hi - k0 - 32 * n - 4 * hh;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float p[8], ds[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 16 * c + 8 * (i >> 2) + (i & 3);
                    const float v = sc.value(x[8 * c + i]);
                    float e = fmaf(v, sc.scale, nl);
                    if constexpr (BIAS) e = fmaf(-slope2, fabsf(far - (float)r), e);
                    p[i] = __builtin_amdgcn_exp2f(e);
                    ds[i] = CAP ? dpd[8 * c + i] * sc.slope(v) : dpd[8 * c + i];
                }
                if (mixed) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int4 kd = *reinterpret_cast<const int4*>(kdoc + buf * BN + 32 * n + 16 * c + 8 * q + 4 * hh);
                        const int id[4] = {kd.x, kd.y, kd.z, kd.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (id[i] != mydoc) p[4 * q + i] = 0.f;
                    }
                }
                if (k0 + BN > hi_low) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (16 * c + 8 * (i >> 2) + (i & 3) >= end) p[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) ds[i] = score_grad<T>(p[i], ds[i], gn);
                const Frag<T> sf = frag_acc<T>(ds);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    dq[d] = mma<T>(COLS ? cf[c][COLS ? d : 0] : TL::col(tk, 32 * n + 16 * c, 32 * d, lane), sf, dq[d]);
            }
        }
        put(buf ^ 1);
    }
    if (j >= g.J) return;
    T* dqp = reinterpret_cast<T*>(g.dq.ptr) + b * g.dq.sb + h * g.dq.sh + (int64_t)j * g.dq.st;
    const float f = g.scaler * sc.SLOPE * gn.dsinv;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = 32 * d + 8 * q + 4 * hh;
            if (e >= g.P) continue;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = dq[d][4 * q + i] * f;
            store4<T>(dqp + e, y);
        }
}

template <typename T, int DP, bool CAP, bool BIAS, int QH>
__global__ __launch_bounds__(NT * QH) void dkv_k(StreamArgs g) {
    __shared__ __attribute__((aligned(16))) char lds[DkvTiles<T, DP, QH>::LDS];
    static_assert(QH == 1 || DkvTiles<T, DP, QH>::LDS >= DP * 1024, "the pairs' sums");
    dkv_block<T, DP, CAP, BIAS, QH>(g, (int)blockIdx.x, lds);
}
template <typename T, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(NT, sizeof(T) == 2 ? 2 : 1) void dq_k(StreamArgs g) {
    __shared__ __attribute__((aligned(16))) char lds[DqTiles<T, DP>::LDS];
    dq_block<T, DP, CAP, BIAS>(g, (int)blockIdx.x, lds);
}
// Both in one launch, so that the end of the one fills with the other:
// blocks 0 .. nk - 1 (the longer ones) do keys, the others rows.  4 x 4096
// tokens in documents of about 700, 16 heads of 64: 333 us, 0.54 PFLOP/s of
// the seven products; 3 x 1531 causal tokens with distances in fp16, 12 heads
// of 64: 70 to 75.
template <typename T, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(NT, DP <= 64 && sizeof(T) == 2 ? 2 : 1) void dkv_dq_k(StreamArgs g, int nk) {
    constexpr int A = DkvTiles<T, DP, 1>::LDS, B = DqTiles<T, DP>::LDS;
    __shared__ __attribute__((aligned(16))) char lds[A > B ? A : B];
    if ((int)blockIdx.x < nk) dkv_block<T, DP, CAP, BIAS, 1>(g, (int)blockIdx.x, lds);
    else dq_block<T, DP, CAP, BIAS>(g, (int)blockIdx.x - nk, lds);
}

// ------------------------------------------------------------- launches
template <typename T, int DP, bool CAP, bool BIAS> void launch_fwd(const StreamArgs& a, bool few, hipStream_t st) {
    const int64_t rows = (int64_t)a.J * a.pack, nz = (int64_t)a.B * (a.H / a.pack) * a.splits;
    if (few)
        fwd_k<T, DP, CAP, BIAS, 1, 1><<<dim3((unsigned)((rows + 31) / 32 * nz)), NT, 0, st>>>(a);
    else
        fwd_k<T, DP, CAP, BIAS, 4, 2><<<dim3((unsigned)((rows + STREAM_BM - 1) / STREAM_BM * nz)), NT, 0, st>>>(a);
}

template <typename T, int DP, bool CAP, bool BIAS> void launch_bwd(const StreamArgs& a, hipStream_t st) {
    const int64_t nk = (int64_t)((a.K + STREAM_KEYS - 1) / STREAM_KEYS) * a.B * a.G;
    const int64_t nq = (int64_t)((a.J + 127) / 128) * a.B * a.H;
    const int64_t nkb = nk * a.hparts;
    if (!stream_apart(DP, nkb + nq)) {
        dkv_dq_k<T, DP, CAP, BIAS><<<dim3((unsigned)(nkb + nq)), NT, 0, st>>>(a, (int)nkb);
    } else if constexpr (DP > 64) {
        constexpr int QH = sizeof(T) == 2 ? 2 : 1;  // (two tiles of float32 keys and rows do not fit LDS together)
        if (nkb > 0) dkv_k<T, DP, CAP, BIAS, QH><<<dim3((unsigned)nkb), NT * QH, 0, st>>>(a);
        if (nq > 0) dq_k<T, DP, CAP, BIAS><<<dim3((unsigned)nq), NT, 0, st>>>(a);
    }
    if (a.hparts > 1) {
        const int64_t n = (int64_t)a.B * a.G * a.K * (2 * a.P / 8);
        dkv_join_k<T><<<dim3((unsigned)((n + NT - 1) / NT)), NT, 0, st>>>(a);
    }
}

// fn(head size, capped, biased) as compile-time values
template <typename Fn> void pick(const StreamArgs& a, Fn fn) {
    auto bias = [&](auto dp, auto cap) {
        if (a.slopes) fn(dp, cap, std::true_type{});
        else fn(dp, cap, std::false_type{});
    };
    auto cap = [&](auto dp) {
        if (a.cap > 0.f) bias(dp, std::true_type{});
        else bias(dp, std::false_type{});
    };
    const int dp = stream_head_pad(a.P);
    if (dp == 32) cap(std::integral_constant<int, 32>{});
    else if (dp == 64) cap(std::integral_constant<int, 64>{});
    else if (dp == 96) cap(std::integral_constant<int, 96>{});
    else cap(std::integral_constant<int, 128>{});
}

}  // namespace stream

// (a launch without blocks is an error: what has no rows or keys is left out)
inline int64_t stream_ranges_n(const StreamArgs& a) {
    return (int64_t)((a.K + STREAM_RANGE - 1) / STREAM_RANGE) * a.B;
}

template <typename T> void stream_fwd(const StreamArgs& a, bool few, hipStream_t st) {
    if (a.doc && a.K > 0) stream::ranges_k<T><<<dim3((unsigned)stream_ranges_n(a)), 64, 0, st>>>(a);
    stream::pick(a, [&](auto dp, auto cap, auto bias) {
        stream::launch_fwd<T, decltype(dp)::value, decltype(cap)::value, decltype(bias)::value>(a, few, st);
    });
    if (a.splits > 1) {
        const int64_t lanes = (int64_t)a.B * a.H * a.J * 16;
        stream::join_k<T><<<dim3((unsigned)((lanes + stream::NT - 1) / stream::NT)), stream::NT, 0, st>>>(a);
    }
}

template <typename T> void stream_bwd(const StreamArgs& a, hipStream_t st) {
    if (a.doc && a.K > 0) stream::ranges_k<T><<<dim3((unsigned)stream_ranges_n(a)), 64, 0, st>>>(a);
    if (a.J > 0) {
        int64_t n = (int64_t)((a.J + STREAM_DROWS - 1) / STREAM_DROWS) * a.B * a.H;
        if constexpr (__is_same(T, half_t)) n += (int64_t)a.vmax_n * a.B * a.G;
        if (a.P <= 32) stream::rows_k<T, 4><<<dim3((unsigned)n), stream::NT, 0, st>>>(a);
        else if (a.P <= 64) stream::rows_k<T, 8><<<dim3((unsigned)n), stream::NT, 0, st>>>(a);
        else stream::rows_k<T, 16><<<dim3((unsigned)n), stream::NT, 0, st>>>(a);
    }
    stream::pick(a, [&](auto dp, auto cap, auto bias) {
        stream::launch_bwd<T, decltype(dp)::value, decltype(cap)::value, decltype(bias)::value>(a, st);
    });
}

}  // namespace dm

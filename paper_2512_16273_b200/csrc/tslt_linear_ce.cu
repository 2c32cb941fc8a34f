// Softmax cross entropy of a linear head over a large vocabulary, with its gradients (tslt_linear_ce,
// tslt_linear_ce_backward), without ever holding the logits [rows, V].
//
// Mathematics.  z = H W^T; lse_n = ln sum_v exp z[n, v]; loss_n = lse_n - z[n, t_n].  With g_n the weight of row n's loss,
// G[n, v] = g_n (exp(z[n, v] - lse_n) - [v = t_n]), dH = G W, dW = G^T H.
//
// Forward: the rows that count are gathered, and the target's logit is an fp32 dot product on the way.  One product whose
// epilogue turns each tile of z, still in tensor memory, into (max, sum) pairs, two a row; the pairs of all tiles (16 bytes
// for 256 logits) go to the workspace and a small kernel joins them.
// Backward, piece by piece of the vocabulary: z of the piece is computed again and its epilogue writes G of the piece in
// bf16 to the workspace (as 64-column panels, contiguous whichever of its axes a product reads along); one kernel with two
// products reads it: the piece's part of dH (summed over the pieces in fp32, in a fixed order) and dW of the piece (complete:
// its sum runs over the rows).  The target's entry of G comes from the gather's fp32 dot product again: where its probability is
// near 1 it is a small difference, which the tensor cores' sum of z would spoil (gradients off by 9 to 470 times what lse's
// own rounding leaves).  2 + 6 rows x V x D operations: z is computed twice, as rows x V logits are not kept between two calls.
//
// Bound by the tensor cores under the power cap (6144 rows, V = 128256, D = 4096, sustained: forward 4.9 ms, a piece of 16128
// entries z and G 655 us, dH and dW 1250 us; cuBLAS for the three products of a piece alone 627, 612 and 591 us).
//
// Rounding.  G is bf16: it is an operand of the tensor cores beside the bf16 weight and hidden rows, and two bf16 parts of it would double
// the two products that bound the call.  It costs about what the outputs' own rounding does (gradients off by 0.0018 to 0.0019 of
// their norm, 0.0017 from their rounding alone).  Powers are ex2.approx (2^-22 relative; 0 below 2^-126), a tile's sums
// of them fp32, their join fp64.  The sums of dH and dW are the tensor cores' fp32: n entries lose n 2^-30 of the sum in the mean
// (as z does below), 1.5e-5 for a piece of 16128 entries and 5e-4 for the longest (524288, up to 256 rows), below the
// bf16 outputs' 2^-8; pieces and cuts are added to nearest.
//
// Ignored rows (negative target) are taken out before anything is multiplied: the rows that count are copied together, in
// their order, and every product runs over those only.  Ignored rows cost nothing and what they hold (padding, NaN) is
// never looked at.
#include "tslt_gemm.cuh"

namespace tslt {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
constexpr int kStatsParts = 2;                         // (max, sum) pairs a row and tile: column halves of the epilogue
constexpr int kTileN = 256;                            // vocabulary entries (or hidden units) of a tile
constexpr long long kPieceBytes = 256ll << 20;         // most bytes of G held at a time

inline long long up(long long x, long long m) { return (x + m - 1) / m * m; }

// ---- workspace ---------------------------------------------------------------------------------------------
// [0, 256): status word, [128]: number of rows that count.  Then, each 256-byte aligned:
struct CeSpace {
    int* status;
    int* count;
    int* row_of;       // [rows_pad] source row of the i-th row that counts
    int* target;       // [rows_pad]
    float* top_weight; // the largest finite |g| of the rows that count, 1 if that is 0   (backward)
    float* lse2;       // [rows_pad] lse * log2(e)                        (backward)
    float* weight;     // [rows_pad] g / top_weight                       (backward)
    float* gtarget;    // [rows_pad] G at the target / top_weight         (backward)
    uint16_t* hidden;  // panels [ds / 64][rows_pad][64]: the rows that count, bf16; zeros up to the next multiple of 256 rows
    float2* part;      // [parts, rows_pad] (max, sum) in base 2          (forward)
    float* ztarget;    // [rows_pad]                                      (forward)
    uint16_t* g;       // panels [piece / 64][rows_pad][64]               (backward)
    float* acc;        // [splits][da / 4][rows_pad][4]                   (backward)
    long long rows_pad, ds, da, tiles, piece;
    int pieces, splits, pair, nt;  // nt: columns of a tile of z (forward)
    int direct;                    // one piece and one cut: dH leaves its product as it is wanted
    size_t bytes;
};

static CeSpace ce_space(void* ws, int rows, int V, int D, bool backward) {
    CeSpace s = {};
    s.rows_pad = up(rows, 256);
    s.ds = up(D, 64);
    s.da = up(D, 4);
    s.pair = rows > 128;
    const long long vt = up(V, kTileN);
    s.nt = gemm::choose_nt((rows + (s.pair ? 255 : 127)) / (s.pair ? 256 : 128), V, s.pair != 0, 32);
    s.tiles = (V + s.nt - 1) / s.nt;
    long long c = kPieceBytes / 2 / s.rows_pad / kTileN * kTileN;
    if (c < kTileN) c = kTileN;
    s.pieces = (int)((vt + c - 1) / c);
    s.piece = up((vt + s.pieces - 1) / s.pieces, kTileN);
    s.pieces = (int)((vt + s.piece - 1) / s.piece);
    // dH's tiles come first on their clusters and dW's fill up behind them (one kernel), so a tile of dH may be as long as a
    // cluster's whole share of both: cut its sum over the piece where it is longer (few rows: few tiles, a long sum).
    // Sums in stages; a tile of dW costs its epilogue, ten stages, where its own sum is shorter.
    const long long tile_rows = s.pair ? 256 : 128, slots = s.pair ? 74 : 148, cols = up(D, kTileN) / kTileN;
    const long long k1 = s.piece / 64, k2 = s.rows_pad / 64 < 10 ? 10 : s.rows_pad / 64;
    const long long tiles1 = up(rows, tile_rows) / tile_rows * cols, share = (tiles1 * k1 + up(s.piece, tile_rows) / tile_rows * cols * k2) / slots;
    const long long most1 = s.pair ? share : share / 4;  // few rows: four tiles of dH to a share, their sums are small (77 rows: 101 us, one: 118)
    s.splits = (int)(most1 < 1 ? k1 : (k1 + most1 - 1) / most1);
    if (s.splits > k1 / 8) s.splits = (int)(k1 / 8);  // eight stages a cut at least
    if (s.splits < 1) s.splits = 1;
    s.direct = s.pieces == 1 && s.splits == 1;
    uint8_t* p = (uint8_t*)ws;
    size_t at = kWsHeaderBytes;
    auto take = [&](size_t n) {
        uint8_t* r = p + at;
        at += align_up256(n);
        return r;
    };
    s.status = (int*)p;
    s.count = (int*)(p + 128);
    s.top_weight = (float*)(p + 132);
    s.row_of = (int*)take(s.rows_pad * 4);
    s.target = (int*)take(s.rows_pad * 4);
    s.hidden = (uint16_t*)take(s.rows_pad * s.ds * 2);
    if (backward) {
        s.lse2 = (float*)take(s.rows_pad * 4);
        s.weight = (float*)take(s.rows_pad * 4);
        s.gtarget = (float*)take(s.rows_pad * 4);
        s.g = (uint16_t*)take(s.rows_pad * s.piece * 2);
        if (!s.direct) s.acc = (float*)take((size_t)s.splits * s.rows_pad * s.da * 4);
    } else {
        s.part = (float2*)take(s.tiles * kStatsParts * s.rows_pad * 8);
        s.ztarget = (float*)take(s.rows_pad * 4);
    }
    s.bytes = at;
    return s;
}

// ---- gathering the rows that count --------------------------------------------------------------------------
struct GatherParams {
    const uint16_t *hidden, *weight;
    const int* target;
    long long h_stride, w_stride;
    int rows, V, D, per;
    const float *lse_in, *weight_in;  // backward (weight_in may be null: 1)
    float *loss, *lse;                // forward: zeroed for ignored rows
    uint16_t* dhidden;                // backward: zeroed for ignored rows
    long long dh_stride;
    CeSpace s;
};
constexpr int kGatherThreads = 256;

__device__ __forceinline__ bool counts(int t, int V) { return t >= 0 && t < V; }

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float acc) {
    float x[8], y[8];
    unpack_vec<bf16_t>(a, x);
    unpack_vec<bf16_t>(b, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = fmaf(x[i], y[i], acc);
    return acc;
}
// The vector of elements [8 i, 8 i + 8) of a row of D, zeros past its end.
__device__ __forceinline__ uint4 row_vec(const uint16_t* row, int i, int D) {
    if (8 * i + 8 <= D) return reinterpret_cast<const uint4*>(row)[i];
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = 8 * i + 2 * j;
        w[j] = (e < D ? (uint32_t)row[e] : 0u) | (e + 1 < D ? (uint32_t)row[e + 1] << 16 : 0u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One warp per row, 8 rows of a CTA at a time; CTA b takes `per` source rows from b * per on.  How many rows count before
// them (and in all) every CTA finds from the targets itself (few bytes next to the rows), so that none waits for another.
__global__ void __launch_bounds__(kGatherThreads) ce_gather_kernel(const __grid_constant__ GatherParams p) {
    __shared__ int s_before, s_all;
    __shared__ uint32_t s_top;
    wait_for_primary_kernel();
    allow_dependent_launch();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int first = min(p.rows, (int)blockIdx.x * p.per), last = min(p.rows, first + p.per);
    if (tid == 0) {
        s_before = s_all = 0;
        s_top = 0u;
    }
    // the loads of a warp's first row are in flight while the targets are counted (an ignored row's are thrown away)
    const int vecs = (int)(p.s.ds / 8), row1 = first + warp;
    const int t1 = row1 < last ? p.target[row1] : -1;
    uint4 v[4], u[4];
    auto load = [&](const uint16_t* h, const uint16_t* w, int i0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = row_vec(h, i0 + 32 * k, p.D);
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = row_vec(w, i0 + 32 * k, p.D);
    };
    if (counts(t1, p.V)) load(p.hidden + row1 * p.h_stride, p.weight + t1 * p.w_stride, lane);
    __syncthreads();
    int before = 0, all = 0, bad = 0;
    float top = 0.f;
#pragma unroll 8
    for (int i = tid; i < p.rows; i += kGatherThreads) {
        const int t = p.target[i];
        const int c = counts(t, p.V);
        bad |= t >= p.V;
        all += c;
        before += i < first ? c : 0;
        if (p.weight_in && c) {
            const float g = fabsf(p.weight_in[i]);
            if (g < INFINITY) top = fmaxf(top, g);  // a NaN or an infinity stays in its own row
        }
    }
    before = __reduce_add_sync(0xffffffffu, before);
    all = __reduce_add_sync(0xffffffffu, all);
    top = warp_max(top);
    bad = __syncthreads_or(bad);
    if (lane == 0) {
        atomicAdd(&s_before, before);
        atomicAdd(&s_all, all);
        atomicMax(&s_top, __float_as_uint(top));  // non-negative floats order as integers
    }
    __syncthreads();
    const float wtop = p.weight_in && s_top ? __uint_as_float(s_top) : 1.f;
    if (blockIdx.x == 0 && tid == 0) {
        *p.s.status = bad ? TSLT_STATUS_BAD_TARGET : 0;
        *p.s.count = s_all;
        *p.s.top_weight = wtop;
    }
    int at0 = s_before;
    for (int r0 = first; r0 < last; r0 += 32) {  // 32 rows: a ballot gives each its place
        const int mine = r0 + lane < last ? p.target[r0 + lane] : -1;
        const uint32_t on = __ballot_sync(0xffffffffu, counts(mine, p.V));
        for (int j = warp; j < 32 && r0 + j < last; j += kGatherThreads / 32) {
            const int row = r0 + j, t = __shfl_sync(0xffffffffu, mine, j);
            if (on >> j & 1) {
                const int at = at0 + __popc(on & ((1u << j) - 1u));
                const uint16_t *h = p.hidden + row * p.h_stride, *w = p.weight + t * p.w_stride;
                uint4* dst = reinterpret_cast<uint4*>(p.s.hidden) + (size_t)at * 8;
                float z = 0.f;
                for (int i0 = lane; i0 < vecs; i0 += 128) {  // eight loads in flight
                    if (row != row1 || i0 != lane) load(h, w, i0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int i = i0 + 32 * k;
                        z = dot8(v[k], u[k], z);
                        if (i < vecs) dst[(size_t)(i >> 3) * p.s.rows_pad * 8 + (i & 7)] = v[k];
                    }
                }
                z = warp_sum(z);
                if (lane == 0) {
                    p.s.row_of[at] = row;
                    p.s.target[at] = t;
                    if (p.loss) {
                        p.s.ztarget[at] = z;
                    } else {
                        p.s.lse2[at] = (float)((double)p.lse_in[row] * 1.4426950408889634);
                        const float g = p.weight_in ? __fdiv_rn(p.weight_in[row], wtop) : 1.f;
                        p.s.weight[at] = g;
                        p.s.gtarget[at] = g * expm1f(z - p.lse_in[row]);
                    }
                }
            } else if (p.loss) {
                if (lane == 0) p.loss[row] = p.lse[row] = 0.f;
            } else {
                uint16_t* o = p.dhidden + row * p.dh_stride;
                for (int i = lane; i < p.D / 8; i += 32) reinterpret_cast<uint4*>(o)[i] = make_uint4(0, 0, 0, 0);
                for (int i = p.D / 8 * 8 + lane; i < p.D; i += 32) o[i] = 0;
            }
        }
        at0 += __popc(on);
    }
    // zeros behind the last row: the products over rows run in steps of 64
    const int end = (s_all + 255) / 256 * 256;
    for (int row = s_all + blockIdx.x * (kGatherThreads / 32) + warp; row < end; row += gridDim.x * (kGatherThreads / 32)) {
        uint4* dst = reinterpret_cast<uint4*>(p.s.hidden) + (size_t)row * 8;
        for (int i = lane; i < vecs; i += 32) dst[(size_t)(i >> 3) * p.s.rows_pad * 8 + (i & 7)] = make_uint4(0, 0, 0, 0);
    }
}

// ---- epilogues ---------------------------------------------------------------------------------------------
// This lane's value in column `col` of the tile (col < 0: none): one warp-wide read per distinct lane that wants one.
__device__ __forceinline__ float pick_column(uint32_t tmem, int col, int lane) {
    float z = 0.f;
    uint32_t want = __ballot_sync(0xffffffffu, col >= 0);
    while (want) {
        const int l = __ffs(want) - 1;
        want &= want - 1;
        const uint32_t v = gemm::tmem_ld1(tmem + __shfl_sync(0xffffffffu, col, l));
        if (lane == l) z = __uint_as_float(v);
    }
    return z;
}

// The tensor cores' fp32 additions truncate: each of the D / 16 that a logit is summed with loses up to 2^-23 of the running
// sum, which is half the logit in the mean where the sum grows evenly.  Such a logit comes out too small by a factor
// 1 - c D / 16 2^-25, where c = 0.72 for half a unit lost at evenly spread mantissas; measured c = 0.51 to 0.55 (D = 512 to 16384;
// normal, positive and shifted inputs, a hundredth of the units twelve times larger).  The factor that makes up for it costs nothing:
// it goes into log2(e), for lse and G alike.  It leaves a mean error of lse of 1e-7 relative at D = 4096 and a largest one of 1e-6,
// which an fp32 product without tensor cores has too.  A sum that is complete after its first columns loses twice as much (c = 1.07),
// one that grows in its last columns or is exact nothing: there the error is that of no factor at all in size, with the sign turned
// (3.3e-5 at D = 4096, z = 8).  Without the factor lse would be 0 to 6.8e-5 too small, with it it is off by -3.5e-5 to 3.3e-5.
static float log2e_for(int D) { return (float)(1.4426950408889634 * (1.0 + (D / 16) * (0.52 / 33554432.0))); }

struct StatsEpilogue {
    static constexpr bool kOutBox = false;
    struct Params {
        float log2e;
        float2* part;
        const float* ztarget;
        const int* target;
        long long rows_pad;
        int V;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int row, int lane, int part, gemm::WarpSmem&) {
        const int n = min(t.nt, p.V - t.col0);
        float m = -INFINITY, s = 0.f;
        for (int c = part * 32; c < n; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            gemm::tmem_wait32(r);
            if (c + 32 > n) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c + j >= n) r[j] = 0xff800000u;  // -inf
            }
            float top = __uint_as_float(r[0]);
#pragma unroll
            for (int j = 1; j < 32; ++j) top = fmaxf(top, __uint_as_float(r[j]));
            top *= p.log2e;
            if (top > m) {
                s *= ex2_approx(m - top);
                m = top;
            }
            float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 32; ++j) add[j & 3] += ex2_approx(fmaf(__uint_as_float(r[j]), p.log2e, -m));
            s += (add[0] + add[1]) + (add[2] + add[3]);
        }
        // The target's logit is known better than the tensor cores sum it, and it is often most of the row's sum: put the
        // better value in its place.
        const bool on = row < t.rows;
        const int col = on ? p.target[row] - t.col0 : -1;
        const bool here = col >= 0 && col < n && (col / 32) % kParts == part;
        const float z = pick_column(tmem, here ? col : -1, lane);
        if (here) s += ex2_approx(fmaf(p.ztarget[row], kLog2e, -m)) - ex2_approx(fmaf(z, p.log2e, -m));
        if (on) p.part[((long long)t.n * kParts + part) * p.rows_pad + row] = make_float2(m, s);
    }
};

struct GradEpilogue {  // G of a piece, bf16; zeros in the rows of a tile, and the columns of a step of 64, that do not exist
    static constexpr bool kOutBox = false;
    struct Params {
        float log2e;
        uint16_t* g;
        const float *lse2, *weight, *gtarget;
        const int* target;
        long long rows_pad;
        int v0, n_real;  // first vocabulary entry of the piece; its entries
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int row, int lane, int part, gemm::WarpSmem&) {
        const bool on = row < t.rows;
        const float lse2 = on ? p.lse2[row] : 0.f, w = on ? p.weight[row] : 0.f;
        const int col = on ? p.target[row] - p.v0 - t.col0 : -1;
        const int n = min(t.nt, p.n_real - t.col0);  // its last columns, up to a multiple of 64, are zeros
        auto at = [&](int c) { return p.g + ((long long)((t.col0 + c) >> 6) * p.rows_pad + row) * 64 + ((t.col0 + c) & 63); };
        const int end = min(t.nt, (p.n_real + 63) / 64 * 64 - t.col0);
        for (int c = part * 32; c < end; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            gemm::tmem_wait32(r);
            uint32_t b[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float lo = ex2_approx(fmaf(__uint_as_float(r[2 * j]), p.log2e, -lse2)) * w;
                float hi = ex2_approx(fmaf(__uint_as_float(r[2 * j + 1]), p.log2e, -lse2)) * w;
                if (!on || c + 2 * j >= n) lo = 0.f;
                if (!on || c + 2 * j + 1 >= n) hi = 0.f;
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b[j]) : "f"(hi), "f"(lo));
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)  // whole sectors
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at(c) + 16 * j), "r"(b[8 * j]), "r"(b[8 * j + 1]),
                             "r"(b[8 * j + 2]), "r"(b[8 * j + 3]), "r"(b[8 * j + 4]), "r"(b[8 * j + 5]), "r"(b[8 * j + 6]), "r"(b[8 * j + 7])
                             : "memory");
        }
        // the target's entry, by the part that wrote its column
        const bool here = col >= 0 && col < n && (col / 32) % kParts == part;
        if (here) {
            uint16_t b;
            asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(b) : "f"(p.gtarget[row]));
            *at(col) = b;
        }
    }
};

// dW of a piece: rows are vocabulary entries.  A warp turns 32 rows x 64 columns at a time through its box of shared memory,
// so that whole 128-byte lines go out (a lane's own 16-byte pieces, 2 KB apart, cost 37 instead of 20 us for 32001 x 1000).
struct WeightEpilogue {
    static constexpr bool kOutBox = true;
    struct Params {
        CUtensorMap out;  // of the piece: its columns up to a multiple of 8 (a copy writes 16 bytes or none)
        uint16_t* rows;   // the same; the columns behind are stored one by one
        long long stride;
        const float* scale;
        int n_real, D;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool zero, const gemm::Tile& t, int row, int lane, int part,
                                               gemm::WarpSmem& own) {
        const float scale = *p.scale;
        for (int c = part * 64; c < t.nt && t.col0 + c < p.D; c += kParts * 64) {
            uint32_t r[32], b[32];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                gemm::tmem_ld32(tmem + c + 32 * half, r);
                gemm::tmem_wait32(r);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;"
                        : "=r"(b[16 * half + j])
                        : "f"(__uint_as_float(r[2 * j + 1]) * scale), "f"(__uint_as_float(r[2 * j]) * scale));
                    if (zero) b[16 * half + j] = 0;
                }
            }
            const int d = t.col0 + c, whole = p.D & ~7;
            if (row - lane < p.n_real && d < whole) gemm::send_box(own, b, lane, &p.out, d, row - lane);
            if (whole < p.D && d + 64 > whole && row < p.n_real) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (d + j >= whole && d + j < p.D) p.rows[row * p.stride + d + j] = (uint16_t)(b[j / 2] >> (16 * (j & 1)));
            }
        }
    }
};

struct HiddenEpilogue {  // a piece's part of dH, added up in fp32 (one buffer per cut of the sum), laid out so that a warp's rows are adjacent
    static constexpr bool kOutBox = false;
    struct Params {
        float4* acc;
        long long rows_pad, da;
        int D, first;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool zero, const gemm::Tile& t, int row, int, int part, gemm::WarpSmem&) {
        const bool on = row < t.rows;
        for (int c = part * 32; c < t.nt && t.col0 + c < p.D; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            const int d = t.col0 + c;
            float4* out = p.acc + (t.split * (p.da / 4) + d / 4) * p.rows_pad + row;
            float4 a[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                a[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (!p.first && on && d + 4 * j < p.D) a[j] = out[j * p.rows_pad];
            }
            gemm::tmem_wait32(r);
            if (on) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!zero) {
                        a[j].x += __uint_as_float(r[4 * j]);
                        a[j].y += __uint_as_float(r[4 * j + 1]);
                        a[j].z += __uint_as_float(r[4 * j + 2]);
                        a[j].w += __uint_as_float(r[4 * j + 3]);
                    }
                    if (d + 4 * j < p.D) out[j * p.rows_pad] = a[j];
                }
            }
        }
    }
};

struct HiddenRowsEpilogue {  // dH itself, where one tile sums a row's whole gradient (one piece, one cut): rows to their places
    static constexpr bool kOutBox = false;
    struct Params {
        uint16_t* out;
        const int* row_of;
        const float* scale;
        long long stride;
        int D, wide;  // wide: rows start on 32-byte boundaries
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool zero, const gemm::Tile& t, int row, int, int part, gemm::WarpSmem&) {
        const bool on = row < t.rows;
        const float scale = *p.scale;
        uint16_t* out = p.out + (on ? p.row_of[row] : 0) * p.stride;
        for (int c = part * 32; c < t.nt && t.col0 + c < p.D; c += kParts * 32) {
            uint32_t r[32], b[16];
            gemm::tmem_ld32(tmem + c, r);
            gemm::tmem_wait32(r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b[j]) : "f"(__uint_as_float(r[2 * j + 1]) * scale), "f"(__uint_as_float(r[2 * j]) * scale));
                if (zero) b[j] = 0;
            }
            const int d = t.col0 + c;
            if (on && p.wide && d + 32 <= p.D) {  // whole sectors
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + d + 16 * j), "r"(b[8 * j]), "r"(b[8 * j + 1]),
                                 "r"(b[8 * j + 2]), "r"(b[8 * j + 3]), "r"(b[8 * j + 4]), "r"(b[8 * j + 5]), "r"(b[8 * j + 6]), "r"(b[8 * j + 7])
                                 : "memory");
            } else if (on) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (d + j < p.D) out[d + j] = (uint16_t)(b[j / 2] >> (16 * (j & 1)));
            }
        }
    }
};

// ---- small kernels -----------------------------------------------------------------------------------------
// Joins the tiles' (max, sum) pairs: a CTA takes 32 rows, its warps the tiles in turn; fp64 sums, a fixed order.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps) ce_join_kernel(CeSpace s, int parts, float* loss, float* lse) {
    __shared__ float s_m[kJoinWarps][32];
    __shared__ double s_s[kJoinWarps][32];
    wait_for_primary_kernel();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + lane, rows = *s.count;
    if ((int)blockIdx.x * 32 >= rows) return;
    const float2* at = s.part + (row < rows ? row : 0);
    const int src = row < rows ? s.row_of[row] : 0;
    const float zt = row < rows ? s.ztarget[row] : 0.f;
    float m = -INFINITY;
    double sum = 0.0;
    for (int t0 = warp; t0 < parts; t0 += 8 * kJoinWarps) {  // eight pairs in flight
        float2 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = t0 + j * kJoinWarps;
            v[j] = t < parts ? at[t * s.rows_pad] : make_float2(-INFINITY, 0.f);
        }
        float top = v[0].x;
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, v[j].x);
        if (top > m) {
            sum *= (double)ex2_approx(m - top);
            m = top;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sum += (double)(v[j].y * ex2_approx(v[j].x - (m == -INFINITY ? 0.f : m)));  // (a part without columns: -inf and 0)
    }
    s_m[warp][lane] = m;
    s_s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && row < rows) {
        float top = s_m[0][lane];
#pragma unroll
        for (int w = 1; w < kJoinWarps; ++w) top = fmaxf(top, s_m[w][lane]);
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w)
            if (s_s[w][lane] != 0.0) all += s_s[w][lane] * (double)ex2_approx(s_m[w][lane] - top);  // (a warp without tiles has -inf and 0)
        const double l = kLn2 * ((double)top + log2(all));
        lse[src] = (float)l;
        loss[src] = (float)(l - (double)zt);
    }
}

// dH: adds the cuts of the sum and puts the rows back in their places, times the largest weight.  A CTA takes 32 rows by 64
// hidden units: read as they lie (rows adjacent), turned in shared memory, written as 128-byte pieces of rows.  With many
// cuts (few rows) kGroups of warps share them, each adding its own in order.
template <int kGroups>
__global__ void __launch_bounds__(256 * kGroups) ce_scatter_kernel(CeSpace s, uint16_t* out, long long stride, int D) {
    __shared__ float4 sums[kGroups > 1 ? kGroups - 1 : 1][16][32];
    __shared__ uint32_t tile[32][33];
    wait_for_primary_kernel();
    allow_dependent_launch();
    const int rows = *s.count, r0 = blockIdx.x * 32, d0 = blockIdx.y * 64;
    if (r0 >= rows) return;
    const float scale = *s.top_weight;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 7, group = threadIdx.x >> 8;
    const float4* acc = reinterpret_cast<const float4*>(s.acc);
    const int from = s.splits * group / kGroups, to = s.splits * (group + 1) / kGroups;
    const long long cut = s.da / 4 * s.rows_pad;
    const float4* a[2];
    bool on[2];
    float4 v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int d = d0 + 4 * (warp + 8 * k);
        on[k] = d < D && r0 + lane < rows;
        a[k] = acc + (long long)(d / 4) * s.rows_pad + r0 + lane;
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int i = from; i < to; i += 4) {  // eight loads in flight
        float4 w[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[k][j] = on[k] && i + j < to ? a[k][(i + j) * cut] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[k] = make_float4(v[k].x + w[k][j].x, v[k].y + w[k][j].y, v[k].z + w[k][j].z, v[k].w + w[k][j].w);
    }
    if (group > 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) sums[group - 1][warp + 8 * k][lane] = v[k];
    }
    if (kGroups > 1) __syncthreads();
    if (group == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c4 = warp + 8 * k;
#pragma unroll
            for (int g = 0; g + 1 < kGroups; ++g) {
                const float4 w = sums[g][c4][lane];
                v[k] = make_float4(v[k].x + w.x, v[k].y + w.y, v[k].z + w.z, v[k].w + w.w);
            }
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(tile[lane][2 * c4]) : "f"(v[k].y * scale), "f"(v[k].x * scale));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(tile[lane][2 * c4 + 1]) : "f"(v[k].w * scale), "f"(v[k].z * scale));
        }
    }
    __syncthreads();
    for (int r = threadIdx.x >> 5; r < 32; r += 8 * kGroups) {
        const int d = d0 + 2 * lane;
        if (r0 + r < rows && d < D) {
            uint16_t* o = out + s.row_of[r0 + r] * stride + d;
            const uint32_t w = tile[r][lane];
            if (d + 1 < D) *reinterpret_cast<uint32_t*>(o) = w;
            else *o = (uint16_t)w;
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------
template <typename... Params, typename... Args>
static int launch_after(void (*kernel)(Params...), dim3 grid, int threads, cudaStream_t st, const Args&... args) {
    return gemm::launch_early(kernel, grid, threads, 0, 1, st, args...) == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
}

static int gather(GatherParams p, cudaStream_t st) {
    p.per = p.rows > 8 * 148 * 8 ? (p.rows + 148 * 8 - 1) / (148 * 8) : 8;
    const int grid = (p.rows + p.per - 1) / p.per;
    return launch_after(ce_gather_kernel, dim3(grid), kGatherThreads, st, p);
}

template <class Epi, int kWarps>
static int product(bool pair, const gemm::Maps& maps, const gemm::Product& p, const typename Epi::Params& ep, cudaStream_t st) {
    return pair ? gemm::launch<false, 2, kWarps, Epi>(maps, p, ep, st) : gemm::launch<false, 1, kWarps, Epi>(maps, p, ep, st);
}

template <class Epi>
static int both(bool pair, const gemm::Maps& maps, const gemm::Product& p, const typename Epi::Params& ep, const gemm::Maps& maps2,
                const gemm::Product& p2, const WeightEpilogue::Params& ep2, cudaStream_t st) {
    return pair ? gemm::launch_two<false, 2, 4, Epi, WeightEpilogue>(maps, p, ep, maps2, p2, ep2, st)
                : gemm::launch_two<false, 1, 4, Epi, WeightEpilogue>(maps, p, ep, maps2, p2, ep2, st);
}

// z of `width` vocabulary entries of the weight, in tiles that reach column `cover` at least: the product that forward and
// backward share.
static int logits_product(const CeSpace& s, int rows, int D, const uint16_t* w, long long w_stride, long long width, long long cover, int nt,
                          gemm::Product* p,
                          gemm::Maps* maps) {
    *p = gemm::Product{};
    const int tile_rows = s.pair ? 256 : 128;
    p->m_tiles = (int)(up(rows, tile_rows) / tile_rows);
    p->nt = nt;
    p->n_tiles = (int)((cover + nt - 1) / nt);
    p->splits = 1;
    p->k_elems = 64;
    p->k_blocks = (D + 63) / 64;
    p->group_m = gemm::rows_in_l2(tile_rows, s.ds * 2);
    p->m_total = rows;
    p->m_limit = s.count;
    p->status = s.status;
    p->a_layout = gemm::kPanelsK;
    p->pitch = (int)s.rows_pad;
    return gemm::encode_map(&maps->a, gemm::kElemBf16, s.hidden, 64, s.ds / 64 * s.rows_pad, 128, 128) &&
                   gemm::encode_map(&maps->b, gemm::kElemBf16, w, D, width, w_stride * 2, s.pair ? nt / 2 : nt)
               ? TSLT_OK
               : TSLT_ERR_CUDA;
}

static int check_common(const void* hidden, long long h_stride, const void* weight, long long w_stride, const int* target, int rows, int V, int D) {
    auto bad = [&](const void* p, long long stride) { return !p || ((uintptr_t)p & 15) || stride < D || stride % 8; };
    if (bad(weight, w_stride)) return TSLT_ERR_INVALID_ARG;
    if (rows > 0 && (bad(hidden, h_stride) || !target)) return TSLT_ERR_INVALID_ARG;
    (void)V;
    return TSLT_OK;
}

static int check_sizes(int rows, int V, int D) {
    if (rows < 0 || V <= 0 || D <= 0) return TSLT_ERR_INVALID_ARG;
    if (D > TSLT_MAX_HIDDEN || rows > TSLT_MAX_LOSS_ROWS || V > TSLT_MAX_VOCAB) return TSLT_ERR_UNSUPPORTED;
    return TSLT_OK;
}

}  // namespace tslt

using namespace tslt;

extern "C" int tslt_linear_ce_workspace_bytes(int rows, int V, int D, size_t* bytes) {
    if (!bytes) return TSLT_ERR_INVALID_ARG;
    if (const int rc = check_sizes(rows, V, D)) return rc;
    *bytes = rows ? ce_space(nullptr, rows, V, D, false).bytes : kWsHeaderBytes;
    return TSLT_OK;
}

extern "C" int tslt_linear_ce_backward_workspace_bytes(int rows, int V, int D, size_t* bytes) {
    if (!bytes) return TSLT_ERR_INVALID_ARG;
    if (const int rc = check_sizes(rows, V, D)) return rc;
    *bytes = rows ? ce_space(nullptr, rows, V, D, true).bytes : kWsHeaderBytes;
    return TSLT_OK;
}

extern "C" int tslt_linear_ce(const void* hidden, long long hidden_stride, const void* weight, long long weight_stride, const int* target,
                              int rows, int V, int D, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (const int rc = check_sizes(rows, V, D)) return rc;
    if (rows == 0) return TSLT_OK;
    if (const int rc = check_common(hidden, hidden_stride, weight, weight_stride, target, rows, V, D)) return rc;
    if (!loss || !lse || !workspace || ((uintptr_t)workspace & 255)) return TSLT_ERR_INVALID_ARG;
    const CeSpace s = ce_space(workspace, rows, V, D, false);
    if (workspace_bytes < s.bytes) return TSLT_ERR_WORKSPACE;
    if (loss == lse || (const void*)loss == target || (const void*)lse == target) return TSLT_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    gemm::Product p;
    gemm::Maps maps;
    if (const int rc = logits_product(s, rows, D, (const uint16_t*)weight, weight_stride, V, V, s.nt, &p, &maps)) return rc;
    const GatherParams g = {(const uint16_t*)hidden, (const uint16_t*)weight, target, hidden_stride, weight_stride, rows, V, D, 0, nullptr,
                            nullptr, loss, lse, nullptr, 0, s};
    if (const int rc = gather(g, st)) return rc;
    const StatsEpilogue::Params ep = {log2e_for(D), s.part, s.ztarget, s.target, s.rows_pad, V};
    if (const int rc = product<StatsEpilogue, 4 * kStatsParts>(s.pair, maps, p, ep, st)) return rc;
    return launch_after(ce_join_kernel, dim3((rows + 31) / 32), 32 * kJoinWarps, st, s, (int)s.tiles * kStatsParts, loss, lse);
}

extern "C" int tslt_linear_ce_backward(const void* hidden, long long hidden_stride, const void* weight, long long weight_stride,
                                       const int* target, const float* lse, const float* dloss, int rows, int V, int D, void* dhidden,
                                       long long dhidden_stride, void* dweight, long long dweight_stride, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    if (const int rc = check_sizes(rows, V, D)) return rc;
    if (const int rc = check_common(hidden, hidden_stride, weight, weight_stride, target, rows, V, D)) return rc;
    auto bad = [&](const void* q, long long stride) { return !q || ((uintptr_t)q & 15) || stride < D || stride % 8; };
    if (bad(dweight, dweight_stride)) return TSLT_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (rows == 0)  // no row contributes
        return cudaMemset2DAsync(dweight, dweight_stride * 2, 0, (size_t)D * 2, V, st) == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
    if (dhidden == hidden || dhidden == weight || dhidden == dweight || dweight == hidden || dweight == weight) return TSLT_ERR_INVALID_ARG;
    if (bad(dhidden, dhidden_stride) || !lse || !workspace || ((uintptr_t)workspace & 255)) return TSLT_ERR_INVALID_ARG;
    const CeSpace s = ce_space(workspace, rows, V, D, true);
    if (workspace_bytes < s.bytes) return TSLT_ERR_WORKSPACE;
    const GatherParams g = {(const uint16_t*)hidden, (const uint16_t*)weight, target, hidden_stride, weight_stride, rows, V, D, 0, lse, dloss,
                            nullptr, nullptr, (uint16_t*)dhidden, dhidden_stride, s};
    if (const int rc = gather(g, st)) return rc;
    const uint16_t* w = (const uint16_t*)weight;
    const int tile_rows = s.pair ? 256 : 128, nt = D > 128 ? 256 : 128;
    for (int c = 0; c < s.pieces; ++c) {
        const long long v0 = c * s.piece, width = v0 + s.piece < V ? s.piece : V - v0;
        gemm::Product p;
        gemm::Maps maps;
        if (const int rc = logits_product(s, rows, D, w + v0 * weight_stride, weight_stride, width, up(width, 64),  // dH sums in steps of 64
                                         gemm::choose_nt((rows + tile_rows - 1) / tile_rows, width, s.pair != 0, 32), &p, &maps)) return rc;
        const GradEpilogue::Params eg = {log2e_for(D), s.g, s.lse2, s.weight, s.gtarget, s.target, s.rows_pad, (int)v0, (int)width};
        if (const int rc = product<GradEpilogue, 8>(s.pair, maps, p, eg, st)) return rc;

        // one kernel for both products that read G.  The piece's part of dH first, while the weight's piece is still in L2 from
        // the product above: its sum runs over the piece's vocabulary entries
        const int ctas = s.pair ? 2 : 1, b_blocks = nt / ctas / 64;
        const uint16_t* wp = w + v0 * weight_stride;
        p.m_tiles = (int)(up(rows, tile_rows) / tile_rows);
        p.n_tiles = (D + nt - 1) / nt;
        p.nt = nt;
        p.k_blocks = (int)((width + 63) / 64);
        p.splits = s.splits;
        p.group_m = 8;
        p.b_layout = D % 64 == 0 ? gemm::kBlocksMN : gemm::kRowsMN;
        if (!gemm::encode_map(&maps.a, gemm::kElemBf16, s.g, 64, s.piece / 64 * s.rows_pad, 128, 128) ||
            !(D % 64 == 0 ? gemm::encode_blocks(&maps.b, wp, width, weight_stride * 2, D / 64, 128, b_blocks)
                          : gemm::encode_map(&maps.b, gemm::kElemBf16, wp, D, width, weight_stride * 2, 64)))
            return TSLT_ERR_CUDA;
        const HiddenEpilogue::Params eh = {(float4*)s.acc, s.rows_pad, s.da, D, c == 0};

        // dW of the piece: rows are vocabulary entries, the sum runs over the rows that count
        gemm::Product p2 = p;
        gemm::Maps maps2;
        p2.m_tiles = (int)(up(width, tile_rows) / tile_rows);
        p2.k_blocks = (int)(s.rows_pad / 64);
        p2.splits = 1;
        p2.group_m = 1;  // a strip of G is read by all column tiles at once, the hidden rows stay in L2 (dW alone, sustained: 594 us; groups of 8: 625)
        p2.a_layout = p2.b_layout = gemm::kBlocksMN;
        p2.m_total = (int)width;
        p2.m_limit = nullptr;
        p2.k_limit = s.count;
        if (!gemm::encode_blocks(&maps2.a, s.g, s.rows_pad, 128, s.piece / 64, s.rows_pad * 128, 2) ||
            !gemm::encode_blocks(&maps2.b, s.hidden, s.rows_pad, 128, s.ds / 64, s.rows_pad * 128, b_blocks))
            return TSLT_ERR_CUDA;
        uint16_t* dw = (uint16_t*)dweight + v0 * dweight_stride;
        WeightEpilogue::Params ew = {{}, dw, dweight_stride, s.top_weight, (int)width, D};
        if (!gemm::encode_map(&ew.out, gemm::kElemBf16, dw, D < 8 ? 8 : D & ~7, width, dweight_stride * 2, 32)) return TSLT_ERR_CUDA;
        const int wide = ((uintptr_t)dhidden & 31) == 0 && dhidden_stride % 16 == 0;
        const HiddenRowsEpilogue::Params er = {(uint16_t*)dhidden, s.row_of, s.top_weight, dhidden_stride, D, wide};
        const int rc = s.direct ? both<HiddenRowsEpilogue>(s.pair, maps, p, er, maps2, p2, ew, st) : both<HiddenEpilogue>(s.pair, maps, p, eh, maps2, p2, ew, st);
        if (rc) return rc;
    }
    if (s.direct) return TSLT_OK;
    const dim3 grid((rows + 31) / 32, (D + 63) / 64);
    return s.splits >= 8 ? launch_after(ce_scatter_kernel<4>, grid, 1024, st, s, (uint16_t*)dhidden, dhidden_stride, D)
                         : launch_after(ce_scatter_kernel<1>, grid, 256, st, s, (uint16_t*)dhidden, dhidden_stride, D);
}

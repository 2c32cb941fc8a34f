// Softmax cross entropy of a linear head over a large vocabulary, with its gradients (tslt_linear_ce,
// tslt_linear_ce_backward), without ever holding the logits [rows, V].
//
// Mathematics.  z = H W^T; lse_n = ln sum_v exp z[n, v]; loss_n = lse_n - z[n, t_n].  With g_n the weight of row n's loss,
// G[n, v] = g_n (exp(z[n, v] - lse_n) - [v = t_n]), dH = G W, dW = G^T H.
//
// Forward: one product whose epilogue turns each 256-column tile of z, still in tensor memory, into a running (max, sum)
// pair per row; the pairs of all tiles (8 bytes for 256 logits) go to the workspace and a small kernel joins them.
// Backward, piece by piece of the vocabulary: z of the piece is computed again and its epilogue writes G of the piece in
// bf16 to the workspace; two products read it, dW of the piece (complete: its sum runs over the rows) and the piece's part
// of dH (summed over the pieces in fp32, in a fixed order).  Bound by the tensor cores: 2 + 6 products of rows x V x D
// multiply-adds (the recomputation is the price of not keeping rows x V logits).
//
// Ignored rows (negative target) are taken out before anything is multiplied: the rows that count are copied together, in
// their order, and every product runs over those only.  Ignored rows cost nothing and what they hold (padding, NaN) is
// never looked at.
#include "tslt_gemm.cuh"

namespace tslt {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
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
    float* lse2;       // [rows_pad] lse * log2(e)                        (backward)
    float* weight;     // [rows_pad] g                                    (backward)
    uint16_t* hidden;  // [rows_pad, ds] the rows that count, bf16; zeros up to the next multiple of 256 rows
    float2* part;      // [tiles, rows_pad] (max, sum) in base 2          (forward)
    float* ztarget;    // [rows_pad]                                      (forward)
    uint16_t* g;       // [rows_pad, piece]                               (backward)
    float* acc;        // [splits, rows_pad, da]                          (backward)
    long long rows_pad, ds, da, tiles, piece;
    int pieces, splits, pair;
    size_t bytes;
};

static CeSpace ce_space(void* ws, int rows, int V, int D, bool backward) {
    CeSpace s = {};
    s.rows_pad = up(rows, 256);
    s.ds = up(D, 64);
    s.da = up(D, 4);
    s.pair = rows > 128;
    const long long vt = up(V, kTileN);
    s.tiles = vt / kTileN;
    long long c = kPieceBytes / 2 / s.rows_pad / kTileN * kTileN;
    if (c < kTileN) c = kTileN;
    s.pieces = (int)((vt + c - 1) / c);
    s.piece = up((vt + s.pieces - 1) / s.pieces, kTileN);
    s.pieces = (int)((vt + s.piece - 1) / s.piece);
    // dH of few rows has few tiles and a long sum: cut it so that the machine is full, 256 vocabulary entries a cut at least
    const long long tile_rows = s.pair ? 256 : 128;
    const long long tiles3 = up(rows, tile_rows) / tile_rows * (up(D, kTileN) / kTileN), slots = s.pair ? 74 : 148;
    long long cuts = slots / tiles3;
    if (cuts > s.piece / 256) cuts = s.piece / 256;
    s.splits = (int)(cuts < 1 ? 1 : cuts);
    uint8_t* p = (uint8_t*)ws;
    size_t at = kWsHeaderBytes;
    auto take = [&](size_t n) {
        uint8_t* r = p + at;
        at += align_up256(n);
        return r;
    };
    s.status = (int*)p;
    s.count = (int*)(p + 128);
    s.row_of = (int*)take(s.rows_pad * 4);
    s.target = (int*)take(s.rows_pad * 4);
    s.hidden = (uint16_t*)take(s.rows_pad * s.ds * 2);
    if (backward) {
        s.lse2 = (float*)take(s.rows_pad * 4);
        s.weight = (float*)take(s.rows_pad * 4);
        s.g = (uint16_t*)take(s.rows_pad * s.piece * 2);
        s.acc = (float*)take((size_t)s.splits * s.rows_pad * s.da * 4);
    } else {
        s.part = (float2*)take(s.tiles * s.rows_pad * 8);
        s.ztarget = (float*)take(s.rows_pad * 4);
    }
    s.bytes = at;
    return s;
}

// ---- gathering the rows that count --------------------------------------------------------------------------
struct GatherParams {
    const uint16_t* hidden;
    const int* target;
    long long h_stride;
    int rows, V, D;
    const float *lse_in, *weight_in;  // backward (weight_in may be null: 1)
    float *loss, *lse;                // forward: zeroed for ignored rows
    uint16_t* dhidden;                // backward: zeroed for ignored rows
    long long dh_stride;
    CeSpace s;
};
constexpr int kGatherThreads = 256;

__device__ __forceinline__ bool counts(int t, int V) { return t >= 0 && t < V; }

__device__ __forceinline__ void copy_row(uint16_t* dst, const uint16_t* src, int D, int tid) {
    const int vecs = D / 8;
    for (int i = tid; i < vecs; i += kGatherThreads)
        reinterpret_cast<uint4*>(dst)[i] = src ? reinterpret_cast<const uint4*>(src)[i] : make_uint4(0, 0, 0, 0);
    for (int i = vecs * 8 + tid; i < D; i += kGatherThreads) dst[i] = src ? src[i] : (uint16_t)0;
}

// CTA b takes `per` source rows from b * per on: it counts the rows that count before them (and in all) from the targets,
// which every CTA reads whole (they are few bytes next to the rows), so that no CTA waits for another.
__global__ void __launch_bounds__(kGatherThreads) ce_gather_kernel(const __grid_constant__ GatherParams p, int per) {
    __shared__ int s_before, s_all;
    const int tid = threadIdx.x, lane = tid & 31;
    const int first = min(p.rows, (int)blockIdx.x * per), last = min(p.rows, first + per);
    if (tid == 0) s_before = s_all = 0;
    __syncthreads();
    int before = 0, all = 0, bad = 0;
    for (int i = tid; i < p.rows; i += kGatherThreads) {
        const int t = p.target[i];
        const int c = counts(t, p.V);
        bad |= t >= p.V;
        all += c;
        before += i < first ? c : 0;
    }
    before = __reduce_add_sync(0xffffffffu, before);
    all = __reduce_add_sync(0xffffffffu, all);
    bad = __syncthreads_or(bad);
    if (lane == 0) {
        atomicAdd(&s_before, before);
        atomicAdd(&s_all, all);
    }
    __syncthreads();
    int at = s_before;
    if (blockIdx.x == 0 && tid == 0) {
        *p.s.status = bad ? TSLT_STATUS_BAD_TARGET : 0;
        *p.s.count = s_all;
    }
    for (int row = first; row < last; ++row) {
        const int t = p.target[row];
        if (counts(t, p.V)) {
            copy_row(p.s.hidden + at * p.s.ds, p.hidden + row * p.h_stride, p.D, tid);
            if (tid == 0) {
                p.s.row_of[at] = row;
                p.s.target[at] = t;
                if (p.lse_in) {
                    p.s.lse2[at] = (float)((double)p.lse_in[row] * 1.4426950408889634);
                    p.s.weight[at] = p.weight_in ? p.weight_in[row] : 1.f;
                }
            }
            ++at;
        } else {
            if (tid == 0 && p.loss) {
                p.loss[row] = 0.f;
                p.lse[row] = 0.f;
            }
            if (p.dhidden) copy_row(p.dhidden + row * p.dh_stride, nullptr, p.D, tid);
        }
    }
    // zeros behind the last row: the products over rows run in steps of 64
    const int end = (s_all + 255) / 256 * 256;
    for (int row = s_all + blockIdx.x; row < end; row += gridDim.x) copy_row(p.s.hidden + row * p.s.ds, nullptr, p.D, tid);
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

struct StatsEpilogue {
    struct Params {
        float2* part;
        float* ztarget;
        const int* target;
        long long rows_pad;
        int V;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int row, int lane, int part) {
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
            top *= kLog2e;
            if (top > m) {
                s *= ex2_approx(m - top);
                m = top;
            }
            float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 32; ++j) add[j & 3] += ex2_approx(fmaf(__uint_as_float(r[j]), kLog2e, -m));
            s += (add[0] + add[1]) + (add[2] + add[3]);
        }
        const bool on = row < t.rows;
        if (on) p.part[((long long)t.n * kParts + part) * p.rows_pad + row] = make_float2(m, s);
        if (part == 0) {
            const int col = on ? __ldg(p.target + row) - t.col0 : -1;
            const bool here = col >= 0 && col < n;
            const float z = pick_column(tmem, here ? col : -1, lane);
            if (here) p.ztarget[row] = z;
        }
    }
};

struct GradEpilogue {  // G of a piece, bf16; zeros in the rows and columns of a tile that do not exist
    struct Params {
        uint16_t* g;
        const float *lse2, *weight;
        const int* target;
        long long stride;
        int v0, n_real;  // first vocabulary entry of the piece; its entries
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int row, int lane, int part) {
        const bool on = row < t.rows;
        const float lse2 = on ? __ldg(p.lse2 + row) : 0.f, w = on ? __ldg(p.weight + row) : 0.f;
        const int col = on ? __ldg(p.target + row) - p.v0 - t.col0 : -1;
        const int n = min(t.nt, p.n_real - t.col0);
        uint16_t* out = p.g + row * p.stride + t.col0;
        for (int c = part * 32; c < t.nt; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            gemm::tmem_wait32(r);
            uint32_t b[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float lo = ex2_approx(fmaf(__uint_as_float(r[2 * j]), kLog2e, -lse2)) * w;
                float hi = ex2_approx(fmaf(__uint_as_float(r[2 * j + 1]), kLog2e, -lse2)) * w;
                if (!on || c + 2 * j >= n) lo = 0.f;
                if (!on || c + 2 * j + 1 >= n) hi = 0.f;
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b[j]) : "f"(hi), "f"(lo));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                reinterpret_cast<uint4*>(out + c)[j] = make_uint4(b[4 * j], b[4 * j + 1], b[4 * j + 2], b[4 * j + 3]);
        }
        // the target's entry, by the part that wrote its column
        const bool here = col >= 0 && col < n && (col / 32) % kParts == part;
        const float z = pick_column(tmem, here ? col : -1, lane);
        if (here) {
            uint16_t b;
            asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(b) : "f"((ex2_approx(fmaf(z, kLog2e, -lse2)) - 1.f) * w));
            out[col] = b;
        }
    }
};

struct WeightEpilogue {  // dW of a piece: rows are vocabulary entries
    struct Params {
        uint16_t* out;  // of the piece's first entry
        long long stride;
        int n_real, D;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool zero, const gemm::Tile& t, int row, int, int part) {
        const bool on = row < p.n_real;
        uint16_t* out = p.out + row * p.stride;
        for (int c = part * 32; c < t.nt && t.col0 + c < p.D; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            gemm::tmem_wait32(r);
            if (zero) {
#pragma unroll
                for (int j = 0; j < 32; ++j) r[j] = 0;
            }
            uint32_t b[16];
#pragma unroll
            for (int j = 0; j < 16; ++j)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b[j]) : "f"(__uint_as_float(r[2 * j + 1])), "f"(__uint_as_float(r[2 * j])));
            const int d = t.col0 + c;
            if (on) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (d + 8 * j + 8 <= p.D) {
                        *reinterpret_cast<uint4*>(out + d + 8 * j) = make_uint4(b[4 * j], b[4 * j + 1], b[4 * j + 2], b[4 * j + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (d + 8 * j + i < p.D) out[d + 8 * j + i] = (uint16_t)(b[4 * j + i / 2] >> (16 * (i & 1)));
                    }
                }
            }
        }
    }
};

struct HiddenEpilogue {  // a piece's part of dH, added up in fp32 (one buffer per cut of the sum)
    struct Params {
        float* acc;
        long long rows_pad, da;
        int D, first;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool zero, const gemm::Tile& t, int row, int, int part) {
        const bool on = row < t.rows;
        float* out = p.acc + ((long long)t.split * p.rows_pad + row) * p.da;
        for (int c = part * 32; c < t.nt && t.col0 + c < p.D; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            gemm::tmem_wait32(r);
            const int d = t.col0 + c;
            if (on) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (d + 4 * j < p.D) {  // da is a multiple of 4: the vector stays inside the row
                        float4* o = reinterpret_cast<float4*>(out + d + 4 * j);
                        float4 v = zero ? make_float4(0.f, 0.f, 0.f, 0.f)
                                        : make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]), __uint_as_float(r[4 * j + 2]),
                                                      __uint_as_float(r[4 * j + 3]));
                        if (!p.first) {
                            const float4 a = *o;
                            v = make_float4(a.x + v.x, a.y + v.y, a.z + v.z, a.w + v.w);
                        }
                        *o = v;
                    }
                }
            }
        }
    }
};

// ---- small kernels -----------------------------------------------------------------------------------------
// Joins the tiles' (max, sum) pairs: a CTA takes 32 rows, its warps the tiles in turn; fp64 sums.
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) ce_join_kernel(CeSpace s, int parts, float* __restrict__ loss, float* __restrict__ lse) {
    __shared__ float s_m[kJoinWarps][32];
    __shared__ double s_s[kJoinWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + lane, rows = *s.count;
    float m = -INFINITY;
    double sum = 0.0;
    if (row < rows) {
        for (int t = warp; t < parts; t += kJoinWarps) {
            const float2 v = s.part[t * s.rows_pad + row];
            if (v.x > m) {
                sum = sum * (double)ex2_approx(m - v.x) + (double)v.y;
                m = v.x;
            } else {
                sum += (double)(v.y * ex2_approx(v.x - m));
            }
        }
    }
    s_m[warp][lane] = m;
    s_s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && row < rows) {
        float top = s_m[0][lane];
        for (int w = 1; w < kJoinWarps; ++w) top = fmaxf(top, s_m[w][lane]);
        double all = 0.0;
        for (int w = 0; w < kJoinWarps; ++w)
            if (s_s[w][lane] != 0.0) all += s_s[w][lane] * exp2((double)s_m[w][lane] - (double)top);
        const double l = kLn2 * ((double)top + log2(all));
        const int src = s.row_of[row];
        lse[src] = (float)l;
        loss[src] = (float)(l - (double)s.ztarget[row]);
    }
}

// dH: adds the cuts of the sum in order and puts the rows back in their places.
__global__ void __launch_bounds__(256) ce_scatter_kernel(CeSpace s, uint16_t* __restrict__ out, long long stride, int D) {
    const int rows = *s.count;
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        uint16_t* o = out + s.row_of[row] * stride;
        const float* a = s.acc + (long long)row * s.da;
        for (int d = threadIdx.x * 4; d < D; d += 1024) {
            float4 v = *reinterpret_cast<const float4*>(a + d);
            for (int i = 1; i < s.splits; ++i) {
                const float4 w = *reinterpret_cast<const float4*>(a + i * s.rows_pad * s.da + d);
                v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
            }
            uint32_t lo, hi;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(v.y), "f"(v.x));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(v.w), "f"(v.z));
            if (d + 4 <= D) {
                *reinterpret_cast<uint2*>(o + d) = make_uint2(lo, hi);
            } else {
                o[d] = (uint16_t)lo;
                if (d + 1 < D) o[d + 1] = (uint16_t)(lo >> 16);
                if (d + 2 < D) o[d + 2] = (uint16_t)hi;
            }
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------
static int gather(const GatherParams& p, cudaStream_t st) {
    const int per = p.rows > 148 * 4 ? (p.rows + 148 * 4 - 1) / (148 * 4) : 1;
    const int grid = (p.rows + per - 1) / per;
    ce_gather_kernel<<<grid, kGatherThreads, 0, st>>>(p, per);
    return cudaGetLastError() == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
}

template <class Epi>
static int product(bool pair, const CUtensorMap& ta, const CUtensorMap& tb, const gemm::Product& p, const typename Epi::Params& ep, cudaStream_t st) {
    return pair ? gemm::launch<false, 2, 4, Epi>(ta, tb, p, ep, st) : gemm::launch<false, 1, 4, Epi>(ta, tb, p, ep, st);
}

// z of `width` vocabulary entries from row v0 of the weight: the product that forward and backward share.
static int logits_product(const CeSpace& s, int rows, int D, const uint16_t* w, long long w_stride, long long width, gemm::Product* p,
                          CUtensorMap* ta, CUtensorMap* tb) {
    *p = gemm::Product{};
    const int tile_rows = s.pair ? 256 : 128;
    p->m_tiles = (int)(up(rows, tile_rows) / tile_rows);
    p->nt = kTileN;
    p->n_tiles = (int)(up(width, kTileN) / kTileN);
    p->splits = 1;
    p->k_elems = 64;
    p->k_blocks = (D + 63) / 64;
    p->group_m = 16;
    p->m_total = rows;
    p->m_limit = s.count;
    p->status = s.status;
    return gemm::encode_map(ta, false, s.hidden, D, s.rows_pad, s.ds * 2, 128) &&
                   gemm::encode_map(tb, false, w, D, width, w_stride * 2, s.pair ? kTileN / 2 : kTileN)
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
    if (D > TSLT_MAX_HIDDEN || rows > TSLT_MAX_LOSS_ROWS || V > TSLT_MAX_LOSS_VOCAB) return TSLT_ERR_UNSUPPORTED;
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
    cudaStream_t st = (cudaStream_t)stream;
    gemm::Product p;
    CUtensorMap ta, tb;
    if (const int rc = logits_product(s, rows, D, (const uint16_t*)weight, weight_stride, V, &p, &ta, &tb)) return rc;
    GatherParams g = {(const uint16_t*)hidden, target, hidden_stride, rows, V, D, nullptr, nullptr, loss, lse, nullptr, 0, s};
    if (const int rc = gather(g, st)) return rc;
    const StatsEpilogue::Params ep = {s.part, s.ztarget, s.target, s.rows_pad, V};
    if (const int rc = product<StatsEpilogue>(s.pair, ta, tb, p, ep, st)) return rc;
    ce_join_kernel<<<(rows + 31) / 32, 32 * kJoinWarps, 0, st>>>(s, (int)s.tiles, loss, lse);
    return cudaGetLastError() == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
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
    if (bad(dhidden, dhidden_stride) || !lse || !workspace || ((uintptr_t)workspace & 255)) return TSLT_ERR_INVALID_ARG;
    const CeSpace s = ce_space(workspace, rows, V, D, true);
    if (workspace_bytes < s.bytes) return TSLT_ERR_WORKSPACE;
    GatherParams g = {(const uint16_t*)hidden, target, hidden_stride, rows, V, D, lse, dloss, nullptr, nullptr, (uint16_t*)dhidden, dhidden_stride, s};
    if (const int rc = gather(g, st)) return rc;
    const uint16_t* w = (const uint16_t*)weight;
    const int tile_rows = s.pair ? 256 : 128, nt = D > 128 ? 256 : 128;
    for (int c = 0; c < s.pieces; ++c) {
        const long long v0 = c * s.piece, width = v0 + s.piece < V ? s.piece : V - v0;
        gemm::Product p;
        CUtensorMap ta, tb;
        if (const int rc = logits_product(s, rows, D, w + v0 * weight_stride, weight_stride, width, &p, &ta, &tb)) return rc;
        const GradEpilogue::Params eg = {s.g, s.lse2, s.weight, s.target, s.piece, (int)v0, (int)width};
        if (const int rc = product<GradEpilogue>(s.pair, ta, tb, p, eg, st)) return rc;

        // dW of the piece: rows are vocabulary entries, the sum runs over the rows that count
        p.m_tiles = (int)(up(width, tile_rows) / tile_rows);
        p.n_tiles = (D + nt - 1) / nt;
        p.nt = nt;
        p.k_blocks = (int)(s.rows_pad / 64);
        p.group_m = 8;
        p.a_mn = p.b_mn = 1;
        p.m_total = (int)width;
        p.m_limit = nullptr;
        p.k_limit = s.count;
        if (!gemm::encode_map(&ta, false, s.g, s.piece, s.rows_pad, s.piece * 2, 64) ||
            !gemm::encode_map(&tb, false, s.hidden, D, s.rows_pad, s.ds * 2, 64))
            return TSLT_ERR_CUDA;
        const WeightEpilogue::Params ew = {(uint16_t*)dweight + v0 * dweight_stride, dweight_stride, (int)width, D};
        if (const int rc = product<WeightEpilogue>(s.pair, ta, tb, p, ew, st)) return rc;

        // the piece's part of dH: the sum runs over its vocabulary entries
        p.m_tiles = (int)(up(rows, tile_rows) / tile_rows);
        p.k_blocks = (int)((width + 63) / 64);
        p.splits = s.splits;
        p.a_mn = 0;
        p.m_total = rows;
        p.m_limit = s.count;
        p.k_limit = nullptr;
        if (!gemm::encode_map(&ta, false, s.g, s.piece, s.rows_pad, s.piece * 2, 128) ||
            !gemm::encode_map(&tb, false, w + v0 * weight_stride, D, width, weight_stride * 2, 64))
            return TSLT_ERR_CUDA;
        const HiddenEpilogue::Params eh = {s.acc, s.rows_pad, s.da, D, c == 0};
        if (const int rc = product<HiddenEpilogue>(s.pair, ta, tb, p, eh, st)) return rc;
    }
    ce_scatter_kernel<<<rows < 148 * 8 ? rows : 148 * 8, 256, 0, st>>>(s, (uint16_t*)dhidden, dhidden_stride, D);
    return cudaGetLastError() == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
}

// The head product in 8-bit integers (tslt_head_logits): z[n, v] = s_n t_v sum_k q[n, k] c[v, k].  The sum is exact (32-bit
// integers); the scales are multiplied in fp32 and the logit is rounded once.
//
// One to four rows (a draft's step): bound by reading the weight once and by how soon that starts.  No tensor cores: warps take
// blocks of four weight rows, each lane 16 bytes of k at a time from all four, and dot products of four bytes (dp4a) with
// the tokens' codes in shared memory.  V = 32000, K = 2048, us with / without this form: 1 row 12.8 / 17.6, 4 rows
// 14.1 / 17.6, 8 rows 23.0 / 17.6 (the dot products are then the bound); V = 128256, K = 4096: 1 row 78 / 87, 4 rows 82 / 88.
//
// Few rows (a decoding step): bound by reading the weight once.  The weight is the operand of the tensor cores' 128 rows and
// the tokens are its columns (16 ... 160), so that the whole weight goes once through shared memory whatever their number
// (V = 128256, K = 4096, 32 rows: 90 us on the device, 0.89 of the copy bandwidth).
//
// Many rows (verification, prompts): bound by the tensor cores.  The tokens are the rows, 256 of them to a pair of CTAs, and a
// lane of the epilogue holds 64 consecutive logits of a token, which leave through shared memory as whole 128-byte lines
// (V = 256000, K = 4096, 2304 rows: 1.77 ms cool, 1.86 to 1.95 ms sustained, 2.5 to 2.7 POPS; cuBLAS's int8 product, which
// leaves 32-bit sums, 1.54 and 1.79 to 1.93 ms).
#include "tslt_gemm.cuh"

namespace tslt {

// Few rows: lanes are vocabulary entries, columns are tokens.
template <typename T> struct HeadEpilogue {
    static constexpr bool kOutBox = false;
    struct Params {
        T* out;
        long long stride;
        const float *row_scale, *weight_scale;
        int rows, V;
    };
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ void put(uint16_t* p, float v) {
        uint16_t b;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(b) : "f"(v));
        *p = b;
    }
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int v, int lane, int part, gemm::WarpSmem&) {
        const bool on = v < p.V;
        const float wv = on ? p.weight_scale[v] : 0.f;
        const int n = min(t.nt, p.rows - t.col0);
        for (int c = part * 32; c < n; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            const float mine = c + lane < n ? p.row_scale[t.col0 + c + lane] : 0.f;  // lane j: the scale of column c + j
            gemm::tmem_wait32(r);
            T* out = p.out + (long long)(t.col0 + c) * p.stride + v;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                // left to right: the product of the scales alone could underflow
                const float z = (float)(int)r[j] * __shfl_sync(0xffffffffu, mine, j) * wv;
                if (on && c + j < n) put(out + j * p.stride, z);
            }
        }
    }
};

// Many rows: lanes are tokens, columns are vocabulary entries.
template <typename T> struct HeadRowsEpilogue {
    static constexpr bool kOutBox = true;
    static constexpr int kCols = 128 / sizeof(T);  // logits of a 128-byte line
    struct Params {
        CUtensorMap out;  // the logits' columns up to a multiple of 16 bytes (a copy writes 16 bytes or none)
        T* rows;          // the same; the columns behind are stored one by one
        long long stride;
        const float *row_scale, *weight_scale;
        int n_rows, V;
    };
    template <int kParts>
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int row, int lane, int part,
                                               gemm::WarpSmem& own) {
        const float scale = row < p.n_rows ? p.row_scale[row] : 0.f;
        constexpr int kStep = 16 / sizeof(T);
        const int whole = p.V / kStep * kStep;
        for (int c = part * kCols; c < t.nt && t.col0 + c < p.V; c += kParts * kCols) {
            const int v0 = t.col0 + c;
            // the columns' scales, a copy for each warp: 64 shuffles or loads would cost more than 16 reads of shared memory
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kCols; i += 32) {
                const float w = v0 + i + lane < p.V ? p.weight_scale[v0 + i + lane] : 0.f;
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(own.scratch + 4 * (i + lane)), "f"(w) : "memory");
            }
            __syncwarp();
            uint32_t b[32];
#pragma unroll
            for (int i = 0; i < kCols; i += 32) {
                uint32_t r[32];
                gemm::tmem_ld32(tmem + c + i, r);
                gemm::tmem_wait32(r);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    float w[4], z[4];
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]) : "r"(own.scratch + 4 * (i + j)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) z[k] = (float)(int)r[j + k] * scale * w[k];  // left to right, as the few-rows form
                    if (sizeof(T) == 4) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) b[(j + k) & 31] = __float_as_uint(z[k]);
                    } else {
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b[((i + j) / 2) & 31]) : "f"(z[1]), "f"(z[0]));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b[((i + j) / 2 + 1) & 31]) : "f"(z[3]), "f"(z[2]));
                    }
                }
            }
            if (row - lane < p.n_rows && v0 < whole) gemm::send_box(own, b, lane, &p.out, v0, row - lane);
            if (whole < p.V && v0 + kCols > whole && row < p.n_rows) {
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    if (v0 + j >= whole && v0 + j < p.V) {
                        if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p.rows)[row * p.stride + v0 + j] = b[j & 31];
                        else reinterpret_cast<uint16_t*>(p.rows)[row * p.stride + v0 + j] = (uint16_t)(b[(j / 2) & 31] >> (16 * (j & 1)));
                    }
                }
            }
        }
    }
};

// One to four rows.  kRows: 1, 2 or 4, the rows of q in shared memory (rows of zeros behind the last).
constexpr int kVecBlock = 4;  // weight rows of a warp at a time
constexpr int kVecThreads = 256;
constexpr int kVecCodes = 40 * 1024;  // most bytes of q in shared memory
struct VecParams {
    const int8_t *q, *w;
    const float *row_scale, *weight_scale;
    void* out;
    long long q_stride, w_stride, out_stride;
    int rows, V, K;
    int* status;
};
// Weight rows v0 ... v0 + 3 by a warp.  What stands between a row's last code and the next row meets zeros; behind the last row there
// may be nothing: kEnd, the block that holds it, takes the codes behind its whole chunks one by one.
template <int kRows, typename T, bool kEnd>
__device__ __forceinline__ void head_vec_block(const VecParams& p, const uint8_t* s_codes, int chunks, long long v0, int lane) {
    const uint4* codes = reinterpret_cast<const uint4*>(s_codes);
    const int whole = kEnd ? p.K / 16 : chunks;
    int acc[kVecBlock][kRows];
#pragma unroll
    for (int b = 0; b < kVecBlock; ++b)
#pragma unroll
        for (int r = 0; r < kRows; ++r) acc[b][r] = 0;
    const int8_t* w[kVecBlock];
#pragma unroll
    for (int b = 0; b < kVecBlock; ++b) w[b] = p.w + (v0 + b < p.V ? v0 + b : p.V - 1) * p.w_stride;
    for (int c0 = lane; c0 < whole; c0 += 64) {  // eight loads in flight
        uint4 x[2][kVecBlock];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < kVecBlock; ++b)
                x[u][b] = c0 + 32 * u < whole ? __ldcs(reinterpret_cast<const uint4*>(w[b]) + c0 + 32 * u) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const uint4 q = codes[r * chunks + (c0 + 32 * u < whole ? c0 + 32 * u : lane)];
#pragma unroll
                for (int b = 0; b < kVecBlock; ++b) {
                    acc[b][r] = __dp4a((int)x[u][b].x, (int)q.x, acc[b][r]);
                    acc[b][r] = __dp4a((int)x[u][b].y, (int)q.y, acc[b][r]);
                    acc[b][r] = __dp4a((int)x[u][b].z, (int)q.z, acc[b][r]);
                    acc[b][r] = __dp4a((int)x[u][b].w, (int)q.w, acc[b][r]);
                }
            }
        }
    }
    if (kEnd && whole * 16 + lane < p.K) {  // fewer than 16 codes: one a lane
#pragma unroll
        for (int b = 0; b < kVecBlock; ++b) {
            const int x = w[b][whole * 16 + lane];
#pragma unroll
            for (int r = 0; r < kRows; ++r) acc[b][r] += x * (int8_t)s_codes[(r * chunks + whole) * 16 + lane];
        }
    }
    // lane 4 r + b ends up with the sum of row r and weight row b
    int mine = 0;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int b = 0; b < kVecBlock; ++b) {
            const int sum = __reduce_add_sync(0xffffffffu, acc[b][r]);
            if (lane == r * kVecBlock + b) mine = sum;
        }
    const int r = lane / kVecBlock;
    const long long v = v0 + lane % kVecBlock;
    if (r < kRows && r < p.rows && v < p.V) {
        const float z = (float)mine * p.row_scale[r] * p.weight_scale[v];
        HeadEpilogue<T>::put(reinterpret_cast<T*>(p.out) + r * p.out_stride + v, z);
    }
}
template <int kRows, typename T>
__global__ void __launch_bounds__(kVecThreads, 4) head_vec_kernel(const __grid_constant__ VecParams p) {
    extern __shared__ __align__(16) uint8_t s_codes[];
    const int tid = threadIdx.x, lane = tid & 31;
    wait_for_primary_kernel();
    allow_dependent_launch();
    const int chunks = (p.K + 15) / 16;
    if (blockIdx.x == 0 && tid == 0) *p.status = 0;  // nothing here waits
    for (int i = tid; i < kRows * chunks; i += kVecThreads) {
        const int r = i / chunks, at = (i - r * chunks) * 16;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < p.rows) {
            const int8_t* q = p.q + r * p.q_stride + at;
            if (at + 16 <= p.K) {
                v = *reinterpret_cast<const uint4*>(q);
            } else {  // zeros behind the last code, and nothing read there: the buffer may end with it
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 15; ++j)
                    if (at + j < p.K) w[j / 4] |= (uint32_t)(uint8_t)q[j] << (8 * (j % 4));
                v = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        reinterpret_cast<uint4*>(s_codes)[i] = v;
    }
    __syncthreads();
    const long long step = (long long)gridDim.x * (kVecThreads / 32) * kVecBlock, end = p.K % 16 ? (p.V - 1) / kVecBlock * kVecBlock : p.V;
    long long v0 = (long long)(blockIdx.x * (kVecThreads / 32) + (tid >> 5)) * kVecBlock;
    for (; v0 < end; v0 += step) head_vec_block<kRows, T, false>(p, s_codes, chunks, v0, lane);
    if (v0 < p.V) head_vec_block<kRows, T, true>(p, s_codes, chunks, v0, lane);  // of a ragged K only: the block that starts at `end`
}

template <int kRows, typename T> static int launch_vec(VecParams p, int* status, cudaStream_t st) {
    p.status = status;
    const long long blocks = ((long long)p.V + kVecBlock * (kVecThreads / 32) - 1) / (kVecBlock * (kVecThreads / 32));
    const int sms = gemm::sm_count();
    if (sms <= 0) return TSLT_ERR_CUDA;
    const long long most = (long long)sms * 4;
    return gemm::launch_early(head_vec_kernel<kRows, T>, dim3((unsigned)(blocks < most ? blocks : most)), kVecThreads,
                              (size_t)kRows * ((p.K + 15) / 16 * 16), 1, st, p) == cudaSuccess
               ? TSLT_OK
               : TSLT_ERR_CUDA;
}

// Rows from which the tokens become the tensor cores' rows: few-rows / many-rows form, us, at V = 128256, K = 4096: 128 rows
// 101 / 110, 160 rows 109 / 112, 192 rows 116 / 115, 256 rows 133 / 117; K = 1024: 128 rows 49 / 52, 192 rows 60 / 57.  (The few-rows
// form has one tile of at most 256 columns, so there is nothing to compare behind 256 rows.  The many-rows form computes whole tiles
// of 256 rows: 257 rows cost what 512 do.)
constexpr int kManyRows = 161;

template <typename T>
static int launch_head(const signed char* q, const float* qs, long long q_stride, const signed char* w, const float* ws, long long w_stride,
                       int rows, int V, int K, T* out, long long out_stride, int* status, cudaStream_t st) {
    const int vec_rows = rows <= 2 ? rows : 4;
    if (rows <= 4 && vec_rows * K <= kVecCodes) {
        const VecParams v = {(const int8_t*)q, (const int8_t*)w, qs, ws, out, q_stride, w_stride, out_stride, rows, V, K};
        return vec_rows == 1 ? launch_vec<1, T>(v, status, st) : vec_rows == 2 ? launch_vec<2, T>(v, status, st) : launch_vec<4, T>(v, status, st);
    }
    gemm::Product p = {};
    p.splits = 1;
    p.k_elems = 128;
    p.k_blocks = (K + 127) / 128;
    p.status = status;
    p.clear_status = 1;
    gemm::Maps maps;
    if (rows >= kManyRows) {
        p.m_tiles = (rows + 255) / 256;
        p.nt = gemm::choose_nt(p.m_tiles, V, true, HeadRowsEpilogue<T>::kCols);
        p.n_tiles = (V + p.nt - 1) / p.nt;
        p.group_m = gemm::rows_in_l2(256, K);
        p.m_total = rows;
        typename HeadRowsEpilogue<T>::Params ep = {{}, out, out_stride, qs, ws, rows, V};
        const int step = 16 / sizeof(T);
        if (!gemm::encode_map(&maps.a, gemm::kElemInt8, q, K, rows, q_stride, 128) || !gemm::encode_map(&maps.b, gemm::kElemInt8, w, K, V, w_stride, p.nt / 2) ||
            !gemm::encode_map(&ep.out, sizeof(T) == 4 ? gemm::kElemFp32 : gemm::kElemBf16, out, V < step ? step : V / step * step, rows,
                              out_stride * (long long)sizeof(T), 32))
            return TSLT_ERR_CUDA;
        return gemm::launch<true, 2, 4, HeadRowsEpilogue<T>>(maps, p, ep, st);
    }
    p.nt = rows <= 16 ? 16 : (rows + 31) / 32 * 32;
    p.n_tiles = 1;
    p.m_tiles = (V + 127) / 128;
    p.group_m = 1;
    p.m_total = V;
    if (!gemm::encode_map(&maps.a, gemm::kElemInt8, w, K, V, w_stride, 128) || !gemm::encode_map(&maps.b, gemm::kElemInt8, q, K, rows, q_stride, p.nt)) return TSLT_ERR_CUDA;
    const typename HeadEpilogue<T>::Params ep = {out, out_stride, qs, ws, rows, V};
    return gemm::launch<true, 1, 8, HeadEpilogue<T>>(maps, p, ep, st);
}

}  // namespace tslt

using namespace tslt;

extern "C" int tslt_head_logits(const signed char* q, const float* q_scale, long long q_stride, const signed char* weight,
                                const float* weight_scale, long long weight_stride, int rows, int V, int D, int logits_dtype, void* logits,
                                long long logits_stride, void* workspace, size_t workspace_bytes, void* stream) {
    if (logits_dtype != TSLT_F32 && logits_dtype != TSLT_BF16) return TSLT_ERR_UNSUPPORTED;
    if (rows < 0 || V <= 0 || D <= 0) return TSLT_ERR_INVALID_ARG;
    if (D > TSLT_MAX_INT8_K || rows > TSLT_MAX_VOCAB || V > TSLT_MAX_VOCAB) return TSLT_ERR_UNSUPPORTED;
    if (rows == 0) return TSLT_OK;
    const int b = logits_dtype == TSLT_F32 ? 4 : 2;
    auto bad = [](const void* p, long long stride_bytes, long long row_bytes) {
        return !p || ((uintptr_t)p & 15) || stride_bytes < row_bytes || stride_bytes % 16;
    };
    if (bad(q, q_stride, D) || bad(weight, weight_stride, D) || bad(logits, logits_stride * b, (long long)V * b) || !q_scale || !weight_scale)
        return TSLT_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255)) return TSLT_ERR_INVALID_ARG;
    if (workspace_bytes < kWsHeaderBytes) return TSLT_ERR_WORKSPACE;
    int* status = (int*)workspace;
    cudaStream_t st = (cudaStream_t)stream;
    return b == 4 ? launch_head<float>(q, q_scale, q_stride, weight, weight_scale, weight_stride, rows, V, D, (float*)logits, logits_stride, status, st)
                  : launch_head<uint16_t>(q, q_scale, q_stride, weight, weight_scale, weight_stride, rows, V, D, (uint16_t*)logits, logits_stride,
                                          status, st);
}

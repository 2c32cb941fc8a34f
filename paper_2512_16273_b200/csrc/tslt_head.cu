// The head product in 8-bit integers (tslt_head_logits): z[n, v] = s_n t_v sum_k q[n, k] c[v, k].  The sum is exact (32-bit
// integers); the scales are multiplied in fp32 and the logit is rounded once.
//
// Few rows (a decoding step): bound by reading the weight once.  The weight is the operand of the tensor cores' 128 rows and
// the tokens are its columns (16 ... 128), so that the whole weight goes once through shared memory whatever their number.
//
// Many rows (verification, prompts): bound by the tensor cores.  The tokens are the rows, 256 of them to a pair of CTAs, and a
// lane of the epilogue holds 64 consecutive logits of a token, which leave through shared memory as whole 128-byte lines.
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
        const float wv = on ? __ldg(p.weight_scale + v) : 0.f;
        const int n = min(t.nt, p.rows - t.col0);
        for (int c = part * 32; c < n; c += kParts * 32) {
            uint32_t r[32];
            gemm::tmem_ld32(tmem + c, r);
            const float mine = c + lane < n ? __ldg(p.row_scale + t.col0 + c + lane) : 0.f;  // lane j: the scale of column c + j
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
        const float scale = row < p.n_rows ? __ldg(p.row_scale + row) : 0.f;
        constexpr int kStep = 16 / sizeof(T);
        const int whole = p.V / kStep * kStep;
        for (int c = part * kCols; c < t.nt && t.col0 + c < p.V; c += kParts * kCols) {
            const int v0 = t.col0 + c;
            // the columns' scales, a copy for each warp: 64 shuffles or loads would cost more than 16 reads of shared memory
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kCols; i += 32) {
                const float w = v0 + i + lane < p.V ? __ldg(p.weight_scale + v0 + i + lane) : 0.f;
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
            if (lane == 0) gemm::store_wait_read<1>();  // the last copy but one, which was of this box, has read it
            __syncwarp();
            const uint32_t box = own.next(), line = box + lane * 128;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(line + ((i ^ (lane & 7)) << 4)), "r"(b[4 * i]), "r"(b[4 * i + 1]),
                             "r"(b[4 * i + 2]), "r"(b[4 * i + 3])
                             : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0 && row < p.n_rows && v0 < whole) gemm::store_box(&p.out, box, v0, row);
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

// Rows from which the tokens become the tensor cores' rows.
constexpr int kManyRows = 129;

template <typename T>
static int launch_head(const signed char* q, const float* qs, long long q_stride, const signed char* w, const float* ws, long long w_stride,
                       int rows, int V, int K, T* out, long long out_stride, int* status, cudaStream_t st) {
    gemm::Product p = {};
    p.splits = 1;
    p.k_elems = 128;
    p.k_blocks = (K + 127) / 128;
    p.status = status;
    p.clear_status = 1;
    CUtensorMap ta, tb;
    if (rows >= kManyRows) {
        p.m_tiles = (rows + 255) / 256;
        p.nt = gemm::choose_nt(p.m_tiles, V, true, HeadRowsEpilogue<T>::kCols);
        p.n_tiles = (V + p.nt - 1) / p.nt;
        p.group_m = 16;
        p.m_total = rows;
        typename HeadRowsEpilogue<T>::Params ep = {{}, out, out_stride, qs, ws, rows, V};
        const int step = 16 / sizeof(T);
        if (!gemm::encode_map(&ta, gemm::kElemInt8, q, K, rows, q_stride, 128) || !gemm::encode_map(&tb, gemm::kElemInt8, w, K, V, w_stride, p.nt / 2) ||
            !gemm::encode_map(&ep.out, sizeof(T) == 4 ? gemm::kElemFp32 : gemm::kElemBf16, out, V < step ? step : V / step * step, rows,
                              out_stride * (long long)sizeof(T), 32))
            return TSLT_ERR_CUDA;
        return gemm::launch<true, 2, 4, HeadRowsEpilogue<T>>(ta, tb, p, ep, false, st);
    }
    p.nt = rows <= 16 ? 16 : (rows + 31) / 32 * 32;
    p.n_tiles = 1;
    p.m_tiles = (V + 127) / 128;
    p.group_m = 1;
    p.m_total = V;
    if (!gemm::encode_map(&ta, gemm::kElemInt8, w, K, V, w_stride, 128) || !gemm::encode_map(&tb, gemm::kElemInt8, q, K, rows, q_stride, p.nt)) return TSLT_ERR_CUDA;
    const typename HeadEpilogue<T>::Params ep = {out, out_stride, qs, ws, rows, V};
    return gemm::launch<true, 1, 8, HeadEpilogue<T>>(ta, tb, p, ep, false, st);
}

}  // namespace tslt

using namespace tslt;

extern "C" int tslt_head_logits(const signed char* q, const float* q_scale, long long q_stride, const signed char* weight,
                                const float* weight_scale, long long weight_stride, int rows, int V, int D, int logits_dtype, void* logits,
                                long long logits_stride, void* workspace, size_t workspace_bytes, void* stream) {
    if (logits_dtype != TSLT_F32 && logits_dtype != TSLT_BF16) return TSLT_ERR_UNSUPPORTED;
    if (rows < 0 || V <= 0 || D <= 0) return TSLT_ERR_INVALID_ARG;
    if (D > TSLT_MAX_INT8_K) return TSLT_ERR_UNSUPPORTED;
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

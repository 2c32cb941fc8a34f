// The head product in 8-bit integers (tslt_head_logits): z[n, v] = s_n t_v sum_k q[n, k] c[v, k].
//
// The weight is the operand of the tensor cores' 128 rows and the tokens are its columns: a decoding step has few tokens
// (16 ... 256 columns), so the whole weight goes once through shared memory whatever their number, and a warp's lanes hold
// consecutive vocabulary entries of one token, which is how the logits lie in memory.  The sum is exact (32-bit integers);
// the scales are multiplied in fp32 and the logit is rounded once.
#include "tslt_gemm.cuh"

namespace tslt {

template <typename T> struct HeadEpilogue {
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
    static __device__ __forceinline__ void run(const Params& p, uint32_t tmem, bool, const gemm::Tile& t, int v, int lane, int part) {
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

template <typename T>
static int launch_head(const signed char* q, const float* qs, long long q_stride, const signed char* w, const float* ws, long long w_stride,
                       int rows, int V, int K, T* out, long long out_stride, int* status, cudaStream_t st) {
    gemm::Product p = {};
    const bool pair = rows > 64;
    const int unit = 32;
    p.n_tiles = (rows + 255) / 256;
    p.nt = ((rows + p.n_tiles - 1) / p.n_tiles + unit - 1) / unit * unit;
    if (rows <= 16) p.nt = 16;
    const int tile_rows = pair ? 256 : 128;
    p.m_tiles = (V + tile_rows - 1) / tile_rows;
    p.splits = 1;
    p.k_elems = 128;
    p.k_blocks = (K + 127) / 128;
    p.group_m = 1;
    p.m_total = V;
    p.status = status;
    p.clear_status = 1;
    CUtensorMap ta, tb;
    if (!gemm::encode_map(&ta, true, w, K, V, w_stride, 128) || !gemm::encode_map(&tb, true, q, K, rows, q_stride, pair ? p.nt / 2 : p.nt))
        return TSLT_ERR_CUDA;
    const typename HeadEpilogue<T>::Params ep = {out, out_stride, qs, ws, rows, V};
    return pair ? gemm::launch<true, 2, 8, HeadEpilogue<T>>(ta, tb, p, ep, st) : gemm::launch<true, 1, 8, HeadEpilogue<T>>(ta, tb, p, ep, st);
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

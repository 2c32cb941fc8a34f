// RMS norm with the residual's addition and an 8-bit output (tslt_rmsnorm_quant), and the same quantiser
// without the norm (tslt_quantize_rows).
//
// Mathematics.  h = x + r in the storage type; v = h w; the normalised row is y = v / rms(h), and its codes are
// q = rint(127 y / max|y|) with scale = max|y| / 127.  The row's 1 / rms cancels out of q: q = rint(127 v / max|v|).
// So the sum of squares and the maximum are needed from ONE pass over the row and one block reduction gives both;
// the row stays in registers between them and is read and written once: 2 + 2 + 2 + 1 bytes an element (bf16 with a
// residual).  Bound by HBM once the arithmetic was on pairs: 16384 x 4096 takes 80 us (5.8 TB/s), with values 94 us
// (6.5 TB/s, 0.98 of the copy bandwidth; outputs reused from call to call); element by element it was 113 us at 42
// instructions an element, and 102 us with 76 registers a thread instead of 64 (six CTAs of 128 threads on an SM instead of
// eight).  fp32: 126 us, 6.9 TB/s.  The quantiser on a 128256 x 4096 weight: fp32 426 us (6.2 TB/s), bf16 472 us (3.3 TB/s: 0.6 of
// the bytes, as many instructions).
//
// Rounding.  t = v * (127 / max|v|) in fp32 is off by at most 1.5 * 2^-23 * 127 = 2.3e-5; where t lies within 1e-4 of
// the border between two codes (one element in 5000), the code is taken from the quotient in fp64 instead, so that
// every code is the nearest one to the exact quotient of the fp32 values v and max|v|.  (For bf16 h and w the product
// v is exact.)  Rows whose sum of squares leaves fp32's range take it in fp64, from a second reading of the row.
#include "tslt_gemm.cuh"

namespace tslt {

struct NormParams {
    const void *x, *r, *w;  // r, w may be null
    void* h;                // may be null; may equal x or r
    uint16_t* y;            // may be null: q * scale in bf16
    int8_t* q;
    float* scale;
    long long xs, rs, hs, ys, qs;  // row strides in elements
    int rows, D;
    float eps;
};

// ---- pairs of fp32: one instruction for two elements (the kernel is bound by instructions before it is bound by memory) ----
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ float lo_of(Pair p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float hi_of(Pair p) { return __uint_as_float((uint32_t)(p >> 32)); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// The largest of |a|, |b| and |c|; a NaN among them is the result (fmaxf drops it).
__device__ __forceinline__ float top3(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {  // lo in the low half
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// A 16-byte vector as pairs, and back (values that came from the storage type).
template <typename T> __device__ __forceinline__ void to_pairs(const uint4& v, Pair* z);
template <> __device__ __forceinline__ void to_pairs<float>(const uint4& v, Pair* z) {
    z[0] = pair(__uint_as_float(v.x), __uint_as_float(v.y));
    z[1] = pair(__uint_as_float(v.z), __uint_as_float(v.w));
}
template <> __device__ __forceinline__ void to_pairs<bf16_t>(const uint4& v, Pair* z) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
// x + r rounded to the storage type, as a vector.
template <typename T> __device__ __forceinline__ uint4 add_vec(const uint4& x, const uint4& r);
template <> __device__ __forceinline__ uint4 add_vec<float>(const uint4& x, const uint4& r) {
    return make_uint4(__float_as_uint(__fadd_rn(__uint_as_float(x.x), __uint_as_float(r.x))), __float_as_uint(__fadd_rn(__uint_as_float(x.y), __uint_as_float(r.y))),
                      __float_as_uint(__fadd_rn(__uint_as_float(x.z), __uint_as_float(r.z))), __float_as_uint(__fadd_rn(__uint_as_float(x.w), __uint_as_float(r.w))));
}
template <> __device__ __forceinline__ uint4 add_vec<bf16_t>(const uint4& x, const uint4& r) {
    Pair a[4], b[4];
    to_pairs<bf16_t>(x, a);
    to_pairs<bf16_t>(r, b);
    uint32_t d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Pair t = add2(a[i], b[i]);
        d[i] = pack_bf16x2(lo_of(t), hi_of(t));
    }
    return make_uint4(d[0], d[1], d[2], d[3]);
}

// Adding 1.5 * 2^23 rounds to the nearest integer, ties to even, at the rate of an addition (the conversion instructions
// run at an eighth of it), and leaves the integer's two's complement in the low bits.
constexpr float kRounder = 12582912.f;
// The exact codes of P values, as bytes.
template <int P> __device__ __noinline__ Pair exact_codes(Pair a, Pair b, Pair c, Pair d, float top) {
    const Pair z[4] = {a, b, c, d};
    Pair bytes = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const double e = rint(127.0 * (double)(i & 1 ? hi_of(z[i / 2]) : lo_of(z[i / 2])) / (double)top);
        const int code = e == e ? (int)fmin(fmax(e, -127.0), 127.0) : 0;
        bytes |= (Pair)(uint8_t)code << (8 * i);
    }
    return bytes;
}

// The vector of elements [at, at + kPerVec) of a row of D; past the row's end (its last vector may be short) zeros.
template <typename T> __device__ __forceinline__ uint4 load_elems(const void* row, int at, int D) {
    constexpr int P = Elt<T>::kPerVec;
    const char* p = (const char*)row + (size_t)at * Elt<T>::kBytes;
    if (at + P <= D) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (at + i < D) {
            if (Elt<T>::kBytes == 4) w[i & 3] = reinterpret_cast<const uint32_t*>(p)[i];
            else w[(i / 2) & 3] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T> __device__ __forceinline__ void store_elems(void* row, int at, int D, const uint4& v) {
    constexpr int P = Elt<T>::kPerVec;
    char* p = (char*)row + (size_t)at * Elt<T>::kBytes;
    if (at + P <= D) {
        *reinterpret_cast<uint4*>(p) = v;
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (at + i < D) {
                if (Elt<T>::kBytes == 4) reinterpret_cast<uint32_t*>(p)[i] = w[i & 3];
                else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[(i / 2) & 3] >> (16 * (i & 1)));
            }
        }
    }
}

// The sum of squares of h over vectors t, t + nth, ... of a row, in fp64: for rows whose fp32 sum overflows or loses its small squares.
// h is read again, from where this thread stored it or from x and r.
template <typename T> __device__ __noinline__ double far_squares(const NormParams& p, long long row, int t, int nth) {
    constexpr int P = Elt<T>::kPerVec;
    const char* x = p.h ? (const char*)p.h + row * p.hs * Elt<T>::kBytes : (const char*)p.x + row * p.xs * Elt<T>::kBytes;
    const char* r = !p.h && p.r ? (const char*)p.r + row * p.rs * Elt<T>::kBytes : nullptr;
    double sum = 0.0;
    for (int at = t * P; at < p.D; at += nth * P) {
        uint4 h = load_elems<T>(x, at, p.D);
        if (r) h = add_vec<T>(h, load_elems<T>(r, at, p.D));
        Pair z[P / 2];
        to_pairs<T>(h, z);
#pragma unroll
        for (int i = 0; i < P / 2; ++i) sum += (double)lo_of(z[i]) * lo_of(z[i]) + (double)hi_of(z[i]) * hi_of(z[i]);
    }
    return warp_sum(sum);
}

// A row is a CTA's, or (kWarpRow, narrow rows) a warp's with nothing to meet for; thread t of it holds vectors t, t + nthreads, ... (NV of them).
template <typename T, int NV, bool kNorm, bool kWarpRow>
__global__ void __launch_bounds__(NV * Elt<T>::kPerVec == 32 ? 512 : 1024, NV * Elt<T>::kPerVec == 32 ? 2 : 0) norm_quant_kernel(const __grid_constant__ NormParams p) {
    constexpr int P = Elt<T>::kPerVec;
    __shared__ float s_sum[32], s_top[32];
    wait_for_primary_kernel();
    allow_dependent_launch();
    const int tid = kWarpRow ? threadIdx.x & 31 : threadIdx.x, nth = kWarpRow ? 32 : blockDim.x, nwarps = nth >> 5;
    const long long row = kWarpRow ? (long long)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    if (kWarpRow && row >= p.rows) return;
    const char* x = (const char*)p.x + row * p.xs * Elt<T>::kBytes;
    const char* r = p.r ? (const char*)p.r + row * p.rs * Elt<T>::kBytes : nullptr;
    uint4 xv[NV], rv[NV], wv[NV];  // every load of the row is in flight before the first is used
#pragma unroll
    for (int j = 0; j < NV; ++j) xv[j] = load_elems<T>(x, (tid + j * nth) * P, p.D);
    if (kNorm && r) {
#pragma unroll
        for (int j = 0; j < NV; ++j) rv[j] = load_elems<T>(r, (tid + j * nth) * P, p.D);
    }
    if (kNorm && p.w) {
#pragma unroll
        for (int j = 0; j < NV; ++j) wv[j] = load_elems<T>(p.w, (tid + j * nth) * P, p.D);
    }
    if (kNorm && r) {
#pragma unroll
        for (int j = 0; j < NV; ++j) xv[j] = add_vec<T>(xv[j], rv[j]);
    }
    if (kNorm && p.h) {
        char* h = (char*)p.h + row * p.hs * Elt<T>::kBytes;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int at = (tid + j * nth) * P;
            if (at < p.D) store_elems<T>(h, at, p.D, xv[j]);
        }
    }
    Pair v[NV][P / 2], squares = pair(0.f, 0.f);
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        to_pairs<T>(xv[j], v[j]);
        if (kNorm) {
#pragma unroll
            for (int i = 0; i < P / 2; ++i) squares = fma2(v[j][i], v[j][i], squares);
        }
        if (kNorm && p.w) {
            Pair w[P / 2];
            to_pairs<T>(wv[j], w);
#pragma unroll
            for (int i = 0; i < P / 2; ++i) v[j][i] = mul2(v[j][i], w[i]);
        }
#pragma unroll
        for (int i = 0; i < P / 2; ++i) top = top3(top, lo_of(v[j][i]), hi_of(v[j][i]));
    }
    float sum = kNorm ? warp_sum(lo_of(squares) + hi_of(squares)) : 0.f;
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));  // not negative: ordered as integers, a NaN above all
    if (!kWarpRow) {
        if ((tid & 31) == 0) {
            s_sum[tid >> 5] = sum;
            s_top[tid >> 5] = top;
        }
        __syncthreads();
        sum = 0.f;
        top = 0.f;
        for (int w = 0; w < nwarps; ++w) {  // the same order in every thread
            sum += s_sum[w];
            top = top3(top, s_top[w], 0.f);
        }
    }
    float s = top / 127.f;
    if (kNorm) {
        const float mean = sum / (float)p.D + p.eps;
        s = top == 0.f ? 0.f : s / sqrtf(mean);
        // below 2^-100 the squares that fp32 rounds to steps of 2^-149 could count (the same in every thread of the row)
        if (top > 0.f && top < INFINITY && !(mean >= 0x1p-100f && mean < INFINITY)) {
            double all = far_squares<T>(p, row, tid, nth);
            if (!kWarpRow) {
                __shared__ double s_far[32];
                if ((tid & 31) == 0) s_far[tid >> 5] = all;
                __syncthreads();
                all = 0.0;
                for (int w = 0; w < nwarps; ++w) all += s_far[w];
            }
            s = (float)((double)top / 127.0 / sqrt(all / p.D + (double)p.eps));
        }
    }
    if (!(top < INFINITY)) s = NAN;  // a NaN or an infinity in the row (top is one whatever the weight) or in the weight
    if (tid == 0) p.scale[row] = s;
    const float inv = top > 0.f ? 127.f / top : 0.f;
    // a row with a NaN or an infinity in it, or so large or small that inv leaves the range, takes the fp64 quotient throughout
    const bool odd = !(inv < 3e38f) || !(top < 3e38f);
    int8_t* q = p.q + row * p.qs;
    const Pair inv2 = pair(inv, inv), up = pair(kRounder, kRounder), down = pair(-kRounder, -kRounder), minus = pair(-1.f, -1.f), s2 = pair(s, s);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int at = (tid + j * nth) * P;
        if (at >= p.D) break;
        Pair c[P / 2];
        uint32_t b[P / 4];
        float border = 0.f;
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
            const Pair t = mul2(v[j][i], inv2), r = add2(t, up);
            c[i] = add2(r, down);
            const Pair d = fma2(c[i], minus, t);
            border = fmaxf(border, fmaxf(fabsf(lo_of(d)), fabsf(hi_of(d))));
            const uint32_t two = __byte_perm(__float_as_uint(lo_of(r)), __float_as_uint(hi_of(r)), 0x0040);
            b[i / 2] = i & 1 ? __byte_perm(b[i / 2], two, 0x5410) : two;
        }
        if (odd || border >= 0.4999f) {
            const Pair e = exact_codes<P>(v[j][0], v[j][1], v[j][P / 2 - 2], v[j][P / 2 - 1], top);
            b[0] = (uint32_t)e;
            if (P == 8) b[P / 4 - 1] = (uint32_t)(e >> 32);
#pragma unroll
            for (int i = 0; i < P / 2; ++i) c[i] = pair((float)(int8_t)(e >> (16 * i)), (float)(int8_t)(e >> (16 * i + 8)));
        }
        if (at + P <= p.D) {
            if (P == 8) *reinterpret_cast<uint2*>(q + at) = make_uint2(b[0], b[P / 4 - 1]);
            else *reinterpret_cast<uint32_t*>(q + at) = b[0];
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (at + i < p.D) q[at + i] = (int8_t)(b[i / 4] >> (8 * (i % 4)));
        }
        if (kNorm && p.y) {
            uint16_t* y = p.y + row * p.ys + at;
            uint32_t o[P / 2];
#pragma unroll
            for (int i = 0; i < P / 2; ++i) {
                const Pair z = mul2(c[i], s2);
                o[i] = pack_bf16x2(lo_of(z), hi_of(z));
            }
            if (at + P <= p.D) {
                if (P == 8) *reinterpret_cast<uint4*>(y) = make_uint4(o[0], o[1], o[P / 2 - 2], o[P / 2 - 1]);
                else *reinterpret_cast<uint2*>(y) = make_uint2(o[0], o[1]);
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i)
                    if (at + i < p.D) y[i] = (uint16_t)(o[i / 2] >> (16 * (i % 2)));
            }
        }
    }
}

constexpr int kMaxHidden = TSLT_MAX_HIDDEN;

template <typename T, bool kNorm> static int launch_norm(const NormParams& p, cudaStream_t st) {
    const int nvec = (p.D + Elt<T>::kPerVec - 1) / Elt<T>::kPerVec;
    // Few rows: latency counts, so a row is spread over as many threads as it has vectors.  Rows enough to fill the
    // machine: four vectors in flight per thread where a row has 512 (16384 x 4096, us, 1 / 2 / 4 vectors: bf16 118 / 107 / 95,
    // fp32 329 / 185 / 150).
    const bool many = p.rows >= 2 * 148;
    if (many && nvec <= 128) {  // a warp holds the row: no barrier, and a quarter of the CTAs to start (16384 x 512 bf16: 18.1 -> 14.6 us; the
    // warp's one row leaves nothing in flight during its arithmetic)
        auto kern = nvec > 64 ? norm_quant_kernel<T, 4, kNorm, true> : nvec > 32 ? norm_quant_kernel<T, 2, kNorm, true> : norm_quant_kernel<T, 1, kNorm, true>;
        return gemm::launch_early(kern, dim3((p.rows + 3) / 4), 128, 0, 1, st, p) == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
    }
    int nv = !many ? 1 : nvec >= 512 ? 4 : nvec >= 256 ? 2 : 1;
    while ((nvec + nv - 1) / nv > 1024) nv *= 2;
    const int threads = ((nvec + nv - 1) / nv + 31) / 32 * 32;
    auto kern = nv == 1 ? norm_quant_kernel<T, 1, kNorm, false> : nv == 2 ? norm_quant_kernel<T, 2, kNorm, false> : norm_quant_kernel<T, 4, kNorm, false>;
    return gemm::launch_early(kern, dim3(p.rows), threads, 0, 1, st, p) == cudaSuccess ? TSLT_OK : TSLT_ERR_CUDA;
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
static int elt_bytes(int dtype) { return dtype == TSLT_F32 ? 4 : 2; }
static bool row_ok(const void* p, long long stride, int D, int bytes) {
    return p && aligned16(p) && stride >= D && stride * bytes % 16 == 0;
}

}  // namespace tslt

using namespace tslt;

extern "C" int tslt_rmsnorm_quant(const void* x, const void* residual, const void* weight, int dtype, int rows, int D,
                                  long long x_stride, long long residual_stride, float eps, void* residual_out,
                                  long long out_stride, void* values, long long values_stride, signed char* q, long long q_stride,
                                  float* scale, void* stream) {
    if (dtype != TSLT_F32 && dtype != TSLT_BF16) return TSLT_ERR_UNSUPPORTED;
    if (rows < 0 || D <= 0 || !(eps >= 0.f)) return TSLT_ERR_INVALID_ARG;
    if (D > kMaxHidden) return TSLT_ERR_UNSUPPORTED;
    if (rows == 0) return TSLT_OK;
    const int b = elt_bytes(dtype);
    if (!row_ok(x, x_stride, D, b) || !row_ok(q, q_stride, D, 1) || !scale) return TSLT_ERR_INVALID_ARG;
    if (residual && !row_ok(residual, residual_stride, D, b)) return TSLT_ERR_INVALID_ARG;
    if (residual_out && !row_ok(residual_out, out_stride, D, b)) return TSLT_ERR_INVALID_ARG;
    if (rows > 1 && residual_out && ((residual_out == x && out_stride != x_stride) || (residual_out == residual && out_stride != residual_stride)))
        return TSLT_ERR_INVALID_ARG;  // a row would go over another that is still to be read
    if (values && !row_ok(values, values_stride, D, 2)) return TSLT_ERR_INVALID_ARG;
    if (weight && !aligned16(weight)) return TSLT_ERR_INVALID_ARG;
    NormParams p = {x, residual, weight, residual_out, (uint16_t*)values, (int8_t*)q, scale, x_stride, residual_stride, out_stride,
                    values_stride, q_stride, rows, D, eps};
    return dtype == TSLT_F32 ? launch_norm<float, true>(p, (cudaStream_t)stream)
                             : launch_norm<bf16_t, true>(p, (cudaStream_t)stream);
}

extern "C" int tslt_quantize_rows(const void* x, int dtype, int rows, int D, long long x_stride, signed char* q,
                                  long long q_stride, float* scale, void* stream) {
    if (dtype != TSLT_F32 && dtype != TSLT_BF16) return TSLT_ERR_UNSUPPORTED;
    if (rows < 0 || D <= 0) return TSLT_ERR_INVALID_ARG;
    if (D > kMaxHidden) return TSLT_ERR_UNSUPPORTED;
    if (rows == 0) return TSLT_OK;
    if (!row_ok(x, x_stride, D, elt_bytes(dtype)) || !row_ok(q, q_stride, D, 1) || !scale) return TSLT_ERR_INVALID_ARG;
    NormParams p = {x, nullptr, nullptr, nullptr, nullptr, (int8_t*)q, scale, x_stride, 0, 0, 0, q_stride, rows, D, 0.f};
    return dtype == TSLT_F32 ? launch_norm<float, false>(p, (cudaStream_t)stream)
                             : launch_norm<bf16_t, false>(p, (cudaStream_t)stream);
}

// Row normalisation with weight, bias and SiLU gate, forward and backward: what follows the layer's output in a model (rows of a head's
// features, RMS, gated) and the layer norm of its blocks (rows of the model's width, mean and variance).
//
//     n = (x - mean) rstd   (GDN_NORM_RMS: mean = 0),   h = n w + b,   y = h silu(z)
//     dh = dy silu(z),  dz = dy h silu'(z),  dw = sum_rows dh n,  db = sum_rows dh,
//     dn = dh w,        dx = rstd (dn - mean(dn) - n mean(dn n))         (GDN_NORM_RMS: without mean(dn))
//
// What bounds it: HBM; every input is read once and every output written once. A row stays in registers between its load and its
// store: 8 elements (16 bytes of bf16) a thread and vector, TPR threads a row, NV vectors a thread. The statistics are taken from the
// registers, the mean first and then the squared distances from it, so nothing cancels. The backward pass forms the statistics again from x, which
// it has to read anyway, instead of reading stored ones. A CTA walks many rows, so that weight and bias are read once per CTA, and in the
// backward pass their gradients stay in registers until the CTA's last row; the CTAs' sums are added by a second small launch in a fixed
// order: the result does not depend on timing.
#include "common.cuh"
#include "sm100_ptx.cuh"

namespace gdn {
namespace {

using namespace sm100;

struct ParamsN {
    const void *dy, *x, *weight, *bias, *gate;  // weight, bias, gate may be null
    void *y, *dx, *dgate;
    float* partial;  // backward: [CTAs][2][width], sums of dw and db
    long long rows;
    int width;
    float eps, inv_width;
    bool rms, param_bf16, want_db;
};

// 8 elements of a row, as they are stored. They are worked on as four packed pairs: the arithmetic is what bounds the kernels beside the HBM.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void get(f2 (&x)[4]) const {
        x[0] = pair2(bf16_lo(w.x), bf16_hi(w.x)), x[1] = pair2(bf16_lo(w.y), bf16_hi(w.y));
        x[2] = pair2(bf16_lo(w.z), bf16_hi(w.z)), x[3] = pair2(bf16_lo(w.w), bf16_hi(w.w));
    }
    __device__ __forceinline__ void set(const f2 (&x)[4]) {
        float a[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpair2(x[i], a[2 * i], a[2 * i + 1]);
        w = make_uint4(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(a[4], a[5]), pack_bf16x2(a[6], a[7]));
    }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void get(f2 (&x)[4]) const { x[0] = pair2(a.x, a.y), x[1] = pair2(a.z, a.w), x[2] = pair2(b.x, b.y), x[3] = pair2(b.z, b.w); }
    __device__ __forceinline__ void set(const f2 (&x)[4]) {
        unpair2(x[0], a.x, a.y), unpair2(x[1], a.z, a.w);
        unpair2(x[2], b.x, b.y), unpair2(x[3], b.z, b.w);
    }
};
__device__ __forceinline__ f2 both(float x) { return pair2(x, x); }
__device__ __forceinline__ float sum2(f2 x) {
    float a, b;
    unpair2(x, a, b);
    return a + b;
}
__device__ __forceinline__ float one(const float* p) { return *p; }
__device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Vector `col .. col + 7` of a row that starts at `row`; elements past the width are zeros. VEC: width a multiple of 8, so every
// vector is whole and aligned; else element by element.
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load8(const T* row, int col, int width, bool active) {
    Raw8<T> r;
    if (VEC && active && col < width) {
        r = *reinterpret_cast<const Raw8<T>*>(row + col);
    } else {
        f2 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = VEC ? both(0.f) : pair2(active && col + 2 * i < width ? one(row + col + 2 * i) : 0.f, active && col + 2 * i + 1 < width ? one(row + col + 2 * i + 1) : 0.f);
        r.set(x);
    }
    return r;
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* row, int col, int width, bool active, const f2 (&x)[4]) {
    if (VEC) {
        if (active && col < width) {
            Raw8<T> r;
            r.set(x);
            *reinterpret_cast<Raw8<T>*>(row + col) = r;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b;
            unpair2(x[i], a, b);
            if (active && col + 2 * i < width) put(row + col + 2 * i, a);
            if (active && col + 2 * i + 1 < width) put(row + col + 2 * i + 1, b);
        }
    }
}
// 8 elements of weight or bias (fp32 or bf16), `none` where there is no such tensor. They are fetched again for every row (from L1), and volatile,
// so that they do not take registers that rows in flight can use: 128 features, backward, 80 registers instead of 96.
template <bool VEC>
__device__ __forceinline__ void load_param(const void* p, bool bf16, int col, int width, float none, f2 (&x)[4]) {
    if (p == nullptr || col >= width) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = both(none);
    } else if (VEC && bf16) {
        Raw8<__nv_bfloat16> r;
        asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w.x), "=r"(r.w.y), "=r"(r.w.z), "=r"(r.w.w) : "l"(static_cast<const __nv_bfloat16*>(p) + col));
        r.get(x);
    } else if (VEC) {
        const float* const q = static_cast<const float*>(p) + col;
        asm volatile("ld.global.nc.v2.u64 {%0,%1}, [%2];" : "=l"(x[0]), "=l"(x[1]) : "l"(q));
        asm volatile("ld.global.nc.v2.u64 {%0,%1}, [%2];" : "=l"(x[2]), "=l"(x[3]) : "l"(q + 4));
    } else {
        const auto at = [&](int c) { return c >= width ? none : bf16 ? one(static_cast<const __nv_bfloat16*>(p) + c) : one(static_cast<const float*>(p) + c); };
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = pair2(at(col + 2 * i), at(col + 2 * i + 1));
    }
}

// Sums of N values over the TPR threads of a row. TPR > 32 (the whole CTA): through `box`, of which two calls in a row use
// different halves, so that one barrier a call is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float2* box, int& turn) {
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], o);
    if (TPR > 32) {
        constexpr int W = TPR / 32;
        float2* const half = box + turn * W;
        turn ^= 1;
        if (threadIdx.x % 32 == 0) half[threadIdx.x / 32] = make_float2(x[0], x[N - 1]);
        __syncthreads();
        f2 s = both(0.f);
#pragma unroll
        for (int i = 0; i < W; ++i) s = add2(s, *reinterpret_cast<const f2*>(half + i));
        float a, b;
        unpair2(s, a, b);
        x[0] = a;
        if (N == 2) x[N - 1] = b;
    }
}

// sigmoid. bf16 rows: four instructions (a product, 2^x, a sum, a reciprocal, the last ones within 2 ulp); exp(-z) = inf gives 0. The gate's
// arithmetic is what the forward kernel issues most of: with __expf and __fdividef 147 us for 1 M rows of 128, so 139. The exponent is rounded before
// 2^x is taken, 2^-18 where |z| is near 80, and log2(e) is: up to 3.8e-6 of the result, a thousandth of its rounding to bf16. fp32 rows: expf, whose
// error is of the result alone (512 K rows of 128, forward / backward: 144 / 218 us, so 140 / 216; with a division too 163 / 259).
template <typename T>
__device__ __forceinline__ float sigmoid(float z) {
    float e, r;
    if (sizeof(T) == 4) e = expf(-z);
    else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}
template <typename T>
__device__ __forceinline__ f2 sigmoid2(f2 z) {
    float a, b;
    unpair2(z, a, b);
    return pair2(sigmoid<T>(a), sigmoid<T>(b));
}

constexpr int kNormThreads = 256;
template <int TPR>
__host__ __device__ constexpr int cta_threads() { return TPR > 32 ? TPR : kNormThreads; }

// The row's values less their mean (past the width: zeros), and one over their deviation
template <typename T, int NV, int TPR, bool VEC>
__device__ __forceinline__ float centred(const Raw8<T> (&raw)[NV], f2 (&x)[NV][4], int t, const ParamsN& p, float2* box, int& turn) {
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v].get(x[v]);
    if (!p.rms) {
#pragma unroll
        for (int v = 0; v < NV; ++v) s[0] += sum2(add2(add2(x[v][0], x[v][1]), add2(x[v][2], x[v][3])));
        row_sums<TPR>(s, box, turn);
        const float mean = s[0] * p.inv_width;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * TPR + t) * 8;
            if (VEC) {
                if (col < p.width) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[v][i] = add2(x[v][i], both(-mean));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[v][i] = add2(x[v][i], pair2(col + 2 * i < p.width ? -mean : 0.f, col + 2 * i + 1 < p.width ? -mean : 0.f));
            }
        }
    }
    f2 q = both(0.f);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) q = fma2(x[v][i], x[v][i], q);
    s[0] = sum2(q);
    row_sums<TPR>(s, box, turn);
    return rsqrtf(s[0] * p.inv_width + p.eps);
}

// N rows' worth of a tensor's vectors for this thread: those of `row`
template <typename T, int NV, int TPR, bool VEC>
__device__ __forceinline__ void load_row(Raw8<T> (&raw)[NV], const void* base, long long row, const ParamsN& p, int t) {
    const bool active = row < p.rows;
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = load8<T, VEC>(static_cast<const T*>(base) + (active ? row : 0) * p.width, (v * TPR + t) * 8, p.width, active);
}

// A thread asks for its next row before it works on the present one.
template <typename T, int NV, int TPR, bool VEC>
__global__ void __launch_bounds__(cta_threads<TPR>()) norm_forward_kernel(const ParamsN p) {
    constexpr int G = cta_threads<TPR>() / TPR;  // rows that a CTA has at a time
    __shared__ float2 box[2 * (TPR > 32 ? TPR / 32 : 1)];
    const int t = threadIdx.x % TPR;
    const long long step = static_cast<long long>(gridDim.x) * G;
    int turn = 0;
    Raw8<T> next[NV], next_gate[NV];
    long long row = static_cast<long long>(blockIdx.x) * G + threadIdx.x / TPR;
    load_row<T, NV, TPR, VEC>(next, p.x, row, p, t);
    if (p.gate != nullptr) load_row<T, NV, TPR, VEC>(next_gate, p.gate, row, p, t);
    for (long long first = static_cast<long long>(blockIdx.x) * G; first < p.rows; first += step, row += step) {
        const bool active = row < p.rows;
        const long long at = (active ? row : 0) * p.width;
        Raw8<T> raw[NV], gate[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = next[v], gate[v] = next_gate[v];
        if (first + step < p.rows) {
            load_row<T, NV, TPR, VEC>(next, p.x, row + step, p, t);
            if (p.gate != nullptr) load_row<T, NV, TPR, VEC>(next_gate, p.gate, row + step, p, t);
        }
        f2 x[NV][4];
        const f2 rstd = both(centred<T, NV, TPR, VEC>(raw, x, t, p, box, turn));
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            f2 w[4];
            load_param<VEC>(p.weight, p.param_bf16, (v * TPR + t) * 8, p.width, 1.f, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[v][i] = mul2(mul2(x[v][i], rstd), w[i]);
            if (p.bias != nullptr) {
                load_param<VEC>(p.bias, p.param_bf16, (v * TPR + t) * 8, p.width, 0.f, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[v][i] = add2(x[v][i], w[i]);
            }
            if (p.gate != nullptr) {
                f2 z[4];
                gate[v].get(z);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[v][i] = mul2(x[v][i], mul2(z[i], sigmoid2<T>(z[i])));
            }
            store8<T, VEC>(static_cast<T*>(p.y) + at, (v * TPR + t) * 8, p.width, active, x[v]);
        }
    }
}

template <typename T, int NV, int TPR, bool VEC>
__global__ void __launch_bounds__(cta_threads<TPR>(), NV == 1 && sizeof(T) == 2 ? 768 / cta_threads<TPR>() : 1) norm_backward_kernel(const ParamsN p) {
    constexpr int G = cta_threads<TPR>() / TPR;
    constexpr int kColumns = NV * TPR * 8;
    __shared__ float2 box[2 * (TPR > 32 ? TPR / 32 : 1)];
    __shared__ float gather[G > 1 ? G * kColumns : 1];
    const int t = threadIdx.x % TPR;
    int turn = 0;
    f2 dw[NV][4], db[NV][4];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[v][i] = db[v][i] = both(0.f);
    const long long step = static_cast<long long>(gridDim.x) * G;
    Raw8<T> next[NV], next_gate[NV], next_up[NV];
    long long row = static_cast<long long>(blockIdx.x) * G + threadIdx.x / TPR;
    const auto ask = [&](long long r) {
        load_row<T, NV, TPR, VEC>(next, p.x, r, p, t);
        load_row<T, NV, TPR, VEC>(next_up, p.dy, r, p, t);
        if (p.gate != nullptr) load_row<T, NV, TPR, VEC>(next_gate, p.gate, r, p, t);
    };
    ask(row);
    for (long long first = static_cast<long long>(blockIdx.x) * G; first < p.rows; first += step, row += step) {
        const bool active = row < p.rows;
        const long long at = (active ? row : 0) * p.width;
        Raw8<T> raw[NV], gate[NV], up[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = next[v], gate[v] = next_gate[v], up[v] = next_up[v];
        if (first + step < p.rows) ask(row + step);
        f2 n[NV][4], dh[NV][4];
        // (a row past the last is a row of zeros, whose rstd is infinite where eps = 0: 0, lest n be NaN)
        const float inv = centred<T, NV, TPR, VEC>(raw, n, t, p, box, turn), rstd = active ? inv : 0.f;
        // dh, its sums, the gate's gradient. Elements past the width, and rows past the last, have dy = 0 and n = 0 and so count for nothing.
        f2 c0 = both(0.f), c1 = both(0.f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            f2 w[4];
            up[v].get(dh[v]);
            load_param<VEC>(p.weight, p.param_bf16, (v * TPR + t) * 8, p.width, 1.f, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) n[v][i] = mul2(n[v][i], both(rstd));
            if (p.gate != nullptr) {
                f2 z[4], b[4];
                gate[v].get(z);
                load_param<VEC>(p.bias, p.param_bf16, (v * TPR + t) * 8, p.width, 0.f, b);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f2 s = sigmoid2<T>(z[i]), zs = mul2(z[i], s);
                    // silu'(z) = s + z s (1 - s)
                    const f2 slope = fma2(zs, fma2(s, both(-1.f), both(1.f)), s), h = fma2(n[v][i], w[i], b[i]);
                    z[i] = mul2(mul2(dh[v][i], h), slope);
                    dh[v][i] = mul2(dh[v][i], zs);
                }
                store8<T, VEC>(static_cast<T*>(p.dgate) + at, (v * TPR + t) * 8, p.width, active, z);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                dw[v][i] = fma2(dh[v][i], n[v][i], dw[v][i]);
                db[v][i] = add2(db[v][i], dh[v][i]);
                dh[v][i] = mul2(dh[v][i], w[i]);
                c0 = add2(c0, dh[v][i]);
                c1 = fma2(dh[v][i], n[v][i], c1);
            }
        }
        float c[2] = {sum2(c0), sum2(c1)};
        row_sums<TPR>(c, box, turn);
        const f2 m0 = both(p.rms ? 0.f : -c[0] * p.inv_width), m1 = both(-c[1] * p.inv_width);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) n[v][i] = mul2(both(rstd), fma2(n[v][i], m1, add2(dh[v][i], m0)));
            store8<T, VEC>(static_cast<T*>(p.dx) + at, (v * TPR + t) * 8, p.width, active, n[v]);
        }
    }
    launch_dependents();
    if (p.partial == nullptr) return;
    float* const mine = p.partial + static_cast<long long>(blockIdx.x) * 2 * p.width;
#pragma unroll 1
    for (int which = 0; which < (p.want_db ? 2 : 1); ++which) {
        if (G > 1) __syncthreads();
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = (v * TPR + t) * 8 + 2 * i;
                float a, b;
                unpair2(which ? db[v][i] : dw[v][i], a, b);
                if (G > 1) {
                    gather[(threadIdx.x / TPR) * kColumns + col] = a, gather[(threadIdx.x / TPR) * kColumns + col + 1] = b;
                } else {
                    if (col < p.width) mine[which * p.width + col] = a;
                    if (col + 1 < p.width) mine[which * p.width + col + 1] = b;
                }
            }
        if (G == 1) continue;
        __syncthreads();
        for (int col = threadIdx.x; col < p.width; col += cta_threads<TPR>()) {
            float s = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) s += gather[g * kColumns + col];
            mine[which * p.width + col] = s;
        }
    }
}

// The CTAs' sums of dw and db, added in order of the CTAs (32 columns a CTA, 32 rows of them at a time)
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* partial, int parts, int width, float* dw, float* db) {
    __shared__ float box[32][33];
    grid_dependency_wait();
    const int col = blockIdx.x * 32 + threadIdx.x;
    float* const out = blockIdx.y ? db : dw;
    if (out == nullptr) return;
    float s = 0.f;
    if (col < width)
#pragma unroll 8
        for (int i = threadIdx.y; i < parts; i += 32) s += partial[(static_cast<long long>(i) * 2 + blockIdx.y) * width + col];
    box[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && col < width) {
        s = 0.f;
        for (int i = 0; i < 32; ++i) s += box[i][threadIdx.x];
        out[col] = s;
    }
}

// Threads that a launch brings per SM, at most: as many as are resident there (80 registers backward, 48 forward) of bf16 rows in whole vectors with one
// vector a thread (up to 256 features and from 513 to 2048), so that no CTA is left for a second round. 1 M rows of 128 (with the sigmoid as it was):
// backward 0.264 ms, with 1024 threads 0.314; forward 0.147, with 1024 0.156, with 1536 0.176. The other instantiations take more registers and the rule
// was not measured for them: some CTAs of theirs come in a second round (resident / launched per SM, backward: fp32 2 / 3 up to 256 features, 1 / 3 to
// 512, 3 or 4 / 6 to 1024, 1 or 2 / 3 to 2048, bf16 1 / 3 from 257 to 512; forward: fp32 3 or 4 / 5 up to 256, 2 / 5 to 512, 1 / 2 above 4096).
constexpr int kForwardThreads = 1280, kBackwardThreads = 768;

// threads of a row; CTAs of a launch
int row_threads(int width) { return width <= 128 ? 16 : width <= 512 ? 32 : width <= 1024 ? 128 : width <= 2048 ? 256 : 512; }
long long cta_count(long long rows, int width, int per_sm) {
    const int tpr = row_threads(width), threads = tpr > 32 ? tpr : kNormThreads, g = threads / tpr;
    const long long need = (rows + g - 1) / g, most = static_cast<long long>(per_sm / threads) * kSMs;
    return need < most ? need : most;
}

template <typename T, int NV, int TPR>
int launch_norm(const ParamsN& p, bool backward, cudaStream_t stream) {
    const bool vec = p.width % 8 == 0;
    const unsigned grid = static_cast<unsigned>(cta_count(p.rows, p.width, backward ? kBackwardThreads : kForwardThreads));
    if (grid > 0) {
        auto* kern = backward ? (vec ? norm_backward_kernel<T, NV, TPR, true> : norm_backward_kernel<T, NV, TPR, false>)
                              : (vec ? norm_forward_kernel<T, NV, TPR, true> : norm_forward_kernel<T, NV, TPR, false>);
        kern<<<grid, cta_threads<TPR>(), 0, stream>>>(p);
        if (cudaGetLastError() != cudaSuccess) return GDN_ERR_LAUNCH;
        count_launch();
    }
    return GDN_OK;
}

template <typename T>
int launch_norm_width(const ParamsN& p, bool backward, cudaStream_t stream) {
    const int w = p.width;
    if (w <= 128) return launch_norm<T, 1, 16>(p, backward, stream);
    if (w <= 256) return launch_norm<T, 1, 32>(p, backward, stream);
    if (w <= 512) return launch_norm<T, 2, 32>(p, backward, stream);
    if (w <= 1024) return launch_norm<T, 1, 128>(p, backward, stream);
    if (w <= 2048) return launch_norm<T, 1, 256>(p, backward, stream);
    if (w <= 4096) return launch_norm<T, 1, 512>(p, backward, stream);
    if (w <= 8192) return launch_norm<T, 2, 512>(p, backward, stream);
    return launch_norm<T, 4, 512>(p, backward, stream);
}

}  // namespace

size_t norm_workspace(long long rows, int width) {
    return static_cast<size_t>(cta_count(rows, width, kBackwardThreads)) * 2 * width * sizeof(float);
}

int launch_layer_norm(const ProblemN& q, bool backward, cudaStream_t stream) {
    ParamsN p{};
    p.dy = q.dy, p.x = q.x, p.weight = q.weight, p.bias = q.bias, p.gate = q.gate;
    p.y = q.y, p.dx = q.dx, p.dgate = q.dgate;
    p.rows = q.rows, p.width = q.width, p.eps = q.eps, p.inv_width = 1.f / static_cast<float>(q.width);
    p.rms = (q.flags & GDN_NORM_RMS) != 0, p.param_bf16 = q.param_dtype == GDN_DTYPE_BF16;
    p.want_db = q.dbias != nullptr;
    const bool sums = backward && (q.dweight != nullptr || q.dbias != nullptr);
    p.partial = sums ? static_cast<float*>(q.workspace) : nullptr;
    const int rc = q.dtype == GDN_DTYPE_BF16 ? launch_norm_width<__nv_bfloat16>(p, backward, stream) : launch_norm_width<float>(p, backward, stream);
    if (rc != GDN_OK || !sums) return rc;  // (without rows there is no workspace, and the sums are zero)
    const int parts = static_cast<int>(cta_count(q.rows, q.width, kBackwardThreads));
    float *const dw = q.dweight, *const db = q.dbias;
    const dim3 grid((q.width + 31) / 32, db != nullptr ? 2 : 1);  // (without a weight there may be a bias)
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(32, 32);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, norm_sum_kernel, static_cast<const float*>(p.partial), parts, q.width, dw, db) != cudaSuccess) {
        cudaGetLastError();
        return GDN_ERR_LAUNCH;
    }
    count_launch();
    return GDN_OK;
}

}  // namespace gdn

// The gated delta rule token by token: decoding one or a few new tokens per sequence on a pool of states.
//
// Per (sequence, value head), with S the state [d_v x d_k] and a_t = exp(g_t):
//     u_t = beta_t (v_t - a_t S k_t),   S <- a_t S + u_t k_t^T,   o_t = scale S q_t
// which is evaluated as two products with the old state and one pass that updates it:
//     x = S k_t,  y = S q_t,  u_t = beta_t (v_t - a_t x),  o_t = scale (a_t y + u_t <k_t, q_t>),  S <- a_t S + u_t k_t^T
// so that both sums over d_k run side by side and nothing waits for the updated state.
//
// What bounds it: the state is read once and written once (128 KB per head in fp32) and everything else is small, so HBM at
// large batches and latency at small ones. A row of the state (one value feature) lies on 8 lanes, 16 bytes a lane and load (a
// warp's load is four runs of 128 bytes), and stays in registers for all tokens of the call: a sum over d_k is 3 shuffles. Rows
// are independent, so a head is cut into slices of rows for as many CTAs as there is need for. All arithmetic is fp32, with a bf16
// state too, which is rounded once, when it is stored.
#include "common.cuh"

namespace gdn {
namespace {

constexpr int kLanes = 8;       // lanes that share a row of the state
constexpr int kStepThreads = 128;
constexpr int kRowsPerPass = kStepThreads / kLanes;

struct Strides {  // of a token tensor, in elements
    long long batch, token, head;
};

struct ParamsStep {
    const void *Q, *K, *V;
    const float *beta, *g;
    void* S;
    const int* slots;  // may be null: sequence b's state is S[b]
    void* O;
    int* status;  // for slots that cannot be used
    Strides q, v, gate;  // q: Q and K; v: V and O
    int H_v, group, T, d_k, d_v, n_slots, slices;
    float scale;
    bool l2norm;
};

// N elements of a row of bf16 or fp32, from an address that is aligned to 16 bytes (8 for four bf16)
template <int N>
__device__ __forceinline__ void load_n(const float* p, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 w = *reinterpret_cast<const float4*>(p + i);
        x[i] = w.x, x[i + 1] = w.y, x[i + 2] = w.z, x[i + 3] = w.w;
    }
}
template <int N>
__device__ __forceinline__ void load_n(const __nv_bfloat16* p, float (&x)[N]) {
    uint32_t w[N / 2];
    if (N == 8) {
        const uint4 t = *reinterpret_cast<const uint4*>(p);
        w[0] = t.x, w[1] = t.y, w[2 % (N / 2)] = t.z, w[3 % (N / 2)] = t.w;
    } else {
        const uint2 t = *reinterpret_cast<const uint2*>(p);
        w[0] = t.x, w[1] = t.y;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void store_n(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store_n(__nv_bfloat16* p, const float (&x)[8]) {
    __nv_bfloat162 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void store_one(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_one(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// TOK: type of the token tensors; ST: of the state; DK: the widest d_k (columns past d_k count as zeros); R: rows of the state
// that a thread holds its part of
template <typename TOK, typename ST, int DK, int R>
__global__ void __launch_bounds__(kStepThreads) recurrent_step_kernel(const ParamsStep p) {
    constexpr int E = 16 / sizeof(ST);        // elements of a 16-byte piece of a row
    constexpr int NP = DK / (E * kLanes);     // pieces of a row that a lane holds
    const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
    const int slice = blockIdx.x % p.slices;
    const int h = (blockIdx.x / p.slices) % p.H_v;
    const int b = blockIdx.x / p.slices / p.H_v;
    const int row0 = slice * (R * kRowsPerPass) + sub;

    int slot = b;
    bool live = true;
    if (p.slots != nullptr) {
        slot = p.slots[b];
        live = slot >= 0;
        // two sequences on one state would race: the first in the batch has it, the others are reported and not computed
        bool bad = slot >= p.n_slots;
        for (int i = threadIdx.x; i < b; i += kStepThreads) bad |= live && p.slots[i] == slot;
        if (__syncthreads_or(bad)) {
            if (threadIdx.x == 0) *p.status = GDN_ERR_INVALID_ARG;
            live = false;
        }
    }
    TOK* const out = static_cast<TOK*>(p.O) + b * p.v.batch + h * p.v.head;
    if (!live) {  // a padded row of the batch: its output is zero
        for (int t = 0; t < p.T; ++t)
            for (int r = 0; r < R; ++r) {
                const int row = row0 + r * kRowsPerPass;
                if (lane == 0 && row < p.d_v) store_one(out + t * p.v.token + row, 0.f);
            }
        return;
    }
    ST* const S = static_cast<ST*>(p.S) + (static_cast<long long>(slot) * p.H_v + h) * p.d_v * p.d_k;
    float s[R][NP][E];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + r * kRowsPerPass;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int col = (j * kLanes + lane) * E;
            if (row < p.d_v && col < p.d_k) {
                load_n<E>(S + static_cast<long long>(row) * p.d_k + col, s[r][j]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) s[r][j][e] = 0.f;
            }
        }
    }
    const TOK* const Q = static_cast<const TOK*>(p.Q) + b * p.q.batch + (h / p.group) * p.q.head;
    const TOK* const K = static_cast<const TOK*>(p.K) + b * p.q.batch + (h / p.group) * p.q.head;
    const TOK* const V = static_cast<const TOK*>(p.V) + b * p.v.batch + h * p.v.head;
    const long long gate0 = b * p.gate.batch + h * p.gate.head;
    for (int t = 0; t < p.T; ++t) {
        float q[NP][E], k[NP][E], v[R];
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int col = (j * kLanes + lane) * E;
            if (col < p.d_k) {
                load_n<E>(Q + t * p.q.token + col, q[j]);
                load_n<E>(K + t * p.q.token + col, k[j]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) q[j][e] = k[j][e] = 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = row0 + r * kRowsPerPass;
            v[r] = row < p.d_v ? to_float(V[t * p.v.token + row]) : 0.f;
        }
        const float beta = p.beta[gate0 + t * p.gate.token], a = expf(p.g[gate0 + t * p.gate.token]);
        float qq = 0.f, kk = 0.f, kq = 0.f;
#pragma unroll
        for (int j = 0; j < NP; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                qq = fmaf(q[j][e], q[j][e], qq);
                kk = fmaf(k[j][e], k[j][e], kk);
                kq = fmaf(k[j][e], q[j][e], kq);
            }
        qq = sum_lanes(qq), kk = sum_lanes(kk), kq = sum_lanes(kq);
        // 1 / ||k||, 1 / ||q||; a row of zeros stays zero
        const float rk = !p.l2norm ? 1.f : (kk == 0.f ? 0.f : rsqrtf(kk)), rq = !p.l2norm ? 1.f : (qq == 0.f ? 0.f : rsqrtf(qq));
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x = 0.f, y = 0.f;
#pragma unroll
            for (int j = 0; j < NP; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x = fmaf(s[r][j][e], k[j][e], x);
                    y = fmaf(s[r][j][e], q[j][e], y);
                }
            x = sum_lanes(x), y = sum_lanes(y);
            const float u = beta * (v[r] - a * rk * x), uk = u * rk;
#pragma unroll
            for (int j = 0; j < NP; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) s[r][j][e] = fmaf(a, s[r][j][e], uk * k[j][e]);
            const int row = row0 + r * kRowsPerPass;
            if (lane == 0 && row < p.d_v) store_one(out + t * p.v.token + row, p.scale * rq * fmaf(a, y, uk * kq));
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + r * kRowsPerPass;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int col = (j * kLanes + lane) * E;
            if (row < p.d_v && col < p.d_k) store_n(S + static_cast<long long>(row) * p.d_k + col, s[r][j]);
        }
    }
}

template <typename TOK, typename ST, int DK>
int launch_step_dk(ParamsStep& p, long long seqs, cudaStream_t stream) {
    constexpr int R = 2;
    p.slices = (p.d_v + R * kRowsPerPass - 1) / (R * kRowsPerPass);
    const long long ctas = seqs * p.H_v * p.slices;
    if (ctas >= (1LL << 31)) return GDN_ERR_UNSUPPORTED;
    recurrent_step_kernel<TOK, ST, DK, R><<<static_cast<unsigned>(ctas), kStepThreads, 0, stream>>>(p);
    if (cudaGetLastError() != cudaSuccess) return GDN_ERR_LAUNCH;
    count_launch();
    return GDN_OK;
}

template <typename TOK, typename ST>
int launch_step_types(ParamsStep& p, long long seqs, cudaStream_t stream) {
    if (p.d_k <= 64) return launch_step_dk<TOK, ST, 64>(p, seqs, stream);
    return p.d_k <= 128 ? launch_step_dk<TOK, ST, 128>(p, seqs, stream) : launch_step_dk<TOK, ST, 256>(p, seqs, stream);
}

}  // namespace

int launch_recurrent_step(const ProblemStep& q, cudaStream_t stream) {
    ParamsStep p{};
    int* const status = device_status_word();
    if (status == nullptr) return GDN_ERR_LAUNCH;
    p.status = status + 1;
    p.Q = q.Q, p.K = q.K, p.V = q.V, p.beta = q.beta, p.g = q.g, p.S = q.S, p.slots = q.slots, p.O = q.O;
    p.H_v = q.H_v, p.group = q.H_v / q.H_k, p.T = q.T, p.d_k = q.d_k, p.d_v = q.d_v, p.n_slots = q.n_slots;
    p.scale = q.scale, p.l2norm = (q.flags & GDN_FLAG_K_L2NORM) != 0;
    const bool token_major = (q.flags & GDN_FLAG_LAYOUT_BTHD) != 0;
    const auto strides = [&](long long H, long long d) {
        return token_major ? Strides{q.T * H * d, H * d, d} : Strides{H * q.T * d, d, q.T * d};
    };
    p.q = strides(q.H_k, q.d_k), p.v = strides(q.H_v, q.d_v), p.gate = strides(q.H_v, 1);
    const bool bf16 = q.dtype == GDN_DTYPE_BF16, s16 = q.state_dtype == GDN_DTYPE_BF16;
    if (bf16) return s16 ? launch_step_types<__nv_bfloat16, __nv_bfloat16>(p, q.B, stream) : launch_step_types<__nv_bfloat16, float>(p, q.B, stream);
    return s16 ? launch_step_types<float, __nv_bfloat16>(p, q.B, stream) : launch_step_types<float, float>(p, q.B, stream);
}

}  // namespace gdn

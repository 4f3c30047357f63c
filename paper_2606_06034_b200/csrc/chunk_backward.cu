// Backward pass of the chunk-wise gated delta rule (C = 64 tokens, d_k = d_v = 128, bf16 tensors, fp32 states and gates).
//
// Forward, per chunk (S: state [d_v x d_k] carried in; k, q of unit length where the caller asks for it; g: cumulative log-gate of the
// chunk; A_ij = beta_i exp(g_i - g_j) <k_i, k_j> below the diagonal; T = (I + A)^-1):
//     z_i = S k_i,   u = T (beta (v - exp(g) z)),   o = scale (exp(g) S q + P u),   P_ij = exp(g_i - g_j) <q_i, k_j>  (j <= i)
//     S' = exp(g_C) S + sum_j exp(g_C - g_j) u_j k_j^T
// Backward (D = dL/dS'). u solves a triangular system, so the gradient r of its right-hand side solves the transposed one, and the gradient
// of A is -r u^T: W = T diag(beta exp(g)) K and the gradient of T never appear.
//     y_j = D k_j,   r = T^T (scale P^T dO + exp(g_C - g) y)
//     dS = exp(g_C) D + sum_i (scale exp(g_i) dO_i q_i^T - beta_i exp(g_i) r_i k_i^T)
//     dv = beta r
//     p_ij = scale exp(g_i - g_j) <dO_i, u_j>  (j <= i),   m_ij = -beta_i exp(g_i - g_j) <r_i, u_j>  (j < i)
//     dq = scale exp(g) (dO S) + p k
//     dk = p^T q + exp(g_C - g) (u D) - beta exp(g) (r S) + (m + m^T) k
//     dbeta_i = <r_i, v_i - exp(g_i) z_i> - sum_{j<i} <r_i, u_j> A_ij / beta_i
//     N_ij = scale P_ij <dO_i, u_j> - A_ij <r_i, u_j>  (j < i)
//     dg_i (cumulative) = sum_j N_ij - sum_j N_ji + scale exp(g_i) <q_i, S^T dO_i> - beta_i exp(g_i) <r_i, z_i> - exp(g_C - g_i) <u_i, y_i>
//                         (at the chunk's end also + sum_i exp(g_C - g_i) <u_i, y_i> + exp(g_C) <D, S>), summed backwards for the raw gates
// Four launches: `chunk_system` (per chunk and key head: T, P and the gates' tables), `chunk_states` (per sequence, value head and
// slice of d_v, forward over the chunks: S, u, z), `chunk_state_grads` (the same backward: D, r), `chunk_grads` (per chunk and key
// head, the value heads that share it in turn: dQ, dK, dV, dbeta, dg). Both chains are independent for each row of S (each value feature), so a head
// is cut into slices for more CTAs than it has heads.
//
// Precision: dbeta, dg and dS_in are fp32 and so is what they are made of. Products run on the tensor cores in tf32 with an fp32
// operand as the sum of its upper 11 bits and the rest (2 products where the other operand is bf16, which tf32 holds exactly, 3 where
// both are fp32): 2^-21 of a product is lost. What only reaches dQ, dK, dV, which are rounded to bf16 (2^-9), takes one product.
#include "common.cuh"
#include "sm100_ptx.cuh"

namespace gdn {
namespace {

using namespace sm100;

constexpr int kC = 64, kD = 128;
constexpr int kSlice = 32;               // value features of a chain's CTA
constexpr int kSlices = kD / kSlice;
constexpr int kThreads = 256;

// workspace of one chunk of one value head, in floats
constexpr int kWsT = 0, kWsP = kWsT + kC * kC, kWsS = kWsP + kC * kC, kWsDS = kWsS + kD * kD, kWsU = kWsDS + kD * kD;
constexpr int kWsZ = kWsU + kC * kD;     // z, then r in its place
constexpr int kWsTab = kWsZ + kC * kD;   // tables of 64 floats each
enum { TAB_EGK = 0, TAB_BETA, TAB_ECK, TAB_BEGK, TAB_SEGQ, TAB_G, TAB_RK, TAB_RQ, kTabs };
constexpr int kWsDots = kWsTab + kTabs * kC;  // per slice: <r, v - exp(g) z>, beta exp(g) <r, z>, exp(g_C - g) <u, y>
constexpr int kDots = 3;
constexpr int kWsChunk = kWsDots + kSlices * kDots * kC;

struct Strides {  // of a token tensor, in elements
    long long seq, token, head;
    __device__ __forceinline__ long long at(int s, int t, int h) const { return s * seq + t * token + h * head; }
};

struct ParamsB {
    const __nv_bfloat16 *Q, *K, *V, *dO;
    const float *beta, *g, *S_in, *dS_out;
    __nv_bfloat16 *dQ, *dK, *dV;
    float *dbeta, *dg, *dS_in;
    float* ws;
    const int* cu;  // packed sequences: their boundaries; null: n_seq sequences of T tokens
    int n_seq, T, H_k, H_v, group, chunks;  // chunks: of a dense sequence
    Strides qk, v, gate;
    float scale;
    bool l2norm;
};

// Sequence s: its first token, its length and the index of its first chunk in the workspace. Packed: sequence s starts at cu[s] / 64 +
// s, which leaves room for the chunks of those before it whatever their lengths, and needs no table.
struct Seq {
    int first, len, slot;
};
__device__ __forceinline__ Seq seq_of(const ParamsB& p, int s) {
    if (p.cu == nullptr) return Seq{0, p.T, s * p.chunks};
    const int a = p.cu[s], b = p.cu[s + 1];
    return Seq{a, b > a ? b - a : 0, a / kC + s};
}
// the sequence and the chunk that a place of the workspace belongs to; false where it belongs to none
__device__ __forceinline__ bool chunk_of(const ParamsB& p, int slot, int& s, int& first, int& rows) {
    if (p.cu == nullptr) {
        s = slot / p.chunks;
        first = (slot % p.chunks) * kC;
        rows = min(kC, p.T - first);
        return true;
    }
    int lo = 0, hi = p.n_seq - 1;
    while (lo < hi) {  // the last sequence whose chunks start at or before `slot`
        const int mid = (lo + hi + 1) / 2;
        if (p.cu[mid] / kC + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    s = lo;
    const Seq q = seq_of(p, s);
    const int t = (slot - q.slot) * kC;
    first = q.first + t;
    rows = min(kC, q.len - t);
    return slot >= q.slot && rows > 0;
}
__device__ __forceinline__ float* chunk_ws(const ParamsB& p, int slot, int h) {
    return p.ws + (static_cast<long long>(slot) * p.H_v + h) * kWsChunk;
}

// ---------------------------------------------------------------- copies into shared memory
__device__ __forceinline__ void cp16(void* dst, const void* src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// 64 rows of `cols` bf16 (a multiple of 8) into rows of LD elements; rows from `rows` on are zeros
template <int LD, int COLS>
__device__ __forceinline__ void copy_rows(__nv_bfloat16* dst, const __nv_bfloat16* src, long long row_stride, int rows) {
    for (int i = threadIdx.x; i < kC * (COLS / 8); i += kThreads) {
        const int r = i / (COLS / 8), c = i % (COLS / 8) * 8;
        cp16(dst + r * LD + c, r < rows ? src + r * row_stride + c : src, r < rows);
    }
}
// ROWS rows of COLS floats
template <int LD, int ROWS, int COLS>
__device__ __forceinline__ void copy_floats(float* dst, const float* src, int src_ld) {
    for (int i = threadIdx.x; i < ROWS * (COLS / 4); i += kThreads) {
        const int r = i / (COLS / 4), c = i % (COLS / 4) * 4;
        cp16(dst + r * LD + c, src + r * src_ld + c, true);
    }
}

// ---------------------------------------------------------------- tensor-core products
// m16n8k8 tf32 and m16n8k16 bf16, fp32 accumulators. The sum index that lane c = lane % 4 holds in its two (four) places is 2c, 2c + 1
// in both operands, which the sum does not notice: neighbours in memory, fetched together. Two tiles of columns are taken as a pair
// that covers 16 columns in turn (even ones, odd ones): B of both is one fetch where the columns are neighbours in memory, and a thread's results are
// four columns in a row: 4c, 4c + 2 in the first tile, 4c + 1, 4c + 3 in the second.
// Row lengths in shared memory (in 32-bit words): 8 mod 32 for operands whose sum index runs along the row, 4 mod 16 for those where it
// runs down the rows: no bank conflicts.
__device__ __forceinline__ void mma_tf32(float (&d)[4], const float (&a)[4], float b0, float b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(__float_as_uint(a[0])), "r"(__float_as_uint(a[1])), "r"(__float_as_uint(a[2])), "r"(__float_as_uint(a[3])),
                   "r"(__float_as_uint(b0)), "r"(__float_as_uint(b1)));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// upper 11 bits of the mantissa (what tf32 holds); the rest
__device__ __forceinline__ float tf_hi(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFFE000u); }
template <int N>
__device__ __forceinline__ void split(const float (&x)[N], float (&hi)[N], float (&lo)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) hi[i] = tf_hi(x[i]), lo[i] = x[i] - hi[i];
}
struct Lane {
    int g, c;  // row of a fragment, place along the sum
    __device__ __forceinline__ Lane() : g((threadIdx.x % 32) / 4), c(threadIdx.x % 4) {}
};
// A[m][k] = x[m * ld + k]
__device__ __forceinline__ void a_rows(const float* x, int ld, int m0, int k0, const Lane& l, float (&a)[4]) {
    const float2 u = *reinterpret_cast<const float2*>(x + (m0 + l.g) * ld + k0 + 2 * l.c);
    const float2 v = *reinterpret_cast<const float2*>(x + (m0 + l.g + 8) * ld + k0 + 2 * l.c);
    a[0] = u.x, a[2] = u.y, a[1] = v.x, a[3] = v.y;
}
__device__ __forceinline__ void a_rows(const __nv_bfloat16* x, int ld, int m0, int k0, const Lane& l, float (&a)[4]) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(x + (m0 + l.g) * ld + k0 + 2 * l.c);
    const uint32_t v = *reinterpret_cast<const uint32_t*>(x + (m0 + l.g + 8) * ld + k0 + 2 * l.c);
    a[0] = bf16_lo(u), a[2] = bf16_hi(u), a[1] = bf16_lo(v), a[3] = bf16_hi(v);
}
// A[m][k] = x[k * ld + m]
__device__ __forceinline__ void a_cols(const float* x, int ld, int m0, int k0, const Lane& l, float (&a)[4]) {
    const float* const q = x + (k0 + 2 * l.c) * ld + m0 + l.g;
    a[0] = q[0], a[1] = q[8], a[2] = q[ld], a[3] = q[ld + 8];
}
// a pair of tiles, B[k][n] = x[k * ld + n]: b[0], b[1] of the first tile, b[2], b[3] of the second
__device__ __forceinline__ void b_cols(const float* x, int ld, int n0, int k0, const Lane& l, float (&b)[4]) {
    const float2 u = *reinterpret_cast<const float2*>(x + (k0 + 2 * l.c) * ld + n0 + 2 * l.g);
    const float2 v = *reinterpret_cast<const float2*>(x + (k0 + 2 * l.c + 1) * ld + n0 + 2 * l.g);
    b[0] = u.x, b[2] = u.y, b[1] = v.x, b[3] = v.y;
}
__device__ __forceinline__ void b_cols(const __nv_bfloat16* x, int ld, int n0, int k0, const Lane& l, float (&b)[4]) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(x + (k0 + 2 * l.c) * ld + n0 + 2 * l.g);
    const uint32_t v = *reinterpret_cast<const uint32_t*>(x + (k0 + 2 * l.c + 1) * ld + n0 + 2 * l.g);
    b[0] = bf16_lo(u), b[2] = bf16_hi(u), b[1] = bf16_lo(v), b[3] = bf16_hi(v);
}
// a pair of tiles, B[k][n] = x[n * ld + k]
__device__ __forceinline__ void b_rows(const float* x, int ld, int n0, int k0, const Lane& l, float (&b)[4]) {
    const float2 u = *reinterpret_cast<const float2*>(x + (n0 + 2 * l.g) * ld + k0 + 2 * l.c);
    const float2 v = *reinterpret_cast<const float2*>(x + (n0 + 2 * l.g + 1) * ld + k0 + 2 * l.c);
    b[0] = u.x, b[1] = u.y, b[2] = v.x, b[3] = v.y;
}
// one pair of tiles += A B, with A, B exact in tf32 / one of them split / both split
__device__ __forceinline__ void pair_1(float (&d)[2][4], const float (&a)[4], const float (&b)[4]) {
    mma_tf32(d[0], a, b[0], b[1]);
    mma_tf32(d[1], a, b[2], b[3]);
}
__device__ __forceinline__ void pair_b2(float (&d)[2][4], const float (&a)[4], const float (&b)[4]) {
    float hi[4], lo[4];
    split(b, hi, lo);
    pair_1(d, a, lo);
    pair_1(d, a, hi);
}
__device__ __forceinline__ void pair_a2(float (&d)[2][4], const float (&a)[4], const float (&b)[4]) {
    float hi[4], lo[4];
    split(a, hi, lo);
    pair_1(d, lo, b);
    pair_1(d, hi, b);
}
__device__ __forceinline__ void pair_3(float (&d)[2][4], const float (&a)[4], const float (&b)[4]) {
    float ah[4], al[4], bh[4], bl[4];
    split(a, ah, al);
    split(b, bh, bl);
    pair_1(d, al, bh);
    pair_1(d, ah, bl);
    pair_1(d, ah, bh);
}
// the four neighbouring results of a thread in row g (half = 0) or g + 8 (half = 1) of a pair
__device__ __forceinline__ float4 pair_row(const float (&d)[2][4], int half) {
    return make_float4(d[0][2 * half], d[1][2 * half], d[0][2 * half + 1], d[1][2 * half + 1]);
}
__device__ __forceinline__ float dot4(float4 a, float4 b) { return a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w; }
__device__ __forceinline__ float4 scaled(float4 a, float s) { return make_float4(a.x * s, a.y * s, a.z * s, a.w * s); }
__device__ __forceinline__ float4 bf16x4(uint2 w) { return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)); }
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

constexpr int kLdX = 136;  // bf16 rows of 128 features: 68 words
constexpr int kLdF = 136;  // fp32 rows of 128, sum index along the row
constexpr int kLdN = 132;  // fp32 rows of 128, sum index down the rows (or pairs of rows)
constexpr int kLdM = 72;   // fp32 rows of 64, sum index along the row
constexpr int kLdV = 68;   // fp32 rows of 64, sum index down the rows
constexpr int kLdS = 36;   // fp32 rows of a slice's 32 features, sum index down the rows
constexpr int kLdO = 40;   // bf16 rows of a slice's 32 features: 20 words

// ---------------------------------------------------------------- T, P and the gates' tables
struct SmemSystem {
    union {
        struct {
            __nv_bfloat16 K[kC * kLdX], Q[kC * kLdX];
        } in;
        float T[kC * kLdV];
    };
    float kk[kC * kLdV], qk[kC * kLdV], A[kC * kLdV];
    float rk[kC], rq[kC], g[kC], beta[kC];
};

__global__ void __launch_bounds__(kThreads) chunk_system_kernel(const ParamsB p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemSystem& sm = *reinterpret_cast<SmemSystem*>(smem_raw);
    const int hk = blockIdx.x % p.H_k, slot = blockIdx.x / p.H_k;
    int s, first, rows;
    if (!chunk_of(p, slot, s, first, rows)) return;
    const int tid = threadIdx.x, warp = tid / 32;
    const Lane l;
    copy_rows<kLdX, kD>(sm.in.K, p.K + p.qk.at(s, first, hk), p.qk.token, rows);
    copy_rows<kLdX, kD>(sm.in.Q, p.Q + p.qk.at(s, first, hk), p.qk.token, rows);
    cp_commit();
    cp_wait<0>();
    __syncthreads();
    {  // lengths of the rows: four threads a row
        const int row = tid / 4, part = tid % 4;
        float nk = 0.f, nq = 0.f;
        for (int i = 0; i < kD / 8; ++i) {
            const int col = (i * 4 + part) * 2;
            const uint32_t a = *reinterpret_cast<const uint32_t*>(sm.in.K + row * kLdX + col), b = *reinterpret_cast<const uint32_t*>(sm.in.Q + row * kLdX + col);
            nk = fmaf(bf16_lo(a), bf16_lo(a), fmaf(bf16_hi(a), bf16_hi(a), nk));
            nq = fmaf(bf16_lo(b), bf16_lo(b), fmaf(bf16_hi(b), bf16_hi(b), nq));
        }
        nk = quad_sum(nk), nq = quad_sum(nq);
        if (part == 0) {
            sm.rk[row] = !p.l2norm ? 1.f : (nk == 0.f ? 0.f : rsqrtf(nk));
            sm.rq[row] = !p.l2norm ? 1.f : (nq == 0.f ? 0.f : rsqrtf(nq));
        }
    }
    const int m0 = warp % 4 * 16, n0 = warp / 4 * 32;
    float kk[4][4] = {}, qk[4][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < kD; k0 += 16) {
        const auto word = [&](const __nv_bfloat16* x, int row, int k) { return *reinterpret_cast<const uint32_t*>(x + row * kLdX + k + 2 * l.c); };
        const uint32_t ak[4] = {word(sm.in.K, m0 + l.g, k0), word(sm.in.K, m0 + l.g + 8, k0), word(sm.in.K, m0 + l.g, k0 + 8), word(sm.in.K, m0 + l.g + 8, k0 + 8)};
        const uint32_t aq[4] = {word(sm.in.Q, m0 + l.g, k0), word(sm.in.Q, m0 + l.g + 8, k0), word(sm.in.Q, m0 + l.g, k0 + 8), word(sm.in.Q, m0 + l.g + 8, k0 + 8)};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint32_t b0 = word(sm.in.K, n0 + n * 8 + l.g, k0), b1 = word(sm.in.K, n0 + n * 8 + l.g, k0 + 8);
            mma_bf16(kk[n], ak, b0, b1);
            mma_bf16(qk[n], aq, b0, b1);
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = m0 + l.g + (e / 2) * 8, j = n0 + n * 8 + 2 * l.c + e % 2;
            sm.kk[i * kLdV + j] = kk[n][e] * sm.rk[i] * sm.rk[j];
            sm.qk[i * kLdV + j] = qk[n][e] * p.scale * sm.rq[i] * sm.rk[j];
        }
    for (int hv = hk * p.group; hv < (hk + 1) * p.group; ++hv) {
        float* const ws = chunk_ws(p, slot, hv);
        if (warp == 0) {  // the gates' prefix sum: lane i has tokens 2i, 2i + 1; gates that are closed (-inf) end at exp(-128) = 0
            const int t = 2 * l.g * 4 + 2 * l.c;
            float x[2], b[2];
            for (int e = 0; e < 2; ++e) {
                const long long at = p.gate.at(s, first + t + e, hv);
                x[e] = t + e < rows ? p.g[at] : 0.f;
                b[e] = t + e < rows ? p.beta[at] : 0.f;
                if (x[e] < -128.f) x[e] = -128.f;
            }
            float sum = x[0] + x[1];
            for (int o = 1; o < 32; o *= 2) {
                const float y = __shfl_up_sync(0xffffffffu, sum, o);
                if (static_cast<int>(threadIdx.x) >= o) sum += y;
            }
            sm.g[t] = sum - x[1], sm.g[t + 1] = sum;
            sm.beta[t] = b[0], sm.beta[t + 1] = b[1];
        }
        __syncthreads();
        if (tid < kC) {
            const float g = sm.g[tid], eg = expf(g), ec = expf(sm.g[kC - 1] - g), beta = sm.beta[tid], rk = sm.rk[tid], rq = sm.rq[tid];
            float* const tab = ws + kWsTab;
            const bool real = tid < rows;
            tab[TAB_EGK * kC + tid] = real ? eg * rk : 0.f;
            tab[TAB_BETA * kC + tid] = beta;
            tab[TAB_ECK * kC + tid] = real ? ec * rk : 0.f;
            tab[TAB_BEGK * kC + tid] = real ? beta * eg * rk : 0.f;
            tab[TAB_SEGQ * kC + tid] = real ? p.scale * eg * rq : 0.f;
            tab[TAB_G * kC + tid] = g;
            tab[TAB_RK * kC + tid] = rk;
            tab[TAB_RQ * kC + tid] = rq;
        }
        for (int i = tid; i < kC * kC / 4; i += kThreads) {
            const int row = i / 16, col = i % 16 * 4;
            float a[4], q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = col + e;
                const float gam = j <= row ? expf(sm.g[row] - sm.g[j]) : 0.f;
                a[e] = j < row ? sm.beta[row] * gam * sm.kk[row * kLdV + j] : 0.f;
                q[e] = j <= row ? gam * sm.qk[row * kLdV + j] : 0.f;
            }
            *reinterpret_cast<float4*>(sm.A + row * kLdV + col) = make_float4(a[0], a[1], a[2], a[3]);
            *reinterpret_cast<float4*>(ws + kWsP + row * kC + col) = make_float4(q[0], q[1], q[2], q[3]);
        }
        __syncthreads();
        {  // column j of T by forward substitution: x_i = [i = j] - sum_k A_ik x_k, four threads a column
            const int j = tid / 4, part = tid % 4;
            float x[16];
#pragma unroll
            for (int m = 0; m < 16; ++m) x[m] = 0.f;
#pragma unroll
            for (int i = 0; i < kC; ++i) {
                float a = 0.f, b = 0.f;
#pragma unroll
                for (int m = 0; m <= i / 4; m += 2) {
                    a = fmaf(sm.A[i * kLdV + 4 * m + part], x[m], a);
                    if (m + 1 <= i / 4) b = fmaf(sm.A[i * kLdV + 4 * m + 4 + part], x[m + 1], b);
                }
                const float xi = (i == j ? 1.f : 0.f) - quad_sum(a + b);
                if (i % 4 == part) x[i / 4] = xi;
            }
#pragma unroll
            for (int m = 0; m < 16; ++m) sm.T[(4 * m + part) * kLdV + j] = x[m];
        }
        __syncthreads();
        for (int i = tid; i < kC * kC / 4; i += kThreads) {
            const int row = i / 16, col = i % 16 * 4;
            *reinterpret_cast<float4*>(ws + kWsT + row * kC + col) = *reinterpret_cast<const float4*>(sm.T + row * kLdV + col);
        }
    }
}

// ---------------------------------------------------------------- the states, forward over the chunks
struct StageF {
    __nv_bfloat16 K[kC * kLdX];
    float T[kC * kLdM];
    float tab[kTabs * kC];
};
struct SmemF {
    StageF stage[2];
    float S[kSlice * kLdN];
    float R[kC * kLdS], U[kC * kLdS];
};

__global__ void __launch_bounds__(kThreads) chunk_states_kernel(const ParamsB p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemF& sm = *reinterpret_cast<SmemF*>(smem_raw);
    const int slice = blockIdx.x % kSlices, h = blockIdx.x / kSlices % p.H_v, s = blockIdx.x / kSlices / p.H_v;
    const Seq seq = seq_of(p, s);
    const int n = (seq.len + kC - 1) / kC;
    const int tid = threadIdx.x, warp = tid / 32;
    const Lane l;
    const int hk = h / p.group;
    const auto load = [&](int c) {
        if (c < n) {
            StageF& st = sm.stage[c % 2];
            const float* const ws = chunk_ws(p, seq.slot + c, h);
            copy_rows<kLdX, kD>(st.K, p.K + p.qk.at(s, seq.first + c * kC, hk), p.qk.token, seq.len - c * kC);
            copy_floats<kLdM, kC, kC>(st.T, ws + kWsT, kC);
            copy_floats<kTabs * kC, 1, kTabs * kC>(st.tab, ws + kWsTab, 0);
        }
        cp_commit();
    };
    load(0);
    // tokens x features: 16 x 16 a warp
    const int m0 = warp % 4 * 16, n0 = warp / 4 * 16;
    const int v0 = slice * kSlice + n0 + 4 * l.c;  // this thread's four features
    // the state: 32 features x 16 keys a warp, in registers (fragments) and, for the first product, in shared memory
    float S[2][2][4];
    const float* const S_in = p.S_in == nullptr ? nullptr : p.S_in + ((static_cast<long long>(s) * p.H_v + h) * kD + slice * kSlice) * kD;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = mt * 16 + half * 8 + l.g, col = warp * 16 + 4 * l.c;
            const float4 x = S_in == nullptr ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(S_in + row * kD + col);
            S[mt][0][2 * half] = x.x, S[mt][1][2 * half] = x.y, S[mt][0][2 * half + 1] = x.z, S[mt][1][2 * half + 1] = x.w;
            *reinterpret_cast<float4*>(sm.S + row * kLdN + col) = x;
        }
    for (int c = 0; c < n; ++c) {
        const StageF& st = sm.stage[c % 2];
        float* const ws = chunk_ws(p, seq.slot + c, h);
        const int t0 = c * kC;
        float4 v[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int t = t0 + m0 + half * 8 + l.g;
            v[half] = t < seq.len ? bf16x4(*reinterpret_cast<const uint2*>(p.V + p.v.at(s, seq.first + t, h) + v0)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<float4*>(ws + kWsS + (slice * kSlice + mt * 16 + half * 8 + l.g) * kD + warp * 16 + 4 * l.c) = pair_row(S[mt], half);
        cp_wait<0>();
        __syncthreads();  // the chunk's operands are there, the state's copy is written, the last chunk's stage is free
        load(c + 1);
        float z[2][4] = {};
#pragma unroll
        for (int k0 = 0; k0 < kD; k0 += 8) {
            float a[4], b[4];
            a_rows(st.K, kLdX, m0, k0, l, a);
            b_rows(sm.S, kLdN, n0, k0, l, b);
            pair_b2(z, a, b);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + half * 8 + l.g;
            const float e = st.tab[TAB_EGK * kC + i], beta = st.tab[TAB_BETA * kC + i];
            const float4 x = scaled(pair_row(z, half), e);  // exp(g_i) S k_i
            *reinterpret_cast<float4*>(ws + kWsZ + i * kD + v0) = x;
            *reinterpret_cast<float4*>(sm.R + i * kLdS + n0 + 4 * l.c) =
                make_float4(beta * (v[half].x - x.x), beta * (v[half].y - x.y), beta * (v[half].z - x.z), beta * (v[half].w - x.w));
        }
        __syncthreads();
        float u[2][4] = {};
        for (int k0 = 0; k0 < m0 + 16; k0 += 8) {  // T is lower triangular
            float a[4], b[4];
            a_rows(st.T, kLdM, m0, k0, l, a);
            b_cols(sm.R, kLdS, n0, k0, l, b);
            pair_3(u, a, b);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + half * 8 + l.g;
            const float4 x = pair_row(u, half);
            *reinterpret_cast<float4*>(ws + kWsU + i * kD + v0) = x;
            *reinterpret_cast<float4*>(sm.U + i * kLdS + n0 + 4 * l.c) = scaled(x, st.tab[TAB_ECK * kC + i]);
        }
        __syncthreads();
        const float decay = expf(st.tab[TAB_G * kC + kC - 1]);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            float d[2][4] = {};
#pragma unroll
            for (int k0 = 0; k0 < kC; k0 += 8) {
                float a[4], b[4];
                a_cols(sm.U, kLdS, mt * 16, k0, l, a);
                b_cols(st.K, kLdX, warp * 16, k0, l, b);
                pair_a2(d, a, b);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) S[mt][x][e] = fmaf(decay, S[mt][x][e], d[x][e]);
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<float4*>(sm.S + (mt * 16 + half * 8 + l.g) * kLdN + warp * 16 + 4 * l.c) = pair_row(S[mt], half);
        }
    }
}

// ---------------------------------------------------------------- their gradients, backward over the chunks
struct StageB {
    __nv_bfloat16 K[kC * kLdX], Q[kC * kLdX], dO[kC * kLdO];
    float T[kC * kLdV], P[kC * kLdV];
    float tab[kTabs * kC];
};
struct SmemB {
    StageB stage[2];
    float D[kSlice * kLdN];
    float du[kC * kLdS], w[2 * kC * kLdS];  // w: scale exp(g) dO, then -beta exp(g) r
    float dots[2][kDots][kC];
};

__global__ void __launch_bounds__(kThreads) chunk_state_grads_kernel(const ParamsB p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemB& sm = *reinterpret_cast<SmemB*>(smem_raw);
    const int slice = blockIdx.x % kSlices, h = blockIdx.x / kSlices % p.H_v, s = blockIdx.x / kSlices / p.H_v;
    const Seq seq = seq_of(p, s);
    const int n = (seq.len + kC - 1) / kC;
    const int tid = threadIdx.x, warp = tid / 32;
    const Lane l;
    const int hk = h / p.group;
    const auto load = [&](int c) {
        if (c >= 0) {
            StageB& st = sm.stage[c % 2];
            const float* const ws = chunk_ws(p, seq.slot + c, h);
            const int t = seq.first + c * kC, rows = seq.len - c * kC;
            copy_rows<kLdX, kD>(st.K, p.K + p.qk.at(s, t, hk), p.qk.token, rows);
            copy_rows<kLdX, kD>(st.Q, p.Q + p.qk.at(s, t, hk), p.qk.token, rows);
            copy_rows<kLdO, kSlice>(st.dO, p.dO + p.v.at(s, t, h) + slice * kSlice, p.v.token, rows);
            copy_floats<kLdV, kC, kC>(st.T, ws + kWsT, kC);
            copy_floats<kLdV, kC, kC>(st.P, ws + kWsP, kC);
            copy_floats<kTabs * kC, 1, kTabs * kC>(st.tab, ws + kWsTab, 0);
        }
        cp_commit();
    };
    load(n - 1);
    const int m0 = warp % 4 * 16, n0 = warp / 4 * 16;
    const int v0 = slice * kSlice + n0 + 4 * l.c;
    float D[2][2][4];
    const long long state = ((static_cast<long long>(s) * p.H_v + h) * kD + slice * kSlice) * kD;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = mt * 16 + half * 8 + l.g, col = warp * 16 + 4 * l.c;
            const float4 x = p.dS_out == nullptr ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(p.dS_out + state + row * kD + col);
            D[mt][0][2 * half] = x.x, D[mt][1][2 * half] = x.y, D[mt][0][2 * half + 1] = x.z, D[mt][1][2 * half + 1] = x.w;
            *reinterpret_cast<float4*>(sm.D + row * kLdN + col) = x;
        }
    for (int c = n - 1; c >= 0; --c) {
        const StageB& st = sm.stage[c % 2];
        float* const ws = chunk_ws(p, seq.slot + c, h);
        const int t0 = c * kC;
        float4 v[2], z[2], uu[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + half * 8 + l.g, t = t0 + i;
            v[half] = t < seq.len ? bf16x4(*reinterpret_cast<const uint2*>(p.V + p.v.at(s, seq.first + t, h) + v0)) : make_float4(0.f, 0.f, 0.f, 0.f);
            z[half] = *reinterpret_cast<const float4*>(ws + kWsZ + i * kD + v0);
            uu[half] = *reinterpret_cast<const float4*>(ws + kWsU + i * kD + v0);
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<float4*>(ws + kWsDS + (slice * kSlice + mt * 16 + half * 8 + l.g) * kD + warp * 16 + 4 * l.c) = pair_row(D[mt], half);
        cp_wait<0>();
        __syncthreads();
        load(c - 1);
        float y[2][4] = {}, x[2][4] = {};
#pragma unroll
        for (int k0 = 0; k0 < kD; k0 += 8) {
            float a[4], b[4];
            a_rows(st.K, kLdX, m0, k0, l, a);
            b_rows(sm.D, kLdN, n0, k0, l, b);
            pair_b2(y, a, b);
        }
        for (int k0 = m0; k0 < kC; k0 += 8) {  // P^T dO: P is lower triangular
            float a[4], b[4];
            a_cols(st.P, kLdV, m0, k0, l, a);
            b_cols(st.dO, kLdO, n0, k0, l, b);
            pair_a2(x, a, b);
        }
        float dot_end[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + half * 8 + l.g;
            const float4 e = scaled(pair_row(y, half), st.tab[TAB_ECK * kC + i]), q = pair_row(x, half);  // exp(g_C - g_i) D k_i
            dot_end[half] = quad_sum(dot4(uu[half], e));
            *reinterpret_cast<float4*>(sm.du + i * kLdS + n0 + 4 * l.c) = make_float4(e.x + q.x, e.y + q.y, e.z + q.z, e.w + q.w);
            const float4 o = bf16x4(*reinterpret_cast<const uint2*>(st.dO + i * kLdO + n0 + 4 * l.c));
            *reinterpret_cast<float4*>(sm.w + i * kLdS + n0 + 4 * l.c) = scaled(o, st.tab[TAB_SEGQ * kC + i]);
        }
        __syncthreads();
        float r[2][4] = {};
        for (int k0 = m0; k0 < kC; k0 += 8) {  // T^T is upper triangular
            float a[4], b[4];
            a_cols(st.T, kLdV, m0, k0, l, a);
            b_cols(sm.du, kLdS, n0, k0, l, b);
            pair_3(r, a, b);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + half * 8 + l.g;
            const float4 e = pair_row(r, half);
            *reinterpret_cast<float4*>(ws + kWsZ + i * kD + v0) = e;
            *reinterpret_cast<float4*>(sm.w + (kC + i) * kLdS + n0 + 4 * l.c) = scaled(e, -st.tab[TAB_BEGK * kC + i]);
            const float rz = quad_sum(dot4(e, z[half]));
            const float rv = quad_sum(dot4(e, make_float4(v[half].x - z[half].x, v[half].y - z[half].y, v[half].z - z[half].z, v[half].w - z[half].w)));
            if (l.c == 0) {
                float(*const dots)[kC] = sm.dots[warp / 4];
                dots[0][i] = rv, dots[1][i] = rz * st.tab[TAB_BETA * kC + i], dots[2][i] = dot_end[half];
            }
        }
        __syncthreads();
        if (tid < kDots * kC) ws[kWsDots + slice * kDots * kC + tid] = sm.dots[0][tid / kC][tid % kC] + sm.dots[1][tid / kC][tid % kC];
        const float decay = expf(st.tab[TAB_G * kC + kC - 1]);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            float d[2][4] = {};
#pragma unroll
            for (int k0 = 0; k0 < kC; k0 += 8) {
                float a[4], b[4];
                a_cols(sm.w, kLdS, mt * 16, k0, l, a);
                b_cols(st.Q, kLdX, warp * 16, k0, l, b);
                pair_a2(d, a, b);
                a_cols(sm.w + kC * kLdS, kLdS, mt * 16, k0, l, a);
                b_cols(st.K, kLdX, warp * 16, k0, l, b);
                pair_a2(d, a, b);
            }
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) D[mt][q][e] = fmaf(decay, D[mt][q][e], d[q][e]);
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<float4*>(sm.D + (mt * 16 + half * 8 + l.g) * kLdN + warp * 16 + 4 * l.c) = pair_row(D[mt], half);
        }
    }
    if (p.dS_in != nullptr) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<float4*>(p.dS_in + state + (mt * 16 + half * 8 + l.g) * kD + warp * 16 + 4 * l.c) = pair_row(D[mt], half);
    }
}

// ---------------------------------------------------------------- the chunks' gradients
struct SmemC {
    __nv_bfloat16 K[kC * kLdX], Q[kC * kLdX], dO[kC * kLdX];
    float u[kC * kLdF], r[kC * kLdF];
    union {
        float S[kD * kLdN];  // the state, then its gradient
        struct {
            float p[kC * kLdV], m[kC * kLdM];
        } pair;
    };
    float tab[kTabs * kC];
    float rowq[4][kC], rown[2][kC], rowb[2][kC], coln[4][kC];
    float ds[kThreads / 32];
};

__global__ void __launch_bounds__(kThreads) chunk_grads_kernel(const ParamsB p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemC& sm = *reinterpret_cast<SmemC*>(smem_raw);
    const int hk = blockIdx.x % p.H_k, slot = blockIdx.x / p.H_k;
    int s, first, rows;
    if (!chunk_of(p, slot, s, first, rows)) return;
    const int tid = threadIdx.x, warp = tid / 32;
    const Lane l;
    copy_rows<kLdX, kD>(sm.K, p.K + p.qk.at(s, first, hk), p.qk.token, rows);
    copy_rows<kLdX, kD>(sm.Q, p.Q + p.qk.at(s, first, hk), p.qk.token, rows);
    // tokens x features: 32 x 32 a warp, two pairs of tiles wide; tokens x tokens: 16 x 32 a warp
    const int wm = warp % 2 * 32, wn = warp / 2 * 32;
    const int pm = warp % 4 * 16, pn = warp / 4 * 32;
    float dq[2][2][2][4] = {}, dk[2][2][2][4] = {};  // [rows][pair][tile][], times 1 / ||q||, 1 / ||k||
    const auto add_scaled = [&](float (&to)[2][2][2][4], const float (&x)[2][2][2][4], const float* tab, float sign) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const float e0 = sign * tab[wm + mt * 16 + l.g], e1 = sign * tab[wm + mt * 16 + 8 + l.g];
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    to[mt][q][t][0] = fmaf(e0, x[mt][q][t][0], to[mt][q][t][0]);
                    to[mt][q][t][1] = fmaf(e0, x[mt][q][t][1], to[mt][q][t][1]);
                    to[mt][q][t][2] = fmaf(e1, x[mt][q][t][2], to[mt][q][t][2]);
                    to[mt][q][t][3] = fmaf(e1, x[mt][q][t][3], to[mt][q][t][3]);
                }
        }
    };
    // rows of `x` times rows of a bf16 tile: this thread's share of row i, summed over the lanes of the row
    const auto row_dot = [&](const float (&x)[2][2][2][4], const __nv_bfloat16* tile, int mt, int half) {
        const int i = wm + mt * 16 + half * 8 + l.g;
        float d = 0.f;
#pragma unroll
        for (int q = 0; q < 2; ++q) d += dot4(pair_row(x[mt][q], half), bf16x4(*reinterpret_cast<const uint2*>(tile + i * kLdX + wn + q * 16 + 4 * l.c)));
        return quad_sum(d);
    };
    for (int hv = hk * p.group; hv < (hk + 1) * p.group; ++hv) {
        const float* const ws = chunk_ws(p, slot, hv);
        copy_rows<kLdX, kD>(sm.dO, p.dO + p.v.at(s, first, hv), p.v.token, rows);
        copy_floats<kLdF, kC, kD>(sm.u, ws + kWsU, kD);
        copy_floats<kLdF, kC, kD>(sm.r, ws + kWsZ, kD);
        copy_floats<kLdN, kD, kD>(sm.S, ws + kWsS, kD);
        copy_floats<kTabs * kC, 1, kTabs * kC>(sm.tab, ws + kWsTab, 0);
        cp_commit();
        cp_wait<0>();
        __syncthreads();
        const float decay = expf(sm.tab[TAB_G * kC + kC - 1]);
        {  // dO S (two products: <q, S^T dO> is part of dg) and r S
            float x[2][2][2][4] = {}, w[2][2][2][4] = {};
#pragma unroll 2
            for (int k0 = 0; k0 < kD; k0 += 8) {
                float o[2][4], r[2][4];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    a_rows(sm.dO, kLdX, wm + mt * 16, k0, l, o[mt]);
                    a_rows(sm.r, kLdF, wm + mt * 16, k0, l, r[mt]);
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float b[4], hi[4], lo[4];
                    b_cols(sm.S, kLdN, wn + q * 16, k0, l, b);
                    split(b, hi, lo);
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        pair_1(x[mt][q], o[mt], lo);
                        pair_1(x[mt][q], o[mt], hi);
                        pair_1(w[mt][q], r[mt], b);
                    }
                }
            }
            float part[2][2][2][4] = {};
            add_scaled(part, x, sm.tab + TAB_SEGQ * kC, 1.f);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float d = row_dot(part, sm.Q, mt, half);
                    if (l.c == 0) sm.rowq[warp / 2][wm + mt * 16 + half * 8 + l.g] = d;
                }
#pragma unroll
            for (int i = 0; i < 32; ++i) (&dq[0][0][0][0])[i] += (&part[0][0][0][0])[i];
            add_scaled(dk, w, sm.tab + TAB_BEGK * kC, -1.f);
        }
        __syncthreads();
        {  // the state's gradient in the state's place, and their product
            float d = 0.f;
            for (int i = tid; i < kD * kD / 4; i += kThreads) {
                float4* const at = reinterpret_cast<float4*>(sm.S + (i / 32) * kLdN + i % 32 * 4);
                const float4 x = *reinterpret_cast<const float4*>(ws + kWsDS + i * 4);
                d += dot4(*at, x);
                *at = x;
            }
            for (int o = 16; o > 0; o /= 2) d += __shfl_xor_sync(0xffffffffu, d, o);
            if (tid % 32 == 0) sm.ds[warp] = d;
        }
        __syncthreads();
        {  // u D
            float x[2][2][2][4] = {};
#pragma unroll 2
            for (int k0 = 0; k0 < kD; k0 += 8) {
                float a[2][4];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) a_rows(sm.u, kLdF, wm + mt * 16, k0, l, a[mt]);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float b[4];
                    b_cols(sm.S, kLdN, wn + q * 16, k0, l, b);
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) pair_1(x[mt][q], a[mt], b);
                }
            }
            add_scaled(dk, x, sm.tab + TAB_ECK * kC, 1.f);
        }
        __syncthreads();
        {  // dO u^T, r u^T, k k^T, q k^T; what they make
            float ou[4][4] = {}, ru[4][4] = {}, kk[4][4] = {}, qk[4][4] = {};
#pragma unroll 2
            for (int k0 = 0; k0 < kD; k0 += 16) {
                const auto word = [&](const __nv_bfloat16* x, int row, int k) { return *reinterpret_cast<const uint32_t*>(x + row * kLdX + k + 2 * l.c); };
                const uint32_t ak[4] = {word(sm.K, pm + l.g, k0), word(sm.K, pm + l.g + 8, k0), word(sm.K, pm + l.g, k0 + 8), word(sm.K, pm + l.g + 8, k0 + 8)};
                const uint32_t aq[4] = {word(sm.Q, pm + l.g, k0), word(sm.Q, pm + l.g + 8, k0), word(sm.Q, pm + l.g, k0 + 8), word(sm.Q, pm + l.g + 8, k0 + 8)};
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t b0 = word(sm.K, pn + n * 8 + l.g, k0), b1 = word(sm.K, pn + n * 8 + l.g, k0 + 8);
                    mma_bf16(kk[n], ak, b0, b1);
                    mma_bf16(qk[n], aq, b0, b1);
                }
#pragma unroll
                for (int k1 = k0; k1 < k0 + 16; k1 += 8) {
                    float o[4], r[4], rh[4], rl[4];
                    a_rows(sm.dO, kLdX, pm, k1, l, o);
                    a_rows(sm.r, kLdF, pm, k1, l, r);
                    split(r, rh, rl);
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const float2 b = *reinterpret_cast<const float2*>(sm.u + (pn + n * 8 + l.g) * kLdF + k1 + 2 * l.c);
                        const float h0 = tf_hi(b.x), h1 = tf_hi(b.y), l0 = b.x - h0, l1 = b.y - h1;
                        mma_tf32(ou[n], o, l0, l1);
                        mma_tf32(ou[n], o, h0, h1);
                        mma_tf32(ru[n], rl, h0, h1);
                        mma_tf32(ru[n], rh, l0, l1);
                        mma_tf32(ru[n], rh, h0, h1);
                    }
                }
            }
            const float* const g = sm.tab + TAB_G * kC;
            const float* const rk = sm.tab + TAB_RK * kC;
            float rown[2] = {}, rowb[2] = {};
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                float coln[2] = {};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = pm + l.g + (e / 2) * 8, j = pn + n * 8 + 2 * l.c + e % 2;
                    const float gam = j <= i ? expf(g[i] - g[j]) : 0.f;
                    const float rr = rk[i] * rk[j];
                    const float qq = p.scale * gam * sm.tab[TAB_RQ * kC + i] * rk[j];
                    // p_ij and m_ij with the lengths of the rows that they will multiply
                    const float pp = j <= i ? ou[n][e] * qq : 0.f;
                    const float kg = j < i ? -gam * rr * ru[n][e] : 0.f, mm = sm.tab[TAB_BETA * kC + i] * kg;
                    const float both = j < i ? fmaf(pp, qk[n][e], mm * kk[n][e]) : 0.f;
                    rown[e / 2] += both;
                    coln[e % 2] += both;
                    if (j < i) rowb[e / 2] = fmaf(kg, kk[n][e], rowb[e / 2]);
                    sm.pair.p[i * kLdV + j] = pp;
                    if (j < i) {
                        sm.pair.m[i * kLdM + j] = mm;
                        sm.pair.m[j * kLdM + i] = mm;
                    } else if (j == i) {
                        sm.pair.m[i * kLdM + i] = 0.f;
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) coln[e] += __shfl_xor_sync(0xffffffffu, coln[e], o);
                    if (l.g == 0) sm.coln[warp % 4][pn + n * 8 + 2 * l.c + e] = coln[e];
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float a = quad_sum(rown[half]), b = quad_sum(rowb[half]);
                if (l.c == 0) sm.rown[warp / 4][pm + half * 8 + l.g] = a, sm.rowb[warp / 4][pm + half * 8 + l.g] = b;
            }
        }
        __syncthreads();
        for (int k0 = 0; k0 < kC; k0 += 8) {  // p k, p^T q, (m + m^T) k
            float bk[2][4], bq[2][4];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                b_cols(sm.K, kLdX, wn + q * 16, k0, l, bk[q]);
                b_cols(sm.Q, kLdX, wn + q * 16, k0, l, bq[q]);
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                float a[4];
                if (k0 <= wm + mt * 16 + 15) {
                    a_rows(sm.pair.p, kLdV, wm + mt * 16, k0, l, a);
                    pair_1(dq[mt][0], a, bk[0]);
                    pair_1(dq[mt][1], a, bk[1]);
                }
                if (k0 + 7 >= wm + mt * 16) {
                    a_cols(sm.pair.p, kLdV, wm + mt * 16, k0, l, a);
                    pair_1(dk[mt][0], a, bq[0]);
                    pair_1(dk[mt][1], a, bq[1]);
                }
                a_rows(sm.pair.m, kLdM, wm + mt * 16, k0, l, a);
                pair_1(dk[mt][0], a, bk[0]);
                pair_1(dk[mt][1], a, bk[1]);
            }
        }
        // dV = beta r
        for (int i = tid; i < kC * kD / 8; i += kThreads) {
            const int row = i / (kD / 8), col = i % (kD / 8) * 8;
            if (row < rows) {
                const float b = sm.tab[TAB_BETA * kC + row];
                const float4 x = scaled(*reinterpret_cast<const float4*>(sm.r + row * kLdF + col), b), y = scaled(*reinterpret_cast<const float4*>(sm.r + row * kLdF + col + 4), b);
                *reinterpret_cast<uint4*>(p.dV + p.v.at(s, first + row, hv) + col) =
                    make_uint4(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w), pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
            }
        }
        if (warp == 0) {  // dbeta, dg: lane i has tokens 2i, 2i + 1
            float d[2], ends = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = 2 * tid + e;
                float direct = 0.f, rz = 0.f, end = 0.f;
#pragma unroll
                for (int x = 0; x < kSlices; ++x) {
                    const float* const dots = ws + kWsDots + x * kDots * kC;
                    direct += dots[i], rz += dots[kC + i], end += dots[2 * kC + i];
                }
                if (i < rows) p.dbeta[p.gate.at(s, first + i, hv)] = direct + sm.rowb[0][i] + sm.rowb[1][i];
                d[e] = sm.rown[0][i] + sm.rown[1][i] - (sm.coln[0][i] + sm.coln[1][i] + sm.coln[2][i] + sm.coln[3][i]) +
                       (sm.rowq[0][i] + sm.rowq[1][i] + sm.rowq[2][i] + sm.rowq[3][i]) - rz - end;
                ends += end;
            }
#pragma unroll
            for (int o = 16; o > 0; o /= 2) ends += __shfl_xor_sync(0xffffffffu, ends, o);
            float dsum = 0.f;
#pragma unroll
            for (int x = 0; x < kThreads / 32; ++x) dsum += sm.ds[x];
            if (tid == 31) d[1] += ends + decay * dsum;
            float sum = d[0] + d[1];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float x = __shfl_down_sync(0xffffffffu, sum, o);
                if (tid + o < 32) sum += x;
            }
            if (2 * tid < rows) p.dg[p.gate.at(s, first + 2 * tid, hv)] = sum;
            if (2 * tid + 1 < rows) p.dg[p.gate.at(s, first + 2 * tid + 1, hv)] = sum - d[0];
        }
        __syncthreads();
    }
    // through the norm of the rows: x - ||row||^-2 <row, x> row
    const auto finish = [&](const float (&x)[2][2][2][4], const __nv_bfloat16* tile, const float* inv, __nv_bfloat16* out) {
        if (p.l2norm) {
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float d = row_dot(x, tile, mt, half);
                    if (l.c == 0) sm.rowq[warp / 2][wm + mt * 16 + half * 8 + l.g] = d;
                }
            __syncthreads();
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = wm + mt * 16 + half * 8 + l.g;
                const float d = p.l2norm ? inv[i] * inv[i] * (sm.rowq[0][i] + sm.rowq[1][i] + sm.rowq[2][i] + sm.rowq[3][i]) : 0.f;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int col = wn + q * 16 + 4 * l.c;
                    const float4 a = pair_row(x[mt][q], half), b = bf16x4(*reinterpret_cast<const uint2*>(tile + i * kLdX + col));
                    if (i < rows)
                        *reinterpret_cast<uint2*>(out + p.qk.at(s, first + i, hk) + col) =
                            make_uint2(pack_bf16x2(a.x - d * b.x, a.y - d * b.y), pack_bf16x2(a.z - d * b.z, a.w - d * b.w));
                }
            }
        __syncthreads();
    };
    finish(dq, sm.Q, sm.tab + TAB_RQ * kC, p.dQ);
    finish(dk, sm.K, sm.tab + TAB_RK * kC, p.dK);
}

template <typename Smem>
bool launch(void (*kern)(ParamsB), long long ctas, const ParamsB& p, cudaStream_t stream) {
    if (ctas == 0) return true;
    static_assert(sizeof(Smem) <= 227 * 1024, "");
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem)) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    kern<<<static_cast<unsigned>(ctas), kThreads, sizeof(Smem), stream>>>(p);
    if (cudaGetLastError() != cudaSuccess) return false;
    count_launch();
    return true;
}

long long chunk_places(int n_seq, long long tokens) { return tokens / kC + n_seq; }

}  // namespace

size_t layer_backward_workspace(int n_seq, long long tokens, int H_v) {
    return static_cast<size_t>(chunk_places(n_seq, tokens)) * H_v * kWsChunk * sizeof(float);
}

int launch_layer_backward(const ProblemB& q, cudaStream_t stream) {
    ParamsB p{};
    p.Q = static_cast<const __nv_bfloat16*>(q.Q), p.K = static_cast<const __nv_bfloat16*>(q.K), p.V = static_cast<const __nv_bfloat16*>(q.V);
    p.dO = static_cast<const __nv_bfloat16*>(q.dO);
    p.beta = q.beta, p.g = q.g, p.S_in = q.S_in, p.dS_out = q.dS_out;
    p.dQ = static_cast<__nv_bfloat16*>(q.dQ), p.dK = static_cast<__nv_bfloat16*>(q.dK), p.dV = static_cast<__nv_bfloat16*>(q.dV);
    p.dbeta = q.dbeta, p.dg = q.dg, p.dS_in = q.dS_in, p.ws = static_cast<float*>(q.workspace), p.cu = q.cu_seqlens;
    p.n_seq = q.n_seq, p.T = q.T, p.H_k = q.H_k, p.H_v = q.H_v, p.group = q.H_v / q.H_k, p.chunks = (q.T + kC - 1) / kC;
    p.scale = q.scale, p.l2norm = (q.flags & GDN_FLAG_K_L2NORM) != 0;
    const bool token_major = (q.flags & GDN_FLAG_LAYOUT_BTHD) != 0, packed = q.cu_seqlens != nullptr;
    const auto strides = [&](long long H, long long d) {
        Strides s = token_major ? Strides{q.T * H * d, H * d, d} : Strides{q.T * H * d, d, q.T * d};
        if (packed) s.seq = 0;
        return s;
    };
    p.qk = strides(q.H_k, kD), p.v = strides(q.H_v, kD), p.gate = strides(q.H_v, 1);
    const long long places = packed ? chunk_places(q.n_seq, q.T) : static_cast<long long>(q.n_seq) * p.chunks;
    const long long chains = static_cast<long long>(q.n_seq) * q.H_v * kSlices;
    if (places * q.H_k >= (1LL << 31) || chains >= (1LL << 31)) return GDN_ERR_UNSUPPORTED;
    const bool ok = launch<SmemSystem>(chunk_system_kernel, places * q.H_k, p, stream) && launch<SmemF>(chunk_states_kernel, chains, p, stream) &&
                    launch<SmemB>(chunk_state_grads_kernel, chains, p, stream) && launch<SmemC>(chunk_grads_kernel, places * q.H_k, p, stream);
    return ok ? GDN_OK : GDN_ERR_LAUNCH;
}

}  // namespace gdn

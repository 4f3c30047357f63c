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
// Four launches: `chunk_system` (per chunk and key head: T, P and the gates' tables), `chunk_states` (per sequence and value head,
// forward over the chunks: S, u, z), `chunk_state_grads` (the same backward: D, r), `chunk_grads` (per chunk and key head, the value
// heads that share it in turn: dQ, dK, dV, dbeta, dg). What the later ones need of the earlier ones goes through the caller's workspace.
//
// Precision: everything between the bf16 inputs and the results is fp32. The tensor cores multiply bf16: an fp32 operand is the sum of three
// bf16 pieces (24 bits), three products where the other operand is bf16 itself, six where both are split (the three smallest of the nine are
// below 2^-24); all sums are fp32. The one rounding to fewer bits is that of dQ, dK, dV to bf16 at their end. Against fp64, relative 2-norms: dbeta
// 1.8e-7 to 2.8e-7, dg 1.6e-7 to 7e-7, dS_in 5e-8 to 2.2e-7 (the formulas in torch fp32: 2.1e-7 to 7e-7, 1.2e-7 to 1.8e-6, 6e-8 to 1.5e-7).
//
// us per launch, 8 x 4096 tokens with 32 heads / one sequence of 32768 tokens with 16 and 32 heads / 61 packed sequences of 16411 tokens
// in all: system 621 / 521 / 297, states 498 / 1512 / 306, their gradients 747 / 2658 / 488, chunks' gradients 1740 / 1526 / 948. (With
// states, p and m of two pieces in the last one, 1507 / 1450 / 852: dg was off by 3.4e-6 where <D, S> is all of it, and three times as many values of
// dQ, dK fell on the other side of a rounding.) On mma.sync with tf32 pieces the four took 742 / 628, 1615 / 2607, 3137 / 3563 and 2945 / 2756.
#include <cuda.h>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace gdn {
namespace {

using namespace sm100;

constexpr int kC = 64, kD = 128;
constexpr int kThreads = 256;

// workspace of one chunk of one value head, in floats. T and P: bf16 tiles of three pieces each (see split3), as the products want them in shared
// memory. The states [v][key] fp32, in blocks of 8 x 8 (see state_at). u, z, r [v][token] fp32: a feature of the value per row, as the
// chains have them in tensor memory, 16-byte pieces of a row out of order (see vt_at).
constexpr int kPieces = 3;
constexpr int kWsT = 0, kWsP = kWsT + kPieces * kC * kC / 2, kWsS = kWsP + kPieces * kC * kC / 2, kWsDS = kWsS + kD * kD, kWsU = kWsDS + kD * kD;
constexpr int kWsZ = kWsU + kC * kD;     // exp(g) z, then r in its place
constexpr int kWsTab = kWsZ + kC * kD;   // tables of 64 floats each
enum { TAB_EGK = 0, TAB_BETA, TAB_ECK, TAB_BEGK, TAB_SEGQ, TAB_G, TAB_GLO, TAB_RK, TAB_RQ, TAB_DECAY, kTabs };  // (G, GLO: see Gates; DECAY: exp(g_C), at 0)
constexpr int kWsDots = kWsTab + kTabs * kC;  // exp(g) <r, z>, exp(g_C - g) <u, y>
constexpr int kDots = 2;
constexpr int kWsChunk = kWsDots + kDots * kC;
static_assert(kWsChunk % 4 == 0, "16-byte pieces");

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
    int* status;
    const int* cu;  // packed sequences: their boundaries; null: n_seq sequences of T tokens
    int n_seq, T, H_k, H_v, group, chunks;  // chunks: of a dense sequence
    long long units;                        // places of chunks in the workspace times key heads
    Strides qk, v, gate;
    float scale;
    bool l2norm, token_major;
};

// The token tensors for the copy engine: [heads][tokens][128], or [batch][tokens][heads x 128] where they are token-major; boxes of 64 x 64
// in the 128-byte swizzle
struct Maps {
    CUtensorMap Q, K, V, dO;
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
// ---------------------------------------------------------------- products in registers (the Gram matrices)
// m16n8k16 bf16, fp32 accumulators
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
struct Lane {
    int g, c;  // row of a fragment, pair of columns
    __device__ __forceinline__ Lane() : g((threadIdx.x % 32) / 4), c(threadIdx.x % 4) {}
};
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

constexpr int kLdX = 136;  // bf16 rows of 128 features: 68 words, no bank conflicts
constexpr int kLdV = 68;   // fp32 rows of 64

// A value as three bf16 pieces, x = h - m + l (the middle one negated: that is how the difference comes out of one instruction): 24 bits
__device__ __forceinline__ float bf16_minus_lo(uint32_t w, float x) {
    float r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tsub.f32.bf16 %0, a, %2;\n\t}" : "=f"(r) : "r"(w), "f"(x));
    return r;
}
__device__ __forceinline__ float bf16_minus_hi(uint32_t w, float x) {
    float r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tsub.f32.bf16 %0, b, %2;\n\t}" : "=f"(r) : "r"(w), "f"(x));
    return r;
}
__device__ __forceinline__ void split3(float x, float y, uint32_t& h, uint32_t& m, uint32_t& l) {
    h = pack_bf16x2(x, y);
    const float a = bf16_minus_lo(h, x), b = bf16_minus_hi(h, y);
    m = pack_bf16x2(a, b);
    l = pack_bf16x2(bf16_minus_lo(m, a), bf16_minus_hi(m, b));
}
// Byte of element (row, col) of a 64 x 64 bf16 tile in the 128-byte swizzle: 16-byte pieces of a row change places with its number mod 8
__device__ __forceinline__ int swizzled(int row, int col) { return row * 128 + ((((col >> 3) ^ row) & 7) << 4) + (col & 7) * 2; }
constexpr int kTile = kC * kC * 2;  // bytes of such a tile
// four neighbours of a row into the three tiles of a matrix
__device__ __forceinline__ void store_pieces(float* tiles, int row, int col, const float (&x)[4]) {
    uint32_t w[kPieces][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) split3(x[2 * e], x[2 * e + 1], w[0][e], w[1][e], w[2][e]);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(tiles) + i * kTile + swizzled(row, col)) = make_uint2(w[i][0], w[i][1]);
}

// ---------------------------------------------------------------- T, P and the gates' tables
// Gates: the sums of a chunk's log-gates reach 50 in ordinary texts and 8192 where gates close, and a sum in fp32 would be off by 2^-19 to 2^-11,
// as would every decay exp(g_i - g_j) between neighbours be, relatively (r, and with it dbeta, by 1.4e-6 for ordinary gates; dbeta and dg
// by 4e-5 to 4e-4 for 8 to 60 closed ones). They are summed in fp64 and kept as hi + lo.
__device__ __forceinline__ float exp_between(float hi, float lo, float hi0, float lo0) { return expf((hi - hi0) + (lo - lo0)); }
__device__ __forceinline__ float exp_of(float hi, float lo) {  // (lo <= 2^-18 where exp is not 0)
    const float e = expf(hi);
    return fmaf(e, lo, e);
}
struct SmemSystem {
    union {
        struct {
            __nv_bfloat16 K[kC * kLdX], Q[kC * kLdX];
        } in;
        struct {
            float T[kC * kLdV], A[kC * kLdV];
        };
    };
    float kk[kC * kLdV], qk[kC * kLdV];
    float rk[kC], rq[kC], g[kC], glo[kC], beta[kC];
};

__global__ void __launch_bounds__(kThreads, 3) chunk_system_kernel(const ParamsB p) {
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
            double sum = static_cast<double>(x[0]) + x[1];
            for (int o = 1; o < 32; o *= 2) {
                const double y = __shfl_up_sync(0xffffffffu, sum, o);
                if (static_cast<int>(threadIdx.x) >= o) sum += y;
            }
            for (int e = 0; e < 2; ++e) {
                const double g = e ? sum : sum - x[1];
                sm.g[t + e] = static_cast<float>(g);
                sm.glo[t + e] = static_cast<float>(g - sm.g[t + e]);
            }
            sm.beta[t] = b[0], sm.beta[t + 1] = b[1];
        }
        __syncthreads();
        if (tid < kC) {
            const float g = sm.g[tid], lo = sm.glo[tid], eg = exp_of(g, lo), ec = exp_between(sm.g[kC - 1], sm.glo[kC - 1], g, lo), beta = sm.beta[tid], rk = sm.rk[tid], rq = sm.rq[tid];
            float* const tab = ws + kWsTab;
            const bool real = tid < rows;
            tab[TAB_EGK * kC + tid] = real ? eg * rk : 0.f;
            tab[TAB_BETA * kC + tid] = beta;
            tab[TAB_ECK * kC + tid] = real ? ec * rk : 0.f;
            tab[TAB_BEGK * kC + tid] = real ? beta * eg * rk : 0.f;
            tab[TAB_SEGQ * kC + tid] = real ? p.scale * eg * rq : 0.f;
            tab[TAB_G * kC + tid] = g;
            tab[TAB_GLO * kC + tid] = lo;
            if (tid == kC - 1) tab[TAB_DECAY * kC] = eg;
            tab[TAB_RK * kC + tid] = rk;
            tab[TAB_RQ * kC + tid] = rq;
        }
        for (int i = tid; i < kC * kC / 4; i += kThreads) {
            const int row = i / 16, col = i % 16 * 4;
            float a[4], q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = col + e;
                const float gam = j <= row ? exp_between(sm.g[row], sm.glo[row], sm.g[j], sm.glo[j]) : 0.f;
                a[e] = j < row ? sm.beta[row] * gam * sm.kk[row * kLdV + j] : 0.f;
                q[e] = j <= row ? gam * sm.qk[row * kLdV + j] : 0.f;
            }
            *reinterpret_cast<float4*>(sm.A + row * kLdV + col) = make_float4(a[0], a[1], a[2], a[3]);
            store_pieces(ws + kWsP, row, col, q);
        }
        __syncthreads();
        // T = (I + A)^-1: the two diagonal blocks of 32 by forward substitution, column j of either x_i = [i = j] - sum_k A_ik x_k, four
        // threads a column; the block below them is -T22 A21 T11. (By substitution alone the kernel, which shared memory bounds, takes 0.77 ms
        // for 16384 chunks, so 0.61.)
        {
            const int j = tid / 4, part = tid % 4, r0 = j & 32;
            float x[8];
#pragma unroll
            for (int m = 0; m < 8; ++m) x[m] = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float a = 0.f, b = 0.f;
#pragma unroll
                for (int m = 0; m <= i / 4; m += 2) {
                    a = fmaf(sm.A[(r0 + i) * kLdV + r0 + 4 * m + part], x[m], a);
                    if (m + 1 <= i / 4) b = fmaf(sm.A[(r0 + i) * kLdV + r0 + 4 * m + 4 + part], x[m + 1], b);
                }
                const float xi = (r0 + i == j ? 1.f : 0.f) - quad_sum(a + b);
                if (i % 4 == part) x[i / 4] = xi;
            }
#pragma unroll
            for (int m = 0; m < 8; ++m) sm.T[(r0 + 4 * m + part) * kLdV + j] = x[m];
        }
        __syncthreads();
        {
            const int i = tid / 8, c = tid % 8 * 4;
            const auto product = [&](const float* row, const float* m) {  // row [32] times m [32][4]
                float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                    const float4 r = *reinterpret_cast<const float4*>(row + k);
                    const float w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 v = *reinterpret_cast<const float4*>(m + (k + e) * kLdV);
                        d.x = fmaf(w[e], v.x, d.x), d.y = fmaf(w[e], v.y, d.y), d.z = fmaf(w[e], v.z, d.z), d.w = fmaf(w[e], v.w, d.w);
                    }
                }
                return d;
            };
            *reinterpret_cast<float4*>(sm.A + i * kLdV + 32 + c) = product(sm.A + (32 + i) * kLdV, sm.T + c);  // (A has nothing above its diagonal)
            *reinterpret_cast<float4*>(sm.T + i * kLdV + 32 + c) = make_float4(0.f, 0.f, 0.f, 0.f);
            __syncthreads();
            const float4 d = product(sm.T + (32 + i) * kLdV + 32, sm.A + 32 + c);
            *reinterpret_cast<float4*>(sm.T + (32 + i) * kLdV + c) = make_float4(-d.x, -d.y, -d.z, -d.w);
        }
        __syncthreads();
        for (int i = tid; i < kC * kC / 4; i += kThreads) {
            const int row = i / 16, col = i % 16 * 4;
            const float4 x = *reinterpret_cast<const float4*>(sm.T + row * kLdV + col);
            const float t[4] = {x.x, x.y, x.z, x.w};
            store_pieces(ws + kWsT, row, col, t);
        }
    }
}

// ---------------------------------------------------------------- the chains over the chunks: tcgen05, the value's features on the lanes
// One CTA has a (sequence, value head). Everything is kept transposed, a feature of the value on each of the 128 lanes of tensor memory: S
// and D [v x key], and z, u, y, r [v x token]. The fp32 operand of a product, split into three bf16 pieces, is A, in tensor memory; B is a tile in
// shared memory: K or Q as they are (both ways round), T or P in pieces. All sums are fp32 in tensor memory; the state itself stays in registers
// (32 values a thread) and takes the chunk's part, summed on its own, with one fma.
// Sixteen warps: four for each quarter of the lanes, each with a quarter of the columns. Registers have the layout of the 16 x 256 bit loads:
// row (lane / 4) and row + 8 of 16 lanes, columns 2 (lane mod 4) and the next of every 8. In it a warp's 8-byte stores fill whole sectors.
constexpr int kWorkers = 512;  // threads that do what lies between the products
constexpr uint32_t kNegA = 1u << 13;  // instruction descriptor: A negated

__device__ __forceinline__ void tm_ld32(uint32_t taddr, float (&x)[16]) {  // 16 lanes x 32 columns
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tm_ld16(uint32_t taddr, float (&x)[8]) {  // 16 lanes x 16 columns
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r[i]);
}
// the reverse for packed pairs: 16 lanes x 8 or 16 columns of pairs
__device__ __forceinline__ void tm_st_pairs(uint32_t taddr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tm_st_pairs(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// 2 N values of 16 lanes, split, into the columns of the three pieces (`apart` columns from one piece to the next)
template <int N>
__device__ __forceinline__ void tm_st_split(uint32_t taddr, uint32_t apart, const float (&x)[2 * N]) {
    uint32_t h[N], m[N], l[N];
#pragma unroll
    for (int i = 0; i < N; ++i) split3(x[2 * i], x[2 * i + 1], h[i], m[i], l[i]);
    tm_st_pairs(taddr, h);
    tm_st_pairs(taddr + apart, m);
    tm_st_pairs(taddr + 2 * apart, l);
}
__device__ __forceinline__ void ldmatrix_turned(uint32_t at, uint32_t (&w)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
}
// [token][feature] rows turned: four 8 x 8 blocks, tokens t0 .. t0 + 15 and features v0 .. v0 + 15, as pairs of tokens: w[0], w[1] features
// v0 .. and v0 + 8 .. of the first 8 tokens, w[2], w[3] of the others (the layout of the accumulators' registers)
__device__ __forceinline__ void turned(const uint8_t* tile, int t0, int v0, uint32_t (&w)[4]) {
    const int lane = threadIdx.x % 32, t = t0 + (lane & 7) + (lane >> 4) * 8, v = v0 + ((lane >> 3) & 1) * 8;
    ldmatrix_turned(smem_u32(tile + v / 64 * kTile + swizzled(t, v % 64)), w);
}
// 64 tokens of 128 bf16 as two 64 x 64 tiles in the 128-byte swizzle; one thread asks. A box takes what lies behind a sequence's end too:
// those rows are cleared when it has come (clear_tail), for 0 times what is there need not be 0.
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap& map, const ParamsB& p, int heads, int s, int t, int h, uint64_t* bar) {
    const int x = p.token_major ? h * kD : 0, z = p.cu != nullptr ? (p.token_major ? 0 : h) : (p.token_major ? s : s * heads + h);
    tma_load_3d(dst, &map, bar, x, t, z);
    tma_load_3d(dst + kTile, &map, bar, x + 64, t, z);
}
// rows from `rows` on of a tile, by N threads
template <int N>
__device__ __forceinline__ void clear_tail(uint8_t* tile, int rows, int me) {
    for (int i = rows * 8 + me; i < kC * 8; i += N) {
        reinterpret_cast<uint4*>(tile)[i] = make_uint4(0u, 0u, 0u, 0u);
        reinterpret_cast<uint4*>(tile + kTile)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}
// whole runs of bytes (multiples of 16): one thread asks, the copy engine does it
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
// brings them into L2
__device__ __forceinline__ void bulk_prefetch(const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<uint64_t>(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* line) { asm volatile("prefetch.global.L2 [%0];" ::"l"(line) : "memory"); }
__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(smem_u32(src)), "r"(bytes) : "memory");
}

// Bounded wait (about a second) of every thread for products in flight
__device__ __forceinline__ bool wait_products(uint64_t* bar, uint32_t parity) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    uint32_t i = 0;
    while (!mbar_try_wait_hint(bar, parity, 2000u))
        if ((++i & 63u) == 0 && clock64() - t0 > 2000000000LL) return false;
    return true;
}
// what a thread has written to tensor memory is there for whoever issues products behind the next barrier
__device__ __forceinline__ void publish() {
    tmem_wait_st();
    tc_fence_before_sync();
}
// hand-offs: the computing warps arrive and go on, N threads wait. Each is passed once a chunk, and a barrier of the whole CTA lies between two chunks.
template <int ID, int N = 32>
__device__ __forceinline__ void arrive() {
    asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(kWorkers + N) : "memory");
}
template <int ID, int N = 32>
__device__ __forceinline__ void await() {
    asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(kWorkers + N) : "memory");
}

// Products of the chains, each issued by one thread. A [128 lanes x K] in three pieces of K / 2 columns at `a`; the small ones first.
__device__ __forceinline__ uint64_t desc_rows(uint32_t tile) { return smem_desc(tile, 16, 1024, SWZ_128B); }      // sum index along the rows
__device__ __forceinline__ uint64_t desc_cols(uint32_t tile) { return smem_desc(tile, kTile, 1024, SWZ_128B); }  // sum index down the rows
constexpr uint32_t kIdescRows = instr_desc(128, 64, 1, 1, 0, 0, 1), kIdescCols = instr_desc(128, 64, 1, 1, 0, 1, 1);
// d = A X^T, X: 64 rows of 128 bf16 (two tiles)
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t x) {
    const uint64_t b = desc_rows(x);
#pragma unroll
    for (int i = kPieces - 1; i >= 0; --i)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            mma_f16_ts(d, a + i * 64 + k * 8, b + ((k >> 2) * kTile + (k & 3) * 32) / 16, kIdescRows | (i == 1 ? kNegA : 0u), i < kPieces - 1 || k > 0);
}
// d (128 columns, += if `more`) = A X, A [128 x 64 tokens], X as above
__device__ __forceinline__ void product_cols(uint32_t d, uint32_t a, uint32_t x, bool more) {
    const uint64_t b = desc_cols(x);
    constexpr uint32_t idesc = instr_desc(128, 128, 1, 1, 0, 1, 1);
#pragma unroll
    for (int i = kPieces - 1; i >= 0; --i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            mma_f16_ts(d, a + i * 32 + k * 8, b + k * 2048 / 16, idesc | (i == 1 ? kNegA : 0u), more || i < kPieces - 1 || k > 0);
}
// d = A M^T (COLS: A M), both in three pieces, M 64 x 64 in three tiles: the six products of pieces that fp32 can hold. (M is triangular, and
// products of only the columns that 16 of the sum have a part in would be 62 % of the work; but a change of an instruction's shape costs more.)
template <bool COLS>
__device__ __forceinline__ void product_system(uint32_t d, uint32_t a, uint32_t tiles) {
    const uint64_t b = COLS ? desc_cols(tiles) : desc_rows(tiles);
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = sum; i >= 0; --i)
#pragma unroll
            for (int k = 0; k < 4; ++k)  // pieces i of A and sum - i of M; one middle piece: negated
                mma_f16_ts(d, a + i * 32 + k * 8, b + ((sum - i) * kTile + k * (COLS ? 2048 : 32)) / 16,
                           (COLS ? kIdescCols : kIdescRows) | ((i == 1) != (sum - i == 1) ? kNegA : 0u), sum < 2 || i < 2 || k > 0);
}
// d = A P, A [128 x 64 tokens] bf16, P in three tiles
__device__ __forceinline__ void product_pairs(uint32_t d, uint32_t a, uint32_t tiles) {
    const uint64_t b = desc_cols(tiles);
#pragma unroll
    for (int i = kPieces - 1; i >= 0; --i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            mma_f16_ts(d, a + k * 8, b + (i * kTile + k * 2048) / 16, kIdescCols | (i == 1 ? kNegA : 0u), i < kPieces - 1 || k > 0);
}

// a value for each of a thread's 8 x 2 rows and columns: `f(row, column, i)` gets the place of x[i], x[i + 1] (neighbouring columns)
template <int N, typename F>
__device__ __forceinline__ void for_pairs(const F& f) {
    const Lane l;
#pragma unroll
    for (int i = 0; i < N; i += 2) f(l.g + ((i >> 1) & 1) * 8, (i >> 2) * 8 + 2 * l.c, i);
}

constexpr int kLoaders = 32;
constexpr int kChainThreads = kWorkers + 32 + kLoaders;  // sixteen warps that compute, one that issues the products, one that asks for tiles and has them stored
constexpr int kImage = kD * kD * 4;  // bytes of a state
// Byte of element (row, col) of a state: blocks of 8 x 8 values, which a warp writes at once
__device__ __forceinline__ int state_at(int row, int col) { return (row / 8 * (kD / 8) + col / 8) * 256 + row % 8 * 32 + col % 8 * 4; }
// Byte of element (row, token) of u, z or r: 16-byte pieces change places, two by two, with the row's number mod 8: what a warp writes at once (8
// rows of 8 tokens) lies on all banks
__device__ __forceinline__ int vt_at(int row, int t) { return row * (kC * 4) + ((((t >> 2) ^ (row << 1)) & 15) << 4) + (t & 3) * 4; }
// this thread's part of such a matrix
__device__ __forceinline__ void put_vt(uint8_t* to, const float (&x)[2][8], int row0, int quarter) {
#pragma unroll
    for (int lh = 0; lh < 2; ++lh)
        for_pairs<8>([&](int row, int col, int i) {
            *reinterpret_cast<float2*>(to + vt_at(row0 + lh * 16 + row, quarter * 16 + col)) = make_float2(x[lh][i], x[lh][i + 1]);
        });
}
// this thread's part of a state (see for_pairs) into the image
__device__ __forceinline__ void put_image(uint8_t* image, const float (&S)[2][16], int row0, int quarter) {
#pragma unroll
    for (int lh = 0; lh < 2; ++lh)
        for_pairs<16>([&](int row, int col, int i) {
            *reinterpret_cast<float2*>(image + state_at(row0 + lh * 16 + row, quarter * 32 + col)) = make_float2(S[lh][i], S[lh][i + 1]);
        });
}

// the sum over the lanes of a column group of four tokens' values; a lane gets that of token place l.g / 2
__device__ __forceinline__ float token_sum(const float (&x)[4], const Lane& l) {
    float a[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float keep = l.g & 4 ? x[2 + i] : x[i], give = l.g & 4 ? x[i] : x[2 + i];
        a[i] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
    }
    const float keep = l.g & 2 ? a[1] : a[0], give = l.g & 2 ? a[0] : a[1];
    const float b = keep + __shfl_xor_sync(0xffffffffu, give, 8);
    return b + __shfl_xor_sync(0xffffffffu, b, 4);
}

// tensor memory: the state's part of the chunk (128 columns), the state's pieces, z or u, the pieces of the right-hand side or of u
constexpr uint32_t kTmDelta = 0, kTmState = 128, kTmAcc = 320, kTmRhs = 384, kTmColumns = 512;

struct Chain {
    uint64_t *done, *full;  // products complete; copies of a chunk's tiles complete
    uint32_t tm, lanes;     // base; this warp's lanes in the address
    uint32_t phase = 0;
    bool failed = false;
    __device__ __forceinline__ void wait() {
        failed = failed || !wait_products(done, phase);
        phase ^= 1;
        tc_fence_after_sync();
    }
};
__device__ __forceinline__ void chain_begin(Chain& ch, uint64_t* bars, uint32_t* base, uint32_t columns) {
    if (threadIdx.x == 0) {
        mbar_init(bars, 1);
        mbar_init(bars + 1, 1);
        mbar_fence_init();
    }
    if (threadIdx.x < 32) {
        tmem_alloc(base, columns);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    ch.done = bars;
    ch.full = bars + 1;
    ch.tm = *base;
    ch.lanes = static_cast<uint32_t>(threadIdx.x / 32 % 4 * 32) << 16;
}
__device__ __forceinline__ void chain_end(Chain& ch, int* status, uint32_t columns) {
    if (ch.failed) *status = GDN_ERR_TIMEOUT;
    tc_fence_before_sync();
    __syncthreads();
    if (threadIdx.x < 32) tmem_dealloc(ch.tm, columns);
}

// Forward: z, u and the state at the start of every chunk. A chunk's chain is three products (24 of 128 x 64 x 16 each, 1000 cycles with their
// completion) and, between them, the splitting of what the next one reads (700 to 1200 cycles): z -> right-hand side -> u -> state, 3.0 us a
// chunk. What goes to memory (the state, z, u) goes while products run, through shared memory and the copy engine: stored by the threads it
// took 4.4 us, because their stores, 8 rows at a time, kept the loads waiting.
struct alignas(1024) StageF {  // (the tiles lie on 1 KB)
    uint8_t K[2 * kTile], V[2 * kTile], T[kPieces * kTile];
    float tab[kTabs * kC];
};
struct SmemF {
    StageF stage[2];
    uint8_t image[kImage];  // (u after it)
    uint8_t z[kD * kC * 4];
};

__global__ void __launch_bounds__(kChainThreads, 1) chunk_states_kernel(const ParamsB p, const __grid_constant__ Maps maps) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemF& sm = *reinterpret_cast<SmemF*>(smem_raw + ((0u - smem_u32(smem_raw)) & 1023u));
    __shared__ uint64_t bars[2];
    __shared__ uint32_t base;
    const int h = blockIdx.x % p.H_v, s = blockIdx.x / p.H_v, hk = h / p.group;
    const Seq seq = seq_of(p, s);
    const int n = (seq.len + kC - 1) / kC;
    const int warp = threadIdx.x / 32;
    Chain ch;
    chain_begin(ch, bars, &base, kTmColumns);
    if (warp == kWorkers / 32) {  // ---- the products
        for (int c = 0; c < n; ++c) {
            StageF& st = sm.stage[c % 2];
            const uint32_t tileK = smem_u32(st.K), tileT = smem_u32(st.T);
            ch.failed |= !wait_products(ch.full, c & 1);  // (before the barrier: behind it the next copies are asked for)
            if (__syncthreads_or(ch.failed)) break;
            tc_fence_after_sync();
            if (elect_one()) {
                product_rows(ch.tm + kTmAcc, ch.tm + kTmState, tileK);
                mma_commit(ch.done);
            }
            __syncwarp();
            await<1>();
            tc_fence_after_sync();
            if (elect_one()) {
                product_system<false>(ch.tm + kTmAcc, ch.tm + kTmRhs, tileT);
                mma_commit(ch.done);
            }
            __syncwarp();
            await<2>();
            tc_fence_after_sync();
            if (elect_one()) {
                product_cols(ch.tm + kTmDelta, ch.tm + kTmRhs, tileK, false);
                mma_commit(ch.done);
            }
            __syncwarp();
        }
    } else if (warp > kWorkers / 32) {  // ---- the tiles
        const int me = threadIdx.x - kWorkers - 32;
        const auto load = [&](int c) {
            if (c < n && me == 0) {
                StageF& st = sm.stage[c % 2];
                const float* const ws = chunk_ws(p, seq.slot + c, h);
                mbar_arrive_expect_tx(ch.full, sizeof(st.K) + sizeof(st.V) + sizeof(st.T) + sizeof(st.tab));
                load_tile(st.K, maps.K, p, p.H_k, s, seq.first + c * kC, hk, ch.full);
                load_tile(st.V, maps.V, p, p.H_v, s, seq.first + c * kC, h, ch.full);
                bulk_load(st.T, ws + kWsT, sizeof(st.T), ch.full);
                bulk_load(st.tab, ws + kWsTab, sizeof(st.tab), ch.full);
            }
            __syncwarp();
        };
        load(0);
        for (int c = 0; c < n; ++c) {
            tma_store_wait_read<0>();  // the image may be written again
            ch.failed |= !wait_products(ch.full, c & 1);
            if (seq.len - c * kC < kC) {
                clear_tail<kLoaders>(sm.stage[c % 2].K, seq.len - c * kC, me);
                clear_tail<kLoaders>(sm.stage[c % 2].V, seq.len - c * kC, me);
                fence_proxy_async_smem();
            }
            if (__syncthreads_or(ch.failed)) break;
            load(c + 1);
            await<3, kLoaders>();
            if (me == 0) {
                bulk_store(chunk_ws(p, seq.slot + c, h) + kWsS, sm.image, kImage);
                tma_store_commit();
            }
            __syncwarp();
            await<4, kLoaders>();
            if (me == 0) {
                bulk_store(chunk_ws(p, seq.slot + c, h) + kWsZ, sm.z, sizeof(sm.z));
                tma_store_commit();
            }
            __syncwarp();
            tma_store_wait_read<1>();  // the image is on its way: u may have its place
            arrive<5, kLoaders>();
            await<6, kLoaders>();
            if (me == 0) {
                bulk_store(chunk_ws(p, seq.slot + c, h) + kWsU, sm.image, sizeof(sm.z));
                tma_store_commit();
            }
            __syncwarp();
        }
        tma_store_wait_all<0>();
    } else {  // ---- what lies between the products
        const int quarter = warp / 4, row0 = warp % 4 * 32;
        float S[2][16];
        const long long state = (static_cast<long long>(s) * p.H_v + h) * kD * kD;
#pragma unroll
        for (int lh = 0; lh < 2; ++lh)
            for_pairs<16>([&](int row, int col, int i) {
                const float2 x = p.S_in == nullptr ? make_float2(0.f, 0.f)
                                                   : *reinterpret_cast<const float2*>(p.S_in + state + (row0 + lh * 16 + row) * kD + quarter * 32 + col);
                S[lh][i] = x.x, S[lh][i + 1] = x.y;
            });
        for (int c = 0; c < n; ++c) {
            const StageF& st = sm.stage[c % 2];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) tm_st_split<8>(ch.tm + ch.lanes + (lh << 20) + kTmState + quarter * 16, 64, S[lh]);
            publish();
            if (__syncthreads_or(ch.failed)) break;
            put_image(sm.image, S, row0, quarter);
            fence_proxy_async_smem();
            arrive<3, kLoaders>();
            uint32_t v[2][4];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) turned(st.V, quarter * 16, row0 + lh * 16, v[lh]);
            ch.wait();
            float z[2][8];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float x[8];
                tm_ld16(ch.tm + ch.lanes + (lh << 20) + kTmAcc + quarter * 16, z[lh]);
                tmem_wait_ld();
                for_pairs<8>([&](int, int col, int i) {
                    const int t = quarter * 16 + col;
                    const float2 e = *reinterpret_cast<const float2*>(st.tab + TAB_EGK * kC + t), b = *reinterpret_cast<const float2*>(st.tab + TAB_BETA * kC + t);
                    z[lh][i] *= e.x, z[lh][i + 1] *= e.y;
                    x[i] = b.x * (bf16_lo(v[lh][i / 2]) - z[lh][i]), x[i + 1] = b.y * (bf16_hi(v[lh][i / 2]) - z[lh][i + 1]);
                });
                tm_st_split<4>(ch.tm + ch.lanes + (lh << 20) + kTmRhs + quarter * 8, 32, x);
            }
            publish();
            arrive<1>();
            put_vt(sm.z, z, row0, quarter);
            fence_proxy_async_smem();
            arrive<4, kLoaders>();
            ch.wait();
            float u[2][8];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float x[8];
                tm_ld16(ch.tm + ch.lanes + (lh << 20) + kTmAcc + quarter * 16, u[lh]);
                tmem_wait_ld();
                for_pairs<8>([&](int, int col, int i) {
                    const float2 e = *reinterpret_cast<const float2*>(st.tab + TAB_ECK * kC + quarter * 16 + col);
                    x[i] = u[lh][i] * e.x, x[i + 1] = u[lh][i + 1] * e.y;
                });
                tm_st_split<4>(ch.tm + ch.lanes + (lh << 20) + kTmRhs + quarter * 8, 32, x);
            }
            publish();
            arrive<2>();
            await<5, kLoaders>();
            put_vt(sm.image, u, row0, quarter);
            fence_proxy_async_smem();
            arrive<6, kLoaders>();
            const float decay = st.tab[TAB_DECAY * kC];
            ch.wait();
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float x[16];
                tm_ld32(ch.tm + ch.lanes + (lh << 20) + kTmDelta + quarter * 32, x);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) S[lh][i] = fmaf(decay, S[lh][i], x[i]);
            }
        }
    }
    chain_end(ch, p.status, kTmColumns);
}

// Backward: r and the state's gradient at the end of every chunk, 5.3 us a chunk: four products on the chain, two more beside it.
struct alignas(1024) StageB {
    uint8_t K[2 * kTile], Q[2 * kTile], dO[2 * kTile];
    float tab[kTabs * kC];
};
struct SmemB {
    StageB stage[2];
    uint8_t T[kPieces * kTile], P[kPieces * kTile];  // (loaded again behind their last product of the chunk)
    uint8_t image[kImage];
    float dots[4][kDots][kC];
};
// tensor memory: the state's part; its gradient's pieces, and when these are used up those of du or -beta exp(g) r (96 columns) and of scale
// exp(g) dO (96); y or r; P^T dO; dO
constexpr uint32_t kTmDu = kTmState, kTmW = kTmState + 96, kTmX = 384, kTmO = 448;

__global__ void __launch_bounds__(kChainThreads, 1) chunk_state_grads_kernel(const ParamsB p, const __grid_constant__ Maps maps) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemB& sm = *reinterpret_cast<SmemB*>(smem_raw + ((0u - smem_u32(smem_raw)) & 1023u));
    __shared__ uint64_t bars[2];
    __shared__ uint32_t base;
    const int h = blockIdx.x % p.H_v, s = blockIdx.x / p.H_v, hk = h / p.group;
    const Seq seq = seq_of(p, s);
    const int n = (seq.len + kC - 1) / kC;
    const int warp = threadIdx.x / 32;
    Chain ch;
    chain_begin(ch, bars, &base, kTmColumns);
    if (warp == kWorkers / 32) {  // ---- the products
        uint32_t turn = 0;
        for (int c = n - 1; c >= 0; --c) {
            StageB& st = sm.stage[c % 2];
            const uint32_t tileK = smem_u32(st.K), tileQ = smem_u32(st.Q);
            ch.failed |= !wait_products(ch.full, turn);
            turn ^= 1;
            if (__syncthreads_or(ch.failed)) break;
            tc_fence_after_sync();
            if (elect_one()) product_rows(ch.tm + kTmAcc, ch.tm + kTmState, tileK);  // D K^T
            __syncwarp();
            await<1>();
            tc_fence_after_sync();
            if (elect_one()) {  // dO^T P
                product_pairs(ch.tm + kTmX, ch.tm + kTmO, smem_u32(sm.P));
                mma_commit(ch.done);
            }
            __syncwarp();
            await<2>();
            tc_fence_after_sync();
            if (elect_one()) {
                product_system<true>(ch.tm + kTmAcc, ch.tm + kTmDu, smem_u32(sm.T));
                mma_commit(ch.done);
            }
            __syncwarp();
            await<3>();
            tc_fence_after_sync();
            if (elect_one()) product_cols(ch.tm + kTmDelta, ch.tm + kTmW, tileQ, false);
            __syncwarp();
            await<4>();
            tc_fence_after_sync();
            if (elect_one()) {
                product_cols(ch.tm + kTmDelta, ch.tm + kTmDu, tileK, true);
                mma_commit(ch.done);
            }
            __syncwarp();
        }
    } else if (warp > kWorkers / 32) {  // ---- the tiles
        const int me = threadIdx.x - kWorkers - 32;
        uint32_t turn = 0;
        // K, Q, dO have two stages; T and P one: they are asked for behind their last product of the chunk before
        const auto load = [&](int c) {
            if (c >= 0 && me == 0) {
                StageB& st = sm.stage[c % 2];
                mbar_arrive_expect_tx(ch.full, sizeof(st.K) + sizeof(st.Q) + sizeof(st.dO) + sizeof(st.tab) + sizeof(sm.T) + sizeof(sm.P));
                load_tile(st.K, maps.K, p, p.H_k, s, seq.first + c * kC, hk, ch.full);
                load_tile(st.Q, maps.Q, p, p.H_k, s, seq.first + c * kC, hk, ch.full);
                load_tile(st.dO, maps.dO, p, p.H_v, s, seq.first + c * kC, h, ch.full);
                bulk_load(st.tab, chunk_ws(p, seq.slot + c, h) + kWsTab, sizeof(st.tab), ch.full);
            }
            __syncwarp();
        };
        const auto load_system = [&](int c) {
            if (c >= 0 && me == 0) bulk_load(sm.T, chunk_ws(p, seq.slot + c, h) + kWsT, sizeof(sm.T) + sizeof(sm.P), ch.full);
            __syncwarp();
        };
        load(n - 1);
        load_system(n - 1);
        for (int c = n - 1; c >= 0; --c) {
            tma_store_wait_read<0>();
            ch.failed |= !wait_products(ch.full, turn);
            turn ^= 1;
            if (seq.len - c * kC < kC) {
                clear_tail<kLoaders>(sm.stage[c % 2].K, seq.len - c * kC, me);
                clear_tail<kLoaders>(sm.stage[c % 2].Q, seq.len - c * kC, me);
                clear_tail<kLoaders>(sm.stage[c % 2].dO, seq.len - c * kC, me);
                fence_proxy_async_smem();
            }
            if (__syncthreads_or(ch.failed)) break;
            load(c - 1);
            await<5, kLoaders>();
            if (me == 0) {
                bulk_store(chunk_ws(p, seq.slot + c, h) + kWsDS, sm.image, kImage);
                tma_store_commit();
            }
            __syncwarp();
            await<6, kLoaders>();  // T and P are used up
            load_system(c - 1);
            if (c > 0 && me == 0) bulk_prefetch(chunk_ws(p, seq.slot + c - 1, h) + kWsU, 2 * sizeof(float) * kC * kD);
            __syncwarp();
        }
        tma_store_wait_all<0>();
    } else {  // ---- what lies between the products
        const int quarter = warp / 4, row0 = warp % 4 * 32;
        const Lane l;
        float D[2][16];
        const long long state = (static_cast<long long>(s) * p.H_v + h) * kD * kD;
#pragma unroll
        for (int lh = 0; lh < 2; ++lh)
            for_pairs<16>([&](int row, int col, int i) {
                const float2 x = p.dS_out == nullptr ? make_float2(0.f, 0.f)
                                                     : *reinterpret_cast<const float2*>(p.dS_out + state + (row0 + lh * 16 + row) * kD + quarter * 32 + col);
                D[lh][i] = x.x, D[lh][i + 1] = x.y;
            });
        for (int c = n - 1; c >= 0; --c) {
            const StageB& st = sm.stage[c % 2];
            float* const ws = chunk_ws(p, seq.slot + c, h);
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) tm_st_split<8>(ch.tm + ch.lanes + (lh << 20) + kTmState + quarter * 16, 64, D[lh]);
            publish();
            if (__syncthreads_or(ch.failed)) break;
            float2 u[2][4];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {  // dO, its features on the lanes
                uint32_t w[4];
                turned(st.dO, quarter * 16, row0 + lh * 16, w);
                tm_st_pairs(ch.tm + ch.lanes + (lh << 20) + kTmO + quarter * 8, w);
            }
            publish();
            arrive<1>();
#pragma unroll
            for (int lh = 0; lh < 2; ++lh)
                for_pairs<8>([&](int row, int col, int i) {
                    u[lh][i / 2] = *reinterpret_cast<const float2*>(reinterpret_cast<const uint8_t*>(ws + kWsU) + vt_at(row0 + lh * 16 + row, quarter * 16 + col));
                });
            put_image(sm.image, D, row0, quarter);
            fence_proxy_async_smem();
            arrive<5, kLoaders>();
            ch.wait();
            float dots[kDots][4] = {};  // of this thread's four tokens: 8 (i / 4) + 2 c + e at [i / 4 * 2 + e]
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float y[8], x[8];
                tm_ld16(ch.tm + ch.lanes + (lh << 20) + kTmAcc + quarter * 16, y);
                tm_ld16(ch.tm + ch.lanes + (lh << 20) + kTmX + quarter * 16, x);
                tmem_wait_ld();
                for_pairs<8>([&](int, int col, int i) {
                    const float2 e = *reinterpret_cast<const float2*>(st.tab + TAB_ECK * kC + quarter * 16 + col);
                    const float y0 = e.x * y[i], y1 = e.y * y[i + 1];
                    dots[1][i / 4 * 2] = fmaf(u[lh][i / 2].x, y0, dots[1][i / 4 * 2]);
                    dots[1][i / 4 * 2 + 1] = fmaf(u[lh][i / 2].y, y1, dots[1][i / 4 * 2 + 1]);
                    x[i] += y0, x[i + 1] += y1;
                });
                tm_st_split<4>(ch.tm + ch.lanes + (lh << 20) + kTmDu + quarter * 8, 32, x);
            }
            publish();
            arrive<2>();
            float2 z[2][4];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh)
                for_pairs<8>([&](int row, int col, int i) {
                    z[lh][i / 2] = *reinterpret_cast<const float2*>(reinterpret_cast<const uint8_t*>(ws + kWsZ) + vt_at(row0 + lh * 16 + row, quarter * 16 + col));
                });
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float x[8];
                uint32_t w[4];
                turned(st.dO, quarter * 16, row0 + lh * 16, w);
                for_pairs<8>([&](int, int col, int i) {
                    const float2 e = *reinterpret_cast<const float2*>(st.tab + TAB_SEGQ * kC + quarter * 16 + col);
                    const uint32_t o = w[i / 2];
                    x[i] = e.x * bf16_lo(o), x[i + 1] = e.y * bf16_hi(o);
                });
                tm_st_split<4>(ch.tm + ch.lanes + (lh << 20) + kTmW + quarter * 8, 32, x);
            }
            publish();
            arrive<3>();
            ch.wait();  // (for r; what was issued behind it may still run)
            arrive<6, kLoaders>();
            float r[2][8];
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float x[8];
                tm_ld16(ch.tm + ch.lanes + (lh << 20) + kTmAcc + quarter * 16, r[lh]);
                tmem_wait_ld();
                for_pairs<8>([&](int, int col, int i) {
                    const float2 e = *reinterpret_cast<const float2*>(st.tab + TAB_BEGK * kC + quarter * 16 + col);
                    x[i] = -e.x * r[lh][i], x[i + 1] = -e.y * r[lh][i + 1];
                });
                tm_st_split<4>(ch.tm + ch.lanes + (lh << 20) + kTmDu + quarter * 8, 32, x);
            }
            publish();
            arrive<4>();
#pragma unroll
            for (int lh = 0; lh < 2; ++lh)
                for_pairs<8>([&](int, int, int i) {
                    dots[0][i / 4 * 2] = fmaf(r[lh][i], z[lh][i / 2].x, dots[0][i / 4 * 2]);
                    dots[0][i / 4 * 2 + 1] = fmaf(r[lh][i + 1], z[lh][i / 2].y, dots[0][i / 4 * 2 + 1]);
                });
            put_vt(reinterpret_cast<uint8_t*>(ws + kWsZ), r, row0, quarter);
#pragma unroll
            for (int d = 0; d < kDots; ++d) {
                const float sum = token_sum(dots[d], l);
                if ((l.g & 1) == 0) sm.dots[warp % 4][d][quarter * 16 + (l.g >> 2) * 8 + 2 * l.c + ((l.g >> 1) & 1)] = sum;
            }
            const float decay = st.tab[TAB_DECAY * kC];
            asm volatile("bar.sync 7, %0;" ::"n"(kWorkers) : "memory");
            if (threadIdx.x < kDots * kC) {
                const float* const at = &sm.dots[0][0][threadIdx.x];
                ws[kWsDots + threadIdx.x] = (at[0] + at[kDots * kC]) + (at[2 * kDots * kC] + at[3 * kDots * kC]);
            }
            ch.wait();
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float x[16];
                tm_ld32(ch.tm + ch.lanes + (lh << 20) + kTmDelta + quarter * 32, x);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) D[lh][i] = fmaf(decay, D[lh][i], x[i]);
            }
        }
        if (p.dS_in != nullptr) {
#pragma unroll
            for (int lh = 0; lh < 2; ++lh)
                for_pairs<16>([&](int row, int col, int i) {
                    *reinterpret_cast<float2*>(p.dS_in + state + (row0 + lh * 16 + row) * kD + quarter * 32 + col) = make_float2(D[lh][i], D[lh][i + 1]);
                });
        }
    }
    chain_end(ch, p.status, kTmColumns);
}

// ---------------------------------------------------------------- the chunks' gradients
// One CTA has a (chunk, key head) and takes the value heads that share it in turn. dQ and dK are summed transposed, a key feature on each of the
// 128 lanes: A is S or D (tiles [v][key], read down the rows) or K or Q (read down the rows), B is dO, r, u, p or m (64 tokens wide). p and m
// come from products of 64 x 64 (rows on 16 lanes of every quarter). Everything fp32 has three pieces. Those of S or D take 96 KB, and 64 are free: the
// third one takes the place of the second when this one's products are done (S), or that of p and m (D). A value head's chunk reads and writes 307 KB
// (6.9 us of an SM's share of the measured HBM rate); it takes 15.7 us, the chain of some twenty phases of 16 warps between 256 products. 208 KB of
// operands leave no room for a second CTA. The products of pairs, which do not need S, run while S is split: 1.87 -> 1.74 ms for 16384 chunks. What
// the next chunk reads comes into L2 meanwhile, and S, u and r of it into shared memory behind this one's last product: without either 20 us.
constexpr int kGradThreads = 512;  // 16 warps, and one that issues the products and the copies of S and D

struct SmemC {
    uint8_t K[2 * kTile], Q[2 * kTile], dO[2 * kTile];
    uint8_t S[kImage];                                     // the state, then its gradient, as they come; then two pieces, tiles [v][64 keys]
    // [v][token] in pieces. Before that u and r as they come, in the first 64 KB; later p and m in the place of r, three pieces each, and
    // the third piece of the state's gradient in the place of p and m; at the end dQ and dK on their way out, in the last 32 KB
    uint8_t u[kPieces][2 * kTile], r[kPieces][2 * kTile];
    float tab[kTabs * kC];
    float rowq[4][kC], rown[4][kC], rowb[4][kC], coln[4][kC], rv[2][kC], norm[2][4][kC];
    float ds[kGradThreads / 32];
};
constexpr int kRaw = kC * kD * 4;  // bytes of u or r
struct Unit {  // what a CTA takes next: a chunk of a key head
    int ok, slot, hk, s, first, rows;
};

template <int ID>
__device__ __forceinline__ void grad_arrive() {
    asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(kGradThreads + 32) : "memory");
}
template <int ID>
__device__ __forceinline__ void grad_await() {
    asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(kGradThreads + 32) : "memory");
}
__device__ __forceinline__ void grad_sync() { asm volatile("bar.sync 5, %0;" ::"n"(kGradThreads) : "memory"); }

// N products over K in steps of 16: A and B advance by their steps (bytes); `half_a`, `half_b`: extra step behind every 64
template <int N>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, int step_a, uint64_t b, int step_b, uint32_t idesc, bool more) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int ka = step_a == 32 ? (k >> 2) * kTile + (k & 3) * 32 : k * step_a, kb = step_b == 32 ? (k >> 2) * kTile + (k & 3) * 32 : k * step_b;
        mma_f16_ss(d, a + ka / 16, b + kb / 16, idesc, more || k > 0);
    }
}
constexpr int kAlong = 32, kDown = 2048;  // steps of an operand whose sum index runs along the rows, down the rows
__host__ __device__ constexpr uint32_t grad_idesc(int m, bool a_down, bool b_down, bool minus) {
    return instr_desc(m, 64, 1, 1, a_down, b_down, 1) | (minus ? kNegA : 0u);
}
constexpr uint32_t kTmDOS = 0, kTmRS = 64, kTmUD = 128, kTmDQ = 192, kTmDK = 256, kTmOU = 320, kTmRU = 384, kTmKK = kTmDQ, kTmQK = kTmDK;

__global__ void __launch_bounds__(kGradThreads + 32, 1) chunk_grads_kernel(const ParamsB p, const __grid_constant__ Maps maps) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SmemC& sm = *reinterpret_cast<SmemC*>(smem_raw + ((0u - smem_u32(smem_raw)) & 1023u));
    __shared__ uint64_t bar_pair, bar_s, bar_l, bar_out, bar_d, bar_load, bar_tile;
    __shared__ uint32_t base;
    __shared__ Unit units[2];
    const int tid = threadIdx.x, warp = tid / 32;
    const Lane l;
    bool failed = false;
    // the unit at or after place `at` of this CTA's (every gridDim.x-th); places that hold no chunk are passed over
    const auto find_unit = [&](long long at) {
        Unit x{0, 0, 0, 0, 0, 0};
        for (; at < p.units; at += gridDim.x) {
            x.slot = static_cast<int>(at / p.H_k), x.hk = static_cast<int>(at % p.H_k);
            if (chunk_of(p, x.slot, x.s, x.first, x.rows)) {
                x.ok = 1;
                break;
            }
        }
        return x;
    };
    if (tid == 0) {
        units[0] = find_unit(blockIdx.x);
        for (uint64_t* b : {&bar_pair, &bar_s, &bar_l, &bar_out, &bar_d, &bar_load, &bar_tile}) mbar_init(b, 1);
        mbar_fence_init();
    }
    if (warp == 0) {
        tmem_alloc(&base, kTmColumns);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = base;
    const int heads = p.group;

    if (warp == kGradThreads / 32) {  // ---- products and the copies of S and D
        const uint32_t K = smem_u32(sm.K), Q = smem_u32(sm.Q), dO = smem_u32(sm.dO), S = smem_u32(sm.S);
        const auto tile_u = [&](int i) { return smem_u32(sm.u[i]); };
        const auto tile_r = [&](int i) { return smem_u32(sm.r[i]); };
        const auto state = [&](int i) { return smem_desc(S + i * (kImage / 2), 2 * kTile, 1024, SWZ_128B); };
        // a state's second piece times the upper two of u or r, and its first one times all three. (The third one's product comes on its own.)
        const auto products_second = [&](uint32_t d, const auto& tile) {
            product<8>(d, state(1), kDown, desc_cols(tile(1)), kDown, grad_idesc(128, true, true, false), false);
            product<8>(d, state(1), kDown, desc_cols(tile(0)), kDown, grad_idesc(128, true, true, true), true);
        };
        const auto products_first = [&](uint32_t d, const auto& tile) {
            product<8>(d, state(0), kDown, desc_cols(tile(2)), kDown, grad_idesc(128, true, true, false), true);
            product<8>(d, state(0), kDown, desc_cols(tile(1)), kDown, grad_idesc(128, true, true, true), true);
            product<8>(d, state(0), kDown, desc_cols(tile(0)), kDown, grad_idesc(128, true, true, false), true);
        };
        // What is asked for next comes into L2 while the products of the present head run: the HBM would idle then, and be what everybody
        // waits for later
        const auto prefetch = [&](const Unit& x, int hv, bool keys) {
            if (!x.ok) return;
            if (elect_one()) bulk_prefetch(chunk_ws(p, x.slot, hv) + kWsS, (kWsTab - kWsS) * 4);
            __syncwarp();
            for (int i = tid % 32; i < 2 * x.rows; i += 32) {
                const long long q = p.qk.at(x.s, x.first + i / 2, x.hk) + i % 2 * 64, v = p.v.at(x.s, x.first + i / 2, hv) + i % 2 * 64;
                if (keys) prefetch_l2(p.K + q), prefetch_l2(p.Q + q);
                prefetch_l2(p.dO + v);
                prefetch_l2(p.V + v);
            }
        };
        const auto load = [&](const float* ws) {  // S, u and r of a value head
            if (elect_one()) {
                mbar_arrive_expect_tx(&bar_load, kImage + 2 * kRaw);
                bulk_load(sm.u, ws + kWsU, 2 * kRaw, &bar_load);
                bulk_load(sm.S, ws + kWsS, kImage, &bar_load);
            }
            __syncwarp();
        };
        const auto load_tiles = [&](const Unit& x, int hv, bool keys) {
            if (elect_one()) {
                mbar_arrive_expect_tx(&bar_tile, (keys ? 3 : 1) * 2 * kTile + sizeof(sm.tab));
                if (keys) {
                    load_tile(sm.K, maps.K, p, p.H_k, x.s, x.first, x.hk, &bar_tile);
                    load_tile(sm.Q, maps.Q, p, p.H_k, x.s, x.first, x.hk, &bar_tile);
                }
                load_tile(sm.dO, maps.dO, p, p.H_v, x.s, x.first, hv, &bar_tile);
                bulk_load(sm.tab, chunk_ws(p, x.slot, hv) + kWsTab, sizeof(sm.tab), &bar_tile);
            }
            __syncwarp();
        };
        uint32_t phase = 0;
        Unit now = units[0];
        if (now.ok) {
            load(chunk_ws(p, now.slot, now.hk * heads));
            load_tiles(now, now.hk * heads, true);
        }
        long long place = blockIdx.x;
        for (int n = 0, it = 0; now.ok;) {
            const int hv = now.hk * heads + it, s = now.s, first = now.first, rows = now.rows;
            float* const ws = chunk_ws(p, now.slot, hv);
            const bool last = it + 1 == heads;
            Unit next = now;
            if (last) {
                place = static_cast<long long>(now.slot) * p.H_k + now.hk + gridDim.x;
                next = find_unit(place);
                if (elect_one()) units[(n + 1) & 1] = next;
                __syncwarp();
            }
            const int next_hv = last ? next.hk * heads : hv + 1;
            grad_await<7>();  // K, Q, dO, u, r are there
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int i = kPieces - 1; i >= 0; --i)
                    product<8>(tm + kTmOU, desc_rows(dO), kAlong, desc_cols(tile_u(i)), kDown, grad_idesc(64, false, true, i == 1), i < kPieces - 1);
#pragma unroll
                for (int sum = 2; sum >= 0; --sum)
#pragma unroll
                    for (int i = sum; i >= 0; --i)
                        product<8>(tm + kTmRU, desc_cols(tile_r(i)), kDown, desc_cols(tile_u(sum - i)), kDown,
                                   grad_idesc(64, true, true, (i == 1) != (sum - i == 1)), sum < 2 || i < 2);
                product<8>(tm + kTmKK, desc_rows(K), kAlong, desc_rows(K), kAlong, grad_idesc(64, false, false, false), false);
                product<8>(tm + kTmQK, desc_rows(Q), kAlong, desc_rows(K), kAlong, grad_idesc(64, false, false, false), false);
                mma_commit(&bar_pair);
            }
            __syncwarp();
            grad_await<1>();  // the state
            tc_fence_after_sync();
            if (elect_one()) {
                product<8>(tm + kTmDOS, state(1), kDown, desc_rows(dO), kAlong, grad_idesc(128, true, false, true), false);
                products_second(tm + kTmRS, tile_r);
                mma_commit(&bar_s);  // the second piece is used up: the third one may have its place
                product<8>(tm + kTmDOS, state(0), kDown, desc_rows(dO), kAlong, grad_idesc(128, true, false, false), true);
                products_first(tm + kTmRS, tile_r);
            }
            __syncwarp();
            prefetch(next, next_hv, last);
            grad_await<3>();  // the state's third piece
            tc_fence_after_sync();
            if (elect_one()) {
                product<8>(tm + kTmDOS, state(1), kDown, desc_rows(dO), kAlong, grad_idesc(128, true, false, false), true);
                product<8>(tm + kTmRS, state(1), kDown, desc_cols(tile_r(0)), kDown, grad_idesc(128, true, true, false), true);
                mma_commit(&bar_l);
            }
            __syncwarp();
            failed = failed || !wait_products(&bar_l, phase);
            if (elect_one()) {  // the state is used up
                mbar_arrive_expect_tx(&bar_load, kImage);
                bulk_load(sm.S, ws + kWsDS, kImage, &bar_load);
            }
            __syncwarp();
            grad_await<2>();  // p, m
            tc_fence_after_sync();
            if (elect_one()) {
                const uint64_t Kd = desc_cols(K), Qd = desc_cols(Q);
#pragma unroll
                for (int i = kPieces - 1; i >= 0; --i) {
                    const uint32_t pt = tile_r(0) + i * kTile, mt = pt + kPieces * kTile;
                    product<4>(tm + kTmDQ, Kd, kDown, desc_rows(pt), kAlong, grad_idesc(128, true, false, i == 1), i < kPieces - 1);
                    product<4>(tm + kTmDK, Qd, kDown, desc_cols(pt), kDown, grad_idesc(128, true, true, i == 1), i < kPieces - 1);
                    product<4>(tm + kTmDK, Kd, kDown, desc_rows(mt), kAlong, grad_idesc(128, true, false, i == 1), true);
                    product<4>(tm + kTmDK, Kd, kDown, desc_cols(mt), kDown, grad_idesc(128, true, true, i == 1), true);
                }
                mma_commit(&bar_out);
            }
            __syncwarp();
            grad_await<6>();  // the state's gradient
            tc_fence_after_sync();
            if (elect_one()) products_second(tm + kTmUD, tile_u), products_first(tm + kTmUD, tile_u);
            __syncwarp();
            grad_await<4>();  // its third piece, where p and m were; every part of dbeta and dg
            tc_fence_after_sync();
            if (elect_one()) {
                product<8>(tm + kTmUD, smem_desc(tile_r(0), 2 * kTile, 1024, SWZ_128B), kDown, desc_cols(tile_u(0)), kDown, grad_idesc(128, true, true, false), true);
                mma_commit(&bar_d);
            }
            __syncwarp();
            failed = failed || !wait_products(&bar_d, phase);
            phase ^= 1;
            if (next.ok) load(chunk_ws(p, next.slot, next_hv));
            // lane i has tokens 2i, 2i + 1
            const int lane = tid % 32;
            float d[2], ends = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = 2 * lane + e;
                const float rz = ws[kWsDots + i], end = ws[kWsDots + kC + i];
                const float sums[4] = {(sm.rown[0][i] + sm.rown[1][i]) + (sm.rown[2][i] + sm.rown[3][i]), (sm.rowb[0][i] + sm.rowb[1][i]) + (sm.rowb[2][i] + sm.rowb[3][i]),
                                       (sm.coln[0][i] + sm.coln[1][i]) + (sm.coln[2][i] + sm.coln[3][i]), (sm.rowq[0][i] + sm.rowq[1][i]) + (sm.rowq[2][i] + sm.rowq[3][i])};
                if (i < rows) p.dbeta[p.gate.at(s, first + i, hv)] = (sm.rv[0][i] + sm.rv[1][i]) - rz + sums[1];
                d[e] = sums[0] - sums[2] + sums[3] - sm.tab[TAB_BETA * kC + i] * rz - end;
                ends += end;
            }
#pragma unroll
            for (int o = 16; o > 0; o /= 2) ends += __shfl_xor_sync(0xffffffffu, ends, o);
            float dsum = 0.f;
#pragma unroll
            for (int x = 0; x < kGradThreads / 32; ++x) dsum += sm.ds[x];
            if (lane == 31) d[1] += ends + sm.tab[TAB_DECAY * kC] * dsum;
            float sum = d[0] + d[1];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float x = __shfl_down_sync(0xffffffffu, sum, o);
                if (lane + o < 32) sum += x;
            }
            if (2 * lane < rows) p.dg[p.gate.at(s, first + 2 * lane, hv)] = sum;
            if (2 * lane + 1 < rows) p.dg[p.gate.at(s, first + 2 * lane + 1, hv)] = sum - d[0];
            __syncthreads();
            if (next.ok) load_tiles(next, next_hv, last);
            now = next;
            it = last ? 0 : it + 1;
            n += last;
        }
    } else {
        const int quad = warp % 4, quarter = warp / 4;  // 32 key features (16 tokens of p, m), 16 tokens
        const uint32_t lanes = tm + (static_cast<uint32_t>(quad * 32) << 16) + quarter * 16;
        const int t0 = quarter * 16 + 2 * l.c;  // this thread's tokens: t0, t0 + 1, t0 + 8, t0 + 9
        // a token's sum over the features of x times K or Q, in four parts
        const auto put_dots = [&](const float (&x)[2][8], const uint8_t* tile, float (*to)[kC]) {
            float d[4] = {};
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                uint32_t w[4];
                turned(tile, quarter * 16, quad * 32 + lh * 16, w);
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    d[i / 4 * 2] = fmaf(x[lh][i], bf16_lo(w[i / 2]), d[i / 4 * 2]);
                    d[i / 4 * 2 + 1] = fmaf(x[lh][i + 1], bf16_hi(w[i / 2]), d[i / 4 * 2 + 1]);
                }
            }
            const float sum = token_sum(d, l);
            if ((l.g & 1) == 0) to[quad][quarter * 16 + (l.g >> 2) * 8 + 2 * l.c + ((l.g >> 1) & 1)] = sum;
        };
        // This thread's part of a state, 8 x 4 values: as it has come, and the places of its pieces. The pieces take the place of the fp32 values, so every
        // thread reads before any of them writes; the third one comes where the second is when that has been used.
        const auto state_of = [&](int i) { return reinterpret_cast<const float4*>(sm.S) + tid + i * kGradThreads; };
        const auto place_of = [&](int i) {
            const int at = tid + i * kGradThreads, row = at / 256 * 8 + at % 16 / 2, col = at / 16 % 16 * 8 + at % 2 * 4;
            return col / 64 * 2 * kTile + swizzled(row, col % 64);
        };
        const auto put_two = [&](const float4 (&x)[8], uint2 (&third)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint2 h, m;
                split3(x[i].x, x[i].y, h.x, m.x, third[i].x);
                split3(x[i].z, x[i].w, h.y, m.y, third[i].y);
                const int place = place_of(i);
                *reinterpret_cast<uint2*>(sm.S + place) = h;
                *reinterpret_cast<uint2*>(sm.S + kImage / 2 + place) = m;
            }
            fence_proxy_async_smem();
        };
        const auto put_third = [&](uint8_t* to, const uint2 (&third)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint2*>(to + place_of(i)) = third[i];
            fence_proxy_async_smem();
        };
        // V for <r, v>, eight tokens a warp and half of the features
        uint32_t v[8];
        const int row_v = warp % 8 * 8 + l.g;
        const auto ask = [&](const Unit& x, int hv) {
            const long long at = p.v.at(x.s, x.first + row_v, hv) + warp / 8 * 64 + 2 * l.c;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = row_v < x.rows ? *reinterpret_cast<const uint32_t*>(p.V + at + i * 8) : 0u;
        };
        float dq[2][8] = {}, dk[2][8] = {};  // [16 lanes][see for_pairs], times 1 / ||q||, 1 / ||k||
        Unit now = units[0];
        if (now.ok) ask(now, now.hk * heads);
        uint32_t turn = 0;
        for (int n = 0, it = 0; now.ok; turn ^= 1) {
            const int hv = now.hk * heads + it, s = now.s, first = now.first, rows = now.rows;
            const bool last = it + 1 == heads;
            failed = failed || !wait_products(&bar_load, 0);
            {  // u and r in pieces
                float4 x[2][4];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][i] = reinterpret_cast<const float4*>(&sm.u[0][0] + t * kRaw)[tid + i * kGradThreads];
                grad_sync();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = tid + i * kGradThreads, place = swizzled(at / 16, ((at ^ (at / 16 << 1)) & 15) * 4);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        uint32_t w[kPieces][2];
                        split3(x[t][i].x, x[t][i].y, w[0][0], w[1][0], w[2][0]);
                        split3(x[t][i].z, x[t][i].w, w[0][1], w[1][1], w[2][1]);
#pragma unroll
                        for (int q = 0; q < kPieces; ++q) *reinterpret_cast<uint2*>((t ? sm.r : sm.u)[q] + place) = make_uint2(w[q][0], w[q][1]);
                    }
                }
            }
            failed = failed || !wait_products(&bar_tile, turn);
            if (rows < kC) {
                if (it == 0) clear_tail<kGradThreads>(sm.K, rows, tid), clear_tail<kGradThreads>(sm.Q, rows, tid);
                clear_tail<kGradThreads>(sm.dO, rows, tid);
            }
            fence_proxy_async_smem();
            grad_arrive<7>();
            uint2 third[8];
            {  // the state in pieces
                float4 x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *state_of(i);
                grad_sync();
                put_two(x, third);
                grad_arrive<1>();
            }
            {  // dV = beta r, turned back, and <r, v>
                const float b = sm.tab[TAB_BETA * kC + row_v];
                const long long at_v = p.v.at(s, first + row_v, hv) + warp / 8 * 64 + 2 * l.c;
                float rv = 0.f;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t w[kPieces][4];
#pragma unroll
                    for (int q = 0; q < kPieces; ++q) ldmatrix_turned(smem_u32(sm.r[q] + swizzled(warp / 8 * 64 + i * 32 + tid % 32, warp % 8 * 8)), w[q]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float x = (bf16_lo(w[0][k]) - bf16_lo(w[1][k])) + bf16_lo(w[2][k]), y = (bf16_hi(w[0][k]) - bf16_hi(w[1][k])) + bf16_hi(w[2][k]);
                        rv = fmaf(x, bf16_lo(v[i * 4 + k]), fmaf(y, bf16_hi(v[i * 4 + k]), rv));
                        if (row_v < rows) *reinterpret_cast<uint32_t*>(p.dV + at_v + i * 32 + k * 8) = pack_bf16x2(b * x, b * y);
                    }
                }
                rv = quad_sum(rv);
                if (l.c == 0) sm.rv[warp / 8][row_v] = rv;
            }
            failed = failed || !wait_products(&bar_s, turn);
            tc_fence_after_sync();
            put_third(sm.S + kImage / 2, third);
            grad_arrive<3>();
            failed = failed || !wait_products(&bar_pair, turn);
            tc_fence_after_sync();
            {  // p, m, and what dbeta and dg have of them
                float ou[8], ru[8], kk[8], qk[8];
                tm_ld16(lanes + kTmOU, ou);
                tm_ld16(lanes + kTmRU, ru);
                tm_ld16(lanes + kTmKK, kk);
                tm_ld16(lanes + kTmQK, qk);
                tmem_wait_ld();
                const float *const g = sm.tab + TAB_G * kC, *const lo = sm.tab + TAB_GLO * kC;
                const float* const rk = sm.tab + TAB_RK * kC;
                float rown[2] = {}, rowb[2] = {}, coln[4] = {};
                float pp[8], mm[8];  // p_ij and m_ij with the lengths of the rows that they will multiply
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int i = quad * 16 + ((x >> 1) & 1) * 8 + l.g, j = t0 + (x >> 2) * 8 + (x & 1);
                    const float gam = j <= i ? exp_between(g[i], lo[i], g[j], lo[j]) * rk[j] : 0.f;
                    pp[x] = j <= i ? ou[x] * (p.scale * gam * sm.tab[TAB_RQ * kC + i]) : 0.f;
                    const float kg = j < i ? -gam * rk[i] * ru[x] : 0.f;
                    mm[x] = sm.tab[TAB_BETA * kC + i] * kg;
                    if (j < i) {
                        const float both = fmaf(pp[x], qk[x], mm[x] * kk[x]);
                        rown[(x >> 1) & 1] += both;
                        coln[(x >> 2) * 2 + (x & 1)] += both;
                        rowb[(x >> 1) & 1] = fmaf(kg, kk[x], rowb[(x >> 1) & 1]);
                    }
                }
                // they take the place of r: every thread had read it when the products that bar_l stands for were asked for, and these were its last
                failed = failed || !wait_products(&bar_l, turn);
                tc_fence_after_sync();
#pragma unroll
                for (int x = 0; x < 8; x += 2) {
                    uint32_t w[kPieces];
                    uint8_t* const at = sm.r[0] + swizzled(quad * 16 + ((x >> 1) & 1) * 8 + l.g, t0 + (x >> 2) * 8);
                    split3(pp[x], pp[x + 1], w[0], w[1], w[2]);
#pragma unroll
                    for (int q = 0; q < kPieces; ++q) *reinterpret_cast<uint32_t*>(at + q * kTile) = w[q];
                    split3(mm[x], mm[x + 1], w[0], w[1], w[2]);
#pragma unroll
                    for (int q = 0; q < kPieces; ++q) *reinterpret_cast<uint32_t*>(at + (kPieces + q) * kTile) = w[q];
                }
                fence_proxy_async_smem();
                tc_fence_before_sync();
                grad_arrive<2>();
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float a = quad_sum(rown[e]), b = quad_sum(rowb[e]);
                    if (l.c == 0) sm.rown[quarter][quad * 16 + e * 8 + l.g] = a, sm.rowb[quarter][quad * 16 + e * 8 + l.g] = b;
                }
                const float sum = token_sum(coln, l);
                if ((l.g & 1) == 0) sm.coln[quad][quarter * 16 + (l.g >> 2) * 8 + 2 * l.c + ((l.g >> 1) & 1)] = sum;
            }
            {  // scale exp(g) dO S, -beta exp(g) r S
                float part[2][8];
#pragma unroll
                for (int lh = 0; lh < 2; ++lh) {
                    float y[8];
                    tm_ld16(lanes + (lh << 20) + kTmDOS, part[lh]);
                    tm_ld16(lanes + (lh << 20) + kTmRS, y);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = t0 + i / 4 * 8 + i % 2;
                        part[lh][i] *= sm.tab[TAB_SEGQ * kC + t];
                        dq[lh][i] += part[lh][i];
                        dk[lh][i] = fmaf(-sm.tab[TAB_BEGK * kC + t], y[i], dk[lh][i]);
                    }
                }
                put_dots(part, sm.Q, sm.rowq);
            }
            {  // <D, S>, both in fp32: S comes again, from L2
                const float4* const again = reinterpret_cast<const float4*>(chunk_ws(p, now.slot, hv) + kWsS) + tid;
                float4 x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = again[i * kGradThreads];
                failed = failed || !wait_products(&bar_load, 1);  // (the second copy of the value head's two)
                float d = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float4 y = *state_of(i);
                    d = fmaf(x[i].x, y.x, d), d = fmaf(x[i].y, y.y, d), d = fmaf(x[i].z, y.z, d), d = fmaf(x[i].w, y.w, d);
                    x[i] = y;
                }
                grad_sync();
                put_two(x, third);
                grad_arrive<6>();
                for (int o = 16; o > 0; o /= 2) d += __shfl_xor_sync(0xffffffffu, d, o);
                if (l.g == 0 && l.c == 0) sm.ds[warp] = d;
            }
            failed = failed || !wait_products(&bar_out, turn);
            put_third(sm.r[0], third);  // (p and m are used up)
            grad_arrive<4>();
            tc_fence_after_sync();
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float a[8], b[8];
                tm_ld16(lanes + (lh << 20) + kTmDQ, a);
                tm_ld16(lanes + (lh << 20) + kTmDK, b);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) dq[lh][i] += a[i], dk[lh][i] += b[i];
            }
            failed = failed || !wait_products(&bar_d, turn);
            tc_fence_after_sync();
#pragma unroll
            for (int lh = 0; lh < 2; ++lh) {
                float y[8];
                tm_ld16(lanes + (lh << 20) + kTmUD, y);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) dk[lh][i] = fmaf(sm.tab[TAB_ECK * kC + t0 + i / 4 * 8 + i % 2], y[i], dk[lh][i]);
            }
            tc_fence_before_sync();
            if (!last) {
                __syncthreads();
                ask(now, hv + 1);
                ++it;
                continue;
            }
            // through the norm of the rows: x - ||row||^-2 <row, x> row; turned back through shared memory
            if (p.l2norm) {
                put_dots(dq, sm.Q, sm.norm[0]);
                put_dots(dk, sm.K, sm.norm[1]);
            }
            grad_sync();
            uint8_t* const out = &sm.r[1][0];  // two tiles of 64 x 128 in the 128-byte swizzle
            const auto finish = [&](const float (&x)[2][8], const uint8_t* tile, const float* inv, const float (*dots)[kC], uint8_t* to) {
                float c[4] = {};
                if (p.l2norm) {
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const int t = t0 + e / 2 * 8;
                        const float2 a = *reinterpret_cast<const float2*>(inv + t);
                        float2 d[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) d[i] = *reinterpret_cast<const float2*>(dots[i] + t);
                        c[e] = a.x * a.x * ((d[0].x + d[1].x) + (d[2].x + d[3].x)), c[e + 1] = a.y * a.y * ((d[0].y + d[1].y) + (d[2].y + d[3].y));
                    }
                }
#pragma unroll
                for (int lh = 0; lh < 2; ++lh) {
                    uint32_t w[4];
                    turned(tile, quarter * 16, quad * 32 + lh * 16, w);
#pragma unroll
                    for (int i = 0; i < 8; i += 2)
                        w[i / 2] = pack_bf16x2(fmaf(-c[i / 4 * 2], bf16_lo(w[i / 2]), x[lh][i]), fmaf(-c[i / 4 * 2 + 1], bf16_hi(w[i / 2]), x[lh][i + 1]));
                    const int lane = tid % 32, t = quarter * 16 + (lane & 7) + (lane >> 4) * 8, f = quad * 32 + lh * 16 + ((lane >> 3) & 1) * 8;
                    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(smem_u32(to + f / 64 * kTile + swizzled(t, f % 64))), "r"(w[0]), "r"(w[1]),
                                 "r"(w[2]), "r"(w[3])
                                 : "memory");
                }
            };
            finish(dq, sm.Q, sm.tab + TAB_RQ * kC, sm.norm[0], out);
            finish(dk, sm.K, sm.tab + TAB_RK * kC, sm.norm[1], out + 2 * kTile);
            __syncthreads();
            const Unit next = units[(n + 1) & 1];
            if (next.ok) ask(next, next.hk * heads);
            const long long at = p.qk.at(s, first, now.hk);
#pragma unroll
            for (int i = tid; i < kC * kD / 8; i += kGradThreads) {
                const int row = i / 16, col = i % 16 * 8, place = col / 64 * kTile + swizzled(row, col % 64);
                if (row < rows) {
                    *reinterpret_cast<uint4*>(p.dQ + at + row * p.qk.token + col) = *reinterpret_cast<const uint4*>(out + place);
                    *reinterpret_cast<uint4*>(p.dK + at + row * p.qk.token + col) = *reinterpret_cast<const uint4*>(out + 2 * kTile + place);
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) (&dq[0][0])[i] = (&dk[0][0])[i] = 0.f;
            now = next;
            it = 0;
            ++n;
        }
    }
    if (failed) *p.status = GDN_ERR_TIMEOUT;
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tm, kTmColumns);
}

template <typename Smem, typename... A>
bool launch(void (*kern)(ParamsB, A...), long long ctas, unsigned threads, cudaStream_t stream, const ParamsB& p, const A&... maps) {
    if (ctas == 0) return true;
    static_assert(sizeof(Smem) + 1024 <= 227 * 1024, "");  // (1 KB to start on a multiple of 1 KB)
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem) + 1024) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    kern<<<static_cast<unsigned>(ctas), threads, sizeof(Smem) + 1024, stream>>>(p, maps...);
    if (cudaGetLastError() != cudaSuccess) return false;
    count_launch();
    return true;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode_fn() {
    static EncodeTiledFn fn = nullptr;
    if (fn == nullptr) {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess)
            return nullptr;
        fn = reinterpret_cast<EncodeTiledFn>(ptr);
    }
    return fn;
}
bool make_map(CUtensorMap* map, const void* base, long long planes, int T, int cols) {
    const EncodeTiledFn enc = get_encode_fn();
    if (enc == nullptr) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(T), static_cast<cuuint64_t>(planes)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(cols) * 2, static_cast<cuuint64_t>(T) * cols * 2};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(kC), 1}, step[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
    p.status = device_status_word();
    if (p.status == nullptr) return GDN_ERR_LAUNCH;
    p.scale = q.scale, p.l2norm = (q.flags & GDN_FLAG_K_L2NORM) != 0;
    const bool token_major = (q.flags & GDN_FLAG_LAYOUT_BTHD) != 0, packed = q.cu_seqlens != nullptr;
    p.token_major = token_major;
    const auto strides = [&](long long H, long long d) {
        Strides s = token_major ? Strides{q.T * H * d, H * d, d} : Strides{q.T * H * d, d, q.T * d};
        if (packed) s.seq = 0;
        return s;
    };
    p.qk = strides(q.H_k, kD), p.v = strides(q.H_v, kD), p.gate = strides(q.H_v, 1);
    const long long places = packed ? chunk_places(q.n_seq, q.T) : static_cast<long long>(q.n_seq) * p.chunks;
    p.units = places * q.H_k;
    const long long chains = static_cast<long long>(q.n_seq) * q.H_v;
    if (places * q.H_k >= (1LL << 31) || chains >= (1LL << 31)) return GDN_ERR_UNSUPPORTED;
    Maps maps{};
    if (q.T > 0) {
        const long long batch = packed ? 1 : q.n_seq;
        const auto map = [&](CUtensorMap* m, const void* base, int H) {
            return make_map(m, base, token_major ? batch : batch * H, q.T, token_major ? H * kD : kD);
        };
        if (!map(&maps.Q, q.Q, q.H_k) || !map(&maps.K, q.K, q.H_k) || !map(&maps.V, q.V, q.H_v) || !map(&maps.dO, q.dO, q.H_v)) return GDN_ERR_LAUNCH;
    }
    const bool ok = launch<SmemSystem>(chunk_system_kernel, places * q.H_k, kThreads, stream, p) &&
                    launch<SmemF>(chunk_states_kernel, chains, kChainThreads, stream, p, maps) &&
                    launch<SmemB>(chunk_state_grads_kernel, chains, kChainThreads, stream, p, maps) &&
                    launch<SmemC>(chunk_grads_kernel, p.units < kSMs ? p.units : kSMs, kGradThreads + 32, stream, p, maps);
    return ok ? GDN_OK : GDN_ERR_LAUNCH;
}

}  // namespace gdn

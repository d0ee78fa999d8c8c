// Hybrid linear attention with a decay for each head (include/mtfm_hla.h) for gfx950: forward, backward, single tokens.
//
// All passes over a user's tokens are one sweep.  With rows a_i that ask, and pairs (b_i, c_i) that enter a state,
//   S <- l S + b_i c_i^T,   o_i = scale a_i S
// is the forward pass for (a, b, c) = (q, k, v); the gradients are the same sweep with the letters exchanged: dq for (dout, v, k)
// in the same direction with the states transposed, and from the last row backwards dv for (k, q, dout) and dk for (v, dout, q).
//
// A workgroup owns a user's head and goes through the tokens in chunks of 64.  Inside a chunk, with i, j counted from its start and
// S the state in front of it,
//   o_i = scale [ l^(i+1) a_i S + sum_(j<=i) l^(i-j) <a_i, b_j> c_j ],    S <- l^n S + sum_j l^(n-1-j) b_j c_j^T:
// four matrix products.  The work is bound by HBM (4 d^2 + 64 d operations per row and head on 8 d bytes), so a row is read once: the
// state stays in registers from chunk to chunk -- wave w owns its columns [16 w, 16 w + 16), whose accumulators are, rounded, the
// operand of the product with a -- and the next chunk's rows are in flight while the current one is worked on.  Backwards the state is
// handed on decayed already (o_i takes l^i, the update l^(n-j)), so that the gradient of S_L enters, and that of S_0 leaves, as it is.
#include "../../include/mtfm_hla.h"
#include "hta_common.h"
#include "hta_mfma.h"

#include <hip/hip_runtime.h>

namespace hla {

using hta::bf16x4;
using hta::bf16x8;
using hta::fast_exp2;
using hta::floatx4;
using hta::swizzle;

constexpr int CHUNK = 64;
constexpr float MIN_LOG2 = -1e4f;  // of a decay: 2^-10000 is 0, and 0 times it is not NaN

struct Pass {
    const __bf16 *a, *b, *c;
    __bf16* out;
    float* partial;         // backwards, where a group's heads are spread over workgroups: [spread][total_kv][Hkv][d]
    const float* state_in;  // null: zero
    float* state_out;       // null: not wanted
    int32_t transposed;     // the state that is read is that of the other sweeps, transposed
};

struct Args {
    Pass pass[2];
    const float* log_decay;
    const int32_t *q_off, *kv_off, *hist_len, *n_targets;
    int64_t total_q, total_kv;
    int32_t batch, Hq, Hkv, ratio, n_pass, spread;  // spread: workgroups that the heads of a group are dealt to
    int32_t full;
    float scale;
};

__device__ inline floatx4 mfma16(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
// Eight float32 values as the sum of two bf16 ones: the upper half of each as it stands, and what that leaves off, rounded
__device__ inline void split8(const float (&x)[8], bf16x8& hi, bf16x8& lo) {
    uintx4 h;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const unsigned a = __builtin_bit_cast(unsigned, x[2 * e]), b = __builtin_bit_cast(unsigned, x[2 * e + 1]);
        h[e] = __builtin_amdgcn_perm(b, a, 0x07060302);
        lo[2 * e] = (__bf16)(x[2 * e] - __builtin_bit_cast(float, a & 0xFFFF0000u));
        lo[2 * e + 1] = (__bf16)(x[2 * e + 1] - __builtin_bit_cast(float, b & 0xFFFF0000u));
    }
    hi = __builtin_bit_cast(bf16x8, h);
}

// Where a user's rows lie, whatever the arrays hold: inside the tensors
struct User {
    int64_t q0, kv0;
    int L, T;
};
__device__ inline int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); }
__device__ inline User user_of(const Args& g, int u) {
    User r;
    r.kv0 = clamp64(g.kv_off[u], 0, g.total_kv);
    r.q0 = clamp64(g.q_off[u], 0, g.total_q);
    const int64_t n_kv = clamp64(g.kv_off[u + 1], r.kv0, g.total_kv) - r.kv0, n_q = clamp64(g.q_off[u + 1], r.q0, g.total_q) - r.q0;
    r.L = (int)clamp64(g.hist_len[u], 0, g.full ? (n_kv < n_q ? n_kv : n_q) : n_kv);
    const int64_t left_kv = n_kv - r.L, left_q = g.full ? n_q - r.L : n_q;
    r.T = (int)clamp64(g.n_targets[u], 0, left_kv < left_q ? left_kv : left_q);
    return r;
}

// waves per SIMD that the registers are to leave room for
constexpr int sweep_waves(int D, int G, int CB) { return D == 32 && G == 1 ? 4 : D * G * CB <= 64 ? 3 : 2; }

// One sweep over a user by a workgroup of D / (16 CB) waves, each with CB blocks of 16 columns.  Forwards a workgroup has one query head, backwards G heads of a group, whose outputs
// (dv or dk of their common key/value head) it sums.  D[m][n] += A[m][k] B[k][n] of 16x16x32: a lane holds row (column) lane % 16 and k = 8 (lane / 16) ..
// + 7 of either operand, and column lane % 16, rows 4 (lane / 16) .. + 3 of the result.
template <int D, int G, int CB, bool BACK>
__global__ __launch_bounds__(D * 4 / CB, sweep_waves(D, G, CB)) void sweep_kernel(const Args args) {
    constexpr int NW = D / 16 / CB, NT = NW * 64, C16 = D / 8, KS = D / 32, PART = NT / C16, LOADS = CHUNK / PART;  // PART: rows that the threads load at a time
    __shared__ __attribute__((aligned(16))) __bf16 a_s[CHUNK * D], b_s[CHUNK * D], c_s[CHUNK * D], p_s[CHUNK * CHUNK];
    __shared__ float dots_s[CHUNK];
    // powers of the heads' decays, as they are and times `scale`: entry ZERO + m holds l^m, m = -64 .. 64, 0 for m < 0
    constexpr int ZERO = CHUNK, POWERS = 2 * CHUNK + 4;
    __shared__ float power_s[G][POWERS], scaled_s[G][POWERS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;

    // which user, heads and pass: those that share rows are neighbours on one XCD
    const int per_pass = BACK ? args.spread : args.ratio, members = per_pass * args.n_pass;
    const int xcd = blockIdx.x % hta::N_XCD, slot = blockIdx.x / hta::N_XCD;
    const int group = (slot / members) * hta::N_XCD + xcd, member = slot % members;
    if (group >= args.batch * args.Hkv) return;
    const int u = group / args.Hkv, kvh = group % args.Hkv, sub = member % per_pass;
    const Pass ps = args.pass[member / per_pass];
    const int qh0 = kvh * args.ratio + sub * G;  // the first of the G query heads
    const User us = user_of(args, u);
    const int nh = (us.L + CHUNK - 1) / CHUNK, nt = (us.T + CHUNK - 1) / CHUNK, chunks = nh + nt;
    const bool full = args.full;

    // state: tile t of head g and block b, register v: row 32 (t / 2) + 8 quad + 4 (t % 2) + v, column 16 (CB wave + b) + l16.  (Rows in this order make the accumulators of
    // two tiles eight consecutive rows: what an operand wants.)
    floatx4 S[G][CB][2 * KS];
#pragma unroll
    for (int g = 0; g < G; g++) {
        const float* in = ps.state_in ? ps.state_in + ((int64_t)u * args.Hq + qh0 + g) * D * D : nullptr;
#pragma unroll
        for (int b = 0; b < CB; b++)
#pragma unroll
            for (int t = 0; t < 2 * KS; t++) {
                const int row = 32 * (t / 2) + 8 * quad + 4 * (t % 2), col = 16 * (CB * wave + b) + l16;
                S[g][b][t] = floatx4{0.f, 0.f, 0.f, 0.f};
                if (in) {
                    if (ps.transposed) S[g][b][t] = *(const floatx4*)(in + col * D + row);
                    else
#pragma unroll
                        for (int v = 0; v < 4; v++) S[g][b][t][v] = in[(row + v) * D + col];
                }
            }
    }

    struct Rows {  // of a chunk: n rows, row r is first + r (backwards through a history: first - r)
        int64_t q, kv;
        int n;
        bool hist;
    };
    const auto rows_of = [&](int c) {
        Rows r;
        r.hist = BACK ? c >= nt : c < nh;
        if (r.hist) {
            const int first = (BACK ? c - nt : c) * CHUNK, at = BACK ? us.L - 1 - first : first;
            r.n = min(CHUNK, us.L - first);
            r.kv = us.kv0 + at, r.q = us.q0 + at;
        } else {
            const int first = (BACK ? c : c - nh) * CHUNK;
            r.n = min(CHUNK, us.T - first);
            r.kv = us.kv0 + us.L + first, r.q = us.q0 + (full ? us.L : 0) + first;
        }
        return r;
    };
    // A chunk's rows in memory: a uniform address, that of its lowest of 64 rows (backwards through a history row 63, which need not be there), and a
    // lane's bytes from there
    const int heads_a = BACK ? args.Hkv : args.Hq, heads_b = BACK ? args.Hq : args.Hkv;
    const unsigned pitch_a = heads_a * (D * 2), pitch_b = heads_b * (D * 2);
    const auto lowest = [](bool down, int64_t first) { return down ? first - (CHUNK - 1) : first; };
    const auto bytes_of = [](bool down, int r, unsigned pitch, int byte) { return __umul24(down ? CHUNK - 1 - r : r, pitch) + byte; };

    // 16-byte words of the three tiles on their way: word tid % C16 of rows tid / C16 + i PART.  Rows that are not there are zero.
    const int row_t = tid / C16, word_t = tid % C16;
    bf16x8 av[LOADS], bv[LOADS], cv[LOADS];
    const auto fetch = [&](int chunk, int g) {
        const Rows r = rows_of(chunk);
        const bool asks = full || !r.hist;  // are there query rows?
        const bool has_a = (BACK || asks) && (G == 1 || g == 0), has_bc = !BACK || asks, down = BACK && r.hist;
        const int head_a = BACK ? kvh : qh0, head_b = BACK ? qh0 + g : kvh;
        const int64_t row_b = lowest(down, BACK ? r.q : r.kv) * heads_b + head_b;
        const char* a = (const char*)(ps.a + (lowest(down, BACK ? r.kv : r.q) * heads_a + head_a) * D);
        const char *b = (const char*)(ps.b + row_b * D), *c = (const char*)(ps.c + row_b * D);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int row = row_t + i * PART;
            const bool there = row < r.n;
            const unsigned at_a = bytes_of(down, row, pitch_a, word_t * 16), at_b = bytes_of(down, row, pitch_b, word_t * 16);
            av[i] = bv[i] = cv[i] = bf16x8{};
            if (there && has_a) av[i] = *(const bf16x8*)(a + at_a);
            if (there && has_bc) bv[i] = *(const bf16x8*)(b + at_b), cv[i] = *(const bf16x8*)(c + at_b);
        }
    };
    const auto word_at = [](const __bf16* tile, int row, int word) { return tile + row * D + ((word ^ swizzle<D>(row)) * 8); };

    if (chunks > 0) fetch(0, 0);
    for (int i = tid; i < G * POWERS; i += NT) {
        const int g = i / POWERS, m = i % POWERS - ZERO;
        const float g2 = fmaxf(fminf(args.log_decay[qh0 + g], 0.f) * hta::LOG2E, MIN_LOG2);
        const float p = m < 0 ? 0.f : fast_exp2(g2 * (float)m);
        power_s[g][m + ZERO] = p, scaled_s[g][m + ZERO] = p * args.scale;
    }
    // (entries of P that a product reads and no chunk writes)
    for (int i = tid; i < CHUNK * CHUNK / 8; i += NT) ((bf16x8*)p_s)[i] = bf16x8{};

    floatx4 acc[CB][4];
    for (int c = 0; c < chunks; c++) {
        const Rows r = rows_of(c);
        const bool asks = full || !r.hist, down = BACK && r.hist;
        const bool has_out = BACK || asks, has_bc = !BACK || asks;
        const bool intra = r.hist && has_out && has_bc, inter = r.hist ? has_out : !BACK, update = r.hist ? has_bc : BACK;
#pragma unroll
        for (int g = 0; g < G; g++) {
            // (the last readers of the tiles are behind the barrier at the end of the turn)
#pragma unroll
            for (int i = 0; i < LOADS; i++) {
                if (g == 0) *(bf16x8*)word_at(a_s, row_t + i * PART, word_t) = av[i];
                *(bf16x8*)word_at(b_s, row_t + i * PART, word_t) = bv[i];
                *(bf16x8*)word_at(c_s, row_t + i * PART, word_t) = cv[i];
            }
            __syncthreads();
            if (g + 1 < G) fetch(c, g + 1);
            else if (c + 1 < chunks) fetch(c + 1, 0);

            if (intra) {
                // P^T = B A^T with the decays, tiles on and below the diagonal, dealt to the waves
#pragma unroll
                for (int t0 = 0; t0 < 10; t0 += NW) {
                    const int t = t0 + wave;
                    if (t >= 10) break;
                    const int it = t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0, jt = t - it * (it + 1) / 2;
                    const int i = 16 * it + l16, j = 16 * jt + 4 * quad;
                    floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < KS; k++)
                        s = mfma16(*(const bf16x8*)word_at(b_s, 16 * jt + l16, 4 * k + quad), *(const bf16x8*)word_at(a_s, i, 4 * k + quad), s);
                    float w[4];
                    const float* power = scaled_s[g] + ZERO + i - j;
#pragma unroll
                    for (int v = 0; v < 4; v++) w[v] = power[-v];
                    bf16x4 p;
#pragma unroll
                    for (int v = 0; v < 4; v++) {
                        s[v] *= w[v];
                        p[v] = (__bf16)(i - j >= v ? s[v] : 0.f);  // (0 times what a later row holds need not be 0)
                    }
                    *(bf16x4*)(p_s + i * CHUNK + (((j / 8) ^ swizzle<64>(i)) * 8) + (j & 4)) = p;
                }
            } else if (!r.hist) {
                // own keys only: <a_i, b_i>, NW lanes to a row
                const int row = tid / NW, part = tid % NW;
                float dot = 0.f;
#pragma unroll
                for (int k = 0; k < C16 / NW; k++)
                    dot = hta::dot_bf16x8(dot, *(const bf16x8*)word_at(a_s, row, C16 / NW * part + k), *(const bf16x8*)word_at(b_s, row, C16 / NW * part + k));
                dot = hta::sum_lanes<NW>(dot);
                if (part == 0) dots_s[row] = dot * args.scale;
            }
            // o^T = S^T A^T, row i of it times l^(i+1) scale (candidates: l scale, backwards: l^i)
            floatx4 o[CB][4];
            if (inter) {
                bf16x8 s[CB][KS];
#pragma unroll
                for (int b = 0; b < CB; b++)
#pragma unroll
                    for (int k = 0; k < KS; k++)
#pragma unroll
                        for (int v = 0; v < 4; v++) s[b][k][v] = (__bf16)S[g][b][2 * k][v], s[b][k][4 + v] = (__bf16)S[g][b][2 * k + 1][v];
#pragma unroll
                for (int it = 0; it < 4; it++)
#pragma unroll
                    for (int k = 0; k < KS; k++) {
                        const bf16x8 a = *(const bf16x8*)word_at(a_s, 16 * it + l16, 4 * k + quad);
#pragma unroll
                        for (int b = 0; b < CB; b++) o[b][it] = mfma16(s[b][k], a, k == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : o[b][it]);
                    }
            }
            __syncthreads();
            // C^T: this wave's columns of c, rows 32 k + 8 quad .. + 7
            bf16x8 ct[CB][2];
#pragma unroll
            for (int b = 0; b < CB; b++)
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    const int row = 32 * k + 8 * quad + (l16 >> 2), word = 2 * (CB * wave + b) + ((l16 & 3) >> 1), off = (l16 & 1) * 4;
                    ct[b][k] = hta::lds_read_tr_pair(word_at(c_s, row, word) + off, word_at(c_s, row + 4, word) + off);
                }
            floatx4 within[CB][4];
#pragma unroll
            for (int b = 0; b < CB; b++)
#pragma unroll
                for (int it = 0; it < 4; it++) within[b][it] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (intra) {
#pragma unroll
                for (int it = 0; it < 4; it++)
#pragma unroll
                    for (int k = 0; k <= it / 2; k++) {
                        const int i = 16 * it + l16;
                        const bf16x8 p = *(const bf16x8*)(p_s + i * CHUNK + (((4 * k + quad) ^ swizzle<64>(i)) * 8));
#pragma unroll
                        for (int b = 0; b < CB; b++) within[b][it] = mfma16(ct[b][k], p, within[b][it]);
                    }
                // An infinity or a NaN in c reaches the rows in front of it as 0 times itself, and the last rows in any case: then row by row.
                float zero = 0.f;
#pragma unroll
                for (int b = 0; b < CB; b++)
#pragma unroll
                    for (int v = 0; v < 4; v++) zero = fmaf(within[b][3][v], 0.f, zero);
                if (__ballot(zero != zero) != 0) {
#pragma unroll
                    for (int b = 0; b < CB; b++)
#pragma unroll
                        for (int it = 0; it < 4; it++) within[b][it] = floatx4{0.f, 0.f, 0.f, 0.f};
                    for (int j = 0; j < CHUNK; j++) {
#pragma unroll
                        for (int b = 0; b < CB; b++) {
                            const bf16x4 cj = *(const bf16x4*)(word_at(c_s, j, 2 * (CB * wave + b) + (quad >> 1)) + (quad & 1) * 4);
#pragma unroll
                            for (int it = 0; it < 4; it++) {
                                const int i = 16 * it + l16;
                                const float p = (float)p_s[i * CHUNK + (((j / 8) ^ swizzle<64>(i)) * 8) + (j & 7)];
#pragma unroll
                                for (int v = 0; v < 4; v++) within[b][it][v] += j <= i ? p * (float)cj[v] : 0.f;
                            }
                        }
                    }
                }
            } else if (!r.hist) {
#pragma unroll
                for (int b = 0; b < CB; b++)
#pragma unroll
                    for (int it = 0; it < 4; it++) {
                        const int i = 16 * it + l16;
                        const bf16x4 ci = *(const bf16x4*)(word_at(c_s, i, 2 * (CB * wave + b) + (quad >> 1)) + (quad & 1) * 4);
#pragma unroll
                        for (int v = 0; v < 4; v++) within[b][it][v] = dots_s[i] * (float)ci[v];
                    }
            }
            if (inter) {
                const float* power = r.hist ? (BACK ? power_s[g] + ZERO : scaled_s[g] + ZERO + 1) + l16 : scaled_s[g] + ZERO + 1;
                const int step = r.hist ? 16 : 0;
#pragma unroll
                for (int it = 0; it < 4; it++) {
                    const float f = power[it * step];
#pragma unroll
                    for (int b = 0; b < CB; b++)
#pragma unroll
                        for (int v = 0; v < 4; v++) within[b][it][v] = fmaf(o[b][it][v], f, within[b][it][v]);
                }
            }
#pragma unroll
            for (int b = 0; b < CB; b++)
#pragma unroll
                for (int it = 0; it < 4; it++) acc[b][it] = g == 0 ? within[b][it] : acc[b][it] + within[b][it];
            if (has_out && g == G - 1) {
                const int64_t base = (lowest(down, BACK ? r.kv : r.q) * heads_a + (BACK ? kvh : qh0)) * D;
                char* out = (char*)(ps.out + base);
                char* partial = (char*)(ps.partial + (int64_t)sub * args.total_kv * args.Hkv * D + base);
#pragma unroll
                for (int it = 0; it < 4; it++) {
                    if (16 * it + l16 < r.n) {
                        const unsigned at = bytes_of(down, 16 * it + l16, pitch_a, (16 * CB * wave + 4 * quad) * 2);
#pragma unroll
                        for (int b = 0; b < CB; b++) {
                            if (BACK && ps.partial) {
                                *(floatx4*)(partial + 2 * at + 64 * b) = acc[b][it];
                            } else {
                                bf16x4 x;
#pragma unroll
                                for (int v = 0; v < 4; v++) x[v] = (__bf16)acc[b][it][v];
                                *(bf16x4*)(out + at + 32 * b) = x;
                            }
                        }
                    }
                }
            }
            // the state behind the chunk: l^n S + B^T (w c), where w c goes in two halves of 8 bits each, so that float32 keeps 16 of it
            if (r.hist) {
                const float keep = power_s[g][ZERO + r.n];
#pragma unroll
                for (int b = 0; b < CB; b++)
#pragma unroll
                    for (int t = 0; t < 2 * KS; t++) S[g][b][t] *= keep;
            }
            if (update) {
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    bf16x8 hi[CB], lo[CB];
                    float w[8];
                    // l^(n-1-j) (backwards l^(n-j) scale); rows that are not there are zero, and so are these behind the table's end
                    const float* p = (BACK ? scaled_s[g] + ZERO + r.n : power_s[g] + ZERO + r.n - 1) - (32 * k + 8 * quad);
#pragma unroll
                    for (int e = 0; e < 8; e++) w[e] = r.hist ? p[-e] : scaled_s[g][ZERO + 1];
#pragma unroll
                    for (int b = 0; b < CB; b++) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; e++) x[e] = w[e] * (float)ct[b][k][e];
                        split8(x, hi[b], lo[b]);
                    }
#pragma unroll
                    for (int t = 0; t < 2 * KS; t++) {
                        const int row = 32 * k + 8 * quad + (l16 >> 2), word = 4 * (t / 2) + (l16 & 3), off = 4 * (t % 2);
                        const bf16x8 bt = hta::lds_read_tr_pair(word_at(b_s, row, word) + off, word_at(b_s, row + 4, word) + off);
#pragma unroll
                        for (int b = 0; b < CB; b++) {
                            S[g][b][t] = mfma16(bt, hi[b], S[g][b][t]);
                            S[g][b][t] = mfma16(bt, lo[b], S[g][b][t]);
                        }
                    }
                }
            }
            __syncthreads();
        }
    }
    if (ps.state_out) {
#pragma unroll
        for (int g = 0; g < G; g++) {
            float* out = ps.state_out + ((int64_t)u * args.Hq + qh0 + g) * D * D;
#pragma unroll
            for (int b = 0; b < CB; b++)
#pragma unroll
                for (int t = 0; t < 2 * KS; t++)
#pragma unroll
                    for (int v = 0; v < 4; v++) out[(32 * (t / 2) + 8 * quad + 4 * (t % 2) + v) * D + 16 * (CB * wave + b) + l16] = S[g][b][t][v];
        }
    }
}

// dk, dv = the sum of a group's shares, for the rows of the users
constexpr int SUM_THREADS = 256, SUM_BLOCKS = 8;  // (per user)
__global__ __launch_bounds__(SUM_THREADS) void sum_kernel(const Args args, int d) {
    const User us = user_of(args, blockIdx.x);
    const Pass& ps = args.pass[blockIdx.z];
    const int64_t row = (int64_t)args.Hkv * d, slab = args.total_kv * row, first = us.kv0 * row, n = (int64_t)(us.L + us.T) * row;
    for (int64_t e = ((int64_t)blockIdx.y * SUM_THREADS + threadIdx.x) * 8; e < n; e += (int64_t)SUM_BLOCKS * SUM_THREADS * 8) {
        floatx4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
        for (int s = 0; s < args.spread; s++) {
            lo += *(const floatx4*)(ps.partial + s * slab + first + e);
            hi += *(const floatx4*)(ps.partial + s * slab + first + e + 4);
        }
        bf16x8 o;
#pragma unroll
        for (int j = 0; j < 4; j++) o[j] = (__bf16)lo[j], o[4 + j] = (__bf16)hi[j];
        *(bf16x8*)(ps.out + first + e) = o;
    }
}

// Single tokens: a workgroup per row and query head, the state in registers between its reading and its writing.  Lane groups of D / 4 lanes
// hold a state row each (16-byte words), so thread t has columns 4 (t % (D / 4)) .. of rows t / (D / 4) + i ROWS.  Bound by HBM: the state in and out.
// While the state is on its way, the workgroup looks at the other rows' slots: the first row of a slot does the work of all that name it.
constexpr int STEP_THREADS = 256;
template <int D>
__global__ __launch_bounds__(STEP_THREADS) void step_kernel(const __bf16* q, const __bf16* k, const __bf16* v, const float* log_decay, const float* state,
                                                            float* new_state, const int32_t* slots, __bf16* out, int n_rows, int n_slots, int Hq, int Hkv, float scale) {
    constexpr int LANES = D / 4, ROWS = STEP_THREADS / LANES, PER = D / ROWS;
    __shared__ int seen_s[2];               // is there an earlier row of this slot; the next later one
    __shared__ float part_s[ROWS * D];
    const int row0 = blockIdx.x / Hq, h = blockIdx.x % Hq, kvh = h / (Hq / Hkv), tid = threadIdx.x;
    const int slot = slots ? slots[row0] : row0;
    const int c4 = 4 * (tid % LANES), r0 = tid / LANES;
    if (slot < 0 || slot >= n_slots) {
        if (tid < D) out[((int64_t)row0 * Hq + h) * D + tid] = (__bf16)0.f;
        return;
    }
    const int64_t at = ((int64_t)slot * Hq + h) * D * D;
    floatx4 S[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) S[i] = __builtin_nontemporal_load((const floatx4*)(state + at + (r0 + i * ROWS) * D + c4));
    const float decay = expf(fminf(log_decay[h], 0.f));
    for (int row = row0; row < n_rows;) {
        if (tid == 0) seen_s[0] = 0, seen_s[1] = n_rows;
        __syncthreads();
        if (slots) {
            for (int j = row == row0 ? tid : row + 1 + tid; j < n_rows; j += STEP_THREADS)
                if (j != row && slots[j] == slot) {
                    if (j < row0) seen_s[0] = 1;
                    else if (j > row) atomicMin(&seen_s[1], j);
                }
        }
        float kr[PER], qr[PER];
        const __bf16* kp = k + ((int64_t)row * Hkv + kvh) * D;
        const __bf16* qp = q + ((int64_t)row * Hq + h) * D;
#pragma unroll
        for (int i = 0; i < PER; i++) kr[i] = (float)kp[r0 + i * ROWS], qr[i] = (float)qp[r0 + i * ROWS];
        const bf16x4 vr = *(const bf16x4*)(v + ((int64_t)row * Hkv + kvh) * D + c4);
        __syncthreads();
        if (seen_s[0]) return;  // (the same in all threads)
        const int next = slots ? seen_s[1] : n_rows;
        floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < PER; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                S[i][j] = decay * S[i][j] + kr[i] * (float)vr[j];
                o[j] += qr[i] * S[i][j];
            }
        *(floatx4*)&part_s[r0 * D + c4] = o;
        __syncthreads();
        if (tid < D) {
            float total = 0.f;
#pragma unroll
            for (int i = 0; i < ROWS; i++) total += part_s[i * D + tid];
            out[((int64_t)row * Hq + h) * D + tid] = (__bf16)(scale * total);
        }
        row = next;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < PER; i++) __builtin_nontemporal_store(S[i], (floatx4*)(new_state + at + (r0 + i * ROWS) * D + c4));
}

// ------------------------------------------------------------------------------------------------------------ host
bool misaligned(const void* p, unsigned a) { return ((uintptr_t)p & (a - 1)) != 0; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

int check_heads(int32_t Hq, int32_t Hkv, int32_t d, int dtype) {
    if (dtype != MTFM_HTA_BF16) {
        if (dtype != MTFM_HTA_FP32) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "dtype must be MTFM_HTA_BF16, got %d", dtype);
        return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "linear attention takes bf16 tokens only");
    }
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "Hq (%d) must be a positive multiple of Hkv (%d)", Hq, Hkv);
    if (d <= 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "head_dim must be positive, got %d", d);
    if (d != 32 && d != 64 && d != 128) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "head_dim %d: linear attention takes 32, 64 and 128", d);
    if ((int64_t)Hq * d > 1 << 22) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "Hq (%d) x head_dim (%d) exceeds 2^22", Hq, d);
    return MTFM_HTA_OK;
}

int check_sizes(int layer, int dtype, int32_t batch, int64_t total_q, int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t d) {
    if (int rc = check_heads(Hq, Hkv, d, dtype)) return rc;
    if (layer != MTFM_HTA_LAYER_FULL && layer != MTFM_HTA_LAYER_TARGET) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "unknown layer kind %d", layer);
    if (batch < 0 || total_q < 0 || total_kv < 0 || max_hist < 0 || max_targets < 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "negative size");
    if (total_q > INT32_MAX || total_kv > INT32_MAX) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "more than 2^31 - 1 rows");
    if ((int64_t)batch * Hq > (int64_t)1 << 26) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "batch (%d) x Hq (%d) exceeds 2^26", batch, Hq);
    return MTFM_HTA_OK;
}

// heads of a group that a backward workgroup holds: what registers allow of the largest power of two that divides the group
int heads_per_workgroup(int ratio, int d) {
    const int most = d == 128 ? 2 : 4;
    int g = 1;
    while (2 * g <= most && ratio % (2 * g) == 0) g *= 2;
    return g;
}

struct Plan {
    int G, spread;
    size_t partial;  // bytes of one slab set (dk or dv)
};
Plan plan_backward(int64_t total_kv, int Hq, int Hkv, int d) {
    Plan p;
    p.G = heads_per_workgroup(Hq / Hkv, d);
    p.spread = Hq / Hkv / p.G;
    p.partial = p.spread > 1 ? align256((size_t)p.spread * total_kv * Hkv * d * sizeof(float)) : 0;
    return p;
}

template <int D, int G, int CB, bool BACK>
hipError_t launch_sweep_as(const Args& a, hipStream_t s) {
    const int64_t members = (int64_t)(BACK ? a.spread : a.ratio) * a.n_pass, groups = (int64_t)a.batch * a.Hkv;
    const int64_t grid = (groups + hta::N_XCD - 1) / hta::N_XCD * hta::N_XCD * members;
    hipLaunchKernelGGL((sweep_kernel<D, G, CB, BACK>), dim3((unsigned)grid), dim3(D * 4 / CB), 0, s, a);
    return hipGetLastError();
}
template <int D>
hipError_t launch_sweep_d(const Args& a, bool back, int G, hipStream_t s) {
    if (!back) return launch_sweep_as<D, 1, 1, false>(a, s);
    if (G == 1) return launch_sweep_as<D, 1, 1, true>(a, s);
    if (G == 2) return launch_sweep_as<D, 2, 1, true>(a, s);
    if constexpr (D < 128) return launch_sweep_as<D, 4, 1, true>(a, s);
    return hipErrorInvalidValue;
}
hipError_t launch_sweep(const Args& a, int d, bool back, int G, hipStream_t s) {
    return d == 32 ? launch_sweep_d<32>(a, back, G, s) : d == 64 ? launch_sweep_d<64>(a, back, G, s) : launch_sweep_d<128>(a, back, G, s);
}

Args args_of(const float* log_decay, const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len, const int32_t* n_targets, int32_t batch,
             int64_t total_q, int64_t total_kv, int32_t Hq, int32_t Hkv, float scale, int layer) {
    Args a = {};
    a.log_decay = log_decay, a.q_off = q_offsets, a.kv_off = kv_offsets, a.hist_len = hist_len, a.n_targets = n_targets;
    a.total_q = total_q, a.total_kv = total_kv, a.batch = batch, a.Hq = Hq, a.Hkv = Hkv, a.ratio = Hq / Hkv, a.n_pass = 1, a.spread = 1;
    a.full = layer == MTFM_HTA_LAYER_FULL, a.scale = scale;
    return a;
}

int check_arrays(std::initializer_list<const void*> rows_q, std::initializer_list<const void*> rows_kv, std::initializer_list<const void*> states,
                 const float* log_decay, std::initializer_list<const int32_t*> ints, int64_t total_q, int64_t total_kv, float scale) {
    if (!(scale > 0.f) || !(scale < INFINITY)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "scale must be positive and finite");
    if (!log_decay) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    for (const int32_t* p : ints)
        if (!p) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    for (const void* p : rows_q)
        if (total_q > 0 && !p) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    for (const void* p : rows_kv)
        if (total_kv > 0 && !p) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    for (const auto& list : {rows_q, rows_kv, states})
        for (const void* p : list)
            if (misaligned(p, 16)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "rows and states must be 16-byte aligned");
    if (misaligned(log_decay, 4)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "log_decay must be 4-byte aligned");
    for (const int32_t* p : ints)
        if (misaligned(p, 4)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "int32 arrays must be 4-byte aligned");
    return MTFM_HTA_OK;
}

int check_workspace(size_t need, const void* workspace, size_t bytes) {
    if (need == 0) return MTFM_HTA_OK;
    if (!workspace || bytes < need)
        return hta::report_error(MTFM_HTA_ERR_WORKSPACE, "this call needs %zu bytes of workspace, got %zu", need, workspace ? bytes : (size_t)0);
    if (misaligned(workspace, 256)) return hta::report_error(MTFM_HTA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    return MTFM_HTA_OK;
}

template <int D>
hipError_t launch_step(const void* q, const void* k, const void* v, const float* log_decay, const float* state, float* new_state, const int32_t* slots, void* out,
                       int n_rows, int n_slots, int Hq, int Hkv, float scale, hipStream_t s) {
    hipLaunchKernelGGL((step_kernel<D>), dim3((unsigned)(n_rows * Hq)), dim3(STEP_THREADS), 0, s, (const __bf16*)q, (const __bf16*)k, (const __bf16*)v, log_decay,
                       state, new_state, slots, (__bf16*)out, n_rows, n_slots, Hq, Hkv, scale);
    return hipGetLastError();
}

}  // namespace hla

extern "C" {

size_t mtfm_hla_workspace_bytes(int layer, int dtype, int is_bwd, int32_t batch, int64_t total_q, int64_t total_kv, int32_t max_hist, int32_t max_targets,
                                int32_t Hq, int32_t Hkv, int32_t head_dim) {
    if (hla::check_sizes(layer, dtype, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, head_dim) != MTFM_HTA_OK) return (size_t)-1;
    if (!is_bwd || batch == 0) return 0;
    return 2 * hla::plan_backward(total_kv, Hq, Hkv, head_dim).partial;
}

int mtfm_hla_fwd(const void* q, const void* k, const void* v, const float* log_decay, const float* state, void* out, float* final_state,
                 const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len, const int32_t* n_targets, int32_t batch, int64_t total_q,
                 int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t head_dim, float scale, int dtype, int layer,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = hla::check_sizes(layer, dtype, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, head_dim)) return rc;
    if (batch == 0) return MTFM_HTA_OK;
    if (int rc = hla::check_arrays({q, out}, {k, v}, {state, final_state}, log_decay, {q_offsets, kv_offsets, hist_len, n_targets}, total_q, total_kv, scale)) return rc;
    hla::Args a = hla::args_of(log_decay, q_offsets, kv_offsets, hist_len, n_targets, batch, total_q, total_kv, Hq, Hkv, scale, layer);
    a.pass[0] = {(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (__bf16*)out, nullptr, state, final_state, 0};
    hipStream_t s = (hipStream_t)stream;
    hta::timing_begin(MTFM_HLA_KERNEL_FWD, s);
    const hipError_t e = hla::launch_sweep(a, head_dim, false, 1, s);
    hta::timing_end(MTFM_HLA_KERNEL_FWD, s);
    if (e != hipSuccess) return hta::report_error(MTFM_HTA_ERR_LAUNCH, "linear attention forward launch: %s", hipGetErrorString(e));
    return MTFM_HTA_OK;
}

int mtfm_hla_bwd(const void* dout, const void* q, const void* k, const void* v, const float* log_decay, const float* state, const float* dfinal_state, void* dq,
                 void* dk, void* dv, float* dstate, const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len, const int32_t* n_targets,
                 int32_t batch, int64_t total_q, int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t head_dim, float scale,
                 int dtype, int layer, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = hla::check_sizes(layer, dtype, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, head_dim)) return rc;
    if (batch == 0) return MTFM_HTA_OK;
    if (int rc = hla::check_arrays({dout, q, dq}, {k, v, dk, dv}, {state, dfinal_state, dstate}, log_decay, {q_offsets, kv_offsets, hist_len, n_targets}, total_q,
                                   total_kv, scale))
        return rc;
    const hla::Plan plan = hla::plan_backward(total_kv, Hq, Hkv, head_dim);
    if (int rc = hla::check_workspace(2 * plan.partial, workspace, workspace_bytes)) return rc;
    hla::Args a = hla::args_of(log_decay, q_offsets, kv_offsets, hist_len, n_targets, batch, total_q, total_kv, Hq, Hkv, scale, layer);
    hipStream_t s = (hipStream_t)stream;
    const auto Q = (const __bf16*)q, K = (const __bf16*)k, V = (const __bf16*)v, dO = (const __bf16*)dout;
    hipError_t e = hipSuccess;
    hta::timing_begin(MTFM_HLA_KERNEL_BWD, s);
    if (total_q > 0) {
        a.pass[0] = {dO, V, K, (__bf16*)dq, nullptr, state, nullptr, 1};
        e = hla::launch_sweep(a, head_dim, false, 1, s);
    }
    if (e == hipSuccess) {
        float* partial = plan.spread > 1 ? (float*)workspace : nullptr;
        a.pass[0] = {K, Q, dO, (__bf16*)dv, partial, dfinal_state, dstate, 0};
        a.pass[1] = {V, dO, Q, (__bf16*)dk, partial ? partial + plan.partial / sizeof(float) : nullptr, dfinal_state, nullptr, 1};
        a.n_pass = 2, a.spread = plan.spread;
        e = hla::launch_sweep(a, head_dim, true, plan.G, s);
    }
    hta::timing_end(MTFM_HLA_KERNEL_BWD, s);
    if (e == hipSuccess && plan.spread > 1 && total_kv > 0) {
        hta::timing_begin(MTFM_HLA_KERNEL_SUM, s);
        hipLaunchKernelGGL(hla::sum_kernel, dim3(batch, hla::SUM_BLOCKS, 2), dim3(hla::SUM_THREADS), 0, s, a, head_dim);
        e = hipGetLastError();
        hta::timing_end(MTFM_HLA_KERNEL_SUM, s);
    }
    if (e != hipSuccess) return hta::report_error(MTFM_HTA_ERR_LAUNCH, "linear attention backward launch: %s", hipGetErrorString(e));
    return MTFM_HTA_OK;
}

int mtfm_hla_step(const void* q, const void* k, const void* v, const float* log_decay, const float* state, float* new_state, const int32_t* slots, void* out,
                  int32_t n_rows, int32_t n_slots, int32_t Hq, int32_t Hkv, int32_t head_dim, float scale, int dtype, void* stream) {
    if (int rc = hla::check_heads(Hq, Hkv, head_dim, dtype)) return rc;
    if (n_rows < 0 || n_slots < 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "negative size");
    if ((int64_t)n_rows * Hq > (int64_t)1 << 26) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "n_rows (%d) x Hq (%d) exceeds 2^26", n_rows, Hq);
    if (n_rows == 0) return MTFM_HTA_OK;
    if (!(scale > 0.f) || !(scale < INFINITY)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "scale must be positive and finite");
    if (!q || !k || !v || !log_decay || !out || (n_slots > 0 && (!state || !new_state))) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    if (!slots && n_slots < n_rows) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "%d rows without slots for %d states", n_rows, n_slots);
    for (const void* p : {q, k, v, (const void*)state, (const void*)new_state, (const void*)out})
        if (hla::misaligned(p, 16)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "rows and states must be 16-byte aligned");
    if (hla::misaligned(slots, 4) || hla::misaligned(log_decay, 4)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "slots and log_decay must be 4-byte aligned");
    hipStream_t s = (hipStream_t)stream;
    hta::timing_begin(MTFM_HLA_KERNEL_STEP, s);
    const auto launch = head_dim == 32 ? hla::launch_step<32> : head_dim == 64 ? hla::launch_step<64> : hla::launch_step<128>;
    const hipError_t e = launch(q, k, v, log_decay, state, new_state, slots, out, n_rows, n_slots, Hq, Hkv, scale, s);
    hta::timing_end(MTFM_HLA_KERNEL_STEP, s);
    if (e != hipSuccess) return hta::report_error(MTFM_HTA_ERR_LAUNCH, "linear attention step launch: %s", hipGetErrorString(e));
    return MTFM_HTA_OK;
}

}  // extern "C"

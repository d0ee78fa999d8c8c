// Hybrid linear attention with a decay for each head (include/mtfm_hla.h) for gfx950: forward, backward, single tokens.
//
// All passes over a user's tokens are one sweep.  With rows a_i that ask, and pairs (b_i, c_i) that enter a state,
//   S <- l S + b_i c_i^T,   o_i = scale a_i S
// is the forward pass for (a, b, c) = (q, k, v); the gradients are the same sweep with the letters exchanged: dq for (dout, v, k)
// in the same direction with the states transposed, and from the last row backwards dv for (k, q, dout) and dk for (v, dout, q), which
// share the state (one has it transposed) and are one kernel.
//
// A workgroup owns a user's head and goes through the tokens in chunks of 64 or 32.  Inside a chunk, with i, j counted from its start and
// S the state in front of it,
//   o_i = scale [ l^(i+1) a_i S + sum_(j<=i) l^(i-j) <a_i, b_j> c_j ],    S <- l^n S + sum_j l^(n-1-j) b_j c_j^T:
// four matrix products.  The floor is HBM's (4 d^2 + 64 d operations per row and head on 8 d bytes), so a row is read once: the
// state stays in registers from chunk to chunk -- wave w owns its columns [16 w, 16 w + 16), whose accumulators are, rounded, the
// operand of the product with a -- and the next chunk's rows are in flight while the current one is worked on.  Backwards the state is
// handed on decayed already (o_i takes l^i, the update l^(n-j)), so that the gradient of S_L enters, and that of S_0 leaves, as it is.
//
// Roundings: operands of a product are bf16 (the state where rows ask it, weights between two products, results), sums float32.  What enters a state keeps 16
// bits, in two parts of bf16, or 24, in three, where the state is what the caller gets: rounded to 8 it would be off by 2^-9 after the first token.
// Long histories of few users are cut into pieces (plan_of): what each adds to a state, the states in front of them, then all of them at once.
#include "../../include/mtfm_hla.h"
#include "hta_common.h"
#include "hta_mfma.h"

#include <hip/hip_runtime.h>

namespace hla {

using hta::bf16x4;
using hta::bf16x8;
using hta::fast_exp2;
using hta::floatx4;

constexpr int MOST_ROWS = 64;  // of a chunk
constexpr float MIN_LOG2 = -1e4f;  // of a decay: 2^-10000 is 0, and 0 times it is not NaN

// A sweep in the tokens' order: the forward pass, or dq
struct Args {
    const __bf16 *a, *b, *c;
    __bf16* out;
    const float* state_in;  // null: zero
    float* state_out;       // null: not wanted
    int32_t transposed;     // the state that is read is that of the forward sweep, transposed
    const float* log_decay;
    const int32_t *q_off, *kv_off, *hist_len, *n_targets;
    int64_t total_q, total_kv;
    int32_t batch, Hq, Hkv, ratio;
    int32_t full, max_hist, max_targets;
    float scale;
    // backwards: dk, dv and the first state's gradient
    const __bf16 *q, *k, *v, *dout;
    __bf16 *dk, *dv;
    float *partial_k, *partial_v;  // where a group's heads are spread over workgroups: [spread][total_kv][Hkv][d] each; null otherwise
    int32_t spread;
    // long histories in pieces (seg > 0): `seg` rows of one kind to a workgroup, at most n_hist pieces of a history and n_tgt of a user's candidates.  The
    // states in front of the pieces lie in [batch][Hq][n_hist + n_tgt + 1][d][d], in the order of the sweep (backwards the candidates' come first), and the one
    // behind them all.
    int32_t seg, n_hist, n_tgt;
    float *states, *states_back;
    const int32_t* order;  // users by decreasing work; null: as they come
};

// What of a user a workgroup has: rows [h0, h1) of the history in the sweep's order, candidates [t0, t1), and the index of the state in front of them (-1, without
// pieces: what the caller gave)
struct Piece {
    int h0, h1, t0, t1, state;
};
__device__ inline int64_t state_index(const Args& g, int u, int h, int i) { return ((int64_t)u * g.Hq + h) * (g.n_hist + g.n_tgt + 1) + i; }
// Which user, key/value head, piece and member (query head, or set of them) a workgroup has: those that share rows are neighbours on one XCD, and pieces go around
// the XCDs.  False: none.
struct Place {
    int u, kvh, member, piece;
};
__device__ inline bool place_of(const Args& g, int members, Place& w) {
    const int pieces = g.seg ? g.n_hist + g.n_tgt : 1, xcd = blockIdx.x % hta::N_XCD, slot = blockIdx.x / hta::N_XCD;
    const int64_t unit = (int64_t)(slot / members) * hta::N_XCD + xcd;
    if (unit >= (int64_t)g.batch * g.Hkv * pieces) return false;
    const int group = (int)(unit / pieces);
    w.u = g.order ? g.order[group / g.Hkv] : group / g.Hkv, w.kvh = group % g.Hkv, w.member = slot % members, w.piece = (int)(unit % pieces);
    return true;
}
__device__ inline Piece piece_of(const Args& g, int id, int L, int T, bool back) {
    if (g.seg == 0) return {0, L, 0, T, -1};
    const int hs = (L + g.seg - 1) / g.seg, ts = (T + g.seg - 1) / g.seg;
    if (id < g.n_hist) return {min(id * g.seg, L), min((id + 1) * g.seg, L), 0, 0, back ? ts + id : id};
    id -= g.n_hist;
    return {0, 0, min(id * g.seg, T), min((id + 1) * g.seg, T), back ? id : hs};
}

// Tiles in LDS lie in rows of D elements without padding; the 16-byte word w of row r is at position w ^ place<D>(r).  A 16-byte read is served in groups of
// 16 lanes, 0 .. 3, 12 .. 15 and 20 .. 27 the first (the bank conflicts of two lanes say so), an 8-byte read in groups of 32: with this order neither has a
// conflict where 16 lanes read a word of 16 rows and the next 16 its neighbour, or a transposing read takes two words of 4 rows and of 4 rows 8 further.
// (Forward, 212 548 rows, 8/2 heads of 64: 4.4 M cycles of conflicts of 31.6 M that LDS works, 14.3 M in the order before it, made for groups of neighbours.)
template <int D>
__device__ inline int place(int row) {
    const int h = (row >> 2) & 3, c = (((h ^ (h >> 1)) & 1) << 1) | (h >> 1);
    return D == 32 ? c : D == 64 ? (((row >> 1) & 1) << 2) | c : ((row & 3) << 2) | c;
}

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

// Where a user's rows lie, whatever the arrays hold: inside the tensors, and no more of them than was said
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
    r.L = (int)clamp64(clamp64(g.hist_len[u], 0, g.max_hist), 0, g.full ? (n_kv < n_q ? n_kv : n_q) : n_kv);
    const int64_t left_kv = n_kv - r.L, left_q = g.full ? n_q - r.L : n_q;
    r.T = (int)clamp64(clamp64(g.n_targets[u], 0, g.max_targets), 0, left_kv < left_q ? left_kv : left_q);
    return r;
}

// Bytes from the start of a tile that a lane's reads go to, for rows and words that differ in nothing that place<>() looks at but the bits that are
// exchanged here.  (Kept out of the compiler's sight in every turn of the loops: it would keep each of the addresses that follow from them in a register.)
template <int D>
struct Lane {
    unsigned stage;  // the word that the thread stages: row tid / (D / 8), word tid % (D / 8)
    unsigned row;    // word quad of row l16: an operand with its contraction along the row, k = 8 quad ..; words 4 k further by ^ 64 k
    unsigned tr;     // the first of two transposing reads: rows 8 quad .. + 3, columns 0 .. 15 of the wave's first block
    unsigned trp;    // the same, columns 8 (l16 & 3) .. + 3: in the order of the state's rows
    __device__ Lane(int tid, int l16, int quad, int first_block) {
        const int r = tid / (D / 8), w = tid % (D / 8), t = 8 * quad + (l16 >> 2);
        stage = r * (D * 2) + ((w ^ place<D>(r)) * 16);
        row = l16 * (D * 2) + ((quad ^ place<D>(l16)) * 16);
        tr = t * (D * 2) + (((2 * first_block + ((l16 & 3) >> 1)) ^ place<D>(t)) * 16) + (l16 & 1) * 8;
        trp = t * (D * 2) + (((l16 & 3) ^ place<D>(t)) * 16);
    }
    __device__ void forget(int& tid, int& l16, int& quad) { asm volatile("" : "+v"(stage), "+v"(row), "+v"(tr), "+v"(trp), "+v"(tid), "+v"(l16), "+v"(quad)); }
};
template <typename T>
__device__ inline T& lds(char* base, unsigned at) {
    return *(T*)(base + at);
}
// rows r .. r + 3 and r + 4 .. r + 7 of a transposing read at `at` (place<>() of a row 4 further differs by 2 words)
template <int D>
__device__ inline bf16x8 read_tr(char* tile, unsigned at) {
    return hta::lds_read_tr_pair((const __bf16*)(tile + at), (const __bf16*)(tile + (at ^ 32) + 4 * D * 2));
}

constexpr int ZERO = MOST_ROWS, POWERS = 2 * MOST_ROWS + 4;  // powers of a decay: entry ZERO + m holds l^m, m = -64 .. 64, 0 for m < 0
// the tables of `heads` heads from h on, [plain | times scale] each
template <int NT>
__device__ inline void fill_powers(float* table, const float* log_decay, int heads, float scale, int tid) {
    for (int i = tid; i < heads * POWERS; i += NT) {
        const int g = i / POWERS, m = i % POWERS - ZERO;
        const float g2 = fmaxf(fminf(log_decay[g], 0.f) * hta::LOG2E, MIN_LOG2);
        const float p = m < 0 ? 0.f : fast_exp2(g2 * (float)m);
        table[2 * g * POWERS + m + ZERO] = p, table[(2 * g + 1) * POWERS + m + ZERO] = p * scale;
    }
}

// One tile of P^T = B A^T with the decays, rows i = 16 it .. of A (queries), rows j = 16 jt .. of B, to P[i][j]
template <int D, int C>
__device__ inline void score_tile(char* a, char* b, char* p_tile, const float* scaled, const Lane<D>& at, const Lane<C>& at_p, int it, int jt, int l16, int quad) {
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < D / 32; k++)
        s = mfma16(lds<bf16x8>(b + jt * (16 * D * 2), at.row ^ (64 * k)), lds<bf16x8>(a + it * (16 * D * 2), at.row ^ (64 * k)), s);
    const int d = 16 * (it - jt) + l16 - 4 * quad;  // i - j
    const float* power = scaled + ZERO + d;
    float w[4];
#pragma unroll
    for (int v = 0; v < 4; v++) w[v] = power[-v];
    bf16x4 p;
#pragma unroll
    for (int v = 0; v < 4; v++) {
        s[v] *= w[v];
        p[v] = (__bf16)(d >= v ? s[v] : 0.f);  // (0 times what a later row holds need not be 0)
    }
    // word 2 jt + quad / 2 of row i, its half quad % 2: from word quad
    const unsigned to = (at_p.row ^ ((quad ^ (quad >> 1)) * 16) ^ (32 * jt)) + (quad & 1) * 8;
    lds<bf16x4>(p_tile + it * (16 * C * 2), to) = p;
}
__device__ inline int tile_row(int t) { return t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0; }  // of the ten tiles on and below the diagonal

// C^T P^T: what a chunk's own rows add, rows 16 it .. to x[it].  An infinity or a NaN in c would reach the rows in front of it as 0 times itself; it reaches the
// last rows in any case, and where those are not finite all of it is done again, row by row.
template <int D, int C>
__device__ inline void within_chunk(floatx4 (&x)[C / 16], const bf16x8 (&ct)[C / 32], char* p_tile, char* c_tile, const Lane<C>& at_p, int block, int l16, int quad) {
    constexpr int IT = C / 16;
#pragma unroll
    for (int it = 0; it < IT; it++) {
        x[it] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k <= it / 2; k++) x[it] = mfma16(ct[k], lds<bf16x8>(p_tile + it * (16 * C * 2), at_p.row ^ (64 * k)), x[it]);
    }
    const float zero = fmaf(x[IT - 1][0], 0.f, x[IT - 1][1] * 0.f) + fmaf(x[IT - 1][2], 0.f, x[IT - 1][3] * 0.f);
    if (__ballot(zero != zero) != 0) {
#pragma unroll
        for (int it = 0; it < IT; it++) x[it] = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < C; j++) {
            const bf16x4 c = lds<bf16x4>(c_tile, j * (D * 2) + (((2 * block + (quad >> 1)) ^ place<D>(j)) * 16) + (quad & 1) * 8);
#pragma unroll
            for (int it = 0; it < IT; it++) {
                const int i = 16 * it + l16;
                const float p = (float)lds<__bf16>(p_tile, i * (C * 2) + (((j / 8) ^ place<C>(i)) * 16) + (j & 7) * 2);
#pragma unroll
                for (int v = 0; v < 4; v++) x[it][v] += j <= i ? p * (float)c[v] : 0.f;
            }
        }
    }
}

// candidates: <a_i, b_i> scale to dots[i], NT / C lanes to a row
template <int D, int C, int NT>
__device__ inline void own_dots(char* a, char* b, float* dots, float scale, int tid) {
    constexpr int LANES = NT / C, WORDS = D / 8 / LANES;
    const int row = tid / LANES, part = tid % LANES;
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < WORDS; k++) {
        const unsigned at = row * (D * 2) + (((WORDS * part + k) ^ place<D>(row)) * 16);
        dot = hta::dot_bf16x8(dot, lds<bf16x8>(a, at), lds<bf16x8>(b, at));
    }
    dot = hta::sum_lanes<LANES>(dot);
    if (part == 0) dots[row] = dot * scale;
}
template <int D>
__device__ inline floatx4 own_term(const float* dots, char* c_tile, int block, int i, int quad) {
    const bf16x4 c = lds<bf16x4>(c_tile, i * (D * 2) + (((2 * block + (quad >> 1)) ^ place<D>(i)) * 16) + (quad & 1) * 8);
    const float dot = dots[i];
    return floatx4{dot * (float)c[0], dot * (float)c[1], dot * (float)c[2], dot * (float)c[3]};
}

// A state's columns, 16 to a wave (block `block`): tile t, register v of a lane: row 32 (t / 2) + 8 quad + 4 (t % 2) + v, column 16 block + l16.  (Rows in this
// order make the accumulators of two tiles eight consecutive rows: what an operand wants.)
template <int D>
struct State {
    static constexpr int TILES = D / 16, KS = D / 32;
    floatx4 t[TILES];
    __device__ static int row(int tile, int quad) { return 32 * (tile / 2) + 8 * quad + 4 * (tile % 2); }
    __device__ void zero() {
#pragma unroll
        for (int i = 0; i < TILES; i++) t[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ void load(const float* in, bool transposed, int block, int l16, int quad) {
        const int col = 16 * block + l16;
#pragma unroll
        for (int i = 0; i < TILES; i++) {
            if (transposed) t[i] = *(const floatx4*)(in + col * D + row(i, quad));
            else
#pragma unroll
                for (int v = 0; v < 4; v++) t[i][v] = in[(row(i, quad) + v) * D + col];
        }
    }
    __device__ void store(float* out, int block, int l16, int quad) const {
        const int col = 16 * block + l16;
#pragma unroll
        for (int i = 0; i < TILES; i++)
#pragma unroll
            for (int v = 0; v < 4; v++) out[(row(i, quad) + v) * D + col] = t[i][v];
    }
    __device__ void keep(float f) {
#pragma unroll
        for (int i = 0; i < TILES; i++) t[i] *= f;
    }
    __device__ void rounded(bf16x8 (&s)[KS]) const {  // operands: rows 32 k + 8 quad .. + 7
#pragma unroll
        for (int k = 0; k < KS; k++)
#pragma unroll
            for (int v = 0; v < 4; v++) s[k][v] = (__bf16)t[2 * k][v], s[k][4 + v] = (__bf16)t[2 * k + 1][v];
    }
    // += B^T (w c): w c goes in as two bf16 values, 16 bits of it, or as three, all of float32's, where the state itself is what the caller gets (`whole`).
    // w[-j]: the weight of row j (rows that are not there are zero, and so are the weights behind the table's end); step 0: the same for all.
    template <int KT, typename Step>
    __device__ void add(char* b_tile, const bf16x8 (&ct)[KT], const float* w, Step, const Lane<D>& at, int quad, bool whole) {
        constexpr int step = Step::value;
#pragma unroll
        for (int k = 0; k < KT; k++) {
            const float* p = w - step * (32 * k + 8 * quad);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = p[-e * step] * (float)ct[k][e];
            bf16x8 hi, lo;
            split8(x, hi, lo);
#pragma unroll
            for (int i = 0; i < TILES; i++) {
                const bf16x8 bt = read_tr<D>(b_tile + 32 * k * (D * 2) + 8 * (i % 2), at.trp ^ (64 * (i / 2)));
                t[i] = mfma16(bt, hi, t[i]);
                t[i] = mfma16(bt, lo, t[i]);
            }
            if (!whole) continue;
            bf16x8 rest;
#pragma unroll
            for (int e = 0; e < 8; e++) rest[e] = (__bf16)(x[e] - (float)hi[e] - (float)lo[e]);
#pragma unroll
            for (int i = 0; i < TILES; i++)
                t[i] = mfma16(read_tr<D>(b_tile + 32 * k * (D * 2) + 8 * (i % 2), at.trp ^ (64 * (i / 2))), rest, t[i]);
        }
    }
};

// A chunk's rows in memory: a uniform address, that of the lowest of C rows (backwards through a history row C - 1, which need not be there), and a lane's
// bytes from there
template <int C>
__device__ inline int64_t lowest(bool down, int64_t first) { return down ? first - (C - 1) : first; }
template <int C>
__device__ inline unsigned bytes_of(bool down, int r, unsigned pitch, int byte) { return __umul24(down ? C - 1 - r : r, pitch) + byte; }

// What a chunk's rows are: a history's that ask, a history's that do not (a target-only layer), candidates.  The loops have a body for each: branches inside a
// body leave accumulators to be moved about.
enum Kind { ASKING, SILENT, CANDIDATES };
template <Kind K>
using KindOf = std::integral_constant<Kind, K>;

struct Rows {  // of a chunk: n rows, row r is first + r (backwards through a history: first - r)
    int64_t q, kv;
    int n;
    bool hist;
};

// One sweep over a user's head in the tokens' order by a workgroup of D / 16 waves, each with 16 of the state's columns.  D[m][n] += A[m][k] B[k][n] of
// 16x16x32: a lane holds row (column) lane % 16 and k = 8 (lane / 16) .. + 7 of either operand, and column lane % 16, rows 4 (lane / 16) .. + 3 of the result.
//
// 212 548 rows of 256 users, 8/2 heads of 64: 152 us = 3.6 TB/s of q, k, v and out (the first form 335; 196 with tables of the powers and 32-bit offsets, 160 with
// one look for what is not finite, behind the product).  364 182 rows, 16/2 of 128: 1015 to 1032 us = 3.3 TB/s (1860, 1540, 1400 on that way; in chunks of 64
// rows 4 % more).  No unit is full: at d = 64 the vector units are busy for 0.46 of the time, LDS for 0.42, the matrix units for 0.19, HBM for 0.7 of what a
// copy reaches; the barriers of a chunk keep them from lying over each other.
template <int D, int C, bool FULL>
__global__ __launch_bounds__(D * 4, 4) void sweep_kernel(const Args args) {
    constexpr int NW = D / 16, NT = NW * 64, C16 = D / 8, KS = D / 32, PART = NT / C16, LOADS = C / PART, TILE = C * D * 2, IT = C / 16, KT = C / 32, TILES = IT * (IT + 1) / 2;
    __shared__ __attribute__((aligned(16))) char a_s[TILE], b_s[TILE], c_s[TILE], p_s[C * C * 2];
    __shared__ float dots_s[C], powers_s[2 * POWERS];
    int tid = threadIdx.x, l16 = tid & 15, quad = (tid >> 4) & 3;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    Place place;
    if (!place_of(args, args.ratio, place)) return;
    const int u = place.u, kvh = place.kvh, qh = kvh * args.ratio + place.member;
    const User us = user_of(args, u);
    const Piece piece = piece_of(args, place.piece, us.L, us.T, false);
    const int nh = (piece.h1 - piece.h0 + C - 1) / C, chunks = nh + (piece.t1 - piece.t0 + C - 1) / C;
    if (args.seg && (chunks == 0 || (nh > 0 && !FULL))) return;

    State<D> S;
    if (piece.state >= 0) S.load(args.states + state_index(args, u, qh, piece.state) * D * D, false, wave, l16, quad);
    else if (args.state_in) S.load(args.state_in + ((int64_t)u * args.Hq + qh) * D * D, args.transposed, wave, l16, quad);
    else S.zero();

    const auto rows_of = [&](int c) {
        Rows r;
        r.hist = c < nh;
        const int first = r.hist ? piece.h0 + c * C : piece.t0 + (c - nh) * C;
        r.n = min(C, (r.hist ? piece.h1 : piece.t1) - first);
        r.kv = us.kv0 + (r.hist ? 0 : us.L) + first, r.q = us.q0 + (!r.hist && FULL ? us.L : 0) + first;
        return r;
    };
    // 16-byte words of the three tiles on their way: word tid % C16 of rows tid / C16 + i PART.  Rows that are not there are zero.
    const unsigned pitch_q = args.Hq * (D * 2), pitch_kv = args.Hkv * (D * 2);
    bf16x8 av[LOADS], bv[LOADS], cv[LOADS];
    const auto fetch = [&](int chunk) {
        const Rows r = rows_of(chunk);
        const bool asks = FULL || !r.hist;
        const char* a = (const char*)(args.a + (r.q * args.Hq + qh) * D);
        const char *b = (const char*)(args.b + (r.kv * args.Hkv + kvh) * D), *c = (const char*)(args.c + (r.kv * args.Hkv + kvh) * D);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int row = tid / C16 + i * PART;
            const unsigned at_a = bytes_of<C>(false, row, pitch_q, tid % C16 * 16), at_b = bytes_of<C>(false, row, pitch_kv, tid % C16 * 16);
            av[i] = bv[i] = cv[i] = bf16x8{};
            if (row < r.n) {
                if (asks) av[i] = *(const bf16x8*)(a + at_a);
                bv[i] = *(const bf16x8*)(b + at_b), cv[i] = *(const bf16x8*)(c + at_b);
            }
        }
    };

    if (chunks > 0) fetch(0);
    fill_powers<NT>(powers_s, args.log_decay + qh, 1, args.scale, tid);
    const float *power = powers_s, *scaled = powers_s + POWERS;
    // (entries of P that a product reads and no chunk writes)
    for (int i = tid; i < C * C / 8; i += NT) ((bf16x8*)p_s)[i] = bf16x8{};
    Lane<D> at(tid, l16, quad, wave);
    Lane<C> at_p(0, l16, quad, 0);

    const auto turn = [&](auto K, int c) {
        constexpr Kind kind = decltype(K)::value;
        const Rows r = rows_of(c);
        at.forget(tid, l16, quad);
        at_p.forget(tid, l16, quad);
        // (the last readers of the tiles are behind the barrier at the end of the turn)
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            if (kind != SILENT) lds<bf16x8>(a_s + i * PART * (D * 2), at.stage) = av[i];
            lds<bf16x8>(b_s + i * PART * (D * 2), at.stage) = bv[i];
            lds<bf16x8>(c_s + i * PART * (D * 2), at.stage) = cv[i];
        }
        __syncthreads();
        if (c + 1 < chunks) fetch(c + 1);
        if (kind == ASKING) {
#pragma unroll
            for (int t0 = 0; t0 < TILES; t0 += NW) {
                const int t = t0 + wave, it = tile_row(t), jt = t - it * (it + 1) / 2;
                if (t0 + NW <= TILES || t < TILES) score_tile<D, C>(a_s, b_s, p_s, scaled, at, at_p, it, jt, l16, quad);
            }
        } else if (kind == CANDIDATES) {
            own_dots<D, C, NT>(a_s, b_s, dots_s, args.scale, tid);
        }
        // o^T = S^T A^T, row i of it times l^(i+1) scale (candidates: l scale)
        floatx4 o[IT];
        if (kind != SILENT) {
            bf16x8 s[KS];
            S.rounded(s);
#pragma unroll
            for (int it = 0; it < IT; it++)
#pragma unroll
                for (int k = 0; k < KS; k++)
                    o[it] = mfma16(s[k], lds<bf16x8>(a_s + it * (16 * D * 2), at.row ^ (64 * k)), k == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : o[it]);
            __syncthreads();
        }
        bf16x8 ct[KT];  // C^T: this wave's columns of c, rows 32 k + 8 quad .. + 7
        if (kind != CANDIDATES)
#pragma unroll
            for (int k = 0; k < KT; k++) ct[k] = read_tr<D>(c_s + 32 * k * (D * 2), at.tr);
        if (kind != SILENT) {
            char* out = (char*)(args.out + (r.q * args.Hq + qh) * D);
            floatx4 x[IT];
            if (kind == ASKING) within_chunk<D, C>(x, ct, p_s, c_s, at_p, wave, l16, quad);
#pragma unroll
            for (int it = 0; it < IT; it++) {
                if (kind == CANDIDATES) x[it] = own_term<D>(dots_s, c_s, wave, 16 * it + l16, quad);
                const float w = scaled[ZERO + 1 + (kind == ASKING ? 16 * it + l16 : 0)];
                bf16x4 y;
#pragma unroll
                for (int v = 0; v < 4; v++) y[v] = (__bf16)fmaf(o[it][v], w, x[it][v]);
                if (16 * it + l16 < r.n) *(bf16x4*)(out + bytes_of<C>(false, 16 * it + l16, pitch_q, 32 * wave + 8 * quad)) = y;
            }
        }
        if (kind != CANDIDATES) {  // the state behind the chunk: l^n S + B^T (w c), w_j = l^(n-1-j)
            S.keep(power[ZERO + r.n]);
            S.add(b_s, ct, power + ZERO + r.n - 1, std::integral_constant<int, 1>{}, at, quad, args.state_out != nullptr);
        }
        __syncthreads();
    };
    int c = 0;
    for (; c < nh; c++) turn(KindOf<FULL ? ASKING : SILENT>{}, c);
    for (; c < chunks; c++) turn(KindOf<CANDIDATES>{}, c);
    if (args.state_out && !args.seg) S.store(args.state_out + ((int64_t)u * args.Hq + qh) * D * D, wave, l16, quad);
}

// dk, dv and the first state's gradient: a sweep from a user's candidates over its history's end to its beginning, for G query heads of a group, whose
// gradients it sums.  With R the state's gradient, rows in the sweep's order, i, j counted from a chunk's start and R handed on decayed already,
//   dv_i = l^i k_i R + scale sum_(j<=i) l^(i-j) <k_i, q_j> dout_j,     dk_i = l^i v_i R^T + scale sum_(j<=i) l^(i-j) <v_i, dout_j> q_j,
//   R <- l^n R + scale sum_j l^(n-j) q_j dout_j^T.
// A wave owns 16 columns of R, and the same columns of dv and of dk; R^T, which the latter needs, is R rounded in LDS, read transposed.
//
// 212 548 rows, 8/2 heads of 64, four heads to a workgroup: 213 us = 3.1 TB/s (dk and dv as two sweeps of their own 460; in one 325; with a body for each kind
// of rows and the sums held where they are formed, 213).  364 182 rows, 16/2 of 128, two heads: 1780 to 2066 us = 3.1 to 3.6 TB/s, half of it the shares of dk
// and dv (3526 and 2870 on that way).  LDS is the busiest unit, 0.47 of the time; at d = 128 its 115 KB leave one workgroup to a compute unit.
template <int D, int G, int C, bool FULL>
__global__ __launch_bounds__(D * 4, 2) void back_kernel(const Args args) {
    constexpr int NW = D / 16, NT = NW * 64, C16 = D / 8, KS = D / 32, PART = NT / C16, LOADS = C / PART, TILE = C * D * 2, IT = C / 16, KT = C / 32, TILES = IT * (IT + 1) / 2;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    char *k_s = smem, *v_s = k_s + TILE, *q_s = v_s + TILE, *g_s = q_s + TILE, *pq_s = g_s + TILE, *pg_s = pq_s + C * C * 2, *r_s = pg_s + C * C * 2;
    float *dots_q = (float*)(r_s + D * D * 2), *dots_g = dots_q + C, *powers_s = dots_g + C;
    int tid = threadIdx.x, l16 = tid & 15, quad = (tid >> 4) & 3;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    Place place;
    if (!place_of(args, args.spread, place)) return;
    const int u = place.u, kvh = place.kvh, sub = place.member, qh0 = kvh * args.ratio + sub * G;
    const User us = user_of(args, u);
    const Piece piece = piece_of(args, place.piece, us.L, us.T, true);
    const int nt = (piece.t1 - piece.t0 + C - 1) / C, chunks = nt + (piece.h1 - piece.h0 + C - 1) / C;
    if (args.seg && chunks == 0) return;

    State<D> R[G];
#pragma unroll
    for (int g = 0; g < G; g++) {
        if (piece.state >= 0) R[g].load(args.states_back + state_index(args, u, qh0 + g, piece.state) * D * D, false, wave, l16, quad);
        else if (args.state_in) R[g].load(args.state_in + ((int64_t)u * args.Hq + qh0 + g) * D * D, false, wave, l16, quad);
        else R[g].zero();
    }
    const auto rows_of = [&](int c) {
        Rows r;
        r.hist = c >= nt;
        const int first = r.hist ? piece.h0 + (c - nt) * C : piece.t0 + c * C, at = r.hist ? us.L - 1 - first : us.L + first;
        r.n = min(C, (r.hist ? piece.h1 : piece.t1) - first);
        r.kv = us.kv0 + at, r.q = us.q0 + (FULL ? at : first);  // (q of a history's rows: only where they ask)
        return r;
    };
    const unsigned pitch_q = args.Hq * (D * 2), pitch_kv = args.Hkv * (D * 2);
    bf16x8 kw[LOADS], vw[LOADS], qw[LOADS], gw[LOADS];
    const auto fetch_kv = [&](int chunk) {
        const Rows r = rows_of(chunk);
        const int64_t first = (lowest<C>(r.hist, r.kv) * args.Hkv + kvh) * D;
        const char *k = (const char*)(args.k + first), *v = (const char*)(args.v + first);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int row = tid / C16 + i * PART;
            const unsigned at = bytes_of<C>(r.hist, row, pitch_kv, tid % C16 * 16);
            kw[i] = vw[i] = bf16x8{};
            if (row < r.n) kw[i] = *(const bf16x8*)(k + at), vw[i] = *(const bf16x8*)(v + at);
        }
    };
    const auto fetch_q = [&](int chunk, int g) {
        const Rows r = rows_of(chunk);
        const int64_t first = (lowest<C>(r.hist, r.q) * args.Hq + qh0 + g) * D;
        const char *q = (const char*)(args.q + first), *dout = (const char*)(args.dout + first);
        const bool asks = FULL || !r.hist;
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int row = tid / C16 + i * PART;
            const unsigned at = bytes_of<C>(r.hist, row, pitch_q, tid % C16 * 16);
            qw[i] = gw[i] = bf16x8{};
            if (row < r.n && asks) qw[i] = *(const bf16x8*)(q + at), gw[i] = *(const bf16x8*)(dout + at);
        }
    };
    if (chunks > 0) fetch_kv(0), fetch_q(0, 0);
    fill_powers<NT>(powers_s, args.log_decay + qh0, G, args.scale, tid);
    for (int i = tid; i < 2 * C * C / 8; i += NT) lds<bf16x8>(pq_s, i * 16) = bf16x8{};
    Lane<D> at(tid, l16, quad, wave);
    Lane<C> at_p(0, l16, quad, 0);

    floatx4 acc_v[IT], acc_k[IT];
    const auto turn = [&](auto K, int c) {
        constexpr Kind kind = decltype(K)::value;
        constexpr bool hist = kind != CANDIDATES;
        const Rows r = rows_of(c);
#pragma unroll
        for (int g = 0; g < G; g++) {
            const float *power = powers_s + 2 * g * POWERS, *scaled = power + POWERS;
            at.forget(tid, l16, quad);
            at_p.forget(tid, l16, quad);
#pragma unroll
            for (int i = 0; i < LOADS; i++) {
                if (g == 0) {
                    lds<bf16x8>(k_s + i * PART * (D * 2), at.stage) = kw[i];
                    lds<bf16x8>(v_s + i * PART * (D * 2), at.stage) = vw[i];
                }
                if (kind != SILENT) {
                    lds<bf16x8>(q_s + i * PART * (D * 2), at.stage) = qw[i];
                    lds<bf16x8>(g_s + i * PART * (D * 2), at.stage) = gw[i];
                }
            }
            bf16x8 s[KS];
            if (hist) {  // R^T for the other waves: row 16 wave + l16 of it, 32 k + 8 quad .. + 7
                R[g].rounded(s);
#pragma unroll
                for (int k = 0; k < KS; k++) lds<bf16x8>(r_s + wave * (16 * D * 2), at.row ^ (64 * k)) = s[k];
            }
            __syncthreads();
            if (g + 1 < G) fetch_q(c, g + 1);
            else if (c + 1 < chunks) fetch_q(c + 1, 0);
            if (g == G - 1 && c + 1 < chunks) fetch_kv(c + 1);

            if (kind == ASKING) {
#pragma unroll
                for (int t0 = 0; t0 < 2 * TILES; t0 += NW) {
                    const int t = t0 + wave, tt = t >= TILES ? t - TILES : t, it = tile_row(tt), jt = tt - it * (it + 1) / 2;
                    if (t0 + NW <= 2 * TILES || t < 2 * TILES)
                        score_tile<D, C>(t >= TILES ? v_s : k_s, t >= TILES ? g_s : q_s, t >= TILES ? pg_s : pq_s, scaled, at, at_p, it, jt, l16, quad);
                }
            } else if (kind == CANDIDATES) {
                own_dots<D, C, NT>(k_s, q_s, dots_q, args.scale, tid);
                own_dots<D, C, NT>(v_s, g_s, dots_g, args.scale, tid);
            }
            if (kind != SILENT) __syncthreads();
            // dv, then dk: at most one of the two's operands in registers
            const auto rows_of_out = [&](floatx4 (&acc)[IT], const bf16x8 (&ct)[KT], const bf16x8 (&state)[KS], char* p_tile, char* c_tile, char* a_tile, const float* dots) {
                floatx4 x[IT];
                if (kind == ASKING) within_chunk<D, C>(x, ct, p_tile, c_tile, at_p, wave, l16, quad);
#pragma unroll
                for (int it = 0; it < IT; it++) {
                    if (kind == CANDIDATES) x[it] = own_term<D>(dots, c_tile, wave, 16 * it + l16, quad);
                    if (kind == SILENT) x[it] = floatx4{0.f, 0.f, 0.f, 0.f};
                    if (hist) {
                        floatx4 o;
#pragma unroll
                        for (int k = 0; k < KS; k++)
                            o = mfma16(state[k], lds<bf16x8>(a_tile + it * (16 * D * 2), at.row ^ (64 * k)), k == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : o);
                        const float f = power[ZERO + 16 * it + l16];
#pragma unroll
                        for (int v = 0; v < 4; v++) x[it][v] = fmaf(o[v], f, x[it][v]);
                    }
                    acc[it] = g == 0 ? x[it] : acc[it] + x[it];
                    asm volatile("" : "+v"(acc[it]));  // (formed here: left to the compiler, it is formed where it is used next, from operands that stay until then)
                }
            };
            bf16x8 gt[KT];  // this wave's columns of dout, rows 32 k + 8 quad .. + 7
            if (kind != SILENT)
#pragma unroll
                for (int k = 0; k < KT; k++) gt[k] = read_tr<D>(g_s + 32 * k * (D * 2), at.tr);
            rows_of_out(acc_v, gt, s, pq_s, g_s, k_s, dots_q);
            __builtin_amdgcn_sched_barrier(0);
            {
                bf16x8 qt[KT], st[KS];  // this wave's columns of q; its rows of R^T
                if (kind != SILENT)
#pragma unroll
                    for (int k = 0; k < KT; k++) qt[k] = read_tr<D>(q_s + 32 * k * (D * 2), at.tr);
                if (hist)
#pragma unroll
                    for (int k = 0; k < KS; k++) st[k] = read_tr<D>(r_s + 32 * k * (D * 2), at.tr);
                rows_of_out(acc_k, qt, st, pg_s, q_s, v_s, dots_g);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (g == G - 1) {
                const int64_t base = (lowest<C>(hist, r.kv) * args.Hkv + kvh) * D, slab = (int64_t)sub * args.total_kv * args.Hkv * D;
#pragma unroll
                for (int it = 0; it < IT; it++) {
                    const int i = 16 * it + l16;
                    if (i >= r.n) continue;
                    const unsigned to = bytes_of<C>(hist, i, pitch_kv, 32 * wave + 8 * quad);
                    if (args.partial_k) {
                        *(floatx4*)((char*)(args.partial_v + slab + base) + 2 * to) = acc_v[it];
                        *(floatx4*)((char*)(args.partial_k + slab + base) + 2 * to) = acc_k[it];
                    } else {
                        bf16x4 x, y;
#pragma unroll
                        for (int v = 0; v < 4; v++) x[v] = (__bf16)acc_v[it][v], y[v] = (__bf16)acc_k[it][v];
                        *(bf16x4*)((char*)(args.dv + base) + to) = x;
                        *(bf16x4*)((char*)(args.dk + base) + to) = y;
                    }
                }
            }
            if (hist) R[g].keep(power[ZERO + r.n]);
            if (kind != SILENT) R[g].add(q_s, gt, scaled + ZERO + (hist ? r.n : 1), std::integral_constant<int, hist ? 1 : 0>{}, at, quad, args.state_out != nullptr);
            __syncthreads();
        }
    };
    int c = 0;
    for (; c < nt; c++) turn(KindOf<CANDIDATES>{}, c);
    for (; c < chunks; c++) turn(KindOf<FULL ? ASKING : SILENT>{}, c);
    if (args.state_out && !args.seg)
#pragma unroll
        for (int g = 0; g < G; g++) R[g].store(args.state_out + ((int64_t)u * args.Hq + qh0 + g) * D * D, wave, l16, quad);
}
template <int D, int G, int C>
constexpr int back_lds() { return 4 * C * D * 2 + 2 * C * C * 2 + D * D * 2 + (2 * C + 2 * G * POWERS) * 4; }

// What each piece adds to a state that starts at zero: forwards sum_j l^(n-1-j) b_j c_j^T over a history's piece, backwards scale times sum_j l^(n-j) q_j dout_j^T
// over either kind (candidates: l).  blockIdx.y: 1 backwards.  A chain of chunks, bound by its latency: one user of 8192 rows, 16/2 heads of 128, pieces of 256
// rows, 24.7 us; 8 users of up to 4096, 8/2 of 64, 12.1 (in chunks of 32 rows 13.3; at d = 128 chunks of 64 do not fit the registers).
template <int D, int C>
__global__ __launch_bounds__(D * 4, 4) void states_kernel(const Args args, int first_job, int whole_jobs) {
    constexpr int NW = D / 16, NT = NW * 64, C16 = D / 8, PART = NT / C16, LOADS = C / PART, TILE = C * D * 2, KT = C / 32;
    __shared__ __attribute__((aligned(16))) char b_s[TILE], c_s[TILE];
    __shared__ float powers_s[2 * POWERS];
    int tid = threadIdx.x, l16 = tid & 15, quad = (tid >> 4) & 3;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool back = (int)blockIdx.y + first_job == 1, whole = whole_jobs & (back ? 2 : 1);

    Place place;
    if (!place_of(args, args.ratio, place)) return;
    const int u = place.u, kvh = place.kvh, qh = kvh * args.ratio + place.member;
    const User us = user_of(args, u);
    const Piece piece = piece_of(args, place.piece, us.L, us.T, back);
    const bool hist = piece.h1 > piece.h0;
    const int from = hist ? piece.h0 : piece.t0, rows = hist ? piece.h1 - piece.h0 : piece.t1 - piece.t0, chunks = (rows + C - 1) / C;
    if (chunks == 0 || (back ? hist && !args.full : !hist)) return;

    const int heads = back ? args.Hq : args.Hkv, head = back ? qh : kvh;
    const unsigned pitch = heads * (D * 2);
    const __bf16 *bg = back ? args.q : args.b, *cg = back ? args.dout : args.c;
    bf16x8 bv[LOADS], cv[LOADS];
    const bool down = back && hist;
    const auto fetch = [&](int c) {
        const int at0 = from + c * C, n = min(C, rows - c * C);
        const int64_t row0 = !back ? us.kv0 + at0 : us.q0 + (hist ? us.L - 1 - at0 : (args.full ? us.L : 0) + at0), first = (lowest<C>(down, row0) * heads + head) * D;
        const char *b = (const char*)(bg + first), *x = (const char*)(cg + first);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int row = tid / C16 + i * PART;
            const unsigned at = bytes_of<C>(down, row, pitch, tid % C16 * 16);
            bv[i] = cv[i] = bf16x8{};
            if (row < n) bv[i] = *(const bf16x8*)(b + at), cv[i] = *(const bf16x8*)(x + at);
        }
    };
    fetch(0);
    fill_powers<NT>(powers_s, args.log_decay + qh, 1, args.scale, tid);
    const float *power = powers_s, *scaled = powers_s + POWERS;
    Lane<D> at(tid, l16, quad, wave);
    State<D> S;
    S.zero();
    for (int c = 0; c < chunks; c++) {
        const int n = min(C, rows - c * C);
        at.forget(tid, l16, quad);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            lds<bf16x8>(b_s + i * PART * (D * 2), at.stage) = bv[i];
            lds<bf16x8>(c_s + i * PART * (D * 2), at.stage) = cv[i];
        }
        __syncthreads();
        if (c + 1 < chunks) fetch(c + 1);
        bf16x8 ct[KT];
#pragma unroll
        for (int k = 0; k < KT; k++) ct[k] = read_tr<D>(c_s + 32 * k * (D * 2), at.tr);
        if (hist) S.keep(power[ZERO + n]);
        if (hist) S.add(b_s, ct, back ? scaled + ZERO + n : power + ZERO + n - 1, std::integral_constant<int, 1>{}, at, quad, whole);
        else S.add(b_s, ct, scaled + ZERO + 1, std::integral_constant<int, 0>{}, at, quad, whole);
        __syncthreads();
    }
    S.store((back ? args.states_back : args.states) + state_index(args, u, qh, piece.state) * D * D, wave, l16, quad);
}

// The states in front of the pieces from what each adds, in the order of the sweep: X <- l^n X + U, in place; the last is the caller's.  blockIdx.z: 1 backwards.
// Bound by its traffic where states are many (16 heads x 33 states of 128 x 128: 69 MB in 13.3 us = 5.2 TB/s), by a trip to memory where they are few (4 us).
constexpr int SCAN_THREADS = 256, SCAN_AHEAD = 16;  // loads in flight: the sum is all latency
template <int D>
__global__ __launch_bounds__(SCAN_THREADS) void scan_kernel(const Args args, int first_job, const float* in_ahead, int transposed, float* out_ahead, const float* in_back,
                                                            float* out_back) {
    const bool back = (int)blockIdx.z + first_job == 1;
    const int u = blockIdx.x / args.Hq, h = blockIdx.x % args.Hq, e = (blockIdx.y * SCAN_THREADS + threadIdx.x) * 4;
    const User us = user_of(args, u);
    const int rows = args.seg, hs = (us.L + rows - 1) / rows, ts = back ? (us.T + rows - 1) / rows : 0, n = hs + ts;
    const float g2 = fmaxf(fminf(args.log_decay[h], 0.f) * hta::LOG2E, MIN_LOG2), all = fast_exp2(g2 * (float)rows);
    const float last = fast_exp2(g2 * (float)(us.L - (hs - 1) * rows));
    const int64_t state = ((int64_t)u * args.Hq + h) * D * D;
    const float* in = back ? in_back : in_ahead;
    float* out = back ? out_back : out_ahead;
    float* p = (back ? args.states_back : args.states) + state_index(args, u, h, 0) * D * D + e;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
    if (in) {
        if (!back && transposed)
#pragma unroll
            for (int v = 0; v < 4; v++) x[v] = in[state + ((e + v) % D) * D + (e + v) / D];
        else x = *(const floatx4*)(in + state + e);
    }
    const bool adds = args.full || !back;  // (backwards through a history that does not ask nothing is added)
    const bool all_wanted = args.full || back;  // (forwards over a history that does not ask: the last alone)
    constexpr int AHEAD = SCAN_AHEAD;
    for (int s = 0; s < n; s += AHEAD) {
        floatx4 y[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; i++) y[i] = s + i < n && (adds || s + i < ts) ? *(const floatx4*)(p + (int64_t)(s + i) * D * D) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
            if (s + i >= n) break;
            const float f = s + i < ts ? 1.f : s + i == n - 1 ? last : all;
            if (all_wanted) *(floatx4*)(p + (int64_t)(s + i) * D * D) = x;
            x = x * f + y[i];
        }
    }
    *(floatx4*)(p + (int64_t)n * D * D) = x;
    if (out) *(floatx4*)(out + state + e) = x;
}

// dk, dv = the sum of a group's shares, for the rows of the users.  Bound by HBM: 364 182 rows, 2 heads of 128, 4 shares: 720 to 765 us = 4.4 to 4.7 TB/s.
constexpr int SUM_THREADS = 256, SUM_BLOCKS = 64;  // (per user)
__global__ __launch_bounds__(SUM_THREADS) void sum_kernel(const Args args, int d) {
    const User us = user_of(args, blockIdx.x);
    const float* partial = blockIdx.z ? args.partial_k : args.partial_v;
    __bf16* out = blockIdx.z ? args.dk : args.dv;
    const int64_t row = (int64_t)args.Hkv * d, slab = args.total_kv * row, first = us.kv0 * row, n = (int64_t)(us.L + us.T) * row;
    for (int64_t e = ((int64_t)blockIdx.y * SUM_THREADS + threadIdx.x) * 4; e < n; e += (int64_t)SUM_BLOCKS * SUM_THREADS * 4) {
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < args.spread; s += 4) {
            floatx4 y[4];
#pragma unroll
            for (int i = 0; i < 4; i++) y[i] = s + i < args.spread ? __builtin_nontemporal_load((const floatx4*)(partial + (s + i) * slab + first + e)) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; i++) x += y[i];
        }
        bf16x4 o;
#pragma unroll
        for (int j = 0; j < 4; j++) o[j] = (__bf16)x[j];
        *(bf16x4*)(out + first + e) = o;
    }
}

// Single tokens: a workgroup per row and query head, the state in registers between its reading and its writing.  Lane groups of D / 4 lanes
// hold a state row each (16-byte words), so thread t has columns 4 (t % (D / 4)) .. of rows t / (D / 4) + i ROWS.  Bound by HBM: the state in and out
// (96 rows, 16/2 heads of 128: 201 MB in 30.2 to 37.2 us, 5.4 TB/s or more; one row, 8/2 of 64: 3.3 us, the launch and two trips to memory).
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

constexpr int64_t MOST_TOKENS = (int64_t)1 << 30;  // (the last piece or chunk may end behind them, in 32 bits)
// A launch has less than 2^32 threads: 4 head_dim to a workgroup, or 256 of the scan; up to 8 groups of heads (2^22 features) may be none.
bool launchable(int64_t workgroups, int d) { return workgroups * std::max(4 * d, 256) < ((int64_t)1 << 32) - ((int64_t)1 << 27); }

int check_sizes(int layer, int dtype, int32_t batch, int64_t total_q, int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t d) {
    if (int rc = check_heads(Hq, Hkv, d, dtype)) return rc;
    if (layer != MTFM_HTA_LAYER_FULL && layer != MTFM_HTA_LAYER_TARGET) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "unknown layer kind %d", layer);
    if (batch < 0 || total_q < 0 || total_kv < 0 || max_hist < 0 || max_targets < 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "negative size");
    if (total_q > MOST_TOKENS || total_kv > MOST_TOKENS) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "more than 2^30 rows");
    if (!launchable((int64_t)batch * Hq, d)) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "batch (%d) x Hq (%d) x head_dim (%d) are too many for a launch", batch, Hq, d);
    return MTFM_HTA_OK;
}

constexpr int MIN_SEG = 128;  // rows of a piece at least; a multiple of what a chunk has
// Rows of a chunk: 64, and 32 where LDS for 64 keeps workgroups off a compute unit that registers would let in.  (us, 64 / 32: forward and backward of 54 users of
// 1090 rows, 4/2 heads of 32, 117 / 103, of 192 of 197 70.4 / 64.0; backward of 239 users of up to 304, 4/4 of 64, 81.1 / 65.9, of 42 of 1016 97 / 103;
// forward of 364 182 rows, 16/2 of 128, 1073 / 1032; at d = 64 the forward pass takes the same, and with four heads to a backward workgroup, or at d = 128, 32
// rows take 1.07 of the time.)
constexpr int sweep_rows(int D, bool FULL) { return D != 64 && FULL ? 32 : 64; }
constexpr int back_rows(int D, int G, bool FULL) { return D == 32 || (D == 64 && G <= 2 && FULL) ? 32 : 64; }
constexpr int states_rows(int D) { return D == 128 ? 32 : 64; }

// heads of a group that a backward workgroup may hold: what registers allow
int most_heads(int d, bool full) { return d == 128 && full ? 2 : 4; }

struct Plan {
    int G, spread;      // backwards: heads of a group to a workgroup, workgroups to a group
    size_t partial;     // bytes of dk's (dv's) shares, 0 for none
    int seg, n_hist, n_tgt;
    size_t states;      // bytes of the pieces' states, one direction
    size_t order;       // bytes of the users' order, 0: as they come
    size_t bytes(bool backward) const { return order + 2 * partial + (backward ? 2 : 1) * states; }
};
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

Plan plan_of(bool backward, bool full, int batch, int64_t total_kv, int max_hist, int max_targets, int Hq, int Hkv, int d) {
    Plan p = {};
    max_hist = (int)std::min((int64_t)max_hist, total_kv), max_targets = (int)std::min((int64_t)max_targets, total_kv);
    // How a call is cut up goes by the time of each way, in us.  A user's head is one workgroup's work, so a sweep lasts as long as the longest history takes by
    // itself, at least; cut into pieces, whose states take another reading of half a sweep's work and two launches, it lasts as long as the chip needs for all
    // rows, in whole pieces to a compute unit (0.85: a user's last one is not whole).  The heads of a group that a backward workgroup does not hold are
    // summed by a launch of its own, over shares that are written and read.  `mean`: rows of a place on a full chip; us of a row there, and of a row of a workgroup that is alone on its compute unit, in a sweep
    // and (of a head) in the sweep for dk and dv: as measured.  (Forward, us, by rows of a piece none / 128 / 256 / 512: one user of 8192, 16/2 heads of 128,
    // 462 / 91 / 77 / 94; 18 users of 360 to 5080, 8/2 of 64, 157 / 62 / 51 / 58; 19 of 438 to 1752 with states, forward and backward, 256 206, 128 150; 256 of
    // 512 to 1024 164 / 357 / 285.  Over 90 calls the choice takes 1.01 of the best one's time; 39 users of 543 to 2424, 8/2 of 64, in pieces of 1024 took 1.8 of that in 256.)
    const int places = 256 * (d == 128 ? 2 : 4), ratio = Hq / Hkv;
    const int64_t whole = (int64_t)batch * Hq;
    const double mean = (double)total_kv * Hq / places;
    const double full_row = full ? (d == 128 ? 0.117 : 0.094) : (d == 128 ? 0.052 : 0.035), lone_row = full ? (d == 128 ? 0.06 : 0.036) : (d == 128 ? 0.035 : 0.016);
    const double full_back = d == 128 ? 0.22 : 0.13, lone_back = full ? (d == 128 ? 0.08 : 0.05) : (d == 128 ? 0.05 : 0.03), start = 6;
    const auto sweep = [&](double rows_of_place, double rows) { return std::max(rows_of_place * full_row, rows * lone_row) + start; };
    double best = 0;
    // pieces of 128 rows, of twice as many and so on; 0: none
    for (int seg = 0; seg <= max_hist / 2; seg = seg ? 2 * seg : MIN_SEG) {
        if (seg && !launchable(whole * (ceil_div(max_hist, seg) + ceil_div(max_targets, seg)), d)) continue;
        const int pieces = seg ? ceil_div(max_hist, seg) : 0;
        const double rows = seg ? seg : max_hist, of_place = seg ? 0.85 * std::ceil(((double)total_kv / seg + batch) * Hq / 256) * 256 * seg / places : mean;
        // (a history that does not ask is nothing but its states, written and read once; the others are written, summed, sixteen in flight, and read)
        const double traffic = seg ? (double)whole * (pieces + 2) * d * d * 8 / 4.9e6 : 0;
        const double states = seg ? (full ? 0.5 : 1.0) * sweep(of_place, rows) + start + 2 * ((pieces - 1) / SCAN_AHEAD) + (full ? 1.0 : 0.5) * traffic : 0;
        const double ahead = (full || !seg ? sweep(of_place, rows + max_targets) : start) + states;
        for (int G = most_heads(d, full); G >= 1; G /= 2) {
            if (ratio % G != 0 || (!backward && G > 1)) continue;
            double time = ahead;
            if (backward) {
                time += std::max((seg ? 1.3 : 1.0) * mean * full_back, (rows + max_targets) * G * lone_back) + start + (full ? states : traffic);
                if (ratio > G) time += start + (double)total_kv * Hq / G * d * 16 / 4.9e6;
            }
            if (best != 0 && time >= best) continue;
            best = time;
            p.G = G, p.seg = seg, p.n_hist = pieces, p.n_tgt = seg ? ceil_div(max_targets, seg) : 0;
        }
    }
    p.spread = ratio / p.G;
    p.partial = backward && p.spread > 1 ? align256((size_t)p.spread * total_kv * Hkv * d * sizeof(float)) : 0;
    if (p.seg) p.states = align256((size_t)whole * (p.n_hist + p.n_tgt + 1) * d * d * sizeof(float));
    // Long users first, where lengths differ and there are more of them than places: the last ones to start are short.  (A launch of 4 us.)
    const bool even = (double)total_kv >= 0.9 * (double)batch * ((double)max_hist + max_targets);
    if (!p.seg && !even && 2 * whole > places && max_hist > 2 * MIN_SEG) p.order = align256(hta::schedule_bytes(batch));
    return p;
}

// the head of the workspace: the users' order
hipError_t launch_order(Args& a, const Plan& plan, void* workspace, hipStream_t s) {
    if (!plan.order) return hipSuccess;
    hta::Params p = {};
    p.hist_len = a.hist_len, p.n_targets = a.n_targets, p.batch = a.batch, p.max_hist = a.max_hist, p.max_targets = a.max_targets;
    a.order = hta::schedule_order(workspace);
    return hta::launch_schedule(p, workspace, s);
}

int64_t grid_of(const Args& a, int members) {
    const int64_t units = (int64_t)a.batch * a.Hkv * (a.seg ? a.n_hist + a.n_tgt : 1);
    return (units + hta::N_XCD - 1) / hta::N_XCD * hta::N_XCD * members;
}

template <int D>
hipError_t launch_sweep_d(const Args& a, hipStream_t s) {
    const dim3 grid((unsigned)grid_of(a, a.ratio));
    if (a.full) hipLaunchKernelGGL((sweep_kernel<D, sweep_rows(D, true), true>), grid, dim3(D * 4), 0, s, a);
    else hipLaunchKernelGGL((sweep_kernel<D, sweep_rows(D, false), false>), grid, dim3(D * 4), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_sweep(const Args& a, int d, hipStream_t s) {
    return d == 32 ? launch_sweep_d<32>(a, s) : d == 64 ? launch_sweep_d<64>(a, s) : launch_sweep_d<128>(a, s);
}

// first_job, jobs: 0, 1 the sweep in the tokens' order; 1, 1 backwards; 0, 2 both
template <int D>
hipError_t launch_states_d(const Args& a, int first_job, int jobs, const float* in_ahead, float* out_ahead, const float* in_back, float* out_back, hipStream_t s) {
    hipLaunchKernelGGL((states_kernel<D, states_rows(D)>), dim3((unsigned)grid_of(a, a.ratio), jobs), dim3(D * 4), 0, s, a, first_job, (out_ahead ? 1 : 0) | (out_back ? 2 : 0));
    hipLaunchKernelGGL((scan_kernel<D>), dim3(a.batch * a.Hq, D * D / (SCAN_THREADS * 4), jobs), dim3(SCAN_THREADS), 0, s, a, first_job, in_ahead, a.transposed,
                       out_ahead, in_back, out_back);
    return hipGetLastError();
}
hipError_t launch_states(const Args& a, int d, int first_job, int jobs, const float* in_ahead, float* out_ahead, const float* in_back, float* out_back, hipStream_t s) {
    const auto launch = d == 32 ? launch_states_d<32> : d == 64 ? launch_states_d<64> : launch_states_d<128>;
    hta::timing_begin(MTFM_HLA_KERNEL_STATES, s);
    const hipError_t e = launch(a, first_job, jobs, in_ahead, out_ahead, in_back, out_back, s);
    hta::timing_end(MTFM_HLA_KERNEL_STATES, s);
    return e;
}

// Lets a kernel use its dynamic LDS; asked for once per kernel and device, not a stream operation (a graph that is being captured does not see it).
template <auto Kernel>
hipError_t allow_lds(int bytes) {
    constexpr int MAX_DEVICES = 64;
    static std::atomic<bool> allowed[MAX_DEVICES];
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    const bool known = dev >= 0 && dev < MAX_DEVICES;
    if (known && allowed[dev].load(std::memory_order_relaxed)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute((const void*)Kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (known && e == hipSuccess) allowed[dev].store(true, std::memory_order_relaxed);
    return e;
}
template <int D, int G, bool FULL>
hipError_t launch_back_as(const Args& a, hipStream_t s) {
    constexpr int C = back_rows(D, G, FULL), lds = back_lds<D, G, C>();
    if (hipError_t e = allow_lds<back_kernel<D, G, C, FULL>>(lds); e != hipSuccess) return e;
    hipLaunchKernelGGL((back_kernel<D, G, C, FULL>), dim3((unsigned)grid_of(a, a.spread)), dim3(D * 4), lds, s, a);
    return hipGetLastError();
}
template <int D, bool FULL>
hipError_t launch_back_layer(const Args& a, int G, hipStream_t s) {
    if (G == 1) return launch_back_as<D, 1, FULL>(a, s);
    if constexpr (D < 128 || !FULL)
        if (G == 4) return launch_back_as<D, 4, FULL>(a, s);
    return launch_back_as<D, 2, FULL>(a, s);
}
template <int D>
hipError_t launch_back_d(const Args& a, int G, hipStream_t s) { return a.full ? launch_back_layer<D, true>(a, G, s) : launch_back_layer<D, false>(a, G, s); }
hipError_t launch_back(const Args& a, int d, int G, hipStream_t s) {
    return d == 32 ? launch_back_d<32>(a, G, s) : d == 64 ? launch_back_d<64>(a, G, s) : launch_back_d<128>(a, G, s);
}

Args args_of(const float* log_decay, const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len, const int32_t* n_targets, int32_t batch,
             int64_t total_q, int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, float scale, int layer) {
    Args a = {};
    a.log_decay = log_decay, a.q_off = q_offsets, a.kv_off = kv_offsets, a.hist_len = hist_len, a.n_targets = n_targets;
    a.total_q = total_q, a.total_kv = total_kv, a.batch = batch, a.Hq = Hq, a.Hkv = Hkv, a.ratio = Hq / Hkv, a.spread = 1;
    a.full = layer == MTFM_HTA_LAYER_FULL, a.max_hist = max_hist, a.max_targets = max_targets, a.scale = scale;
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
    if (batch == 0) return 0;
    const hla::Plan plan = hla::plan_of(is_bwd, layer == MTFM_HTA_LAYER_FULL, batch, total_kv, max_hist, max_targets, Hq, Hkv, head_dim);
    return plan.bytes(is_bwd);
}

int mtfm_hla_fwd(const void* q, const void* k, const void* v, const float* log_decay, const float* state, void* out, float* final_state,
                 const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len, const int32_t* n_targets, int32_t batch, int64_t total_q,
                 int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t head_dim, float scale, int dtype, int layer,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = hla::check_sizes(layer, dtype, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, head_dim)) return rc;
    if (batch == 0) return MTFM_HTA_OK;
    if (int rc = hla::check_arrays({q, out}, {k, v}, {state, final_state}, log_decay, {q_offsets, kv_offsets, hist_len, n_targets}, total_q, total_kv, scale)) return rc;
    const hla::Plan plan = hla::plan_of(false, layer == MTFM_HTA_LAYER_FULL, batch, total_kv, max_hist, max_targets, Hq, Hkv, head_dim);
    if (int rc = hla::check_workspace(plan.bytes(false), workspace, workspace_bytes)) return rc;
    hla::Args a = hla::args_of(log_decay, q_offsets, kv_offsets, hist_len, n_targets, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, scale, layer);
    a.seg = plan.seg, a.n_hist = plan.n_hist, a.n_tgt = plan.n_tgt, a.states = (float*)((char*)workspace + plan.order);
    a.a = (const __bf16*)q, a.b = (const __bf16*)k, a.c = (const __bf16*)v, a.out = (__bf16*)out, a.state_in = state, a.state_out = final_state;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = hla::launch_order(a, plan, workspace, s);
    if (e == hipSuccess && plan.seg) e = hla::launch_states(a, head_dim, 0, 1, state, final_state, nullptr, nullptr, s);
    if (e == hipSuccess && (total_q > 0 || !plan.seg)) {
        hta::timing_begin(MTFM_HLA_KERNEL_FWD, s);
        e = hla::launch_sweep(a, head_dim, s);
        hta::timing_end(MTFM_HLA_KERNEL_FWD, s);
    }
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
    const hla::Plan plan = hla::plan_of(true, layer == MTFM_HTA_LAYER_FULL, batch, total_kv, max_hist, max_targets, Hq, Hkv, head_dim);
    if (int rc = hla::check_workspace(plan.bytes(true), workspace, workspace_bytes)) return rc;
    hla::Args a = hla::args_of(log_decay, q_offsets, kv_offsets, hist_len, n_targets, batch, total_q, total_kv, max_hist, max_targets, Hq, Hkv, scale, layer);
    hipStream_t s = (hipStream_t)stream;
    const auto Q = (const __bf16*)q, K = (const __bf16*)k, V = (const __bf16*)v, dO = (const __bf16*)dout;
    hipError_t e = hla::launch_order(a, plan, workspace, s);
    a.q = Q, a.k = K, a.v = V, a.dout = dO, a.dk = (__bf16*)dk, a.dv = (__bf16*)dv, a.b = V, a.c = K, a.transposed = 1;
    a.seg = plan.seg, a.n_hist = plan.n_hist, a.n_tgt = plan.n_tgt;
    a.states = (float*)((char*)workspace + plan.order + 2 * plan.partial), a.states_back = a.states + plan.states / sizeof(float);
    if (e == hipSuccess && plan.seg) e = hla::launch_states(a, head_dim, total_q > 0 ? 0 : 1, total_q > 0 ? 2 : 1, state, nullptr, dfinal_state, dstate, s);
    hta::timing_begin(MTFM_HLA_KERNEL_BWD, s);
    if (e == hipSuccess && total_q > 0) {
        a.a = dO, a.out = (__bf16*)dq, a.state_in = state;
        e = hla::launch_sweep(a, head_dim, s);
    }
    if (e == hipSuccess) {
        a.state_in = dfinal_state, a.state_out = dstate, a.spread = plan.spread;
        if (plan.spread > 1) a.partial_k = (float*)((char*)workspace + plan.order), a.partial_v = a.partial_k + plan.partial / sizeof(float);
        e = hla::launch_back(a, head_dim, plan.G, s);
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
    if (!hla::launchable((int64_t)n_rows * Hq, 32)) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "n_rows (%d) x Hq (%d) are too many for a launch", n_rows, Hq);
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

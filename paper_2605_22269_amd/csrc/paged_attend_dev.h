// Attention of new tokens over the rows of a paged cache (or of packed sequences), for any number of tokens a sequence, any payload type
// and head size.
//
//   out[token][h] = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s_j - m),  s_j = log2(e) / sqrt(D) q.k_j,  m = max_j s_j
//
// over the rows j of the token's sequence that it sees.  One pass over the rows with the running maximum and sum; rows shared by
// chunks of a sequence are joined by the last of its workgroups to finish.
#pragma once

#include <climits>
#include <type_traits>

#include "eight_dev.h"
#include "paged_dev.h"

namespace mukv {

namespace {

constexpr int kPWaves = 4; // of a workgroup, which has kPQ queries

// Keys of 8 bits as the rows of a score: a lane of four has D / 4 neighbouring codes (or two such runs of 16), which are one operand after
// the other.
template <typename T, int D>
struct KeyCodes {
    static constexpr int E = 16 / (int)sizeof(T), KK = sizeof(T) == 2 ? (D + 31) / 32 : D / 16; // features of an operand, operands
    static constexpr int kRun = KK * E < 16 ? KK * E : 16, kRuns = KK * E / kRun;               // bytes
    // the 16-byte piece of a query that operand kk of lane `of_four` belongs to
    __device__ static __forceinline__ int piece_of(int of_four, int kk) {
        return (kRun * (of_four + 4 * (kk * E / kRun)) + kk * E % kRun) / E;
    }
    struct Codes {
        uint32_t w[KK * E / 4];
        __device__ __forceinline__ void load(const unsigned char *row, int of_four) {
            typedef __attribute__((ext_vector_type(kRun / 4))) unsigned int raw_c;
#pragma unroll
            for (int j = 0; j < kRuns; ++j) {
                const raw_c x = *reinterpret_cast<const raw_c *>(row + kRun * (of_four + 4 * j));
#pragma unroll
                for (int i = 0; i < kRun / 4; ++i) w[j * (kRun / 4) + i] = x[i];
            }
        }
        __device__ __forceinline__ void spread(float scale, raw16 (&k)[KK]) const {
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if constexpr (E == 8)
                    k[kk] = bf16_piece(w[2 * kk], w[2 * kk + 1], scale);
                else
                    k[kk] = f32_piece(w[kk], scale);
            }
        }
    };
};

// Scores of 16 fp32 rows, k, and 16 queries, q(piece): sums of four terms each, joined pair by pair, which is nearer to 64 bits than
// one sum of D terms.  Two pieces at a time: the compiler starts all 4 KK products at once otherwise, in as many registers, and puts
// requested rows aside as they come (22 prompts of 700 to 1500 tokens, 16/4 heads of 128: 6140 us so, 1776 in pairs, 60 TFLOP/s).
template <int KK, typename Q>
__device__ __forceinline__ f32x4 scores_f32(const raw16 (&k)[KK], Q q) {
    f32x4 part[4]; // of 1, 2, 4 and 8 pieces
    f32x4 x;
#pragma unroll
    for (int k0 = 0; k0 < KK; k0 += 2) {
        raw16 y[2] = {k[k0], k[k0 + 1 < KK ? k0 + 1 : k0]};
        if (k0 > 0) asm volatile("" : "+v"(x), "+v"(y[0]), "+v"(y[1]));
#pragma unroll
        for (int kk = k0; kk < k0 + 2 && kk < KK; ++kk) {
            f32x4 c[4];
            const raw16 z = q(kk);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                c[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(y[kk - k0][e]), __uint_as_float(z[e]), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            x = (c[0] + c[1]) + (c[2] + c[3]);
            int level = 0;
#pragma unroll
            for (int n = kk; n & 1; n >>= 1) x = part[level++] + x;
            part[level] = x;
        }
    }
    return x;
}

// Eight fp32 numbers as three bf16 each, which add up to it: 8 of its 24 bits after the other, cut off, so that nothing can overflow.
// (An infinity is the first part; NaN stays NaN in one of them.)
__device__ __forceinline__ void three_parts(const raw16 (&x)[2], raw16 (&part)[3]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t a = x[e / 2][2 * e % 4], b = x[e / 2][2 * e % 4 + 1];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            part[j][e] = a >> 16 | (b & 0xFFFF0000u);
            auto rest = [](uint32_t y) {
                const float f = __uint_as_float(y);
                return fabsf(f) == INFINITY ? 0u : __float_as_uint(f - __uint_as_float(y & 0xFFFF0000u));
            };
            a = rest(a);
            b = rest(b);
        }
    }
}

// Scores of 16 bf16 rows and 16 queries in three parts: sums of 32 terms of each part, the least first, joined pair by pair.
template <int KK>
__device__ __forceinline__ f32x4 scores_of_parts(const raw16 (&k)[KK], const raw16 (&part)[KK][3]) {
    f32x4 c[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        c[kk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 2; j >= 0; --j)
            c[kk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[kk]), __builtin_bit_cast(bf16x8, part[kk][j]), c[kk], 0, 0, 0);
    }
    if constexpr (KK == 4) return (c[0] + c[1]) + (c[2] + c[3]);
    if constexpr (KK == 2) return c[0] + c[1];
    return c[0];
}

// The rows of a tile, in blocks of 32 (bf16, EIGHT) or 16 (fp32), dealt to the waves in turn; nothing crosses the waves until the end.
//   rows     a lane works out where one row lives, from a table entry that was requested a block earlier; the others fetch that by
//            lane permutes.  Keys and values go straight to registers, the next block's requested as soon as this one's are used up.
//   scores   S^T = K Q^T (16x16x32 bf16, 16x16x4 fp32): a lane holds ONE query (lane % 16) and the rows 4 (lane / 16) + r of every 16.
//   values   O^T += V^T P^T: the weights are the B operand as they stand in the lane.  bf16: pairs hi + lo, 16 of the fp32
//            weight's 24 bits; the value rows pass through LDS the wave has to itself and the transpose read.  fp32: no transpose needed.
// EIGHT: rows of 8 bits (eight_dev.h) become bf16 as they are used, which changes no bit of them: keys in registers, where a
// lane's codes are neighbours, so an operand's features are others than without (the queries' are, too); values on their way to LDS.
// fp32 payloads go the same way: queries and weights are three bf16 each, all 24 bits, whose products with a row are exact and are
// added in fp32.  Three matrix instructions so take the place of eight that are twice as long (us a call: 64 users over 200 to 12000
// rows, 64/8 heads of 128, 236, in fp32 522; 12 users, 5 tokens, 28/4 heads of 64, 42 for 90; prompts of 700 to 1500 tokens 698 for 1632).
// As many workgroups to a compute unit as the registers allow (us a launch, two / as now: 100 users of 3 rows, 12 heads of 64 bf16, 13.7 / 10.2;
// 12 users, 5 tokens over 1000 to 9000 rows, 28/4 heads of 64 bf16, 26.5 / 22.3; 6 prompts of 700 to 1500 tokens, 28/4 heads of 32 bf16, 148 / 94;
// of fp32 252 / 218; 1500 tokens, 16/4 heads of 64 fp32, 103 / 92).
// SHARED: one of a call's two launches, over rows that groups of sequences share and over the sequences' own (SharedResults).
template <typename T, int D, bool EIGHT, bool SHARED>
__global__ __launch_bounds__(64 * kPWaves) __attribute__((amdgpu_waves_per_eu(D <= 32 ? 4 : D == 64 ? 3 : 2, D <= 32 ? 5 : D == 64 ? 3 : 2))) void paged_attend_kernel(PagedAttendArgs a) {
    constexpr int W = kPWaves;
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr bool kNarrow = kBf16 || EIGHT; // rows are multiplied as bf16, queries and weights perhaps in parts
    constexpr int kQParts = kBf16 ? 1 : 3, kWParts = kBf16 ? 2 : 3;
    constexpr int kRowB = D * (kNarrow ? 2 : 4), kPieces = kRowB / 16;
    constexpr int kRows = kNarrow ? 32 : 16;             // rows of a block
    constexpr int kTiles = kRows / 16;                 // 16-row tiles of the scores
    constexpr int KK = kNarrow ? (D + 31) / 32 : D / 16; // 16-byte pieces of a key row (and of a query) per lane
    constexpr int NF = D / 16;                         // 16-feature tiles of the output
    // bf16: value pieces per lane, each load of the wave kRowsPerLoad whole rows.  fp32: per 4-row step D / 16 floats.  (EIGHT, bf16: a
    // load is two pieces, where a row has more than two)
    constexpr int kVH = kNarrow ? (EIGHT && D > 16 ? 2 : 1) : (D == 128 ? 2 : 1); // pieces, or loads, per row
    constexpr int kRowsPerLoad = 64 * (kNarrow ? kVH : 1) / kPieces, NV = kNarrow ? kRows / kRowsPerLoad : 4;
    constexpr int kVW = kNarrow ? 4 : (D >= 64 ? 4 : D / 16); // dwords of a piece
    constexpr int kValueLanes = kNarrow ? kPieces / kVH : 16; // of a row
    typedef __attribute__((ext_vector_type(kVW))) unsigned int raw_v;
    using Keys = KeyCodes<std::conditional_t<kNarrow, uint16_t, T>, D>;
    // words of codes of a load of values
    constexpr int kVC = kNarrow ? 2 * kVH : kVH;
    // per wave: staged value rows (bf16), at the end its outputs [16 queries][D]
    __shared__ __align__(1024) unsigned char s_buf[W][64 * D];
    __shared__ float s_m[W][kPQ], s_l[W][kPQ];
    constexpr bool kQueryLds = !kBf16 && D == 128; // fp32, 128 features: the queries' operands wait in LDS
    __shared__ raw16 s_q[!kQueryLds ? 1 : EIGHT ? KK * kQParts : KK][kQueryLds ? 64 : 1];
    const PagedView &v = a.view;
    if (SHARED && a.shared.mode == SharedResults::kLeave) tell_fit(v, a.shared);
    Unit u;
    if (!find_unit(v, a.plan, blockIdx.x, &u)) return;
    const int g = u.g, b = u.b, G = v.G, n_new = u.s.n_new;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int n_queries = n_new * G; // of this KV head: (token, head in group), token-major
    const float scale = a.scale_log2e * (1.f / query_factor<T, D>());
    // the lane's query as a matrix operand: 16-byte pieces lg, lg + 4, ... of its row
    const int my_q = u.tile * kPQ + lr;
    const bool q_ok = my_q < n_queries;
    const int my_tok = q_ok ? my_q / G : 0;
    raw16 qb[kQueryLds ? 1 : EIGHT ? KK * kQParts : KK];
    const bool has_piece = kPieces >= 4 || lg < kPieces; // (rows of 32 bytes have two pieces)
    const int my_piece = kPieces >= 4 ? lg : lg & (kPieces - 1);
    {
        const unsigned char *qp = a.q + (int64_t)(u.s.first + my_tok) * a.q_token + (int64_t)(g * G + (q_ok ? my_q - my_tok * G : 0)) * a.q_head;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kQueryLds && wave != 0) break; // the same in all waves
            if constexpr (EIGHT && !kBf16) {
                const raw16 *const at = reinterpret_cast<const raw16 *>(qp + 32 * Keys::piece_of(my_piece, kk));
                raw16 x[2] = {brought_down<T, D>(at[0]), brought_down<T, D>(at[1])}, part[kQParts];
                if (!q_ok || !has_piece) x[0] = x[1] = raw16{0u, 0u, 0u, 0u};
                three_parts(x, part);
#pragma unroll
                for (int j = 0; j < kQParts; ++j) {
                    if constexpr (kQueryLds)
                        s_q[kk * kQParts + j][lane] = part[j];
                    else
                        qb[kk * kQParts + j] = part[j];
                }
                continue;
            }
            raw16 x = *reinterpret_cast<const raw16 *>(qp + 16 * (EIGHT ? Keys::piece_of(my_piece, kk) : my_piece + 4 * kk));
            x = q_ok && has_piece ? brought_down<T, D>(x) : raw16{0u, 0u, 0u, 0u};
            if constexpr (kQueryLds)
                s_q[kk][lane] = x;
            else
                qb[kk] = x;
        }
    }
    const int first_tok = u.tile * kPQ / G;
    const int last_q = u.tile * kPQ + kPQ - 1 < n_queries ? u.tile * kPQ + kPQ - 1 : n_queries - 1, last_tok = last_q / G;
    const int past = u.s.length - n_new; // token i sees row j iff j <= past + i (it may be negative)
    int n_rows = u.s.rows;               // up to the last one that a query of the tile sees
    if (a.causal && past + last_tok + 1 < n_rows) n_rows = past + last_tok + 1 > 0 ? past + last_tok + 1 : 0;
    // the workgroup's blocks of rows, dealt to its waves
    constexpr int kBlocks = 4; // to one of the plan's
    const int n_blk = (n_rows + kRows - 1) / kRows;
    const int64_t lo = (int64_t)u.lo * kBlocks, hi = (int64_t)u.hi * kBlocks;
    // (the same in all lanes: scalar registers, and branches that are)
    const int b_lo = __builtin_amdgcn_readfirstlane(lo < n_blk ? (int)lo : n_blk);
    const int b_hi = __builtin_amdgcn_readfirstlane(hi < n_blk ? (int)hi : n_blk);
    const unsigned char *const kb = v.k + g * v.stride_head, *const vb = v.v + g * v.stride_head;

    // Row lane % kRows of a block: the page it is on, requested early, where it lives, and the first token that sees it (INT_MAX: it
    // lives nowhere).  Loads are unconditional: a row that lives nowhere reads the first page's first row; what was read instead
    // of a value row becomes zeros (its weights are zero, but zero times anything must stay zero).
    auto page_at = [&](int blk) __attribute__((always_inline)) {
        const int r = blk * kRows + (lane & (kRows - 1));
        return v.table && blk < b_hi && r < n_rows ? v.table[entry_of(v, b, r)] : 0;
    };
    int64_t scale_off = 0; // of its scales
    auto find = [&](int blk, int page, int64_t *off, int *ft) __attribute__((always_inline)) {
        const int r = blk * kRows + (lane & (kRows - 1));
        const bool there = blk < b_hi && r < n_rows && is_page(v, page);
        if constexpr (EIGHT) scale_off = there ? scale_offset_of(v, page, r) : 0;
        *off = !there ? 0 : v.table ? offset_of(v, page, r) : (int64_t)(u.s.first + r) * v.stride_row;
        *ft = there ? (a.causal ? r - past : 0) : INT_MAX;
    };
    auto from_lane = [&](int64_t x, int from) __attribute__((always_inline)) {
        return (int64_t)((uint64_t)(unsigned)__shfl((int)(x >> 32), from) << 32 | (unsigned)__shfl((int)x, from));
    };
    auto value_row = [&](int i) { return kNarrow ? i * kRowsPerLoad + lane / kValueLanes : 4 * lg + i; }; // of the lane's load i
    raw16 kx[kTiles][KK];
    raw_v vx[NV][kVH];
    typename Keys::Codes kc[EIGHT ? kTiles : 1]; // EIGHT: as they come from memory
    uint32_t vc[EIGHT ? NV : 1][EIGHT ? kVC : 1];
    uint32_t k_scale = 0, v_scale = 0; // EIGHT: the bytes of row lane % kRows of the block
    const unsigned char *const ksb = EIGHT ? v.scales.k + g * v.scales.stride_head : nullptr, *const vsb = EIGHT ? v.scales.v + g * v.scales.stride_head : nullptr;
    auto request_keys = [&](int64_t off) __attribute__((always_inline)) {
        if constexpr (EIGHT) {
            k_scale = ksb[scale_off];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) kc[t].load(kb + from_lane(off, 16 * t + lr), my_piece);
            return;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const unsigned char *p = kb + from_lane(off, 16 * t + lr) + 16 * my_piece;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kx[t][kk] = *reinterpret_cast<const raw16 *>(p + 64 * kk);
        }
    };
    auto request_values = [&](int64_t off) __attribute__((always_inline)) {
        if constexpr (EIGHT) {
            v_scale = vsb[scale_off];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const unsigned char *p = vb + from_lane(off, value_row(i));
                typedef __attribute__((ext_vector_type(kVC))) unsigned int raw_c;
                const raw_c x = *reinterpret_cast<const raw_c *>(p + (lane % kValueLanes) * 4 * kVC);
#pragma unroll
                for (int w = 0; w < kVC; ++w) vc[i][w] = x[w];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const unsigned char *p = vb + from_lane(off, value_row(i)) + (kBf16 ? lane % kPieces : lr) * 4 * kVW;
#pragma unroll
            for (int h = 0; h < kVH; ++h) vx[i][h] = *reinterpret_cast<const raw_v *>(p + 256 * h);
        }
    };

    float m_run = -INFINITY, l_run = 0.f; // of query lr; l_run: over the rows this lane holds
    f32x4 acc[NF]; // of query lr.  kNarrow: tile f, features 16 f + 4 lg + r.  fp32: tile (h, e), features 64 h + kVW (4 lg + r) + e
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned char *const buf = s_buf[wave];
    int64_t off; // of the block in hand
    int ft, page_next = 0;
    if constexpr (kQueryLds) __syncthreads(); // the queries are there
    // One block; the next one's keys and values are requested as soon as the registers of this one's are free.
    auto step = [&](auto more, int next) __attribute__((always_inline)) {
        // ---- scores S^T = K Q^T: query lr, rows 16 t + 4 lg + r ----
        f32x4 sc[kTiles];
        if constexpr (kQueryLds) asm volatile("" ::: "memory"); // (the queries are read again, not held)
        if constexpr (EIGHT && !kBf16) { // sums of 32 terms, of the queries' parts the least first, joined pair by pair
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                kc[t].spread(scale_of((uint32_t)__shfl((int)k_scale, 16 * t + lr)), kx[t]);
                if (!has_piece) kx[t][0] = raw16{0u, 0u, 0u, 0u}; // (16 features: KK is 1)
            }
            f32x4 pair[kTiles];
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                f32x4 c[kTiles];
#pragma unroll
                for (int t = 0; t < kTiles; ++t) c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = kQParts - 1; j >= 0; --j) {
                    const raw16 z = kQueryLds ? s_q[kQueryLds ? kk * kQParts + j : 0][kQueryLds ? lane : 0] : qb[kQueryLds ? 0 : kk * kQParts + j];
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
                        c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[t][kk]), __builtin_bit_cast(bf16x8, z), c[t], 0, 0, 0);
                }
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    pair[t] = kk % 2 ? pair[t] + c[t] : c[t];
                    if (kk == (KK > 1 ? 1 : 0)) sc[t] = pair[t];
                    if (kk == 3) sc[t] += pair[t];
                }
            }
        } else if constexpr (kBf16) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
                if constexpr (EIGHT) {
                    if (t > 0) asm volatile("" : "+v"(sc[t - 1])); // (one tile's rows at a time, for the registers' sake)
                    kc[t].spread(scale_of((uint32_t)__shfl((int)k_scale, 16 * t + lr)), kx[t]);
                }
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    if (!has_piece) kx[t][kk] = raw16{0u, 0u, 0u, 0u};
                    sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[t][kk]),
                                                                    __builtin_bit_cast(bf16x8, qb[kk]), sc[t], 0, 0, 0);
                }
            }
        } else {
            sc[0] = scores_f32<KK>(kx[0], [&](int kk) { return kQueryLds ? s_q[kk][lane] : qb[kQueryLds ? 0 : kk]; });
        }
        int64_t off_next = 0;
        int ft_next = 0;
        if constexpr (more.value) {
            __builtin_amdgcn_sched_barrier(0);
            find(next, page_next, &off_next, &ft_next);
            request_keys(off_next);
            page_next = page_at(next + W);
            __builtin_amdgcn_sched_barrier(0);
        }
        const bool late = __builtin_amdgcn_ballot_w64(ft > first_tok) != 0; // somebody does not see some row
        auto first_to_see = [&](int e) { return __shfl(ft, 16 * (e / 4) + 4 * lg + e % 4); }; // row 16 t + 4 lg + r, e = 4 t + r
        if (late) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) sc[t][r] = my_tok >= first_to_see(4 * t + r) ? sc[t][r] : -INFINITY;
        }
        // ---- statistics and weights, all of query lr (a NaN score is in no maximum and makes the sum one).  What the
        // exponents subtract is a whole number, so that bringing sums from one to another multiplies by a power of two ----
        float mx = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3]));
        if constexpr (kTiles == 2) mx = fmaxf(mx, fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        mx = ceilf(xrow_max(mx) * scale);
        if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) { // a maximum moved: bring what was summed to it
            const float m_new = fmaxf(m_run, mx);
            const float corr = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= corr;
#pragma unroll
            for (int f = 0; f < NF; ++f) acc[f] *= corr;
        }
        const float ref = m_run == -INFINITY ? 0.f : m_run;
        float p[4 * kTiles];
        if (__builtin_amdgcn_ballot_w64(fabsf(ref) > kLargeRef) != 0) { // somebody's is so large that its rounding shows
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if constexpr (kBf16)
                        p[4 * t + r] = __builtin_amdgcn_exp2f(fabsf(ref) > kLargeRef ? scaled_apart(sc[t][r], scale, ref) : fmaf(sc[t][r], scale, -ref));
                    else
                        p[4 * t + r] = weight_of_any(sc[t][r], scale, ref);
        } else {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) // (bf16 payloads: the output's own rounding is four orders above the difference's)
                    p[4 * t + r] = kBf16 ? __builtin_amdgcn_exp2f(fmaf(sc[t][r], scale, -ref)) : weight_of(sc[t][r], scale, ref);
        }
        float sum = (p[0] + p[1]) + (p[2] + p[3]);
        if constexpr (kTiles == 2) sum += (p[4] + p[5]) + (p[6] + p[7]);
        l_run += sum;
        // A value that is no number, in a row that a token of the tile does not see, must not reach that token: its weight is zero,
        // the product is not.  Such blocks (rare) are multiplied token by token, hidden rows as zeros.
        bool apart = false;
        auto spread_values = [&](int i) __attribute__((always_inline)) { // EIGHT
            const float s = scale_of((uint32_t)__shfl((int)v_scale, value_row(i)));
#pragma unroll
            for (int h = 0; h < kVH; ++h) {
                const raw16 x = bf16_piece(vc[i][EIGHT ? 2 * h : 0], vc[i][EIGHT ? 2 * h + 1 : 0], s);
#pragma unroll
                for (int e = 0; e < kVW; ++e) vx[i][h][e] = x[e];
            }
        };
        if (EIGHT && late) { // (the one thing that a code can be and no number is 7F; a scale that is none, FF)
            bool none = false;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool nowhere = __shfl(ft, value_row(i)) == INT_MAX;
                const int scale = __shfl((int)v_scale, value_row(i));
                none |= !nowhere && scale == 255;
#pragma unroll
                for (int w = 0; w < kVC; ++w) {
                    const uint32_t x = nowhere ? 0u : vc[i][w];
                    vc[i][w] = x;
                    none |= (((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0u;
                }
            }
            // (zero times a scale that is none is one as well: rows that live nowhere get another)
            if (ft == INT_MAX) v_scale = 127;
            apart = first_tok != last_tok && __builtin_amdgcn_ballot_w64(none) != 0;
        } else if (late) {
            unsigned worst = 0; // (only whether it reaches the exponent of infinities)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool nowhere = __shfl(ft, value_row(i)) == INT_MAX; // zeros in the place of what was read
#pragma unroll
                for (int h = 0; h < kVH; ++h)
#pragma unroll
                    for (int e = 0; e < kVW; ++e) {
                        const unsigned x = nowhere ? 0u : vx[i][h][e];
                        vx[i][h][e] = x;
                        const unsigned upper = x & 0x7F800000u, lower = kBf16 ? (x & 0x7F80u) << 16 : 0u;
                        worst = worst > upper ? worst : upper;
                        worst = worst > lower ? worst : lower;
                    }
            }
            apart = first_tok != last_tok && __builtin_amdgcn_ballot_w64(worst == 0x7F800000u) != 0;
        }
        // ---- O^T += V^T P^T: the weights are the B operand as they stand in the lane ----
        if constexpr (kNarrow) {
            raw16 hi, lo, least;
            if constexpr (kBf16) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    hi[e] = bf16_pair(p[2 * e], p[2 * e + 1]);
                    lo[e] = bf16_pair(p[2 * e] - __uint_as_float(hi[e] << 16), p[2 * e + 1] - __uint_as_float(hi[e] & 0xFFFF0000u));
                }
            } else {
                raw16 x[2], part[kWParts];
#pragma unroll
                for (int e = 0; e < 4 * kTiles; ++e) x[e / 4][e % 4] = __float_as_uint(p[e]);
                three_parts(x, part);
                hi = part[0];
                lo = part[1];
                least = part[2];
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int row = value_row(i);
                if constexpr (EIGHT) spread_values(i);
#pragma unroll
                for (int h = 0; h < kVH; ++h)
                    *reinterpret_cast<raw_v *>(buf + row * kRowB + 16 * ((kVH * (lane % kValueLanes) + h) ^ row_swizzle<D>(row))) = vx[i][h];
            }
            if constexpr (more.value) request_values(off_next);
            asm volatile("" ::: "memory"); // a wave's LDS accesses keep their order; no other wave reads these rows
            const int q4 = lr >> 2, piece = (lane & 3) >> 1, sub = 8 * (lane & 1);
            auto values_of = [&](int f) __attribute__((always_inline)) { // rows 4 lg + t and 16 + 4 lg + t of feature 16 f + lr
                const int r0 = 4 * lg + q4, r1 = r0 + 16;
                const i16x4 v0 = lds_read_tr16(buf + r0 * kRowB + 16 * ((2 * f + piece) ^ row_swizzle<D>(r0)) + sub);
                const i16x4 v1 = lds_read_tr16(buf + r1 * kRowB + 16 * ((2 * f + piece) ^ row_swizzle<D>(r1)) + sub);
                return i16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            };
            auto product_of_parts = [&](bf16x8 x) __attribute__((always_inline)) { // the least first
                f32x4 c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, least), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, lo), c, 0, 0, 0);
                return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, hi), c, 0, 0, 0);
            };
            if (__builtin_expect(!apart, 1)) {
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    const bf16x8 av = __builtin_bit_cast(bf16x8, values_of(f));
                    if constexpr (kWParts == 3) {
                        acc[f] += product_of_parts(av);
                        continue;
                    }
                    acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, hi), acc[f], 0, 0, 0);
                    acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, lo), acc[f], 0, 0, 0);
                }
            } else {
#pragma unroll 1
                for (int tok = first_tok; tok <= last_tok; ++tok)
#pragma unroll
                    for (int f = 0; f < NF; ++f) {
                        i16x8 x = values_of(f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = tok >= first_to_see(e) ? x[e] : (short)0;
                        f32x4 c = acc[f];
                        if constexpr (kWParts == 3) {
                            c += product_of_parts(__builtin_bit_cast(bf16x8, x));
                        } else {
                            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, hi), c, 0, 0, 0);
                            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, lo), c, 0, 0, 0);
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[f][r] = tok == my_tok ? c[r] : acc[f][r];
                    }
            }
            asm volatile("" ::: "memory"); // the next block's rows take their place
        } else {
            __builtin_amdgcn_sched_barrier(0);
            auto product = [&](int h, int e, auto seen) __attribute__((always_inline)) { // four rows at a time, joined pair by pair
                f32x4 d[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    d[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(seen(i) ? __uint_as_float(vx[i][h][e]) : 0.f, p[i], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                return (d[0] + d[1]) + (d[2] + d[3]);
            };
            if (__builtin_expect(!apart, 1)) {
#pragma unroll
                for (int h = 0; h < kVH; ++h)
#pragma unroll
                    for (int e = 0; e < kVW; ++e) {
                        acc[kVW * h + e] += product(h, e, [](int) { return true; });
                        if (e % 2) // (two at a time, for the registers' sake)
                            asm volatile("" : "+v"(acc[kVW * h + e]), "+v"(p[0]), "+v"(p[1]), "+v"(p[2]), "+v"(p[3]));
                    }
            } else {
#pragma unroll 1
                for (int tok = first_tok; tok <= last_tok; ++tok)
#pragma unroll
                    for (int h = 0; h < kVH; ++h)
#pragma unroll
                        for (int e = 0; e < kVW; ++e) {
                            const f32x4 d = product(h, e, [&](int i) { return tok >= first_to_see(i); });
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[kVW * h + e][r] += tok == my_tok ? d[r] : 0.f;
                            asm volatile("" : "+v"(acc[kVW * h + e]), "+v"(p[0]), "+v"(p[1]), "+v"(p[2]), "+v"(p[3]));
                        }
            }
            if constexpr (more.value) {
                __builtin_amdgcn_sched_barrier(0);
                request_values(off_next);
            }
        }
        off = off_next;
        ft = ft_next;
    };
    if (b_lo + wave < b_hi) {
        int blk = b_lo + wave;
        page_next = page_at(blk + W);
        find(blk, page_at(blk), &off, &ft);
        request_keys(off);
        request_values(off);
        // the last block apart: a branch around the loads would make every wait in the loop one for all of them
        for (; blk + W < b_hi; blk += W) step(std::true_type{}, blk + W);
        step(std::false_type{}, 0);
    }
    // What the other launch left, but for the values: to LDS, by the wave that has the fewest rows.  (Asked for before its rows, three loads one
    // after the other hold them up: 48 users' tokens in three rooms 44.9 us a call, so 43.5.)
    __shared__ Taken s_taken[SHARED ? kPQ : 1];
    __shared__ float s_by[SHARED ? kPlanChunks : 1][kPQ];
    __shared__ int s_fit;
    if (SHARED && a.shared.mode == SharedResults::kTake && wave == W - 1 && lane < kPQ) {
        const int qq = u.tile * kPQ + lane, tok = u.s.first + qq / G;
        if (qq < n_queries)
            s_taken[lane] = take_left(a.shared, tok, (int64_t)tok * v.Hq + g * G + (qq - (qq / G) * G), [&](int c, float x) { s_by[c][lane] = x; });
        if (lane == 0) s_fit = *a.shared.fit;
    }
    // ---- the waves' results join in LDS ----
    const float l_sum = xrow_sum(l_run);
    if (lg == 0) {
        // (maxima leave NaN scores out: where there was nothing else the sum is still to be looked at)
        s_m[wave][lr] = m_run == -INFINITY && l_sum != 0.f ? 0.f : m_run;
        s_l[wave][lr] = l_sum;
    }
    constexpr int kQuads = D / 4; // 4-feature pieces of an output row, piece c of query n at c ^ (n % kQuads)
    f32x4(*const s_o)[kQuads] = reinterpret_cast<f32x4(*)[kQuads]>(buf);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        if constexpr (kNarrow) {
            s_o[lr][(4 * f + lg) ^ (lr & (kQuads - 1))] = acc[f];
        } else if constexpr (kVW == 4) { // register r of the four tiles of h: features 64 h + 16 lg + 4 r ..
            const int h = f / 4, r = f % 4;
            s_o[lr][(16 * h + 4 * lg + r) ^ (lr & (kQuads - 1))] =
                f32x4{acc[4 * h][r], acc[4 * h + 1][r], acc[4 * h + 2][r], acc[4 * h + 3][r]};
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = kVW * (4 * lg + r) + f;
                s_o[lr][(d / 4) ^ (lr & (kQuads - 1))][d % 4] = acc[f][r];
            }
        }
    }
    __syncthreads();
    T *const out = static_cast<T *>(a.out);
    const int n_q_here = n_queries - u.tile * kPQ < kPQ ? n_queries - u.tile * kPQ : kPQ;
    auto row_of = [&](int n) { // of the tile's query n among the outputs
        const int qq = u.tile * kPQ + n, tok = qq / G;
        return (int64_t)(u.s.first + tok) * v.Hq + g * G + (qq - tok * G);
    };
    auto finish = [&](int n, int c, float m, float l, f32x4 o) {
        const int64_t row = row_of(n);
        float l_all = l; // (the other launch's weights may have been rounded)
        if constexpr (SHARED) {
            if (!s_fit) return;
            const Taken t = s_taken[n];
            if (t.chunks > 0) {
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                const float *const values = a.shared.values + (int64_t)t.place * D + 4 * c;
#pragma unroll 8
                for (int k = 0; k < t.chunks; ++k) {
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(values + (int64_t)k * t.stride * D);
                    const float by = s_by[k][n];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = by < 0.f ? x[e] : fmaf(y[e], by, x[e]);
                }
                const JoinBy by = join_by(m, l, t.at, t.sum);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = by.other < 0.f ? o[e] : fmaf(x[e], by.other, counted(o[e], by.own));
                l_all = counted(l, by.own) + counted(t.sum_all, by.other);
                l = counted(l, by.own) + counted(t.sum, by.other);
                m = by.at;
            }
        }
        const bool seen = l != 0.f; // no row that the query sees: zeros (a NaN or +inf score makes l a NaN, and the output with it)
        o = seen ? o / l : f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (kBf16)
            *reinterpret_cast<u32x2 *>(out + row * D + 4 * c) = u32x2{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
        else
            *reinterpret_cast<f32x4 *>(out + row * D + 4 * c) = o;
        if (a.pairs && c == 0) *reinterpret_cast<f32x2 *>(a.pairs + 2 * row) = seen ? f32x2{m, 1.f / l_all} : f32x2{0.f, 0.f};
    };
    for (int i = tid; i < n_q_here * kQuads; i += 64 * W) {
        const int n = i / kQuads, c = i - n * kQuads;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, s_m[w][n]);
        float l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float lw = s_l[w][n];
            if (lw != 0.f) { // a wave none of whose rows the query sees has nothing to add (a NaN has)
                const float x = __builtin_amdgcn_exp2f(s_m[w][n] - m);
                l = fmaf(lw, x, l);
                const f32x4 ow = reinterpret_cast<const f32x4(*)[kQuads]>(s_buf[w])[n][c ^ (n & (kQuads - 1))];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(ow[e], x, o[e]);
            }
        }
        if (SHARED && a.shared.mode == SharedResults::kLeave) {
            const int64_t row = row_of(n), place = place_left(a.shared, u, kPQ, n, row);
            *reinterpret_cast<f32x4 *>(a.shared.values + place * D + 4 * c) = o;
            if (c == 0) {
                *reinterpret_cast<f32x4 *>(a.shared.stats + 4 * place) = f32x4{m, l, l, 0.f};
                leave_head(a.shared, u, kPQ, n, row);
                if (a.pairs) *reinterpret_cast<f32x2 *>(a.pairs + 2 * row) = f32x2{0.f, 0.f}; // (stays so if it is no sequence's)
            }
        } else if (u.chunks > 1) {
            if (c == 0) store_far(a.records.stats + ((int64_t)(u.record + u.chunk) * kPQ + n) * 2, m, l);
            store_far4(chunk_values<kPQ, D>(a.records, u.record + u.chunk), n * D + 4 * c, o);
        } else {
            finish(n, c, m, l, o);
        }
    }
    if (u.chunks == 1 || (SHARED && a.shared.mode == SharedResults::kLeave)) return;
    __shared__ int s_last;
    if (!last_to_arrive(a.counts + u.record, u.chunks, &s_last)) return;
    __shared__ float s_join[join_scratch(kPlanChunks, kPQ)];
    join_chunks<kPQ, D, 64 * W, kPlanChunks, 1, 16>(a.records, u.record, u.chunks, n_q_here, s_join, finish);
}

// What each row receives: weights_out[b][g][j] = decay * weights_in[b][g][j] + sum over the tokens and the group's heads of p_j / sum p.
// Grid (rows, sequence, KV head).  A wave keeps the keys of kTiles times 16 rows (the A operand) in registers and the sequence's queries
// stream past it, 16 at a time and requested one tile ahead, with what their weights subtract and the sum they are divided by: S^T
// leaves a lane one query and four rows of every 16, so the sums over the queries run in the lane until the end, where 16 lanes join.
// SPLIT: the four waves have the same rows and a quarter of the queries each, where there are few rows and many queries, as groups have them.
template <typename T, int D, bool EIGHT, int kTiles, bool SPLIT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) void paged_weights_kernel(PagedAttendArgs a, int n_groups) {
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr bool kNarrow = kBf16 || EIGHT, kInParts = EIGHT && !kBf16; // as in paged_attend_kernel
    constexpr int kRowB = D * (kNarrow ? 2 : 4), kPieces = kRowB / 16;
    constexpr int KK = kNarrow ? (D + 31) / 32 : D / 16;
    using Keys = KeyCodes<std::conditional_t<kNarrow, uint16_t, T>, D>;
    const PagedView &v = a.view;
    const int g = blockIdx.z, b = blockIdx.y;
    const SeqShape s = shape_of(v, a.plan, b);
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, G = v.G;
    const int n_w = s.rows < a.weights_rows ? s.rows : a.weights_rows; // rows that have a weight
    const int past = s.length - s.n_new, n_queries = s.n_new * G;
    const float scale = a.scale_log2e * (1.f / query_factor<T, D>());
    const bool padded = a.shared.mode == SharedResults::kLeave; // a group's tokens may be no sequence's: see no row, whatever stands there
    const bool has_piece = kPieces >= 4 || lg < kPieces;
    const int my_piece = kPieces >= 4 ? lg : lg & (kPieces - 1);
    constexpr int kRows = 16 * kTiles; // of a wave
    constexpr int kApart = SPLIT ? 1 : 4; // rows of the workgroup, in those of a wave
    __shared__ float s_sum[SPLIT ? 4 : 1][SPLIT ? kRows : 1];
    for (int r0 = kRows * ((int)blockIdx.x * kApart + (SPLIT ? 0 : (int)(threadIdx.x >> 6))); r0 < n_w; r0 += kApart * kRows * n_groups) {
        raw16 kx[kTiles][KK];
        typename Keys::Codes kc[EIGHT ? kTiles : 1];
        uint32_t k_scale[EIGHT ? kTiles : 1];
        int from[kTiles][4]; // first token that sees row 16 t + 4 lg + e
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int r = r0 + 16 * t + lr;
            const int page = r < n_w ? (v.table ? v.table[entry_of(v, b, r)] : 0) : -1;
            const bool there = is_page(v, page);
            const int64_t off = !there ? 0 : v.table ? offset_of(v, page, r) : (int64_t)(s.first + r) * v.stride_row;
            if constexpr (EIGHT) {
                kc[t].load(v.k + g * v.stride_head + off, my_piece);
                k_scale[t] = (v.scales.k + g * v.scales.stride_head + (there ? scale_offset_of(v, page, r) : 0))[0];
            }
            const unsigned char *kp = v.k + g * v.stride_head + off + 16 * my_piece;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if constexpr (EIGHT) break;
                kx[t][kk] = *reinterpret_cast<const raw16 *>(kp + 64 * kk);
                if (!has_piece) kx[t][kk] = raw16{0u, 0u, 0u, 0u};
            }
            const int ft = there ? (a.causal ? r - past : 0) : INT_MAX;
#pragma unroll
            for (int e = 0; e < 4; ++e) from[t][e] = __shfl(ft, 4 * lg + e);
        }
        if constexpr (EIGHT)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) { // (requested together before)
                kc[t].spread(scale_of(k_scale[t]), kx[t]);
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    if (!has_piece) kx[t][kk] = raw16{0u, 0u, 0u, 0u};
            }
        float sum[kTiles][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[t][e] = 0.f;
        raw16 qx[2][kInParts ? 2 * KK : KK];
        f32x2 pair[2];
        int tok[2];
        auto request = [&](int q0, int at) __attribute__((always_inline)) {
            const int qq = q0 + lr < n_queries ? q0 + lr : n_queries - 1, h = g * G + qq % G;
            tok[at] = qq / G;
            const unsigned char *qp = a.q + (int64_t)(s.first + tok[at]) * a.q_token + (int64_t)h * a.q_head;
            pair[at] = *reinterpret_cast<const f32x2 *>(a.pairs + 2 * ((int64_t)(s.first + tok[at]) * v.Hq + h));
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if constexpr (kInParts) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) qx[at][2 * kk + i] = reinterpret_cast<const raw16 *>(qp + 32 * Keys::piece_of(my_piece, kk))[i];
                    continue;
                }
                qx[at][kk] = *reinterpret_cast<const raw16 *>(qp + 16 * (EIGHT ? Keys::piece_of(my_piece, kk) : my_piece + 4 * kk));
            }
            if (q0 + lr >= n_queries) tok[at] = -1; // sees nothing
        };
        // EIGHT: most rows are seen by all tokens, where nothing has to be looked at
        bool late = false;
        if constexpr (EIGHT) {
            int last = INT_MIN;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) last = last > from[t][e] ? last : from[t][e];
            late = __builtin_amdgcn_ballot_w64(last > 0) != 0;
        }
        auto add = [&](int at, int q0) __attribute__((always_inline)) {
            raw16 q[kInParts ? 1 : KK], part[kInParts ? KK : 1][3];
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if constexpr (kInParts) {
                    raw16 x[2] = {brought_down<T, D>(qx[at][2 * kk]), brought_down<T, D>(qx[at][2 * kk + 1])};
                    if (!has_piece) x[0] = x[1] = raw16{0u, 0u, 0u, 0u};
                    three_parts(x, part[kk]);
                    continue;
                }
                q[kInParts ? 0 : kk] = has_piece ? brought_down<T, D>(qx[at][kk]) : raw16{0u, 0u, 0u, 0u};
            }
            const float ref = pair[at][0], inv = pair[at][1];
            const bool none = padded && inv == 0.f;
            const bool large = __builtin_amdgcn_ballot_w64(none || fabsf(ref) > kLargeRef) != 0; // (its rounding shows)
            if (EIGHT && kBf16 && !late && !large && q0 + 16 <= n_queries) {
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk)
                        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[t][kk]), __builtin_bit_cast(bf16x8, q[kk]), sc, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[t][e] = fmaf(__builtin_amdgcn_exp2f(fmaf(sc[e], scale, -ref)), inv, sum[t][e]);
                }
                return;
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 sc = {0.f, 0.f, 0.f, 0.f};
                if constexpr (kInParts) {
                    sc = scores_of_parts<KK>(kx[t], part);
                } else if constexpr (kBf16) {
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk)
                        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[t][kk]), __builtin_bit_cast(bf16x8, q[kk]), sc, 0, 0, 0);
                } else {
                    sc = scores_f32<KK>(kx[t], [&](int kk) { return q[kk]; });
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (bf16 payloads: rounded at the size of the difference, 2^-21 of a weight that matters.  The prompt kernel's references
                    // are no whole numbers, so weight_of is not for them, whatever the neighbours' are)
                    float w;
                    if constexpr (kBf16)
                        w = __builtin_amdgcn_exp2f(large && fabsf(ref) > kLargeRef ? scaled_apart(sc[e], scale, ref) : fmaf(sc[e], scale, -ref));
                    else
                        w = large ? weight_of_any(sc[e], scale, ref) : weight_of(sc[e], scale, ref);
                    sum[t][e] += tok[at] >= from[t][e] && tok[at] >= 0 && !none ? w * inv : 0.f;
                }
            }
        };
        // queries before the first row's first token see none of these rows
        int q0 = a.causal && r0 - past > 0 ? (r0 - past < s.n_new ? (r0 - past) * G & ~15 : n_queries) : 0;
        constexpr int kStep = SPLIT ? 128 : 32;
        if constexpr (SPLIT) q0 += 32 * (int)(threadIdx.x >> 6);
        if (q0 < n_queries) request(q0, 0);
        for (; q0 < n_queries; q0 += kStep) {
            if (q0 + 16 < n_queries) request(q0 + 16, 1);
            add(0, q0);
            if (q0 + kStep < n_queries) request(q0 + kStep, 0);
            if (q0 + 16 < n_queries) add(1, q0 + 16);
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[t][e] = row16_sum(sum[t][e]);
            const int row = r0 + 16 * t + 4 * lg + (lr & 3);
            if constexpr (SPLIT) {
                if (lr < 4) s_sum[threadIdx.x >> 6][row - r0] = lr == 0 ? sum[t][0] : lr == 1 ? sum[t][1] : lr == 2 ? sum[t][2] : sum[t][3];
            } else if (lr < 4 && row < n_w) {
                const int64_t at = b * a.weights_seq + g * a.weights_head + row;
                const float got = lr == 0 ? sum[t][0] : lr == 1 ? sum[t][1] : lr == 2 ? sum[t][2] : sum[t][3];
                a.weights_out[at] = a.weights_in ? fmaf(a.decay, a.weights_in[at], got) : got;
            }
        }
        if constexpr (SPLIT) {
            __syncthreads();
            const int row = r0 + (int)threadIdx.x;
            if (threadIdx.x < kRows && row < n_w) {
                const int64_t at = b * a.weights_seq + g * a.weights_head + row;
                const float got = (s_sum[0][threadIdx.x] + s_sum[1][threadIdx.x]) + (s_sum[2][threadIdx.x] + s_sum[3][threadIdx.x]);
                a.weights_out[at] = a.weights_in ? fmaf(a.decay, a.weights_in[at], got) : got;
            }
            __syncthreads(); // the next rows' sums take their place
        }
    }
}

template <typename T, int D, bool EIGHT, int kTiles, bool SPLIT = false>
hipError_t launch_weights(const PagedAttendArgs &a, hipStream_t st) {
    constexpr int kRows = (SPLIT ? 1 : 4) * 16 * kTiles; // of a workgroup
    const int64_t room = a.view.table ? room_of(a.view) : a.view.page_rows, rows = room < a.weights_rows ? room : a.weights_rows;
    const int groups = weight_groups(rows, kRows, (int64_t)a.view.Hkv * a.view.n_seqs);
    if (groups < 1) return hipSuccess;
    hipLaunchKernelGGL((paged_weights_kernel<T, D, EIGHT, kTiles, SPLIT>), dim3((unsigned)groups, a.view.n_seqs, a.view.Hkv), dim3(256), 0, st, a, groups);
    return hipGetLastError();
}

template <typename T, int D, bool EIGHT, bool SHARED>
hipError_t launch_typed(const PagedAttendArgs &a, hipStream_t st) {
    const unsigned grid = (unsigned)units_bound(a.view, a.plan);
    if (grid > 0) {
        hipError_t e;
        if (a.plan.queries != kPQ) {
            if constexpr (SHARED)
                e = EIGHT ? launch_shared_flash8(a, D, st) : launch_shared_flash(a, D, st);
            else
                e = EIGHT ? launch_paged_flash8(a, D, st) : launch_paged_flash(a, D, st);
        } else {
            hipLaunchKernelGGL((paged_attend_kernel<T, D, EIGHT, SHARED>), dim3(grid), dim3(64 * kPWaves), 0, st, a);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    return a.weights_out ? EIGHT ? launch_paged_weights8(a, D, sizeof(T) == 2, st) : launch_paged_weights(a, D, sizeof(T) == 2, st) : hipSuccess;
}

// What rows receive, where the attention of the call has left a.pairs.
template <typename T, int D, bool EIGHT>
hipError_t launch_weights_typed(const PagedAttendArgs &a, hipStream_t st) {
    // Queries that stream past are shared by the rows a wave holds; where there are few of them it is more waves that count (us a
    // launch, 16 / 64 rows a wave: 64 users, one token, 2000 rows, 64/8 heads 61 / 70; 6 users, 16 tokens, 36000 rows in all, 28/4 heads 38 / 29).
    if ((int64_t)a.view.n_tokens * a.view.G <= 32 * (int64_t)a.view.n_seqs) return launch_weights<T, D, EIGHT, 1>(a, st);
    if (EIGHT || a.shared.mode != SharedResults::kNone) { // (other calls' sums stay in the order that they have been in)
        const int64_t room = a.view.table ? room_of(a.view) : a.view.page_rows, rows = room < a.weights_rows ? room : a.weights_rows;
        // (us a call, without / with: 64/8 heads of 128 over 6272 shared rows in bf16, 256 tokens 222 / 188, 16 tokens 53 / 57; 128 tokens over 1548, heads
        // of 64, 93 / 62; 16 tokens over 20000 rows in 8 bits, 28/4 heads, 53.5 / 56.5.  With few queries not all four waves have some: 5 tokens,
        // 35 queries to a KV head, over 1500, 4000 and 8000 rows 19.6 / 18.0, 21.7 / 20.1 and 25.7 / 25.7; 16 tokens 22.9 / 19.8, 26.5 / 23.1, 32.0 / 29.6)
        const int64_t groups = div_up(rows, 64) * a.view.n_seqs * a.view.Hkv, queries = (int64_t)a.view.n_tokens * a.view.G / a.view.n_seqs;
        if (groups < 512 || (groups < 2048 && queries >= 512)) return launch_weights<T, D, EIGHT, EIGHT || sizeof(T) == 2 ? 4 : 2, true>(a, st);
    }
    return launch_weights<T, D, EIGHT, EIGHT || sizeof(T) == 2 ? 4 : 2>(a, st);
}

template <typename T, bool EIGHT>
hipError_t launch_weights_by_dim(const PagedAttendArgs &a, int D, hipStream_t st) {
    switch (D) {
    case 16: return launch_weights_typed<T, 16, EIGHT>(a, st);
    case 32: return launch_weights_typed<T, 32, EIGHT>(a, st);
    case 64: return launch_weights_typed<T, 64, EIGHT>(a, st);
    default: return launch_weights_typed<T, 128, EIGHT>(a, st);
    }
}

template <typename T, bool EIGHT, bool SHARED>
hipError_t launch_by_dim(const PagedAttendArgs &a, int D, hipStream_t st) {
    switch (D) {
    case 16: return launch_typed<T, 16, EIGHT, SHARED>(a, st);
    case 32: return launch_typed<T, 32, EIGHT, SHARED>(a, st);
    case 64: return launch_typed<T, 64, EIGHT, SHARED>(a, st);
    default: return launch_typed<T, 128, EIGHT, SHARED>(a, st);
    }
}

} // namespace

} // namespace mukv

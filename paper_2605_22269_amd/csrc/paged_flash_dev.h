// Attention of many new tokens a sequence over a paged cache, or over packed sequences, on the matrix cores: bf16 rows of 64 or 128
// features.  How rows are shared out and joined is as in paged_attend_dev.h.  The softmax differs in two things: what exponents subtract (the
// largest score of a unit's first rows, see below), and the weights, which enter the product rounded to bf16, as the matrix cores take
// them: as the pairs that paged_attend_dev.h multiplies by they would be twice the products.  Each weight is off by 2^-9 of itself at
// most, no more than an output is by its own rounding: outputs are 0.0019-0.0023 off (2-norm, normal numbers), 0.0017 with that rounding alone.
#pragma once

#include <climits>
#include <type_traits>

#include "eight_dev.h"
#include "paged_dev.h"

namespace mukv {

namespace {

constexpr int kFRows = 64; // rows of a step
constexpr int kRing = 8;                       // steps whose rows' places are held
// 2^24: sums of weights past this are worked out again (see below).
constexpr float kMostSum = 16777216.f;

// sum of two bf16 and x, in fp32
__device__ __forceinline__ float add_pair(uint32_t pair, float x) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), bf16x2{(__bf16)1.f, (__bf16)1.f}, x, false);
}

// One unit by a workgroup of four or eight waves; a wave owns 32 kQB queries from the scores to the output.
// Eight waves (rows in 8 bits or shared, tiles of 256 queries, 128 features) hide in each other what four hide in themselves, by having two
// halves of a step in flight: so a half is worked through in order (kPlain), in half the registers.  A step of 64 rows takes 4100
// clocks of the compute unit for 4470, 2048 of them products (us a call: 1568 tokens over 7840 rows in 8 bits 185 for 197, 8192 over themselves 514 for 543).
// EIGHT: rows of 8 bits (eight_dev.h) come through registers, where they become bf16, and lie in LDS as the others do: a step's codes are
// requested where its rows would be, and put down between the products of the half in which they have to be there (half a step earlier they are
// waited for: 8 users, 16 tokens over 8000 rows, 46.0 us a call for 45.1; 1568 tokens over 7840 rows, 28/4 heads of 64, 136 for 131).
// SHARED: one of two launches, as in paged_attend_dev.h.
template <int D, int kQB, int W, bool PAIRS, bool EIGHT, bool SHARED>
__device__ __forceinline__ void flash_unit(const PagedAttendArgs &a, const Unit &u) {
    using T = uint16_t;
    constexpr int kRowB = D * 2, kPieces = kRowB / 16, kRowsPerLoad = 64 / kPieces; // rows one load of a wave brings
    constexpr int kWaveRows = kFRows / W, kLoads = kWaveRows / kRowsPerLoad;        // rows of a step a wave brings, in such loads
    constexpr int KK = D / 16, NF = D / 32; // 16-feature steps of the scores, 32-feature blocks of the output
    constexpr int kBuf = kFRows * kRowB;
    constexpr bool kPlain = W == 8;
    constexpr int kValues = kPlain ? 2 : 3; // steps whose values are there
    constexpr int kFQ = 32 * kQB * W; // queries of the workgroup, kQB blocks of 32 a wave
    __shared__ __align__(1024) unsigned char s_kv[(2 + kValues) * kBuf]; // keys of two steps, and values
    __shared__ int64_t s_off[kRing][kFRows];                 // byte offset of a row
    __shared__ int64_t s_scale_off[EIGHT ? kRing : 1][EIGHT ? kFRows : 1]; // and of its scales
    __shared__ __align__(16) int s_ft[kRing][kFRows];        // first token that sees it
    __shared__ int s_masked[kRing][2];                       // some query of the tile may not see some row of that half of the step
    __shared__ int s_bad[2], s_any, s_again;
    __shared__ unsigned s_inf[2][kFQ][D / 32]; // outputs that a value of +inf, of -inf reaches (both: NaN), where s_any says so
    __shared__ int s_last;
    const PagedView &v = a.view;
    if (threadIdx.x == 0) s_again = 0;
    const int g = u.g, b = u.b, G = v.G, n_new = u.s.n_new;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid)); // (what follows from it is worked out for every unit, not kept in registers from one to the next)
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, lq = lane & 31, half = lane >> 5;
    const int n_queries = n_new * G;
    const int q0 = u.tile * kFQ + 32 * kQB * wave; // the wave's first
    const float scale = a.scale_log2e;
    // the wave's queries as a matrix operand (column lane % 32, 8 features from 8 * half of every 16)
    bf16x8 qb[kQB][KK];
    int my_tok[kQB];
#pragma unroll
    for (int i = 0; i < kQB; ++i) { // nothing is visible to a query that does not exist
        const int qq = q0 + 32 * i + lq;
        my_tok[i] = qq < n_queries ? qq / G : INT_MIN;
    }
    auto load_queries = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kQB; ++i) {
            const bool ok = my_tok[i] >= 0;
            const int tok = ok ? my_tok[i] : 0;
            const unsigned char *qp =
                a.q + (int64_t)(u.s.first + tok) * a.q_token + (int64_t)(g * G + (ok ? q0 + 32 * i + lq - tok * G : 0)) * a.q_head + 16 * half;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                raw16 x = *reinterpret_cast<const raw16 *>(qp + 32 * kk);
                // (EIGHT, SHARED: another query's in the place of none will do, and nothing waits for it here)
                if (!EIGHT && !SHARED && !ok) x = raw16{0u, 0u, 0u, 0u};
                qb[i][kk] = __builtin_bit_cast(bf16x8, x);
            }
        }
    };
    const int first_tok = u.tile * kFQ / G;
    const int last_q = u.tile * kFQ + kFQ - 1 < n_queries ? u.tile * kFQ + kFQ - 1 : n_queries - 1, last_tok = last_q / G;
    const int past = u.s.length - n_new;
    int n_rows = u.s.rows;
    if (a.causal && past + last_tok + 1 < n_rows) n_rows = past + last_tok + 1 > 0 ? past + last_tok + 1 : 0;
    // the unit's steps (a step is one of the plan's blocks)
    n_rows = __builtin_amdgcn_readfirstlane(n_rows); // (the same in all lanes: scalar registers, and branches that are)
    const int all_steps = (n_rows + kFRows - 1) / kFRows;
    const int t_lo = __builtin_amdgcn_readfirstlane(u.lo < all_steps ? u.lo : all_steps);
    const int n_steps = __builtin_amdgcn_readfirstlane((u.hi < all_steps ? u.hi : all_steps) - t_lo);
    const int row0 = t_lo * kFRows;                                                     // the unit's first row
    const int n_halves = n_steps == 0 ? 0 : ((row0 + n_steps * kFRows < n_rows ? row0 + n_steps * kFRows : n_rows) - row0 + 31) / 32;
    const int all_halves = (n_halves + 1) & ~1;
    const unsigned char *const kb = v.k + g * v.stride_head, *const vb = v.v + g * v.stride_head;

    // ---- where rows live ----
    // Row `lane` of a step: the page it is on, requested four steps early, and its place.  A row that lives nowhere is seen by nobody and
    // reads the first page's first row.
    auto page_at = [&](int t) {
        const int r = row0 + t * kFRows + lane;
        return v.table && t < n_steps && r < n_rows ? v.table[entry_of(v, b, r)] : 0;
    };
    auto tabulate = [&](int t, int page) {
        const int r = row0 + t * kFRows + lane;
        const bool there = t < n_steps && r < n_rows && is_page(v, page);
        s_off[t & (kRing - 1)][lane] = !there ? 0 : v.table ? offset_of(v, page, r) : (int64_t)(u.s.first + r) * v.stride_row;
        if constexpr (EIGHT) s_scale_off[t & (kRing - 1)][lane] = !there ? 0 : scale_offset_of(v, page, r);
        const int ft = there ? (a.causal ? r - past : 0) : INT_MAX;
        s_ft[t & (kRing - 1)][lane] = ft;
        const uint64_t late = __builtin_amdgcn_ballot_w64(ft > first_tok);
        if (lane < 2) s_masked[t & (kRing - 1)][lane] = (uint32_t)(late >> (32 * lane)) != 0u;
    };
    // A wave brings rows 16 wave .. 16 wave + 15 of a step, kRowsPerLoad at a time.  A row's 16-byte pieces are stored permuted, so
    // that neither the reads of key operands nor the transpose reads of values meet in a bank.
    const int ld_row = kWaveRows * wave + lane / kPieces, ld_piece = lane % kPieces;
    unsigned k_piece = 0, v_piece = 0; // where in its row the lane's piece of load i comes from, a byte each
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        k_piece |= 16u * key_slot<D>(ld_piece, ld_row + i * kRowsPerLoad) << (8 * i);
        v_piece |= 16u * val_slot<D>(ld_piece, ld_row + i * kRowsPerLoad) << (8 * i);
    }
    // EIGHT: a lane has 16 codes, two pieces of a row, of each load
    constexpr int kCodeLanes = D / 16, kCodeRows = 64 / kCodeLanes, kCodeLoads = EIGHT ? kWaveRows / kCodeRows : 1;
    struct Codes {
        raw16 k[kCodeLoads], v[kCodeLoads];
        uint32_t k_scale[kCodeLoads], v_scale[kCodeLoads];
    };
    Codes next; // requested
    const unsigned char *const ksb = EIGHT ? v.scales.k + g * v.scales.stride_head : nullptr, *const vsb = EIGHT ? v.scales.v + g * v.scales.stride_head : nullptr;
    const int c_row = kWaveRows * wave + lane / kCodeLanes, c_piece = lane % kCodeLanes;
    auto put_down = [&](int t, const Codes &x) __attribute__((always_inline)) { // the rows of step t, requested before
        if (!EIGHT || t >= n_steps) return;
        unsigned char *const dk = s_kv + (t & 1) * kBuf, *const dv = s_kv + (2 + t % kValues) * kBuf;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) {
            const int row = c_row + i * kCodeRows;
            const float ks = scale_of(x.k_scale[i]), vs = scale_of(x.v_scale[i]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                *reinterpret_cast<raw16 *>(dk + row * kRowB + 16 * key_slot<D>(2 * c_piece + h, row)) = bf16_piece(x.k[i][2 * h], x.k[i][2 * h + 1], ks);
                *reinterpret_cast<raw16 *>(dv + row * kRowB + 16 * val_slot<D>(2 * c_piece + h, row)) = bf16_piece(x.v[i][2 * h], x.v[i][2 * h + 1], vs);
            }
        }
    };
    auto request_codes = [&](int t, Codes &x) __attribute__((always_inline)) {
        if (!EIGHT || t >= n_steps) return;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) {
            const int64_t off = s_off[t & (kRing - 1)][c_row + i * kCodeRows], scale = s_scale_off[t & (kRing - 1)][c_row + i * kCodeRows];
            x.k[i] = *reinterpret_cast<const raw16 *>(kb + off + 16 * c_piece);
            x.v[i] = *reinterpret_cast<const raw16 *>(vb + off + 16 * c_piece);
            x.k_scale[i] = ksb[scale];
            x.v_scale[i] = vsb[scale];
        }
    };
    auto request = [&](int t) __attribute__((always_inline)) { // the rows of step t
        if (t >= n_steps) return;
        if constexpr (EIGHT) {
            request_codes(t, next);
            return;
        }
        unsigned char *const dk = s_kv + (t & 1) * kBuf, *const dv = s_kv + (2 + t % kValues) * kBuf;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int64_t off = s_off[t & (kRing - 1)][ld_row + i * kRowsPerLoad];
            const int lds = (kWaveRows * wave + i * kRowsPerLoad) * kRowB; // the wave's 1024 bytes, lane order
            load_to_lds(kb + (off + (k_piece >> (8 * i) & 255u)), dk + lds);
            load_to_lds(vb + (off + (v_piece >> (8 * i) & 255u)), dv + lds);
        }
    };

    // ---- state ----
    // what exponents subtract; sums of the weights over the rows this lane holds, as they enter the product, and with PAIRS as they were
    float ref[kQB], l_run[kQB], l_whole[kQB];
    f32x16 o[kQB][NF];          // features 32 f + 8 (j / 4) + 4 half + j % 4 of query lq
    f32x16 sc[2][kQB];          // scores of two halves of a step: rows 8 (j / 4) + 4 half + j % 4
    float s_scale = scale, s_ref[kQB]; // a weight is 2^(score * s_scale - s_ref)
    bool large = false;             // some ref is so large that the product's rounding shows
    bf16x8 ak[KK], av[2][NF];       // operands on their way: keys of a half, values of its two 16 rows
    // Where this lane reads its operands of a step's first half: keys of 16-feature step kk, values of feature block f (rows 4 half +
    // (lane % 16) / 4 and 8 later of every 16, 4 features).  The walkers go from step to step with the buffers.
    unsigned k_at[KK], v_at[NF][2];
    auto first_operands = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) k_at[kk] = lq * kRowB + 16 * key_slot<D>(2 * kk + half, lq);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int row = 4 * half + ((lane & 15) >> 2), piece = 4 * f + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), sub = 8 * (lane & 1);
            v_at[f][0] = 2 * kBuf + row * kRowB + 16 * val_slot<D>(piece, row) + sub;
            v_at[f][1] = 2 * kBuf + (row + 8) * kRowB + 16 * val_slot<D>(piece, row + 8) + sub;
        }
    };
    auto next_keys = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) k_at[kk] ^= kBuf;
    };
    auto next_values = [&](int t) __attribute__((always_inline)) { // from those of step t
        const unsigned by = t % kValues == kValues - 1 ? 0u - (kValues - 1u) * kBuf : (unsigned)kBuf;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            v_at[f][0] += by;
            v_at[f][1] += by;
        }
    };
    auto load_k = [&](auto second, int kk) { return *reinterpret_cast<const bf16x8 *>(s_kv + k_at[kk] + second.value * 32 * kRowB); };
    auto load_v = [&](auto second, int grp, int f) { // of 16 rows
        const int at = (second.value * 32 + grp * 16) * kRowB;
        const i16x4 x = lds_read_tr16(s_kv + v_at[f][0] + at), y = lds_read_tr16(s_kv + v_at[f][1] + at);
        return __builtin_bit_cast(bf16x8, i16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
    };
    auto values_of = [&](int h) { return s_kv + (2 + (h >> 1) % kValues) * kBuf + (h & 1) * 32 * kRowB; };
    // weights of query block i and 16 rows as a matrix operand
    auto weights_of = [&](const f32x16 &s, int i, int grp) __attribute__((always_inline)) {
        raw16 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[8 * grp + 2 * e], s_scale, -s_ref[i]));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[8 * grp + 2 * e + 1], s_scale, -s_ref[i]));
            w[e] = bf16_pair(x, y);
            // (outputs are divided by the sum of the weights as they enter the product, so that a row that has nearly all of it keeps its
            // value; what rows receive, in 32 bits, by that before the rounding)
            l_run[i] = add_pair(w[e], l_run[i]);
            if (PAIRS) l_whole[i] += x + y;
        }
        return __builtin_bit_cast(bf16x8, w);
    };

    auto scores_of = [&](auto second, f32x16 *s) __attribute__((always_inline)) { // of a half of the step that k_at is at
#pragma unroll
        for (int i = 0; i < kQB; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) s[i][j] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const bf16x8 x = load_k(second, kk);
#pragma unroll
            for (int i = 0; i < kQB; ++i) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qb[i][kk], s[i], 0, 0, 0);
        }
    };
    auto is_masked = [&](int h) { return __builtin_amdgcn_readfirstlane(s_masked[(h >> 1) & (kRing - 1)][h & 1]) != 0; };
    auto hide = [&](int h, f32x16 *s) __attribute__((always_inline)) { // scores of rows that the query does not see: -inf
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
            const i32x4 ft = *reinterpret_cast<const i32x4 *>(&s_ft[(h >> 1) & (kRing - 1)][32 * (h & 1) + 8 * jj + 4 * half]);
#pragma unroll
            for (int i = 0; i < kQB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[i][4 * jj + r] = my_tok[i] >= ft[r] ? s[i][4 * jj + r] : -INFINITY;
        }
    };
    auto largest = [&](const f32x16 &s) __attribute__((always_inline)) { // over both halves of the lanes, scaled
        float m4[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) m4[c] = fmaxf(fmaxf(s[c], s[4 + c]), fmaxf(s[8 + c], s[12 + c]));
        return half_max(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]))) * scale;
    };
    auto base_of = [&](int i) { return ref[i] == -INFINITY ? 0.f : ref[i]; };
    auto set_ref = [&]() __attribute__((always_inline)) {
        bool any = false;
#pragma unroll
        for (int i = 0; i < kQB; ++i) any |= fabsf(base_of(i)) > kLargeRef;
        large = __builtin_amdgcn_ballot_w64(any) != 0;
        s_scale = large ? 1.f : scale;
#pragma unroll
        for (int i = 0; i < kQB; ++i) s_ref[i] = large ? 0.f : base_of(i);
    };
    // For step(h), with v_at at h's step and k_at at that of half h + 1.
    auto load_ahead = [&](auto par) __attribute__((always_inline)) {
        using Here = std::integral_constant<int, par.value>;
        using There = std::integral_constant<int, 1 - par.value>;
#pragma unroll
        for (int kk = 0; kk < KK / 2; ++kk) ak[kk] = load_k(There{}, kk);
#pragma unroll
        for (int f = 0; f < NF; ++f) av[0][f] = load_v(Here{}, 0, f);
    };
    // The scores of half h, before their weights are taken.
    auto look = [&](auto par, int h, int flag) __attribute__((always_inline)) { // flag: s_masked of the half
        constexpr int P = kPlain ? 0 : par.value;
        const int slot = (h >> 1) & (kRing - 1);
        const bool masked = h < all_halves && __builtin_amdgcn_readfirstlane(flag) != 0;
        if (masked) hide(h, sc[P]);
        if (__builtin_expect(large, 0)) {
#pragma unroll
            for (int i = 0; i < kQB; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[P][i][j] = scaled_apart(sc[P][i][j], scale, base_of(i));
        }
        // A value that is no number must not reach a token that does not see its row: the weight is zero, the product is not.
        if (masked) {
            unsigned char *const vs = values_of(h);
            const raw16 *own = reinterpret_cast<const raw16 *>(vs + wave * (32 / W) * kRowB);
            unsigned worst = 0;
#pragma unroll
            for (int i = 0; i < 32 / W * kPieces / 64; ++i) {
                const raw16 x = own[lane + 64 * i];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned upper = x[e] & 0x7F800000u, lower = (x[e] & 0x7F80u) << 16;
                    worst = worst > upper ? worst : upper;
                    worst = worst > lower ? worst : lower;
                }
            }
            static_assert(32 / W * kPieces >= 64, "whole waves");
            if (__builtin_amdgcn_ballot_w64(worst == 0x7F800000u) != 0 && lane == 0) s_bad[h & 1] = 1;
            __syncthreads();
            if (__builtin_expect(s_bad[h & 1] != 0, 0)) {
                // Whatever else is summed, such a value decides the outputs of the tokens that see it: which they are is written
                // down, and the value becomes a zero.
                unsigned sees[kQB], weighs[kQB]; // rows 8 (j / 4) + 4 half + j % 4, bit j
#pragma unroll
                for (int i = 0; i < kQB; ++i) {
                    sees[i] = weighs[i] = 0;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float w = __builtin_amdgcn_exp2f(fmaf(sc[P][i][j], s_scale, -s_ref[i]));
                        sees[i] |= (unsigned)(my_tok[i] >= s_ft[slot][32 * (h & 1) + 8 * (j / 4) + 4 * half + j % 4]) << j;
                        weighs[i] |= (unsigned)(w != 0.f) << j;
                    }
                }
#pragma unroll 1
                for (int j = 0; j < 16; ++j) {
                    const int row = 8 * (j / 4) + 4 * half + j % 4;
#pragma unroll 1
                    for (int d = 0; d < D; ++d) {
                        const unsigned x = *reinterpret_cast<const uint16_t *>(vs + row * kRowB + 16 * val_slot<D>(d / 8, row) + 2 * (d % 8));
                        if ((x & 0x7F80u) != 0x7F80u) continue;
#pragma unroll
                        for (int i = 0; i < kQB; ++i) {
                            if (!(sees[i] >> j & 1)) continue;
                            const bool nan = (x & 0x7Fu) != 0 || !(weighs[i] >> j & 1); // (zero times infinity)
                            const int n = 32 * (kQB * wave + i) + lq;
                            if (nan || !(x >> 15)) atomicOr(&s_inf[0][n][d / 32], 1u << d % 32);
                            if (nan || x >> 15) atomicOr(&s_inf[1][n][d / 32], 1u << d % 32);
                        }
                    }
                }
                __syncthreads(); // every wave has looked at the values
                for (int i = tid; i < 32 * D; i += 64 * W) {
                    uint16_t *const x = reinterpret_cast<uint16_t *>(vs) + i;
                    if ((*x & 0x7F80u) == 0x7F80u) *x = 0;
                }
                if (tid == 0) {
                    s_bad[h & 1] = 0;
                    s_any = 1;
                }
                __syncthreads();
                if constexpr (!kPlain) load_ahead(par); // (they were there already)
            }
        }
    };

    // Eight waves: half h, its scores, weights and values one after the other; the other wave of the SIMD does its weights meanwhile.
    auto plain_step = [&](auto par, int h) __attribute__((always_inline)) {
        const int flag = s_masked[(h >> 1) & (kRing - 1)][par.value];
        scores_of(par, sc[0]);
        look(par, h, flag);
        bf16x8 pw[2];
#pragma unroll
        for (int grp = 0; grp < 2; ++grp) pw[grp] = weights_of(sc[0][0], 0, grp);
#pragma unroll
        for (int grp = 0; grp < 2; ++grp)
#pragma unroll
            for (int f = 0; f < NF; ++f) o[0][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(load_v(par, grp, f), pw[grp], o[0][f], 0, 0, 0);
    };
    // Half h: its weights and values, and the scores of half h + 1 between them.  Operands are in registers a section before their products.
    constexpr int K1 = KK * 3 / 4; // products of the scores in the first section
    auto step = [&](auto par, int h) __attribute__((always_inline)) {
        constexpr int P = par.value;
        using Here = std::integral_constant<int, P>;
        using There = std::integral_constant<int, 1 - P>;
        f32x16 *const nxt = sc[1 - P];
        bf16x8 pw[2][kQB];
        const int flag = s_masked[((h + 1) >> 1) & (kRing - 1)][1 - P];
        // ---- most of the scores; weights of the first 16 rows ----
#pragma unroll
        for (int i = 0; i < kQB; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) nxt[i][j] = 0.f;
#pragma unroll
        for (int kk = KK / 2; kk < KK; ++kk) ak[kk] = load_k(There{}, kk);
#pragma unroll
        for (int f = 0; f < NF; ++f) av[1][f] = load_v(Here{}, 1, f);
#pragma unroll
        for (int kk = 0; kk < K1; ++kk)
#pragma unroll
            for (int i = 0; i < kQB; ++i) nxt[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[kk], qb[i][kk], nxt[i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kQB; ++i) pw[0][i] = weights_of(sc[P][i], i, 0);
#pragma unroll
        for (int n = 0; n < K1 * kQB; ++n) {
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0); // reads of LDS
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);   // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x402, D == 128 ? 5 : 10, 0); // vector instructions beside it
        }
        __builtin_amdgcn_sched_barrier(0);
        if (P == 0 && h > 0) put_down((h >> 1) + 1, next); // (requested a step before)
        // ---- the rest of the scores; values of the first 16 rows, weights of the others ----
#pragma unroll
        for (int kk = K1; kk < KK; ++kk)
#pragma unroll
            for (int i = 0; i < kQB; ++i) nxt[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[kk], qb[i][kk], nxt[i], 0, 0, 0);
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < kQB; ++i) o[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[0][f], pw[0][i], o[i][f], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kQB; ++i) pw[1][i] = weights_of(sc[P][i], i, 1);
#pragma unroll
        for (int n = 0; n < (KK - K1 + NF) * kQB; ++n) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, D == 128 ? 5 : 10, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (P == 0) { // the rows of the next step are there; the next but one's take the place of this one's keys
            if constexpr (!EIGHT) rows_landed();
            __syncthreads();
            request((h >> 1) + 2);
            next_keys();
        } else {
            next_values(h >> 1);
        }
        // ---- values of the other 16 rows; the scores go to where vector instructions reach them ----
        load_ahead(There{});
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                o[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[1][f], pw[1][i], o[i][f], 0, 0, 0);
                if (f == NF / 2) asm volatile("" : "+v"(nxt[i]));
            }
        return flag;
    };

    int page;
    auto stage = [&]() __attribute__((always_inline)) { // the first two steps' rows
        const int p0 = page_at(wave), p1 = W == 4 ? page_at(wave + 4) : 0;
        page = page_at(wave + 8);
        __syncthreads(); // everybody is done with what was there
        tabulate(wave, p0);
        if (W == 4) tabulate(wave + 4, p1);
        __syncthreads();
        if constexpr (EIGHT) {
            Codes first;
            request_codes(0, first);
            request_codes(1, next);
            first_operands();
            put_down(0, first);
            put_down(1, next);
        } else {
            request(0);
            request(1);
            first_operands();
            rows_landed();
        }
        __syncthreads();
    };
    auto next_places = [&](int h) __attribute__((always_inline)) {
        // places of the steps up to this one are free: four new ones every four steps (which are read from two steps on)
        if ((h & 7) == 7 && (W == 4 || wave < 4)) {
            tabulate((h >> 1) + 5 + wave, page);
            page = page_at((h >> 1) + 9 + wave);
        }
    };
    T *const out = static_cast<T *>(a.out);
    float l_sum[kQB], l_all[kQB], at[kQB]; // the sums of weights, and what they are relative to
    // o over the sums of weights to `out`.  past: becomes a NaN where an output is none, or past what fp32 holds
    auto put_results = [&](float(*past)[kQB]) __attribute__((always_inline)) {
        if constexpr (SHARED) {
            if (*a.shared.fit == 0) return; // (leaving does not come here)
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                const int qq = q0 + 32 * i + lq, tok = u.s.first + (qq < n_queries ? my_tok[i] : 0);
                const int64_t row = (int64_t)tok * v.Hq + g * G + (qq < n_queries ? qq - my_tok[i] * G : 0);
                if (qq >= n_queries) continue;
                const Taken t = take_left(a.shared, tok, row, [](int, float) {});
                f32x4 x[NF][4];
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj) x[f][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
                // chunks requested together, where there are registers (718 tokens of 16 users over 6272 shared rows 106.2 us a call, one by one 110.3)
                constexpr int kTogether = W == 8 ? 1 : 2;
#pragma unroll 1
                for (int c0 = 0; c0 < t.chunks; c0 += kTogether) {
                    f32x4 y[kTogether][NF][4];
                    f32x2 st[kTogether];
#pragma unroll
                    for (int n = 0; n < kTogether; ++n) {
                        const int64_t place = t.place + (int64_t)(c0 + n < t.chunks ? c0 + n : c0) * t.stride;
                        st[n] = *reinterpret_cast<const f32x2 *>(a.shared.stats + 4 * place);
#pragma unroll
                        for (int f = 0; f < NF; ++f)
#pragma unroll
                            for (int jj = 0; jj < 4; ++jj) y[n][f][jj] = *reinterpret_cast<const f32x4 *>(a.shared.values + place * D + 4 * half + 32 * f + 8 * jj);
                    }
#pragma unroll
                    for (int n = 0; n < kTogether; ++n) {
                        const float by = c0 + n < t.chunks && st[n][1] != 0.f ? __builtin_amdgcn_exp2f(st[n][0] - t.at) : -1.f;
#pragma unroll
                        for (int f = 0; f < NF; ++f)
#pragma unroll
                            for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                                for (int e = 0; e < 4; ++e) x[f][jj][e] = by < 0.f ? x[f][jj][e] : fmaf(y[n][f][jj][e], by, x[f][jj][e]);
                    }
                }
                const JoinBy by = join_by(at[i], l_sum[i], t.at, t.sum);
                if (by.other < 0.f) continue;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][f][j] = fmaf(x[f][j / 4][j % 4], by.other, counted(o[i][f][j], by.own));
                l_sum[i] = fmaf(t.sum, by.other, counted(l_sum[i], by.own));
                if (PAIRS) l_all[i] = fmaf(t.sum_all, by.other, counted(l_all[i], by.own));
                at[i] = by.at;
            }
        }
#pragma unroll
        for (int i = 0; i < kQB; ++i) {
            const int qq = q0 + 32 * i + lq;
            const bool ok = qq < n_queries, seen = l_sum[i] != 0.f; // a query that saw nothing gets zeros; NaN stays NaN
            const float inv = 1.f / l_sum[i];
            const int tok = ok ? my_tok[i] : 0;
            const int64_t row = (int64_t)(u.s.first + tok) * v.Hq + g * G + (ok ? qq - tok * G : 0);
            T *const op = out + row * D + 8 * half;
            if (PAIRS && ok && half == 0) *reinterpret_cast<f32x2 *>(a.pairs + 2 * row) = seen ? f32x2{at[i], 1.f / l_all[i]} : f32x2{0.f, 0.f};
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int jj = 0; jj < 4; jj += 2) { // a lane holds features 8 jj + 4 half .. + 3: the halves swap, and it stores 16 bytes
                    raw16 w;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t pk[2];
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float y0 = o[i][f][4 * (jj + x) + 2 * e], y1 = o[i][f][4 * (jj + x) + 2 * e + 1];
                            pk[x] = bf16_pair(y0 * inv, y1 * inv);
                            if (past) (*past)[i] = fmaf(y1, 0.f, fmaf(y0, 0.f, (*past)[i]));
                        }
                        auto sw = __builtin_amdgcn_permlane32_swap(pk[0], pk[1], false, false);
                        w[e] = sw[0];
                        w[2 + e] = sw[1];
                    }
                    if (!seen) w = raw16{0u, 0u, 0u, 0u};
                    if (ok) *reinterpret_cast<raw16 *>(op + 32 * f + 8 * jj) = w;
                }
        }
    };
    // The chunk's record: values as they stand in the lanes, so that every access is a kilobyte in a row (query by query they were
    // 16-byte pieces of lines: a call of 220 tiles in two chunks 122 us, unsplit 70).  The last workgroup of the tile to get here
    // joins them, in their order.
    auto piece = [&](int i, int f, int jj) { return (((wave * kQB + i) * NF + f) * 4 + jj) * 256 + 4 * lane; };
    // What exponents subtract is the largest score of the unit's first half, and stays: weights then are what they are, not at most
    // 1, and floating point holds them as well, so nothing in the loop waits for a maximum or brings sums to another one.  Sums that
    // grow large (a later score larger by 24 log2 units or so), or take an output past what fp32 holds, are worked out again with the
    // largest score of all rows.  Outputs are looked at on their way out, where they are in reach of vector instructions anyway.
    for (bool again = false;; again = true) {
        load_queries();
        if (n_halves > 0) {
            if (__builtin_expect(again, 0)) {
                stage();
#pragma unroll
                for (int i = 0; i < kQB; ++i) ref[i] = -INFINITY;
                auto max_of = [&](auto par, int h) __attribute__((always_inline)) {
                    scores_of(par, sc[0]);
                    if (is_masked(h)) hide(h, sc[0]);
#pragma unroll
                    for (int i = 0; i < kQB; ++i) ref[i] = fmaxf(ref[i], largest(sc[0][i]));
                };
#pragma unroll 1
                for (int h = 0; h < n_halves; h += 2) {
                    max_of(std::integral_constant<int, 0>{}, h);
                    max_of(std::integral_constant<int, 1>{}, h + 1);
                    if constexpr (!EIGHT) rows_landed(); // of the next step; this one's keys are done with
                    __syncthreads();
                    request((h >> 1) + 2);
                    put_down((h >> 1) + 2, next);
                    next_keys();
                    next_places(h + 1);
                }
            }
            stage();
            if (tid < 2) s_bad[tid] = 0;
            if (tid == 0) s_any = 0;
            for (int i = tid; i < 2 * kFQ * (D / 32); i += 64 * W) (&s_inf[0][0][0])[i] = 0u;
            scores_of(std::integral_constant<int, 0>{}, sc[0]);
            if (!again) {
                f32x16 s[kQB];
#pragma unroll
                for (int i = 0; i < kQB; ++i) s[i] = sc[0][i];
                if (is_masked(0)) hide(0, s);
#pragma unroll
                for (int i = 0; i < kQB; ++i) ref[i] = largest(s[i]);
            }
            set_ref();
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                l_run[i] = l_whole[i] = 0.f;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][f][j] = 0.f;
            }
            __syncthreads(); // the flags are cleared
            if constexpr (kPlain) {
#pragma unroll 1
                for (int h = 0; h < n_halves; h += 2) { // (an odd half out is joined by one whose rows nobody sees)
                    plain_step(std::integral_constant<int, 0>{}, h);
                    if (h > 0) put_down((h >> 1) + 1, next);
                    plain_step(std::integral_constant<int, 1>{}, h + 1);
                    if constexpr (!EIGHT) rows_landed();
                    __syncthreads(); // the next step's rows are there; the next but one's take the place of this one's
                    request((h >> 1) + 2);
                    next_keys();
                    next_values(h >> 1);
                    next_places(h + 1);
                }
            }
            if constexpr (!kPlain) {
                load_ahead(std::integral_constant<int, 0>{});
#pragma unroll
                for (int i = 0; i < kQB; ++i) asm volatile("" : "+v"(sc[0][i]));
                look(std::integral_constant<int, 0>{}, 0, s_masked[0][0]);
            }
#pragma unroll 1
            for (int h = 0; !kPlain && h < n_halves; h += 2) { // (an odd half out is joined by one whose rows nobody sees)
                const int odd = step(std::integral_constant<int, 0>{}, h);
                look(std::integral_constant<int, 1>{}, h + 1, odd);
                const int even = step(std::integral_constant<int, 1>{}, h + 1);
                next_places(h + 1);
                look(std::integral_constant<int, 0>{}, h + 2, even);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                ref[i] = l_run[i] = l_whole[i] = 0.f;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][f][j] = 0.f;
            }
        }
        // ---- results ----
        if (n_halves > 0 && __builtin_expect(s_any != 0, 0)) {
#pragma unroll
            for (int i = 0; i < kQB; ++i)
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    const unsigned up = s_inf[0][32 * (kQB * wave + i) + lq][f], down = s_inf[1][32 * (kQB * wave + i) + lq][f];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int d = 8 * (j / 4) + 4 * half + j % 4;
                        if (up >> d & 1) o[i][f][j] += INFINITY;
                        if (down >> d & 1) o[i][f][j] -= INFINITY;
                    }
                }
        }
        float past_it[kQB];
#pragma unroll
        for (int i = 0; i < kQB; ++i) {
            l_sum[i] = half_sum(l_run[i]);
            l_all[i] = PAIRS ? half_sum(l_whole[i]) : 0.f;
            at[i] = base_of(i);
            past_it[i] = 0.f;
        }
        if (SHARED && a.shared.mode == SharedResults::kLeave) {
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                const int qq = q0 + 32 * i + lq;
                if (qq >= n_queries) continue;
                const int64_t row = (int64_t)(u.s.first + my_tok[i]) * v.Hq + g * G + (qq - my_tok[i] * G);
                const int64_t place = place_left(a.shared, u, kFQ, qq - u.tile * kFQ, row);
                float *const vp = a.shared.values + place * D + 4 * half;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj) {
                        const f32x4 y = {o[i][f][4 * jj], o[i][f][4 * jj + 1], o[i][f][4 * jj + 2], o[i][f][4 * jj + 3]};
                        *reinterpret_cast<f32x4 *>(vp + 32 * f + 8 * jj) = y;
#pragma unroll
                        for (int e = 0; e < 4; ++e) past_it[i] = fmaf(y[e], 0.f, past_it[i]);
                    }
                if (half == 0) {
                    *reinterpret_cast<f32x4 *>(a.shared.stats + 4 * place) = f32x4{at[i], l_sum[i], PAIRS ? l_all[i] : l_sum[i], 0.f};
                    leave_head(a.shared, u, kFQ, qq - u.tile * kFQ, row);
                    if (PAIRS) *reinterpret_cast<f32x2 *>(a.pairs + 2 * row) = f32x2{0.f, 0.f}; // (stays so if it is no sequence's)
                }
            }
        } else if (u.chunks > 1) {
            const auto values = chunk_values<kFQ, D>(a.records, u.record + u.chunk);
            float *const stats = a.records.stats + (int64_t)(u.record + u.chunk) * kFQ * 2;
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                const int n = 32 * (kQB * wave + i) + lq;
                if (half == 0) store_far(stats + 2 * n, at[i], l_sum[i]);
                if (PAIRS && half == 0) store_far1(a.records.sums + (int64_t)(u.record + u.chunk) * kFQ + n, l_all[i]);
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj) {
                        const f32x4 y = {o[i][f][4 * jj], o[i][f][4 * jj + 1], o[i][f][4 * jj + 2], o[i][f][4 * jj + 3]};
                        store_far4(values, piece(i, f, jj), y);
#pragma unroll
                        for (int e = 0; e < 4; ++e) past_it[i] = fmaf(y[e], 0.f, past_it[i]);
                    }
            }
        } else {
            put_results(&past_it);
        }
        if (again || n_halves == 0) break;
        bool out_of_range = false;
#pragma unroll
        for (int i = 0; i < kQB; ++i) { // (no row of the first half seen, but perhaps others: not with all pages there)
            out_of_range |= l_run[i] > kMostSum || (ref[i] == -INFINITY && n_halves > 1 && my_tok[i] >= (a.causal ? row0 + 32 - past : 0));
            out_of_range |= past_it[i] != past_it[i] && l_sum[i] == l_sum[i];
        }
        if (__builtin_amdgcn_ballot_w64(out_of_range) != 0 && lane == 0) s_again = 1;
        __syncthreads();
        if (__builtin_expect(s_again == 0, 1)) break;
    }
    if (SHARED && a.shared.mode == SharedResults::kLeave) return;
    if (u.chunks == 1 || !last_to_arrive(a.counts + u.record, u.chunks, &s_last)) return;
    const float *const stats = a.records.stats + ((int64_t)u.record * kFQ + 32 * kQB * wave + lq) * 2;
#pragma unroll
    for (int i = 0; i < kQB; ++i) {
        at[i] = -INFINITY;
        l_sum[i] = l_all[i] = 0.f;
#pragma unroll 8
        for (int c = 0; c < u.chunks; ++c) {
            const f32x2 st = load_far(stats + ((int64_t)c * kFQ + 32 * i) * 2);
            at[i] = st[1] != 0.f ? fmaxf(at[i], st[0]) : at[i]; // (else none of the chunk's rows is seen; a NaN is)
        }
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][f][j] = 0.f;
    }
#pragma unroll 1
    for (int c = 0; c < u.chunks; ++c) {
        const auto values = chunk_values<kFQ, D>(a.records, u.record + c);
        f32x2 st[kQB];
#pragma unroll
        for (int i = 0; i < kQB; ++i) st[i] = load_far(stats + ((int64_t)c * kFQ + 32 * i) * 2);
#pragma unroll
        for (int i = 0; i < kQB; ++i) {
            f32x4 x[NF][4];
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int jj = 0; jj < 4; ++jj) x[f][jj] = load_far4(values, piece(i, f, jj));
            const bool some = st[i][1] != 0.f;
            const float by = some ? __builtin_amdgcn_exp2f(st[i][0] - at[i]) : 0.f;
            if (some) l_sum[i] = fmaf(st[i][1], by, l_sum[i]);
            if (PAIRS && some) l_all[i] = fmaf(load_far1(a.records.sums + (int64_t)(u.record + c) * kFQ + 32 * (kQB * wave + i) + lq), by, l_all[i]);
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][f][j] = some ? fmaf(x[f][j / 4][j % 4], by, o[i][f][j]) : o[i][f][j];
        }
    }
    put_results(nullptr);
}

// A workgroup takes a unit; of one sequence's perhaps the units of its stretch, one after the other (us a launch, 28/4 heads of 128, chunks
// alone / shares where they cost less: 1568 tokens over 6272 rows 239 / 177, 2000 over 10000 361 / 327; 1500 over 3000, 16/4 heads of 64, 63 / 55).
template <int D, int kQB, int W, bool PAIRS, bool SHARES, bool EIGHT, bool SHARED>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(W / 4, W / 4))) void paged_flash_kernel(PagedAttendArgs a) {
    if (SHARED && a.shared.mode == SharedResults::kLeave) tell_fit(a.view, a.shared);
    Unit u;
    if constexpr (SHARES) {
        Share share;
        bool there = false;
        const bool even = find_share(a.view, a.plan, blockIdx.x, gridDim.x, &share, &u, &there);
        if (even ? share.at == share.end : !there) return;
        for (;;) {
            if (even) next_unit(a.view, a.plan, &share, &u);
            make_scalar(u);
            flash_unit<D, kQB, W, PAIRS, EIGHT, SHARED>(a, u);
            if (!even || share.at == share.end) return;
            __syncthreads(); // the next unit takes this one's LDS
        }
    } else {
        if (find_unit(a.view, a.plan, blockIdx.x, &u)) flash_unit<D, kQB, W, PAIRS, EIGHT, SHARED>(a, u);
    }
}

} // namespace

template <int D, int kQB, int W, bool PAIRS, bool EIGHT, bool SHARED>
static void start_flash(const PagedAttendArgs &a, unsigned grid, hipStream_t st) {
    if (may_share(a.view, a.plan))
        hipLaunchKernelGGL((paged_flash_kernel<D, kQB, W, PAIRS, true, EIGHT, SHARED>), dim3(grid), dim3(64 * W), 0, st, a);
    else
        hipLaunchKernelGGL((paged_flash_kernel<D, kQB, W, PAIRS, false, EIGHT, SHARED>), dim3(grid), dim3(64 * W), 0, st, a);
}
template <int D, int kQB, int W, bool EIGHT, bool SHARED>
static hipError_t launch_flash(const PagedAttendArgs &a, hipStream_t st) {
    const unsigned grid = (unsigned)units_bound(a.view, a.plan);
    if (a.pairs)
        start_flash<D, kQB, W, true, EIGHT, SHARED>(a, grid, st);
    else
        start_flash<D, kQB, W, false, EIGHT, SHARED>(a, grid, st);
    return hipGetLastError();
}

template <bool EIGHT, bool SHARED>
static hipError_t launch_flash_by_dim(const PagedAttendArgs &a, int D, hipStream_t st) {
    const bool wide = a.plan.queries == 256;
    // tiles of 256: in eight waves, where those of 128 features have the registers
    if (D == 128 && wide) {
        if constexpr (EIGHT || SHARED)
            return launch_flash<128, 1, 8, EIGHT, SHARED>(a, st);
        else
            return launch_flash<128, 2, 4, EIGHT, SHARED>(a, st);
    }
    if (D == 128) return launch_flash<128, 1, 4, EIGHT, SHARED>(a, st);
    return wide ? launch_flash<64, 2, 4, EIGHT, SHARED>(a, st) : launch_flash<64, 1, 4, EIGHT, SHARED>(a, st);
}

} // namespace mukv

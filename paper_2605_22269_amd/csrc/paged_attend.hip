// Attention of new tokens over the rows of a paged cache (or of packed sequences), for any number of tokens a sequence, any payload type
// and head size.
//
//   out[token][h] = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s_j - m),  s_j = log2(e) / sqrt(D) q.k_j,  m = max_j s_j
//
// over the rows j of the token's sequence that it sees.  One pass over the rows with the running maximum and sum; rows shared by
// chunks of a sequence are joined by the last of its workgroups to finish.
#include <climits>
#include <type_traits>

#include "attend_dev.h"
#include "paged_dev.h"

namespace mukv {

namespace {

constexpr int kPQ = 16, kPWaves = 4; // queries and waves of a workgroup

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

// The rows of a tile, in blocks of 32 (bf16) or 16 (fp32), dealt to the waves in turn; nothing crosses the waves until the end.
//   rows     a lane works out where one row lives, from a table entry that was requested a block earlier; the others fetch that by
//            lane permutes.  Keys and values go straight to registers, the next block's requested as soon as this one's are used up.
//   scores   S^T = K Q^T (16x16x32 bf16, 16x16x4 fp32): a lane holds ONE query (lane % 16) and the rows 4 (lane / 16) + r of every 16.
//   values   O^T += V^T P^T: the weights are the B operand as they stand in the lane.  bf16: pairs hi + lo, 16 of the fp32
//            weight's 24 bits; the value rows pass through LDS the wave has to itself and the transpose read.  fp32: no transpose needed.
// As many workgroups to a compute unit as the registers allow (us a launch, two / as now: 100 users of 3 rows, 12 heads of 64 bf16, 13.7 / 10.2;
// 12 users, 5 tokens over 1000 to 9000 rows, 28/4 heads of 64 bf16, 26.5 / 22.3; 6 prompts of 700 to 1500 tokens, 28/4 heads of 32 bf16, 148 / 94;
// of fp32 252 / 218; 1500 tokens, 16/4 heads of 64 fp32, 103 / 92).
template <typename T, int D>
__global__ __launch_bounds__(64 * kPWaves) __attribute__((amdgpu_waves_per_eu(D <= 32 ? 4 : D == 64 ? 3 : 2, D <= 32 ? 5 : D == 64 ? 3 : 2))) void paged_attend_kernel(PagedAttendArgs a) {
    constexpr int W = kPWaves;
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int kRowB = D * (int)sizeof(T), kPieces = kRowB / 16;
    constexpr int kRows = kBf16 ? 32 : 16;             // rows of a block
    constexpr int kTiles = kRows / 16;                 // 16-row tiles of the scores
    constexpr int KK = kBf16 ? (D + 31) / 32 : D / 16; // 16-byte pieces of a key row (and of a query) per lane
    constexpr int NF = D / 16;                         // 16-feature tiles of the output
    // bf16: value pieces per lane, each load of the wave kRowsPerLoad whole rows.  fp32: per 4-row step D / 16 floats
    constexpr int kRowsPerLoad = 64 / kPieces, NV = kBf16 ? kRows / kRowsPerLoad : 4;
    constexpr int kVW = kBf16 ? 4 : (D >= 64 ? 4 : D / 16), kVH = kBf16 ? 1 : (D == 128 ? 2 : 1); // dwords per load, loads per row
    typedef __attribute__((ext_vector_type(kVW))) unsigned int raw_v;
    // per wave: staged value rows (bf16), at the end its outputs [16 queries][D]
    __shared__ __align__(1024) unsigned char s_buf[W][64 * D];
    __shared__ float s_m[W][kPQ], s_l[W][kPQ];
    constexpr bool kQueryLds = !kBf16 && D == 128; // fp32, 128 features: the queries' operands wait in LDS
    __shared__ raw16 s_q[kQueryLds ? KK : 1][kQueryLds ? 64 : 1];
    const PagedView &v = a.view;
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
    raw16 qb[kQueryLds ? 1 : KK];
    const bool has_piece = kPieces >= 4 || lg < kPieces; // (rows of 32 bytes have two pieces)
    const int my_piece = kPieces >= 4 ? lg : lg & (kPieces - 1);
    {
        const unsigned char *qp = a.q + (int64_t)(u.s.first + my_tok) * a.q_token + (int64_t)(g * G + (q_ok ? my_q - my_tok * G : 0)) * a.q_head;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kQueryLds && wave != 0) break; // the same in all waves
            raw16 x = *reinterpret_cast<const raw16 *>(qp + 16 * (my_piece + 4 * kk));
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
    auto find = [&](int blk, int page, int64_t *off, int *ft) __attribute__((always_inline)) {
        const int r = blk * kRows + (lane & (kRows - 1));
        const bool there = blk < b_hi && r < n_rows && is_page(v, page);
        *off = !there ? 0 : v.table ? offset_of(v, page, r) : (int64_t)(u.s.first + r) * v.stride_row;
        *ft = there ? (a.causal ? r - past : 0) : INT_MAX;
    };
    auto from_lane = [&](int64_t x, int from) __attribute__((always_inline)) {
        return (int64_t)((uint64_t)(unsigned)__shfl((int)(x >> 32), from) << 32 | (unsigned)__shfl((int)x, from));
    };
    auto value_row = [&](int i) { return kBf16 ? i * kRowsPerLoad + lane / kPieces : 4 * lg + i; }; // of the lane's load i
    raw16 kx[kTiles][KK];
    raw_v vx[NV][kVH];
    auto request_keys = [&](int64_t off) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const unsigned char *p = kb + from_lane(off, 16 * t + lr) + 16 * my_piece;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kx[t][kk] = *reinterpret_cast<const raw16 *>(p + 64 * kk);
        }
    };
    auto request_values = [&](int64_t off) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const unsigned char *p = vb + from_lane(off, value_row(i)) + (kBf16 ? lane % kPieces : lr) * 4 * kVW;
#pragma unroll
            for (int h = 0; h < kVH; ++h) vx[i][h] = *reinterpret_cast<const raw_v *>(p + 256 * h);
        }
    };

    float m_run = -INFINITY, l_run = 0.f; // of query lr; l_run: over the rows this lane holds
    f32x4 acc[NF]; // of query lr.  bf16: tile f, features 16 f + 4 lg + r.  fp32: tile (h, e), features 64 h + kVW (4 lg + r) + e
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
        if constexpr (kBf16) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
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
        if (late) {
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
        if constexpr (kBf16) {
            raw16 hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hi[e] = bf16_pair(p[2 * e], p[2 * e + 1]);
                lo[e] = bf16_pair(p[2 * e] - __uint_as_float(hi[e] << 16), p[2 * e + 1] - __uint_as_float(hi[e] & 0xFFFF0000u));
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int row = value_row(i);
                *reinterpret_cast<raw_v *>(buf + row * kRowB + 16 * ((lane % kPieces) ^ row_swizzle<D>(row))) = vx[i][0];
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
            if (__builtin_expect(!apart, 1)) {
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    const bf16x8 av = __builtin_bit_cast(bf16x8, values_of(f));
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
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, hi), c, 0, 0, 0);
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, lo), c, 0, 0, 0);
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
        if constexpr (kBf16) {
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
        const bool seen = l != 0.f; // no row that the query sees: zeros (a NaN or +inf score makes l a NaN, and the output with it)
        o = seen ? o / l : f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (kBf16)
            *reinterpret_cast<u32x2 *>(out + row * D + 4 * c) = u32x2{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
        else
            *reinterpret_cast<f32x4 *>(out + row * D + 4 * c) = o;
        if (a.pairs && c == 0) *reinterpret_cast<f32x2 *>(a.pairs + 2 * row) = seen ? f32x2{m, 1.f / l} : f32x2{0.f, 0.f};
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
        if (u.chunks > 1) {
            if (c == 0) store_far(a.records.stats + ((int64_t)(u.record + u.chunk) * kPQ + n) * 2, m, l);
            store_far4(chunk_values<kPQ, D>(a.records, u.record + u.chunk), n * D + 4 * c, o);
        } else {
            finish(n, c, m, l, o);
        }
    }
    if (u.chunks == 1) return;
    __shared__ int s_last;
    if (!last_to_arrive(a.counts + u.record, u.chunks, &s_last)) return;
    __shared__ float s_join[join_scratch(kPlanChunks, kPQ)];
    join_chunks<kPQ, D, 64 * W, kPlanChunks, 1, 16>(a.records, u.record, u.chunks, n_q_here, s_join, finish);
}

// What each row receives: weights_out[b][g][j] = decay * weights_in[b][g][j] + sum over the tokens and the group's heads of p_j / sum p.
// Grid (rows, sequence, KV head).  A wave keeps the keys of kTiles times 16 rows (the A operand) in registers and the sequence's queries
// stream past it, 16 at a time and requested one tile ahead, with what their weights subtract and the sum they are divided by: S^T
// leaves a lane one query and four rows of every 16, so the sums over the queries run in the lane until the end, where 16 lanes join.
template <typename T, int D, int kTiles>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) void paged_weights_kernel(PagedAttendArgs a, int n_groups) {
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int kRowB = D * (int)sizeof(T), kPieces = kRowB / 16;
    constexpr int KK = kBf16 ? (D + 31) / 32 : D / 16;
    const PagedView &v = a.view;
    const int g = blockIdx.z, b = blockIdx.y;
    const SeqShape s = shape_of(v, a.plan, b);
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4, G = v.G;
    const int n_w = s.rows < a.weights_rows ? s.rows : a.weights_rows; // rows that have a weight
    const int past = s.length - s.n_new, n_queries = s.n_new * G;
    const float scale = a.scale_log2e * (1.f / query_factor<T, D>());
    const bool has_piece = kPieces >= 4 || lg < kPieces;
    const int my_piece = kPieces >= 4 ? lg : lg & (kPieces - 1);
    constexpr int kRows = 16 * kTiles; // of a wave
    for (int r0 = kRows * ((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)); r0 < n_w; r0 += 4 * kRows * n_groups) {
        raw16 kx[kTiles][KK];
        int from[kTiles][4]; // first token that sees row 16 t + 4 lg + e
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int r = r0 + 16 * t + lr;
            const int page = r < n_w ? (v.table ? v.table[entry_of(v, b, r)] : 0) : -1;
            const bool there = is_page(v, page);
            const int64_t off = !there ? 0 : v.table ? offset_of(v, page, r) : (int64_t)(s.first + r) * v.stride_row;
            const unsigned char *kp = v.k + g * v.stride_head + off + 16 * my_piece;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                kx[t][kk] = *reinterpret_cast<const raw16 *>(kp + 64 * kk);
                if (!has_piece) kx[t][kk] = raw16{0u, 0u, 0u, 0u};
            }
            const int ft = there ? (a.causal ? r - past : 0) : INT_MAX;
#pragma unroll
            for (int e = 0; e < 4; ++e) from[t][e] = __shfl(ft, 4 * lg + e);
        }
        float sum[kTiles][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[t][e] = 0.f;
        raw16 qx[2][KK];
        f32x2 pair[2];
        int tok[2];
        auto request = [&](int q0, int at) __attribute__((always_inline)) {
            const int qq = q0 + lr < n_queries ? q0 + lr : n_queries - 1, h = g * G + qq % G;
            tok[at] = qq / G;
            const unsigned char *qp = a.q + (int64_t)(s.first + tok[at]) * a.q_token + (int64_t)h * a.q_head + 16 * my_piece;
            pair[at] = *reinterpret_cast<const f32x2 *>(a.pairs + 2 * ((int64_t)(s.first + tok[at]) * v.Hq + h));
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qx[at][kk] = *reinterpret_cast<const raw16 *>(qp + 64 * kk);
            if (q0 + lr >= n_queries) tok[at] = -1; // sees nothing
        };
        auto add = [&](int at) __attribute__((always_inline)) {
            raw16 q[KK];
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) q[kk] = has_piece ? brought_down<T, D>(qx[at][kk]) : raw16{0u, 0u, 0u, 0u};
            const float ref = pair[at][0], inv = pair[at][1];
            const bool large = __builtin_amdgcn_ballot_w64(fabsf(ref) > kLargeRef) != 0; // (its rounding shows)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 sc = {0.f, 0.f, 0.f, 0.f};
                if constexpr (kBf16) {
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
                    sum[t][e] += tok[at] >= from[t][e] && tok[at] >= 0 ? w * inv : 0.f;
                }
            }
        };
        // queries before the first row's first token see none of these rows
        int q0 = a.causal && r0 - past > 0 ? (r0 - past < s.n_new ? (r0 - past) * G & ~15 : n_queries) : 0;
        if (q0 < n_queries) request(q0, 0);
        for (; q0 < n_queries; q0 += 32) {
            if (q0 + 16 < n_queries) request(q0 + 16, 1);
            add(0);
            if (q0 + 32 < n_queries) request(q0 + 32, 0);
            if (q0 + 16 < n_queries) add(1);
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[t][e] = row16_sum(sum[t][e]);
            const int row = r0 + 16 * t + 4 * lg + (lr & 3);
            if (lr < 4 && row < n_w) {
                const int64_t at = b * a.weights_seq + g * a.weights_head + row;
                const float got = lr == 0 ? sum[t][0] : lr == 1 ? sum[t][1] : lr == 2 ? sum[t][2] : sum[t][3];
                a.weights_out[at] = a.weights_in ? fmaf(a.decay, a.weights_in[at], got) : got;
            }
        }
    }
}

template <typename T, int D, int kTiles>
hipError_t launch_weights(const PagedAttendArgs &a, hipStream_t st) {
    constexpr int kRows = 4 * 16 * kTiles; // of a workgroup
    const int64_t room = a.view.table ? room_of(a.view) : a.view.page_rows, rows = room < a.weights_rows ? room : a.weights_rows;
    int64_t groups = (rows + kRows - 1) / kRows, most = 8192 / ((int64_t)a.view.Hkv * a.view.n_seqs);
    if (most < 16) most = 16;
    if (groups > most) groups = most; // (a workgroup goes round: a table is often wider than its sequences)
    if (groups < 1) return hipSuccess;
    hipLaunchKernelGGL((paged_weights_kernel<T, D, kTiles>), dim3((unsigned)groups, a.view.n_seqs, a.view.Hkv), dim3(256), 0, st, a, (int)groups);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_typed(const PagedAttendArgs &a, hipStream_t st) {
    const unsigned grid = (unsigned)units_bound(a.view, a.plan);
    if (grid > 0) {
        hipError_t e;
        if (a.plan.queries != kPQ) {
            e = launch_paged_flash(a, D, st);
        } else {
            hipLaunchKernelGGL((paged_attend_kernel<T, D>), dim3(grid), dim3(64 * kPWaves), 0, st, a);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    if (!a.weights_out) return hipSuccess;
    // Queries that stream past are shared by the rows a wave holds; where there are few of them it is more waves that count (us a
    // launch, 16 / 64 rows a wave: 64 users, one token, 2000 rows, 64/8 heads 61 / 70; 6 users, 16 tokens, 36000 rows in all, 28/4 heads 38 / 29).
    if ((int64_t)a.view.n_tokens * a.view.G <= 32 * (int64_t)a.view.n_seqs) return launch_weights<T, D, 1>(a, st);
    return launch_weights<T, D, sizeof(T) == 2 ? 4 : 2>(a, st);
}

template <typename T>
hipError_t launch_by_dim(const PagedAttendArgs &a, int D, hipStream_t st) {
    switch (D) {
    case 16: return launch_typed<T, 16>(a, st);
    case 32: return launch_typed<T, 32>(a, st);
    case 64: return launch_typed<T, 64>(a, st);
    default: return launch_typed<T, 128>(a, st);
    }
}

} // namespace

// Which kernel takes a call, by what is known on the host; us a call, 28/4 heads of 128, what the rule takes marked.
// The kernel for any shape reads a sequence's rows once for every 16 queries of a KV head, the one for prompts once for 128 or 256, but its
// units are large and start slowly: it takes calls with more queries than that (any / prompts in tiles of 128 / of 256: one user, 16 tokens
// over 8000 rows 19.5* / 34 / 50, over 32000 59* / 58 / 87, 32 tokens over 8000 28.6* / 35 / 51, 64 tokens over 8000 52 / 36 / 52*, over 1000
// 14.0 / 19.5* / 28.8; 8 users over 8000 rows, 4 tokens 31.5* / 42 / 61, 8 tokens 55 / 42* / 61, 16 tokens 89 / 43* / 62).
// Tiles of 128 or of 256 queries: the wide ones read operands for twice the products, so they are faster where there is enough to
// do for every compute unit, and slower where a tile is half empty or the last tiles' rows are what the call waits for (128 / 256: 6
// users, 16 tokens over 3000 to 9000 rows 39* / 56; 300 tokens 14.6* / 20.2; 2000 tokens 55* / 71; 8192 tokens 650 / 493*; 1568 over 6272 rows
// 277 / 238*; 8 users, 64 tokens over 8000 rows 135 / 101*).  What a table has room for stands in for the rows that are there, which the
// host does not know: one user's 64 tokens over 8000 rows are the case above where that takes the slower tile.
int paged_prompt_tile(const PagedView &v, int dtype, int D, int64_t new_hint) {
    if (dtype != MUKV_BF16 || D < 64) return 0;
    const int64_t queries = new_hint * v.G; // of a sequence and KV head
    if (queries < 48 || (int64_t)v.n_tokens * v.Hq < 1500) return 0;
    const int64_t room = v.table ? room_of(v) : new_hint, tiles = div_up(queries, 256) * v.n_seqs * v.Hkv;
    return queries <= 128 || (tiles <= 256 && room <= 4096) ? 128 : 256;
}

PlanShape paged_plan(int dtype, int prompt_tile, bool causal) {
    PlanShape p;
    p.causal = causal;
    p.most = kPlanChunks;
    if (prompt_tile) {
        p.queries = prompt_tile;
        p.rows = 64; // a step of the workgroup
        p.records = 704;
        p.places = 256;
        p.start = 3;
        p.join = 0.8f;
        p.record = 0.06f;
    } else {
        p.queries = kPQ;
        p.rows = dtype == MUKV_BF16 ? 128 : 64; // a block of every wave
        p.records = 2048;
        p.places = 512;
        p.start = 0;
        p.join = p.record = 0.f;
    }
    p.log_queries = p.queries == 256 ? 8 : p.queries == 128 ? 7 : 4;
    p.log_rows = p.rows == 128 ? 7 : 6;
    return p;
}

hipError_t launch_paged_attend(const PagedAttendArgs &a, int D, int dtype, hipStream_t st) {
    return dtype == MUKV_BF16 ? launch_by_dim<uint16_t>(a, D, st) : launch_by_dim<float>(a, D, st);
}

} // namespace mukv

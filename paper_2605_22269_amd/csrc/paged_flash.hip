// Attention of many new tokens a sequence over a paged cache, or over packed sequences, on the matrix cores: bf16 rows of 64 or 128
// features.  The mathematics, and how rows are shared out and joined, are those of paged_attend.hip.
#include <climits>
#include <type_traits>

#include "paged_dev.h"

namespace mukv {

namespace {

constexpr int kFQ = 256, kFRows = 64, kQB = 2; // queries of a workgroup, rows of a step, blocks of 32 queries of a wave
constexpr int kRing = 8;                       // steps whose rows' places are held
constexpr float kLag = 8.f;                    // how far (in log2 units) the running maximum may be ahead of what exponents subtract

// sum of two bf16 and x, in fp32
__device__ __forceinline__ float add_pair(uint32_t pair, float x) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), bf16x2{(__bf16)1.f, (__bf16)1.f}, x, false);
}

// One workgroup of four waves per unit; a wave owns 64 queries from the scores to the output.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void paged_flash_kernel(PagedAttendArgs a) {
    using T = uint16_t;
    constexpr int kRowB = D * 2, kPieces = kRowB / 16, kRowsPerLoad = 64 / kPieces; // rows one load of a wave brings
    constexpr int kLoads = kFRows / 4 / kRowsPerLoad;                               // such loads per wave and step
    constexpr int KK = D / 16, NF = D / 32; // 16-feature steps of the scores, 32-feature blocks of the output
    constexpr int kBuf = kFRows * kRowB;
    __shared__ __align__(1024) unsigned char s_kv[5 * kBuf]; // keys of two steps, values of three
    __shared__ int64_t s_off[kRing][kFRows];                 // byte offset of a row
    __shared__ __align__(16) int s_ft[kRing][kFRows];        // first token that sees it
    __shared__ int s_masked[kRing][2];                       // some query of the tile may not see some row of that half of the step
    __shared__ int s_bad[2], s_any;
    __shared__ unsigned s_inf[2][kFQ][D / 32]; // outputs that a value of +inf, of -inf reaches (both: NaN), where s_any says so
    __shared__ int s_last;
    const PagedView &v = a.view;
    Unit u;
    if (!find_unit(v, a.plan, blockIdx.x, &u)) return;
    const int g = u.g, b = u.b, G = v.G, n_new = u.s.n_new;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, lq = lane & 31, half = lane >> 5;
    const int n_queries = n_new * G;
    const int q0 = u.tile * kFQ + 32 * kQB * wave; // the wave's first
    const float scale = a.scale_log2e;
    // the wave's queries as a matrix operand (column lane % 32, 8 features from 8 * half of every 16)
    bf16x8 qb[kQB][KK];
    int my_tok[kQB];
#pragma unroll
    for (int i = 0; i < kQB; ++i) {
        const int qq = q0 + 32 * i + lq;
        const bool ok = qq < n_queries;
        const int tok = ok ? qq / G : 0;
        my_tok[i] = ok ? tok : INT_MIN; // nothing is visible to a query that does not exist
        const unsigned char *qp = a.q + (int64_t)(u.s.first + tok) * a.q_token + (int64_t)(g * G + (ok ? qq - tok * G : 0)) * a.q_head + 16 * half;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            raw16 x = *reinterpret_cast<const raw16 *>(qp + 32 * kk);
            if (!ok) x = raw16{0u, 0u, 0u, 0u};
            qb[i][kk] = __builtin_bit_cast(bf16x8, x);
        }
    }
    const int first_tok = u.tile * kFQ / G;
    const int last_q = u.tile * kFQ + kFQ - 1 < n_queries ? u.tile * kFQ + kFQ - 1 : n_queries - 1, last_tok = last_q / G;
    const int past = u.s.length - n_new;
    int n_rows = u.s.rows;
    if (a.causal && past + last_tok + 1 < n_rows) n_rows = past + last_tok + 1 > 0 ? past + last_tok + 1 : 0;
    // the unit's steps (a step is one of the plan's blocks)
    const int all_steps = (n_rows + kFRows - 1) / kFRows;
    const int64_t lo = (int64_t)u.chunk * u.per, hi = lo + u.per;
    const int t_lo = lo < all_steps ? (int)lo : all_steps, n_steps = (hi < all_steps ? (int)hi : all_steps) - t_lo;
    const int row0 = t_lo * kFRows;                                                     // the unit's first row
    const int n_halves = n_steps == 0 ? 0 : ((row0 + n_steps * kFRows < n_rows ? row0 + n_steps * kFRows : n_rows) - row0 + 31) / 32;
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
        const int ft = there ? (a.causal ? r - past : 0) : INT_MAX;
        s_ft[t & (kRing - 1)][lane] = ft;
        const uint64_t late = __builtin_amdgcn_ballot_w64(ft > first_tok);
        if (lane < 2) s_masked[t & (kRing - 1)][lane] = (uint32_t)(late >> (32 * lane)) != 0u;
    };
    // A wave brings rows 16 wave .. 16 wave + 15 of a step, kRowsPerLoad at a time.  A row's 16-byte pieces are stored permuted, so
    // that neither the reads of key operands nor the transpose reads of values meet in a bank.
    const int ld_row = 16 * wave + lane / kPieces, ld_piece = lane % kPieces;
    const unsigned char *k_from[kLoads], *v_from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        k_from[i] = kb + 16 * key_slot<D>(ld_piece, ld_row + i * kRowsPerLoad);
        v_from[i] = vb + 16 * val_slot<D>(ld_piece, ld_row + i * kRowsPerLoad);
    }
    auto request = [&](int t) __attribute__((always_inline)) { // the rows of step t
        if (t >= n_steps) return;
        unsigned char *const dk = s_kv + (t & 1) * kBuf, *const dv = s_kv + (2 + t % 3) * kBuf;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int64_t off = s_off[t & (kRing - 1)][ld_row + i * kRowsPerLoad];
            const int lds = (16 * wave + i * kRowsPerLoad) * kRowB; // the wave's 1024 bytes, lane order
            load_to_lds(k_from[i] + off, dk + lds);
            load_to_lds(v_from[i] + off, dv + lds);
        }
    };

    // ---- state ----
    float ref[kQB], l_run[kQB]; // what exponents subtract; sum of the weights over the rows this lane holds
    f32x16 o[kQB][NF];          // features 32 f + 8 (j / 4) + 4 half + j % 4 of query lq
    f32x16 sc[2][kQB];          // scores of two halves of a step: rows 8 (j / 4) + 4 half + j % 4
    float s_scale[kQB], s_ref[kQB]; // a weight is 2^(score * s_scale - s_ref)
#pragma unroll
    for (int i = 0; i < kQB; ++i) {
        ref[i] = -INFINITY;
        l_run[i] = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][f][j] = 0.f;
    }
    int koff[KK]; // this lane's key operand of 16-feature step kk in a half of a staged step
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) koff[kk] = lq * kRowB + 16 * key_slot<D>(2 * kk + half, lq);
    // its value operand of feature block f: rows 4 half + (lane % 16) / 4 and 8 later of every 16, 4 features
    int voff[NF][2];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        const int row = 4 * half + ((lane & 15) >> 2), piece = 4 * f + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), sub = 8 * (lane & 1);
        voff[f][0] = row * kRowB + 16 * val_slot<D>(piece, row) + sub;
        voff[f][1] = (row + 8) * kRowB + 16 * val_slot<D>(piece, row + 8) + sub;
    }
    auto keys_of = [&](int h) { return s_kv + (h >> 1 & 1) * kBuf + (h & 1) * 32 * kRowB; };
    auto values_of = [&](int h) { return s_kv + (2 + (h >> 1) % 3) * kBuf + (h & 1) * 32 * kRowB; };
    auto load_k = [&](const unsigned char *ks, int kk) { return *reinterpret_cast<const bf16x8 *>(ks + koff[kk]); };
    auto load_v = [&](const unsigned char *vs, int grp, int f) { // of 16 rows
        const i16x4 x = lds_read_tr16(vs + grp * 16 * kRowB + voff[f][0]), y = lds_read_tr16(vs + grp * 16 * kRowB + voff[f][1]);
        return i16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    };
    // weights of query block i and 16 rows as a matrix operand
    auto weights_of = [&](const f32x16 &s, int i, int grp, float *sum) __attribute__((always_inline)) {
        raw16 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[8 * grp + 2 * e], s_scale[i], -s_ref[i]));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[8 * grp + 2 * e + 1], s_scale[i], -s_ref[i]));
            w[e] = bf16_pair(x, y);
            *sum = add_pair(w[e], *sum); // (the weights as they enter the product: a row that has nearly all of it keeps its value)
        }
        return __builtin_bit_cast(bf16x8, w);
    };

    // ---- the scores of half h are there: mask, maximum, what the exponents subtract ----
    auto look = [&](auto par, int h) __attribute__((always_inline)) {
        constexpr int P = par.value;
        const int slot = (h >> 1) & (kRing - 1);
        const bool masked = __builtin_amdgcn_readfirstlane(s_masked[slot][h & 1]) != 0;
        if (masked) {
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                const i32x4 ft = *reinterpret_cast<const i32x4 *>(&s_ft[slot][32 * (h & 1) + 8 * jj + 4 * half]);
#pragma unroll
                for (int i = 0; i < kQB; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[P][i][4 * jj + r] = my_tok[i] >= ft[r] ? sc[P][i][4 * jj + r] : -INFINITY;
            }
        }
        float mx[kQB];
        bool ahead = false, large = false;
#pragma unroll
        for (int i = 0; i < kQB; ++i) {
            float m4[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) m4[c] = fmaxf(fmaxf(sc[P][i][c], sc[P][i][4 + c]), sc[P][i][8 + c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) m4[c] = fmaxf(m4[c], sc[P][i][12 + c]);
            mx[i] = half_max(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]))) * scale;
            ahead |= mx[i] > ref[i] + kLag;
        }
        if (__builtin_amdgcn_ballot_w64(ahead) != 0) { // bring what was summed to the new maximum
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
                const float to = mx[i] > ref[i] + kLag ? mx[i] : ref[i];
                const float corr = __builtin_amdgcn_exp2f(ref[i] - (to == -INFINITY ? 0.f : to));
                ref[i] = to;
                l_run[i] *= corr;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][f][j] *= corr;
            }
        }
#pragma unroll
        for (int i = 0; i < kQB; ++i) {
            s_scale[i] = scale;
            s_ref[i] = ref[i] == -INFINITY ? 0.f : ref[i];
            large |= fabsf(s_ref[i]) > kLargeRef;
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(large) != 0, 0)) { // so large that the product's rounding shows
#pragma unroll
            for (int i = 0; i < kQB; ++i) {
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[P][i][j] = scaled_apart(sc[P][i][j], s_scale[i], s_ref[i]);
                s_scale[i] = 1.f;
                s_ref[i] = 0.f;
            }
        }
        // A value that is no number must not reach a token that does not see its row: the weight is zero, the product is not.
        if (masked) {
            unsigned char *const vs = values_of(h);
            const raw16 *own = reinterpret_cast<const raw16 *>(vs + wave * 8 * kRowB);
            unsigned worst = 0;
#pragma unroll
            for (int i = 0; i < 8 * kPieces / 64; ++i) {
                const raw16 x = own[lane + 64 * i];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned upper = x[e] & 0x7F800000u, lower = (x[e] & 0x7F80u) << 16;
                    worst = worst > upper ? worst : upper;
                    worst = worst > lower ? worst : lower;
                }
            }
            if (8 * kPieces < 64 && lane >= 8 * kPieces) worst = 0;
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
                        const float w = __builtin_amdgcn_exp2f(fmaf(sc[P][i][j], s_scale[i], -s_ref[i]));
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
                for (int i = tid; i < 32 * D; i += 256) {
                    uint16_t *const x = reinterpret_cast<uint16_t *>(vs) + i;
                    if ((*x & 0x7F80u) == 0x7F80u) *x = 0;
                }
                if (tid == 0) {
                    s_bad[h & 1] = 0;
                    s_any = 1;
                }
                __syncthreads();
            }
        }
    };

    // Half h: its weights and values, and the scores of half h + 1 between them.
    auto step = [&](auto par, int h) __attribute__((always_inline)) {
        constexpr int P = par.value;
        if constexpr (P == 1) { // the rows of the next step are there; the next but one's take the place of this one's keys
            rows_landed();
            __syncthreads();
            const int t = h >> 1;
            request(t + 2);
        }
        const unsigned char *const ks = keys_of(h + 1), *const vs = values_of(h); // (past the last half: whatever is there)
        f32x16 *const cur = sc[P], *const nxt = sc[1 - P];
#pragma unroll
        for (int i = 0; i < kQB; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) nxt[i][j] = 0.f;
        bf16x8 pw[2][kQB], ak[2], av[2][NF];
        ak[0] = load_k(ks, 0);
#pragma unroll
        for (int kk = 0; kk < KK / 2; ++kk) { // weights of the first 16 rows beside the first features of the scores
            ak[(kk + 1) & 1] = load_k(ks, kk + 1);
            if (kk >= KK / 2 - 2) {
#pragma unroll
                for (int f = 0; f < NF / 2; ++f) av[0][NF / 2 * (kk - KK / 2 + 2) + f] = __builtin_bit_cast(bf16x8, load_v(vs, 0, NF / 2 * (kk - KK / 2 + 2) + f));
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kQB; ++i) nxt[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[kk & 1], qb[i][kk], nxt[i], 0, 0, 0);
            if (kk % (KK / 4) == 0) pw[0][kk / (KK / 4)] = weights_of(cur[kk / (KK / 4)], kk / (KK / 4), 0, &l_run[kk / (KK / 4)]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int kk = KK / 2; kk < KK; ++kk) { // weights of the other 16 beside the other features and the first rows' values
            if (kk + 1 < KK) ak[(kk + 1) & 1] = load_k(ks, kk + 1);
            const int s = kk - KK / 2;
            if (s >= KK / 2 - 2) {
#pragma unroll
                for (int f = 0; f < NF / 2; ++f) av[1][NF / 2 * (s - KK / 2 + 2) + f] = __builtin_bit_cast(bf16x8, load_v(vs, 1, NF / 2 * (s - KK / 2 + 2) + f));
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kQB; ++i) nxt[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[kk & 1], qb[i][kk], nxt[i], 0, 0, 0);
            {
                const int f = s; // KK / 2 == NF
#pragma unroll
                for (int i = 0; i < kQB; ++i) o[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[0][f], pw[0][i], o[i][f], 0, 0, 0);
            }
            if (s % (KK / 4) == 0) pw[1][s / (KK / 4)] = weights_of(cur[s / (KK / 4)], s / (KK / 4), 1, &l_run[s / (KK / 4)]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < kQB; ++i) o[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[1][f], pw[1][i], o[i][f], 0, 0, 0);
    };

    if (n_halves > 0) {
        if (tid < 2) s_bad[tid] = 0;
        if (tid == 0) s_any = 0;
        for (int i = tid; i < 2 * kFQ * (D / 32); i += 256) (&s_inf[0][0][0])[i] = 0u;
        {
            const int p0 = page_at(wave), p1 = page_at(wave + 4);
            tabulate(wave, p0);
            tabulate(wave + 4, p1);
        }
        int page = page_at(wave + 8);
        __syncthreads();
        request(0);
        request(1);
        rows_landed();
        __syncthreads();
        {
            const unsigned char *const ks = keys_of(0);
#pragma unroll
            for (int i = 0; i < kQB; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[0][i][j] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int i = 0; i < kQB; ++i) sc[0][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(load_k(ks, kk), qb[i][kk], sc[0][i], 0, 0, 0);
        }
        look(std::integral_constant<int, 0>{}, 0);
        for (int h = 0; h < n_halves; h += 2) {
            step(std::integral_constant<int, 0>{}, h);
            if (h + 1 >= n_halves) break;
            look(std::integral_constant<int, 1>{}, h + 1);
            step(std::integral_constant<int, 1>{}, h + 1);
            if (h + 2 >= n_halves) break;
            look(std::integral_constant<int, 0>{}, h + 2);
            // places of the steps up to this one are free: four new ones every four steps (which are read from two steps on)
            const int t = h >> 1;
            if ((t & 3) == 3) {
                tabulate(t + 5 + wave, page);
                page = page_at(t + 9 + wave);
            }
        }
    }
    // ---- results ----
    T *const out = static_cast<T *>(a.out);
#pragma unroll
    for (int i = 0; i < kQB; ++i) {
        const float l_sum = half_sum(l_run[i]);
        const int qq = q0 + 32 * i + lq;
        const bool ok = qq < n_queries;
        if (n_halves > 0 && __builtin_expect(s_any != 0, 0)) {
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
        if (u.chunks > 1) { // the chunk's record: [0] what exponents subtracted, [1] sum of the weights, [2..] unnormalised output
            if (!ok) continue;
            float *rec = a.records + ((int64_t)(u.record + u.chunk) * kFQ + (qq - u.tile * kFQ)) * (D + 2);
            if (half == 0) store_far(rec, ref[i] == -INFINITY ? 0.f : ref[i], l_sum);
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) store_far(rec + 2 + 32 * f + 8 * jj + 4 * half + r, o[i][f][4 * jj + r], o[i][f][4 * jj + r + 1]);
        } else {
            const bool seen = l_sum != 0.f; // a query that saw nothing gets zeros; NaN stays NaN
            const float inv = 1.f / l_sum;
            const int tok = ok ? my_tok[i] : 0;
            T *const op = out + ((int64_t)(u.s.first + tok) * v.Hq + g * G + (ok ? qq - tok * G : 0)) * D + 8 * half;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int jj = 0; jj < 4; jj += 2) { // a lane holds features 8 jj + 4 half .. + 3: the halves swap, and it stores 16 bytes
                    raw16 w;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t pk[2];
#pragma unroll
                        for (int x = 0; x < 2; ++x) pk[x] = bf16_pair(o[i][f][4 * (jj + x) + 2 * e] * inv, o[i][f][4 * (jj + x) + 2 * e + 1] * inv);
                        auto sw = __builtin_amdgcn_permlane32_swap(pk[0], pk[1], false, false);
                        w[e] = sw[0];
                        w[2 + e] = sw[1];
                    }
                    if (!seen) w = raw16{0u, 0u, 0u, 0u};
                    if (ok) *reinterpret_cast<raw16 *>(op + 32 * f + 8 * jj) = w;
                }
        }
    }
    if (u.chunks == 1) return;
    // ---- the chunks' records: the last workgroup of the tile to get here joins them, in their order ----
    if (!last_to_arrive(a.counts + u.record, u.chunks, &s_last)) return;
    constexpr int kQuads = D / 4;
    const int n_q_here = n_queries - u.tile * kFQ < kFQ ? n_queries - u.tile * kFQ : kFQ;
    for (int i = tid; i < n_q_here * kQuads; i += 256) {
        const int n = i / kQuads, c = i - n * kQuads, qq = u.tile * kFQ + n, tok = qq / G;
        const float *rec = a.records + ((int64_t)u.record * kFQ + n) * (D + 2);
        constexpr int64_t kNext = (int64_t)kFQ * (D + 2);
        constexpr int kAhead = 4; // records requested together
        float m = -INFINITY, l = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int s0 = 0; s0 < u.chunks; s0 += kAhead) {
            f32x2 st[kAhead], x0[kAhead], x1[kAhead];
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
                if (s0 + s >= u.chunks) break;
                st[s] = load_far(rec + (s0 + s) * kNext);
                x0[s] = load_far(rec + (s0 + s) * kNext + 2 + 4 * c);
                x1[s] = load_far(rec + (s0 + s) * kNext + 4 + 4 * c);
            }
            float m_new = m;
#pragma unroll
            for (int s = 0; s < kAhead; ++s)
                if (s0 + s < u.chunks && st[s][1] != 0.f) m_new = fmaxf(m_new, st[s][0]);
            const float corr = l != 0.f ? __builtin_amdgcn_exp2f(m - m_new) : 0.f;
            l *= corr;
            x *= corr;
            m = m_new;
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
                if (s0 + s >= u.chunks) break;
                if (st[s][1] == 0.f) continue; // none of its rows is seen
                const float y = __builtin_amdgcn_exp2f(st[s][0] - m);
                l = fmaf(st[s][1], y, l);
                x = f32x4{fmaf(x0[s][0], y, x[0]), fmaf(x0[s][1], y, x[1]), fmaf(x1[s][0], y, x[2]), fmaf(x1[s][1], y, x[3])};
            }
        }
        x = l != 0.f ? x / l : f32x4{0.f, 0.f, 0.f, 0.f};
        *reinterpret_cast<u32x2 *>(out + ((int64_t)(u.s.first + tok) * v.Hq + g * G + (qq - tok * G)) * D + 4 * c) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    }
}

} // namespace

hipError_t launch_paged_flash(const PagedAttendArgs &a, int D, hipStream_t st) {
    const unsigned grid = (unsigned)units_bound(a.view, a.plan);
    if (D == 128)
        hipLaunchKernelGGL((paged_flash_kernel<128>), dim3(grid), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((paged_flash_kernel<64>), dim3(grid), dim3(256), 0, st, a);
    return hipGetLastError();
}

} // namespace mukv

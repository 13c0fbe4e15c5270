// The way of new rows into a paged cache of 8 bits, and back (eight_dev.h says what a row is held as).
//
// Both kernels only move rows: what bounds them is memory, and a launch where there are few rows.  Of a row that is written a lane has 8
// neighbouring features, D / 8 neighbouring lanes the row, so a row's largest feature takes log2(D / 8) exchanges between lanes and its codes leave
// as one line of 8 bytes a lane.  A pair's other feature, where halves are rotated, is in the lane n_rot / 16 further on.
#include <climits>

#include "eight_dev.h"
#include "rope_dev.h"

namespace mukv {

namespace {

constexpr int kThreads = 256;
constexpr int kWriteTokens = 4;  // most tokens of a workgroup that writes
constexpr int kReadTokens = 64;  // of one that reads
constexpr int kAhead = 4;        // pieces a thread requests at a time

// The rows of tokens t0 .. t0 + nt - 1 (at most 64), by one wave, lane t token t0 + t: byte offset of the row in the pages and of its
// scale in theirs, -1 if it has none.
__device__ __forceinline__ void places_of(const PagedView &v, int t0, int nt, int64_t *place, int64_t *scale_place) {
    const int lane = threadIdx.x & 63, tok = t0 + lane;
    int b = 0;
    if (v.offsets) { // the last sequence that starts at or before the token: as many start there, or before, but the first
        for (int b0 = 1; b0 < v.n_seqs; b0 += 64) {
            const int starts = b0 + lane < v.n_seqs ? v.offsets[b0 + lane] : INT_MAX;
            for (int t = 0; t < nt; ++t) {
                const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(starts <= t0 + t));
                if (lane == t) b += n;
            }
            if (__builtin_amdgcn_readlane(starts, 63) >= t0 + nt) break; // (where offsets ascend, none of the others counts)
        }
    } else if (v.per_seq > 0) {
        b = tok / v.per_seq;
    }
    *place = *scale_place = -1;
    if (lane >= nt || b >= v.n_seqs) return;
    int first, count;
    tokens_of(v, b, &first, &count);
    const int i = tok - first, length = length_of(v, b, count), row = length - count + i;
    if (i < 0 || i >= count || row < 0 || row >= rows_of(v, first, length)) return;
    const int page = v.table[entry_of(v, b, row)];
    if (!is_page(v, page)) return;
    *place = offset_of(v, page, row);
    *scale_place = scale_offset_of(v, page, row);
}

// Keys and values come first and are requested before anything is worked out; queries, of which there are more, go on as they would to a
// cache of 16 bits, both features of a pair in one lane (1568 tokens, 28/4 heads of 128: 8.3 us a call; all rows alike 14.1).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void write8_kernel(RopeArgs a, int per_wg) {
    constexpr int L = D / 8, N = (int)sizeof(T) / 2; // lanes of a row, 16-byte pieces of a lane's features
    constexpr int kAtOnce = kThreads / L;            // rows
    constexpr int E = 16 / (int)sizeof(T);           // features of a piece
    __shared__ float2 s_turn[kWriteTokens][D / 2];
    __shared__ int64_t s_place[kWriteTokens], s_scale[kWriteTokens];
    const int tid = threadIdx.x, piece = tid % L;
    const int t0 = blockIdx.x * per_wg, nt = a.n_tokens - t0 < per_wg ? a.n_tokens - t0 : per_wg;
    const int n_pairs = a.rotate ? a.n_rot / 2 : 0;
    const int heads = a.k.heads, rows_per = 2 * heads, n_rows = nt * rows_per;
    constexpr int kRounds = 2; // of keys and values, requested together
    raw16 x[kRounds][N];
    auto request = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRounds; ++u) {
            const int r = r0 + u * kAtOnce + tid / L;
            if (r >= n_rows) continue;
            const int t = r / rows_per, h = r - t * rows_per;
            const RopeArgs::Rows &m = h < heads ? a.k : a.v;
            const unsigned char *p = m.x + (int64_t)(t0 + t) * m.token + (h < heads ? h : h - heads) * m.head + piece * 16 * N;
#pragma unroll
            for (int n = 0; n < N; ++n) x[u][n] = *reinterpret_cast<const raw16 *>(p + 16 * n);
        }
    };
    request(0);
    // queries: the first `joint` items of a row are two pieces half a rotated part apart, the others one piece
    const int joint = a.neighbours ? 0 : n_pairs / E, items = D / E - joint;
    const int q_rows = nt * a.q.heads, q_at_once = kThreads / items, my_item = tid % items, my_first = tid < q_at_once * items ? tid / items : q_rows;
    const bool both = my_item < joint;
    raw16 qx[kAhead], qy[kAhead];
    auto request_queries = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + my_first + u * q_at_once;
            if (r >= q_rows) break;
            const int t = r / a.q.heads, h = r - t * a.q.heads;
            const unsigned char *p = a.q.x + (int64_t)(t0 + t) * a.q.token + h * a.q.head;
            qx[u] = *reinterpret_cast<const raw16 *>(p + 16 * (both ? my_item : my_item + joint));
            if (both) qy[u] = *reinterpret_cast<const raw16 *>(p + 16 * (my_item + joint));
        }
    };
    request_queries(0);
    if (tid >= kThreads - 64) { // the last wave, beside the first one's cosines
        int64_t place, scale;
        places_of(a.view, t0, nt, &place, &scale);
        const int lane = tid & 63;
        if (lane < nt) {
            s_place[lane] = place;
            s_scale[lane] = scale;
        }
    }
    for (int i = tid; i < nt * n_pairs; i += kThreads) {
        const int t = i / n_pairs, p = i - t * n_pairs;
        s_turn[t][p] = turn_of(a, t0 + t, p);
    }
    __syncthreads();
    for (int r0 = 0; r0 < n_rows; r0 += kRounds * kAtOnce) { // (the same rounds in all threads: lanes exchange what they have)
        if (r0 > 0) request(r0);
#pragma unroll
        for (int u = 0; u < kRounds; ++u) {
            if (r0 + u * kAtOnce >= n_rows) break;
            const int r = r0 + u * kAtOnce + tid / L;
            const int t = r < n_rows ? r / rows_per : 0, h = r < n_rows ? r - t * rows_per : heads;
            const bool is_k = h < heads, turned = is_k && 8 * piece < 2 * n_pairs;
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = piece_get<T>(x[u][e / E], e % E);
            if (a.neighbours) {
                if (turned)
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float2 c = s_turn[t][4 * piece + e / 2];
                        const float y0 = f[e] * c.x - f[e + 1] * c.y, y1 = f[e + 1] * c.x + f[e] * c.y;
                        f[e] = y0;
                        f[e + 1] = y1;
                    }
            } else if (n_pairs > 0) {
                const bool upper = 8 * piece >= n_pairs; // of the rotated half
                const int away = n_pairs / 8;            // lanes
                const int other = (tid & 63) + (turned ? upper ? -away : away : 0);
                raw16 y[N];
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int w = 0; w < 4; ++w) y[n][w] = (unsigned)__shfl((int)x[u][n][w], other);
                if (turned)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 c = s_turn[t][8 * piece + e - (upper ? n_pairs : 0)];
                        const float g = piece_get<T>(y[e / E], e % E);
                        f[e] = upper ? f[e] * c.x + g * c.y : f[e] * c.x - g * c.y;
                    }
            }
            // the row's largest finite feature
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fabsf(f[e]) < INFINITY ? fmaxf(most, fabsf(f[e])) : most;
#pragma unroll
            for (int m = 1; m < L; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
            if (r >= n_rows || s_place[t] < 0) continue;
            const int g = is_k ? h : h - heads;
            const int byte = scale_byte(most);
            const float by = inverse_scale((uint32_t)byte);
            const u32x2 w = {codes_of(f[0] * by, f[1] * by, f[2] * by, f[3] * by), codes_of(f[4] * by, f[5] * by, f[6] * by, f[7] * by)};
            unsigned char *p = (is_k ? a.view.k : a.view.v) + s_place[t] + g * a.view.stride_head + 8 * piece;
            __builtin_nontemporal_store(w, reinterpret_cast<u32x2 *>(p));
            if (piece == 0) ((is_k ? a.view.scales.k : a.view.scales.v) + s_scale[t] + g * a.view.scales.stride_head)[0] = (unsigned char)byte;
        }
    }
    for (int r0 = 0; r0 < q_rows; r0 += kAhead * q_at_once) {
        if (r0 > 0) request_queries(r0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + my_first + u * q_at_once;
            if (r >= q_rows) break;
            const int t = r / a.q.heads, h = r - t * a.q.heads;
            unsigned char *p = a.q.out + (int64_t)(t0 + t) * a.q.out_token + h * a.q.out_head;
            if (both) {
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 c0 = s_turn[t][E * my_item + e], c1 = s_turn[t][E * my_item + e + 1];
                    const float x0 = piece_get<T>(qx[u], e), y0 = piece_get<T>(qy[u], e), x1 = piece_get<T>(qx[u], e + 1), y1 = piece_get<T>(qy[u], e + 1);
                    piece_put<T>(qx[u], e, x0 * c0.x - y0 * c0.y, x1 * c1.x - y1 * c1.y);
                    piece_put<T>(qy[u], e, y0 * c0.x + x0 * c0.y, y1 * c1.x + x1 * c1.y);
                }
                put_piece(p + 16 * my_item, qx[u]);
                put_piece(p + 16 * (my_item + joint), qy[u]);
                continue;
            }
            if (a.neighbours && E * my_item < 2 * n_pairs) {
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 c = s_turn[t][(E * my_item + e) / 2];
                    const float x0 = piece_get<T>(qx[u], e), y0 = piece_get<T>(qx[u], e + 1);
                    piece_put<T>(qx[u], e, x0 * c.x - y0 * c.y, y0 * c.x + x0 * c.y);
                }
            }
            put_piece(p + 16 * (my_item + joint), qx[u]);
        }
    }
}

// Rows of the sequences' last tokens as they were written: k.out and v.out [token][head][D].  A row that does not exist is zeros.  A lane writes one
// piece, so that neighbouring lanes' are neighbours in memory.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void read8_kernel(RopeArgs a, int per_wg) {
    constexpr int E = 16 / (int)sizeof(T), L = D / E, kAtOnce = kThreads / L; // features of a lane, lanes of a row, rows
    __shared__ int64_t s_place[kReadTokens], s_scale[kReadTokens];
    const int tid = threadIdx.x, piece = tid % L;
    const int t0 = blockIdx.x * per_wg, nt = a.n_tokens - t0 < per_wg ? a.n_tokens - t0 : per_wg;
    if (tid < 64) {
        int64_t place, scale;
        places_of(a.view, t0, nt, &place, &scale);
        if (tid < nt) {
            s_place[tid] = place;
            s_scale[tid] = scale;
        }
    }
    __syncthreads();
    const int heads = a.k.heads, rows_per = 2 * heads, n_rows = nt * rows_per;
    for (int r0 = tid / L; r0 < n_rows; r0 += kAhead * kAtOnce) {
        uint32_t x[kAhead][E / 4];
        uint32_t byte[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + u * kAtOnce;
#pragma unroll
            for (int w = 0; w < E / 4; ++w) x[u][w] = 0u;
            byte[u] = 127u;
            if (r >= n_rows) continue;
            const int t = r / rows_per, h = r - t * rows_per, g = h < heads ? h : h - heads;
            if (s_place[t] < 0) continue;
            const unsigned char *p = (h < heads ? a.view.k : a.view.v) + s_place[t] + g * a.view.stride_head + E * piece;
            if constexpr (E == 8) {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
                x[u][0] = w[0];
                x[u][1] = w[1];
            } else {
                x[u][0] = *reinterpret_cast<const uint32_t *>(p);
            }
            byte[u] = ((h < heads ? a.view.scales.k : a.view.scales.v) + s_scale[t] + g * a.view.scales.stride_head)[0];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + u * kAtOnce;
            if (r >= n_rows) continue;
            const int t = r / rows_per, h = r - t * rows_per, g = h < heads ? h : h - heads;
            const RopeArgs::Rows &m = h < heads ? a.k : a.v;
            unsigned char *p = m.out + (int64_t)(t0 + t) * m.out_token + g * m.out_head + 16 * piece;
            const float scale = scale_of(byte[u]);
            if constexpr (E == 8)
                put_piece(p, bf16_piece(x[u][0], x[u][1], scale));
            else
                put_piece(p, f32_piece(x[u][0], scale));
        }
    }
}

template <typename T, int D>
hipError_t launch_typed(const RopeArgs &a, bool read, hipStream_t st) {
    int per_wg;
    if (read) {
        per_wg = a.n_tokens / 2048;
        per_wg = per_wg < 1 ? 1 : per_wg > kReadTokens ? kReadTokens : per_wg;
    } else {
        per_wg = a.n_tokens / 768;
        per_wg = per_wg < 1 ? 1 : per_wg > kWriteTokens ? kWriteTokens : per_wg;
    }
    const unsigned grid = (unsigned)((a.n_tokens + per_wg - 1) / per_wg);
    if (read)
        hipLaunchKernelGGL((read8_kernel<T, D>), dim3(grid), dim3(kThreads), 0, st, a, per_wg);
    else
        hipLaunchKernelGGL((write8_kernel<T, D>), dim3(grid), dim3(kThreads), 0, st, a, per_wg);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_by_dim(const RopeArgs &a, bool read, hipStream_t st) {
    switch (a.D) {
    case 16: return launch_typed<T, 16>(a, read, st);
    case 32: return launch_typed<T, 32>(a, read, st);
    case 64: return launch_typed<T, 64>(a, read, st);
    default: return launch_typed<T, 128>(a, read, st);
    }
}

} // namespace

hipError_t launch_rows8(const RopeArgs &a, int dtype, bool read, hipStream_t st) {
    return dtype == MUKV_BF16 ? launch_by_dim<uint16_t>(a, read, st) : launch_by_dim<float>(a, read, st);
}

} // namespace mukv

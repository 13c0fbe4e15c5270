// Rotary positions with several axes, and the way of new rows into a paged cache.
//
// Pair i of a token turns by angle(token, i) = position[axis[i]][token] * inv_freq[i].  What all heads of a token share -- cosine and
// sine of its pairs, the row of the cache it becomes -- is worked out once a workgroup, in LDS; the rows themselves go from memory to
// memory in 16-byte pieces, both pieces of a pair in one thread.
// The angle in turns, position * inv_freq / 2 pi, is formed and reduced in 64 bits: at position 10^6 fp32 would be off by 0.06 rad.
#include "rope_dev.h"

namespace mukv {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;   // most tokens of a workgroup
constexpr int kRopePairs = 256;  // most pairs of a head
constexpr int kRopeAhead = 4;    // rows a thread requests at a time

template <typename T, bool NEIGHBOURS>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a, int per_wg) {
    constexpr int E = 16 / (int)sizeof(T); // elements of a piece
    __shared__ float2 s_turn[kRopeTokens][kRopePairs];
    __shared__ int64_t s_place[kRopeTokens]; // byte offset of the token's row in the pages, -1: it has none
    const int tid = threadIdx.x;
    const int t0 = blockIdx.x * per_wg, nt = a.n_tokens - t0 < per_wg ? a.n_tokens - t0 : per_wg;
    const int n_pairs = a.rotate ? a.n_rot / 2 : 0;
    // HALVES: the first `joint` items of a row are two pieces half a rotated part apart, the others one piece that is only moved
    const int joint = NEIGHBOURS ? 0 : n_pairs / E, items = a.D / E - joint;
    const int rows_per = a.q.heads + a.k.heads, n_rows = nt * rows_per;
    const int at_once = kRopeThreads / items, my_item = tid % items, my_first = tid < at_once * items ? tid / items : n_rows;
    const int v_items = a.D / E, v_at_once = kRopeThreads / v_items, v_item = tid % v_items;
    const int n_v = nt * a.v.heads, v_first = tid < v_at_once * v_items ? tid / v_items : n_v;

    auto worked_out = [&]() {
        for (int i = tid; i < nt * n_pairs; i += kRopeThreads) {
            const int t = i / n_pairs, p = i - t * n_pairs;
            s_turn[t][p] = turn_of(a, t0 + t, p);
        }
    };
    // by the last wave, beside the first one's cosines
    auto placed = [&]() {
        const int mine = tid - (kRopeThreads - 64);
        if (mine >= 0 && mine < nt && a.v.heads) {
            const PagedView &v = a.view;
            const int tok = t0 + mine;
            int b;
            if (v.offsets) { // the last sequence that starts at or before the token
                int lo = 0, hi = v.n_seqs - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if (v.offsets[mid] <= tok)
                        lo = mid;
                    else
                        hi = mid - 1;
                }
                b = lo;
            } else {
                b = tok / v.per_seq;
            }
            int first, count;
            tokens_of(v, b, &first, &count);
            const int i = tok - first, length = length_of(v, b, count), row = length - count + i;
            int64_t place = -1;
            if (i >= 0 && i < count && row >= 0 && row < rows_of(v, first, length)) {
                const int page = v.table[entry_of(v, b, row)];
                if (is_page(v, page)) place = offset_of(v, page, row);
            }
            s_place[mine] = place;
        }
    };

    raw16 vx;
    if (v_first < n_v) { // (one row a thread is what most calls have)
        const int t = v_first / a.v.heads, h = v_first - t * a.v.heads;
        vx = *reinterpret_cast<const raw16 *>(a.v.x + (t0 + t) * a.v.token + h * a.v.head + 16 * v_item);
    }
    for (int r0 = 0;; r0 += kRopeAhead * at_once) {
        raw16 x[kRopeAhead], y[kRopeAhead];
#pragma unroll
        for (int u = 0; u < kRopeAhead; ++u) {
            const int r = r0 + my_first + u * at_once;
            if (r >= n_rows) break;
            const int t = r / rows_per, h = r - t * rows_per;
            const bool is_q = h < a.q.heads;
            const unsigned char *p = (is_q ? a.q.x + (t0 + t) * a.q.token + h * a.q.head : a.k.x + (t0 + t) * a.k.token + (h - a.q.heads) * a.k.head);
            const bool pair = my_item < joint;
            x[u] = *reinterpret_cast<const raw16 *>(p + 16 * (pair ? my_item : my_item + joint));
            if (pair) y[u] = *reinterpret_cast<const raw16 *>(p + 16 * (my_item + joint));
        }
        if (r0 == 0) {
            placed();
            worked_out();
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kRopeAhead; ++u) {
            const int r = r0 + my_first + u * at_once;
            if (r >= n_rows) break;
            const int t = r / rows_per, h = r - t * rows_per;
            const bool is_q = h < a.q.heads, pair = my_item < joint;
            const int64_t place = is_q ? 0 : s_place[t];
            if (place < 0) continue;
            unsigned char *p = is_q ? a.q.out + (t0 + t) * a.q.out_token + h * a.q.out_head
                                    : a.view.k + place + (h - a.q.heads) * a.view.stride_head;
            if (pair) {
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 c0 = s_turn[t][E * my_item + e], c1 = s_turn[t][E * my_item + e + 1];
                    const float x0 = piece_get<T>(x[u], e), y0 = piece_get<T>(y[u], e), x1 = piece_get<T>(x[u], e + 1), y1 = piece_get<T>(y[u], e + 1);
                    piece_put<T>(x[u], e, x0 * c0.x - y0 * c0.y, x1 * c1.x - y1 * c1.y);
                    piece_put<T>(y[u], e, y0 * c0.x + x0 * c0.y, y1 * c1.x + x1 * c1.y);
                }
                put_piece(p + 16 * my_item, x[u]);
                put_piece(p + 16 * (my_item + joint), y[u]);
            } else {
                if (NEIGHBOURS && E * my_item < 2 * n_pairs) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const float2 c = s_turn[t][(E * my_item + e) / 2];
                        const float x0 = piece_get<T>(x[u], e), y0 = piece_get<T>(x[u], e + 1);
                        piece_put<T>(x[u], e, x0 * c.x - y0 * c.y, y0 * c.x + x0 * c.y);
                    }
                }
                put_piece(p + 16 * (my_item + joint), x[u]);
            }
        }
        if (r0 + kRopeAhead * at_once >= n_rows) break;
    }
    for (int r = v_first; r < n_v; r += v_at_once) {
        const int t = r / a.v.heads, h = r - t * a.v.heads;
        if (r != v_first) vx = *reinterpret_cast<const raw16 *>(a.v.x + (t0 + t) * a.v.token + h * a.v.head + 16 * v_item);
        if (s_place[t] >= 0) put_piece(a.view.v + s_place[t] + h * a.view.stride_head + 16 * v_item, vx);
    }
}

template <typename T>
hipError_t launch_rope_typed(const RopeArgs &a, hipStream_t st) {
    // 1568 tokens: 10.0 us a launch with a token a workgroup, 8.8 with two, 9.2 with three
    int per_wg = a.n_tokens / 768;
    per_wg = per_wg < 1 ? 1 : per_wg > kRopeTokens ? kRopeTokens : per_wg;
    const unsigned grid = (unsigned)((a.n_tokens + per_wg - 1) / per_wg);
    if (a.neighbours || !a.rotate)
        hipLaunchKernelGGL((rope_kernel<T, true>), dim3(grid), dim3(kRopeThreads), 0, st, a, per_wg);
    else
        hipLaunchKernelGGL((rope_kernel<T, false>), dim3(grid), dim3(kRopeThreads), 0, st, a, per_wg);
    return hipGetLastError();
}

} // namespace

hipError_t launch_rope(const RopeArgs &a, int dtype, hipStream_t st) {
    return dtype == MUKV_BF16 ? launch_rope_typed<uint16_t>(a, st) : launch_rope_typed<float>(a, st);
}

} // namespace mukv

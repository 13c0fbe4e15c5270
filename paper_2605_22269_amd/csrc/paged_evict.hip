// Eviction from a paged cache by the weight its rows have received: per (layer, sequence, KV head) the best rows stay, in their order.
//
// evict_select_kernel ranks the rows, evict_move_kernel packs the chosen rows' keys and values.  A row's rank is a 32-bit key: 0 for
// rows that do not exist (never kept), 1 for NaN weights, the weight's bits in an order that compares as the weights do, all ones
// for the rows that stay whatever they weigh.  The m-th largest key is found by its digits (8 bits, counts in LDS); once the rows that
// share its upper half are few, by counting among them.  Of the rows that equal it the first ones stay.
#include "attend_dev.h"
#include "paged_internal.h"

namespace mukv {

namespace {

constexpr int kSelRows = 4;      // rows a thread takes at a time when the list is written
constexpr int kSelCache = 32768; // keys that wait in LDS; those of further rows are worked out again on every pass
constexpr int kSelCopies = 4;    // of the counts: lanes that count the same digit at once share an address less often
constexpr int kSelCand = 512;    // rows that share the upper half of the key and are ranked by counting, as one number each (56 lists
                                 // of 1172 rows, 350 of them equal: 15 us, with key and row compared apart 46)

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 1u;
    const uint32_t u = __float_as_uint(w + 0.f); // (-0 is 0)
    return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u); // -inf: 0x007FFFFF
}

// One workgroup per (layer, sequence, KV head).  What bounds it: with a few thousand rows the barriers of the four digits.
template <int kSelThreads>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a, int cache_keys) {
    constexpr int kSelWaves = kSelThreads / 64;
    extern __shared__ __align__(16) uint32_t s_key[]; // [cache_keys]
    __shared__ __align__(16) int s_hist[kSelCopies][256];
    __shared__ int s_found[3]; // the digit, how many keys are above it, how many share it
    __shared__ int s_sum[2][kSelWaves];
    __shared__ __align__(16) uint64_t s_cand[kSelCand]; // key, then ~row: larger ones come first
    __shared__ int s_n_cand, s_last_row;
    const PagedView &v = a.view;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = blockIdx.x % v.Hkv, b = blockIdx.x / v.Hkv % v.n_seqs, layer = blockIdx.x / v.Hkv / v.n_seqs;
    const int n = rows_of(v, 0, length_of(v, b, 0));
    const int64_t at = (int64_t)layer * a.w_layer + (int64_t)b * a.w_seq + (int64_t)g * a.w_head;
    const float *w_in = a.w_in + at;
    float *w_out = a.w_out + at;
    int32_t *kept = a.kept + (int64_t)blockIdx.x * a.budget;
    auto key_of = [&](int j) -> uint32_t {
        if (j >= n || !is_page(v, v.table[entry_of(v, b, j)])) return 0u;
        if (j < a.n_sink || j >= n - a.n_recent) return 0xFFFFFFFFu;
        return weight_key(j < a.w_rows ? w_in[j] : 0.f);
    };
    auto get = [&](int j) { return j < cache_keys ? s_key[j] : key_of(j); };

    // ---- the m-th largest key, digit by digit ----
    uint32_t prefix = 0; // of the digits found
    int m = 0, need = 0;
    int last_row = -1;   // counted among few: the last row that stays of those that equal the m-th
    if (tid == 0) s_n_cand = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < kSelCopies * 256; i += kSelThreads) (&s_hist[0][0])[i] = 0;
        __syncthreads();
        int there = 0;
        constexpr int kAhead = 4; // rows a thread asks for together
        for (int j0 = tid; j0 < n; j0 += kAhead * kSelThreads) {
            uint32_t k[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const int j = j0 + e * kSelThreads;
                k[e] = j >= n ? 0u : shift == 24 ? key_of(j) : get(j);
            }
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const int j = j0 + e * kSelThreads;
                if (shift == 24) {
                    if (j < n && j < cache_keys) s_key[j] = k[e];
                    there += k[e] != 0u;
                }
                if (k[e] != 0u && (shift == 24 || k[e] >> (shift + 8) == prefix)) atomicAdd(&s_hist[lane & (kSelCopies - 1)][k[e] >> shift & 255u], 1);
            }
        }
        if (shift == 24) {
            there = wave_sum(there);
            if (lane == 0) s_sum[0][wave] = there;
        }
        __syncthreads();
        if (shift == 24) {
            for (int w = 0; w < kSelWaves; ++w) m += s_sum[0][w];
            m = m < a.budget ? m : a.budget;
            need = m;
            if (m == 0) break; // (the same in all threads)
        }
        if (wave == 0) { // lane: digits 255 - 4 lane .. 252 - 4 lane, the largest first
            i32x4 all = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < kSelCopies; ++c) all += *reinterpret_cast<const i32x4 *>(&s_hist[c][252 - 4 * lane]);
            const int h[4] = {all[3], all[2], all[1], all[0]}, sum = (h[0] + h[1]) + (h[2] + h[3]);
            const int upto = wave_prefix(sum);
            int before = upto - sum;
            if (before < need && need <= upto) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (before < need && need <= before + h[e]) {
                        s_found[0] = 255 - 4 * lane - e;
                        s_found[1] = before;
                        s_found[2] = h[e];
                    }
                    before += h[e];
                }
            }
        }
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)s_found[0];
        need -= s_found[1];
        const bool whole = need == s_found[2]; // all that share the digits so far stay: nothing is left to tell apart
        __syncthreads();
        if (whole) {
            prefix <<= shift;
            need = -1;
            break;
        }
        if (shift == 16 && s_found[2] <= kSelCand) { // (the same in all threads)
            for (int j = tid; j < n; j += kSelThreads) {
                const uint32_t k = get(j);
                if (k >> 16 != prefix) continue;
                s_cand[atomicAdd(&s_n_cand, 1)] = (uint64_t)k << 32 | ~(uint32_t)j;
            }
            constexpr int kTogether = 8;
            const int n_cand = s_found[2], n_read = (n_cand + kTogether - 1) & ~(kTogether - 1);
            if (n_cand + tid < n_read) s_cand[n_cand + tid] = 0; // before nobody
            __syncthreads();
            if (tid < n_cand) {
                const uint64_t mine = s_cand[tid];
                int ahead = 0;
                for (int i = 0; i < n_read; i += kTogether)
#pragma unroll
                    for (int e = 0; e < kTogether; ++e) ahead += s_cand[i + e] > mine;
                if (ahead == need - 1) {
                    s_last_row = (int)~(uint32_t)mine;
                    s_found[0] = (int)(uint32_t)(mine >> 32);
                }
            }
            __syncthreads();
            prefix = (uint32_t)s_found[0];
            last_row = s_last_row;
            need = 0;
            break;
        }
    }
    // Rows above `prefix` stay, and the first `need` of those that equal it (-1: all that are not below it).  (Rows that stay whatever
    // they weigh are no more than the budget: where their key is the m-th largest, all of them are within it, and need is -1.)
    const uint32_t least = need < 0 ? prefix : prefix + 1;
    const int quota = need > 0 ? need : 0;
    auto stays = [&](uint32_t k, int j) { return k >= least || (k == prefix && j <= last_row); };
    // ---- the list, ascending: kSelRows neighbouring rows a thread ----
    int over0 = 0, equal0 = 0; // before this round
    for (int base = 0; m > 0 && base < n; base += kSelThreads * kSelRows) {
        const int j0 = base + tid * kSelRows;
        uint32_t k[kSelRows];
        float w[kSelRows];
        int over = 0, equal = 0;
#pragma unroll
        for (int e = 0; e < kSelRows; ++e) {
            k[e] = j0 + e < n ? get(j0 + e) : 0u;
            w[e] = j0 + e < n && j0 + e < a.w_rows ? w_in[j0 + e] : 0.f;
            if (k[e] == 0u) continue;
            over += stays(k[e], j0 + e);
            equal += need > 0 && k[e] == prefix;
        }
        const int both = wave_prefix(over | equal << 16);
        if (lane == 63) s_sum[1][wave] = both;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // (the weights may be written where they were read)
        __syncthreads();
        int start = 0, all = 0;
#pragma unroll
        for (int x = 0; x < kSelWaves; ++x) {
            if (x < wave) start += s_sum[1][x];
            all += s_sum[1][x];
        }
        start += both - (over | equal << 16);
        int o = over0 + (start & 0xFFFF), q = equal0 + (start >> 16);
#pragma unroll
        for (int e = 0; e < kSelRows; ++e) {
            if (k[e] == 0u) continue;
            const bool is_equal = need > 0 && k[e] == prefix, is_over = stays(k[e], j0 + e);
            if (is_over || (is_equal && q < quota)) {
                const int pos = o + (q < quota ? q : quota);
                kept[pos] = j0 + e;
                if (pos < a.w_rows) w_out[pos] = w[e];
            }
            o += is_over;
            q += is_equal;
        }
        over0 += all & 0xFFFF;
        equal0 += all >> 16;
        __syncthreads();
    }
    for (int i = m + tid; i < a.budget; i += kSelThreads) kept[i] = -1;
    const int n_w = n < a.w_rows ? n : a.w_rows;
    for (int i = m + tid; i < n_w; i += kSelThreads) w_out[i] = 0.f;
}

constexpr int kMoveThreads = 256, kMoveRows = kMoveThreads; // most rows of a workgroup

// What stays of sequence b, the same in all its lists: the entries of one of them before the padding.  (12 lists of 31921 rows: read from
// end to end the kernel took 62 us for it, 16 so.)
__device__ __forceinline__ void write_length(const EvictArgs &a, const int32_t *kept, int b) {
    int lo = 0, len = a.budget; // the first entry of the padding is in lo .. lo + len; every round leaves 1 / kMoveThreads of that
    while (len > 0) {
        const int step = (len + kMoveThreads - 1) / kMoveThreads, i = (int)threadIdx.x * step;
        const int n = __syncthreads_count(i < len && kept[lo + i] >= 0);
        if (n == 0) break;
        const int at = (n - 1) * step + 1; // past the last one that is not padding
        lo += at;
        len = len - at < step - 1 ? len - at : step - 1;
    }
    if (threadIdx.x == 0) a.lengths_out[b] = lo;
}

// Onto other pages: every row on its own.  Grid (layer x sequence x KV head, n_rows rows).
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, int row_bytes, int n_rows) {
    __shared__ int64_t s_from[kMoveRows], s_to[kMoveRows]; // byte offsets in the layer's pages, -1: nothing to move
    const PagedView &v = a.view;
    const int tid = threadIdx.x, list = blockIdx.x;
    const int g = list % v.Hkv, b = list / v.Hkv % v.n_seqs, layer = list / v.Hkv / v.n_seqs;
    const int32_t *kept = a.kept + (int64_t)list * a.budget;
    if (blockIdx.y == 0 && layer == 0 && g == 0) write_length(a, kept, b);
    const int pieces = row_bytes / 16, rows_at_once = kMoveThreads / pieces, piece = tid % pieces, r0 = tid / pieces;
    unsigned char *const bases[2] = {v.k + layer * a.stride_layer + g * v.stride_head + 16 * piece, v.v + layer * a.stride_layer + g * v.stride_head + 16 * piece};
    for (int64_t i0 = (int64_t)blockIdx.y * n_rows; i0 < a.budget; i0 += (int64_t)gridDim.y * n_rows) {
        if (tid < n_rows) {
            const int i = (int)i0 + tid, row = i < a.budget ? kept[i] : -1;
            int64_t from = -1, to = -1;
            if (row >= 0 && i / v.page_rows < a.into_width) {
                const int page = v.table[entry_of(v, b, row)], dst = a.into[(int64_t)b * a.into_width + i / v.page_rows];
                if (is_page(v, page) && is_page(v, dst)) {
                    from = offset_of(v, page, row);
                    to = offset_of(v, dst, i);
                }
            }
            s_from[tid] = from;
            s_to[tid] = to;
        }
        __syncthreads();
        constexpr int kAhead = 4;
        for (int r = r0; r < n_rows; r += kAhead * rows_at_once) {
            raw16 x[kAhead][2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int rr = r + u * rows_at_once;
                if (rr >= n_rows || s_from[rr] < 0) continue;
#pragma unroll
                for (int t = 0; t < 2; ++t) x[u][t] = *reinterpret_cast<const raw16 *>(bases[t] + s_from[rr]);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int rr = r + u * rows_at_once;
                if (rr >= n_rows || s_from[rr] < 0) continue;
#pragma unroll
                for (int t = 0; t < 2; ++t) __builtin_nontemporal_store(x[u][t], reinterpret_cast<raw16 *>(bases[t] + s_to[rr]));
            }
        }
        __syncthreads(); // the next rows' places take these ones'
    }
}

// In place: row i of the result is row kept[i] >= i, so whatever is overwritten in ascending order has been read.  A workgroup takes all
// rows of one tensor in turn, but only 64 bytes of each: the slices of a row do not meet, so there are several workgroups to a list.
// Grid (list, slice, keys or values).
__global__ __launch_bounds__(kMoveThreads) void evict_pack_kernel(EvictArgs a, int row_bytes) {
    const PagedView &v = a.view;
    const int tid = threadIdx.x, list = blockIdx.x;
    const int g = list % v.Hkv, b = list / v.Hkv % v.n_seqs, layer = list / v.Hkv / v.n_seqs;
    const int32_t *kept = a.kept + (int64_t)list * a.budget;
    const int pieces = row_bytes < 64 ? row_bytes / 16 : 4, rows_at_once = kMoveThreads / pieces, r0 = tid / pieces;
    unsigned char *const base = (blockIdx.z ? v.v : v.k) + layer * a.stride_layer + g * v.stride_head + 64 * blockIdx.y + 16 * (tid % pieces);
    constexpr int kAhead = 4;
    raw16 x[2][kAhead];
    int64_t to[2][kAhead]; // -1: nothing to move
    auto request = [&](int i0, raw16(&y)[kAhead], int64_t(&dst)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * rows_at_once + r0, row = i < a.budget ? kept[i] : -1;
            dst[u] = -1;
            if (row <= i) continue; // (-1, or where it stays)
            const int page = v.table[entry_of(v, b, row)], d = v.table[entry_of(v, b, i)];
            if (!is_page(v, page) || !is_page(v, d)) continue;
            dst[u] = offset_of(v, d, i);
            y[u] = *reinterpret_cast<const raw16 *>(base + offset_of(v, page, row));
        }
    };
    auto put = [&](const raw16(&y)[kAhead], const int64_t(&dst)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (dst[u] >= 0) *reinterpret_cast<raw16 *>(base + dst[u]) = y[u];
    };
    const int step = kAhead * rows_at_once;
    auto landed = [] { // every wave's rows are in registers before any is overwritten
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    request(0, x[0], to[0]);
    for (int i0 = 0; i0 < a.budget; i0 += 2 * step) {
        landed();
        request(i0 + step, x[1], to[1]); // (rows after all that is overwritten now)
        put(x[0], to[0]);
        landed();
        request(i0 + 2 * step, x[0], to[0]);
        put(x[1], to[1]);
    }
    if (blockIdx.y == 0 && blockIdx.z == 0 && layer == 0 && g == 0) write_length(a, kept, b);
}

template <int kSelThreads>
hipError_t launch_select(const EvictArgs &a, int lists, int keys, int device, hipStream_t st) {
    static bool allowed[kMaxDevices];
    if (keys * sizeof(uint32_t) > 32 * 1024) {
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(&evict_select_kernel<kSelThreads>), kSelCache * sizeof(uint32_t), device, allowed);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((evict_select_kernel<kSelThreads>), dim3(lists), dim3(kSelThreads), keys * sizeof(uint32_t), st, a, keys);
    return hipGetLastError();
}

} // namespace

hipError_t launch_paged_evict(const EvictArgs &a, int n_layers, int row_bytes, int device, hipStream_t st) {
    const int lists = n_layers * a.view.n_seqs * a.view.Hkv;
    const int64_t room = room_of(a.view);
    const int keys = (int)(room < kSelCache ? room : kSelCache);
    // Few lists: a workgroup each has a compute unit to itself.  (us a launch, 1024 / 512 threads: 112 lists of 8200 rows 24 / 30, 768 of 900
    // to 6000 rows 45 / 28.)
    hipError_t e = lists <= 256 ? launch_select<1024>(a, lists, keys, device, st) : launch_select<512>(a, lists, keys, device, st);
    if (e != hipSuccess) return e;
    if (a.into) {
        // (a workgroup's threads ask for four pieces each, together)
        const int rows = 1024 / (row_bytes / 16) < 64 ? 64 : 1024 / (row_bytes / 16) > kMoveRows ? kMoveRows : 1024 / (row_bytes / 16);
        const int chunks = (a.budget + rows - 1) / rows;
        hipLaunchKernelGGL(evict_move_kernel, dim3(lists, chunks < 65535 ? chunks : 65535), dim3(kMoveThreads), 0, st, a, row_bytes, rows);
    } else {
        hipLaunchKernelGGL(evict_pack_kernel, dim3(lists, row_bytes < 64 ? 1 : row_bytes / 64, 2), dim3(kMoveThreads), 0, st, a, row_bytes);
    }
    return hipGetLastError();
}

} // namespace mukv

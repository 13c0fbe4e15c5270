// Device side of an attention call's plan, shared by the kernels over a paged cache.
#pragma once

#include "attend_dev.h"
#include "paged_internal.h"

namespace mukv {

struct Unit {
    SeqShape s;
    int b, g, tile, chunk, chunks;
    int lo, hi; // blocks of its rows
    int record; // of the tile's first chunk
};

// Blocks of a chunk: the number of chunks that costs least, a lane a number, and what it costs.
__device__ __forceinline__ int chunk_by_cost(const PlanShape &p, const PlanSums &x, bool one_sequence, float *least = nullptr) {
    const int chunks = (threadIdx.x & 63) + 1;
    const float cost = chunks <= p.most ? cost_of(p, x, one_sequence, chunks) : 1e30f, low = -wave_max(-cost);
    const int best = 1 + (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(cost == low));
    if (least) *least = low;
    return best == 1 ? kWhole : div_up32((int)x.longest, best);
}

// Unit `id` of those of u->s.
__device__ __forceinline__ void place_unit(const PagedView &v, int id, Unit *u) {
    // KV heads next to each other: workgroups go to the eight XCDs in turn, so an XCD meets few heads' rows
    u->g = id % v.Hkv;
    id /= v.Hkv;
    u->chunk = id % u->chunks;
    u->lo = u->chunk * u->hi; // (chunks are of hi blocks, all but the last)
    u->hi += u->lo;
    const int rank = id / u->chunks;
    u->record += (rank * v.Hkv + u->g) * u->chunks;
    u->tile = u->s.tiles - 1 - rank; // under the mask the last ones have the most to do: they start first
}
// The same of the only sequence; false: there is none.
__device__ __forceinline__ bool only_unit(const PagedView &v, const PlanShape &p, int id, int per, Unit *u) {
    u->b = 0;
    u->chunks = chunks_of(p, u->s, per);
    u->hi = chunk_of(p, u->s, per);
    u->record = 0;
    if (id >= u->s.tiles * v.Hkv * u->chunks) return false;
    place_unit(v, id, u);
    return true;
}

// In scalar registers (the compiler does not see that all lanes have the same).
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ void make_scalar(SeqShape &s) {
    s = SeqShape{same(s.first), same(s.n_new), same(s.length), same(s.rows), same(s.tiles), same(s.blocks)};
}
__device__ __forceinline__ void make_scalar(Unit &u) {
    make_scalar(u.s);
    u.b = same(u.b), u.g = same(u.g), u.tile = same(u.tile), u.chunk = same(u.chunk), u.chunks = same(u.chunks);
    u.lo = same(u.lo), u.hi = same(u.hi), u.record = same(u.record);
}

// The stretch of this workgroup where one sequence's tiles are shared out evenly.
struct Share {
    SeqShape s;
    uint32_t at, end, head, line, workers; // the next step and the last one's; steps of a KV head, of all
};
// false: chunks of equal size cost no more, and *u is one if *there.
__device__ __forceinline__ bool find_share(const PagedView &v, const PlanShape &p, uint32_t id, uint32_t groups, Share *x, Unit *u, bool *there) {
    const int lane = threadIdx.x & 63;
    x->s = shape_of(v, p, 0);
    make_scalar(x->s);
    const uint32_t workers = (uint32_t)p.places < groups ? (uint32_t)p.places : groups;
    const int64_t tiles = (int64_t)x->s.tiles * v.Hkv;
    const PlanSums sums = sums_of(v, p, x->s);
    float least;
    const int per = chunk_by_cost(p, sums, true, &least);
    bool even = tiles >= 1 && tiles + workers <= p.records && tiles * x->s.blocks <= kMostSteps;
    even = even && shares_fit(p, (uint32_t)tiles, workers);
    even = even && cost_of_shares(p, sums.tiles, sums.seen, (float)workers) < least;
    if (even) {
        int head = 0;
        for (int t0 = 0; t0 < x->s.tiles; t0 += 64) {
            const int t = t0 + lane;
            head += t < x->s.tiles ? steps_of_tile(v, p, x->s, t) : 0;
        }
        x->head = (uint32_t)same(wave_sum(head));
        x->line = x->head * (uint32_t)v.Hkv;
        x->workers = workers;
        even = x->line >= workers; // (a worker without a step would be missed where chunks are counted)
    }
    if (!even) {
        u->s = x->s;
        *there = only_unit(v, p, (int)id, per, u);
        return false;
    }
    // workgroups go to the eight XCDs in turn: neighbouring stretches, which read the same rows, to one of them
    const uint32_t worker = workers % 8 ? id : id % 8 * (workers / 8) + id / 8;
    x->at = id < workers ? stretch_of(worker, workers, x->line) : 0;
    x->end = id < workers ? stretch_of(worker + 1, workers, x->line) : 0;
    return true;
}
// The stretch's next unit.
__device__ __forceinline__ void next_unit(const PagedView &v, const PlanShape &p, Share *x, Unit *u) {
    const int lane = threadIdx.x & 63;
    u->s = x->s;
    u->b = 0;
    u->g = (int)(x->at / x->head);
    const int step = (int)(x->at - (uint32_t)u->g * x->head);
    int before = 0;
    for (int t0 = 0;; t0 += 64) { // the tile that the step is in (it is in one: step < head)
        const int steps = t0 + lane < x->s.tiles ? steps_of_tile(v, p, x->s, t0 + lane) : 0;
        const int upto = before + wave_prefix(steps);
        const uint64_t here = __builtin_amdgcn_ballot_w64(step < upto);
        if (here || t0 + 64 >= x->s.tiles) {
            const int at = here ? __builtin_ctzll(here) : 0;
            const int n = __builtin_amdgcn_readlane(steps, at), first = __builtin_amdgcn_readlane(upto, at) - n;
            u->tile = t0 + at;
            u->lo = step - first;
            const uint32_t left = x->end - x->at;
            u->hi = (uint32_t)(n - u->lo) < left ? n : u->lo + (int)left;
            const uint32_t start = (uint32_t)u->g * x->head + (uint32_t)first, me = worker_at(x->at, x->workers, x->line);
            const uint32_t first_worker = worker_at(start, x->workers, x->line);
            u->chunks = (int)(worker_at(start + (uint32_t)n - 1, x->workers, x->line) - first_worker) + 1;
            u->chunk = (int)(me - first_worker);
            u->record = record_of(first_worker, u->g * x->s.tiles + u->tile);
            x->at += (uint32_t)(u->hi - u->lo);
            return;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
}

// The unit of this workgroup, the same in all lanes; false: there is none (nobody has one where offsets do not ascend).
__device__ __forceinline__ bool find_unit(const PagedView &v, const PlanShape &p, int id, Unit *u) {
    const int lane = threadIdx.x & 63;
    if (v.n_seqs == 1) {
        u->s = shape_of(v, p, 0);
        const PlanSums x = sums_of(v, p, u->s);
        return only_unit(v, p, id, p.start ? chunk_by_cost(p, x, true) : chunk_by_room(p, x), u);
    } else {
        const SeqShape none = {0, 0, 0, 0, 0, 1};
        SeqShape s = none;
        PlanSums all = {0.f, 0.f, 0.f, 0.f};
        bool fit = true;
        for (int b0 = 0; b0 < v.n_seqs; b0 += 64) {
            s = b0 + lane < v.n_seqs ? shape_of(v, p, b0 + lane) : none;
            fit = fit && (b0 + lane >= v.n_seqs || offsets_fit(v, b0 + lane));
            const PlanSums x = sums_of(v, p, s);
            all.tiles += x.tiles;
            all.blocks += x.blocks;
            all.seen += x.seen;
            all.longest = fmaxf(all.longest, x.longest);
        }
        if (__builtin_amdgcn_ballot_w64(!fit) != 0) return false;
        all.blocks = wave_sum(all.blocks);
        all.tiles = wave_sum(all.tiles);
        all.longest = wave_max(all.longest);
        int per;
        if (p.start) {
            all.seen = wave_sum(all.seen);
            per = chunk_by_cost(p, all, false);
        } else {
            per = chunk_by_room(p, all);
        }
        int units0 = 0, records0 = 0, b0 = 0;
        for (;; b0 += 64) {
            if (b0 >= v.n_seqs) return false;
            if (v.n_seqs > 64) s = b0 + lane < v.n_seqs ? shape_of(v, p, b0 + lane) : none;
            const int chunks = chunks_of(p, s, per), units = s.tiles * v.Hkv * chunks, records = chunks > 1 ? units : 0;
            const int units1 = units0 + wave_prefix(units), records1 = records0 + wave_prefix(records);
            const uint64_t here = __builtin_amdgcn_ballot_w64(id < units1);
            if (here) {
                const int at = __builtin_ctzll(here);
                auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
                u->s = SeqShape{of(s.first), of(s.n_new), of(s.length), of(s.rows), of(s.tiles), of(s.blocks)};
                u->b = b0 + at;
                u->hi = chunk_of(p, u->s, per);
                u->chunks = of(chunks);
                u->record = of(records1 - records);
                id -= of(units1 - units);
                break;
            }
            units0 = __builtin_amdgcn_readlane(units1, 63);
            records0 = __builtin_amdgcn_readlane(records1, 63);
        }
    }
    place_unit(v, id, u);
    return true;
}

// ---- results of shared rows ----
// Whether the groups' offsets ascend, for the other launch: by the first wave of workgroup 0.
__device__ __forceinline__ void tell_fit(const PagedView &v, const SharedResults &r) {
    if (blockIdx.x != 0 || threadIdx.x >= 64) return;
    bool fit = true;
    for (int b = threadIdx.x; b < v.n_seqs; b += 64) fit = fit && offsets_fit(v, b);
    if (__builtin_amdgcn_ballot_w64(!fit) == 0) {
        if (threadIdx.x == 0) *r.fit = 1;
    } else if (threadIdx.x == 0) {
        *r.fit = 0;
    }
}
__device__ __forceinline__ bool in_a_group(const SharedResults &r, int token) {
    return !r.offsets || (token >= r.offsets[0] && token < r.offsets[r.n_groups]);
}
// How two parts of a row's softmax become one: what each is multiplied by, and what weights are relative to then.  A part without
// weights (their sum is zero; a NaN is not) counts for nothing: -1.  One that weighs so little that its factor is zero is multiplied by that all
// the same, so that what is no number in it still reaches the output, as in a sum over all rows.
struct JoinBy {
    float at, own, other;
};
__device__ __forceinline__ JoinBy join_by(float at, float sum, float other_at, float other_sum) {
    const bool some = sum != 0.f, others = other_sum != 0.f;
    JoinBy j;
    j.at = some && others ? fmaxf(at, other_at) : others ? other_at : at;
    j.own = some ? (others ? __builtin_amdgcn_exp2f(at - j.at) : 1.f) : -1.f;
    j.other = others ? (some ? __builtin_amdgcn_exp2f(other_at - j.at) : 1.f) : -1.f;
    return j;
}
// x, which is zero where by, a factor of one of the two, is -1
__device__ __forceinline__ float counted(float x, float by) { return by < 0.f ? 0.f : x * by; }

// What a lane leaves of a unit's query n (query `row` among the outputs): where.
__device__ __forceinline__ int place_left(const SharedResults &r, const Unit &u, int queries, int n, int64_t row) {
    return u.chunks == 1 ? r.single + (int)row : (u.record + u.chunk) * queries + n;
}
__device__ __forceinline__ void leave_head(const SharedResults &r, const Unit &u, int queries, int n, int64_t row) {
    if (u.chunk == 0) *reinterpret_cast<i32x4 *>(r.heads + 4 * row) = i32x4{u.chunks, place_left(r, u, queries, n, row), queries, 0};
}
// What was left of query `row`: chunks, where, and in the chunks' order what each is multiplied by (by(c, x), -1: it counts for nothing).
struct Taken {
    int chunks, place, stride; // of the chunks' values
    float at, sum, sum_all;
};
template <typename F>
__device__ __forceinline__ Taken take_left(const SharedResults &r, int token, int64_t row, F by) {
    Taken t = {0, 0, 0, -INFINITY, 0.f, 0.f};
    const i32x4 head = *reinterpret_cast<const i32x4 *>(r.heads + 4 * row); // (read whether or not it has been written)
    if (*r.fit == 0 || !in_a_group(r, token)) return t;
    t.chunks = head[0];
    t.place = head[1];
    t.stride = head[2];
    const float *const stats = r.stats + 4 * (int64_t)head[1];
#pragma unroll 8
    for (int c = 0; c < head[0]; ++c) {
        const f32x2 st = *reinterpret_cast<const f32x2 *>(stats + 4 * (int64_t)c * head[2]);
        t.at = st[1] != 0.f ? fmaxf(t.at, st[0]) : t.at; // (else none of the chunk's rows is seen; a NaN is)
    }
#pragma unroll 8
    for (int c = 0; c < head[0]; ++c) {
        const f32x4 st = *reinterpret_cast<const f32x4 *>(stats + 4 * (int64_t)c * head[2]);
        const bool some = st[1] != 0.f;
        const float x = some ? __builtin_amdgcn_exp2f(st[0] - t.at) : -1.f;
        t.sum = some ? fmaf(st[1], x, t.sum) : t.sum;
        t.sum_all = some ? fmaf(st[2], x, t.sum_all) : t.sum_all;
        by(c, x);
    }
    return t;
}

// ---- joining a tile's chunks ----
// Records are written through to, and read from, the memory that all XCDs share.
constexpr int kFar = 16; // cache policy of a buffer access: the scope of the whole GPU (sc1)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t far_buffer(float *p, int64_t floats) {
    return __builtin_amdgcn_make_buffer_rsrc(p, 0, (int)(4 * floats), 0x00027000);
}
__device__ __forceinline__ f32x4 load_far4(__amdgpu_buffer_rsrc_t r, int floats) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, 4 * floats, 0, kFar));
}
__device__ __forceinline__ void store_far4(__amdgpu_buffer_rsrc_t r, int floats, f32x4 x) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(raw16, x), r, 4 * floats, 0, kFar);
}
__device__ __forceinline__ void store_far1(float *p, float x) {
    __hip_atomic_store(reinterpret_cast<uint32_t *>(p), __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float load_far1(const float *p) {
    return __uint_as_float(__hip_atomic_load(reinterpret_cast<const uint32_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// the values of one chunk of a tile
template <int kQueries, int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_values(const ChunkRecords &r, int record) {
    return far_buffer(r.values + (int64_t)record * kQueries * D, kQueries * D);
}

// LDS that join_chunks wants, in floats
constexpr int join_scratch(int chunks, int queries) { return (chunks + 2) * queries; }

// The last workgroup of a tile joins its chunks, in their order.  put(n, c, m, l, x): features 4 c .. 4 c + 3 of query n, x the sum of
// the outputs that belongs to the reference m and the sum of weights l.  kAhead chunks of kItems pieces of 16 bytes are requested
// together, the first of them before anything else is known; there are at most kChunks.
template <int kQueries, int D, int kThreads, int kChunks, int kItems, int kAhead, typename Put>
__device__ __forceinline__ void join_chunks(const ChunkRecords &r, int record, int chunks, int n_q, float *scratch, Put put) {
    const int tid = threadIdx.x;
    float(*const s_by)[kQueries] = reinterpret_cast<float(*)[kQueries]>(scratch); // what a chunk's output is multiplied by, -1: nothing seen
    float *const s_m = s_by[chunks], *const s_l = s_by[chunks + 1];
    constexpr int kQuads = D / 4;
    const int n_items = n_q * kQuads;
    const auto values = far_buffer(r.values + (int64_t)record * kQueries * D, (int64_t)chunks * kQueries * D);
    f32x4 y[kItems][kAhead];
    auto request = [&](int i0, int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kItems; ++u)
#pragma unroll
            for (int c = 0; c < kAhead; ++c)
                if (c0 + c < chunks && i0 + u * kThreads < n_items) y[u][c] = load_far4(values, (c0 + c) * kQueries * D + 4 * (i0 + u * kThreads));
    };
    request(tid, 0);
    const float *stats = r.stats + (int64_t)record * kQueries * 2;
    constexpr int kLanes = kThreads / kQueries, kEach = (kChunks + kLanes - 1) / kLanes; // lanes of a query, chunks of a lane
    static_assert(kLanes == 16 || kLanes == 1, "a row of lanes, or one");
    const int n_here = tid / kLanes, first = tid % kLanes;
    f32x2 st[kEach]; // the lane's chunks: reference, sum of weights
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int c = first + k * kLanes;
        st[k] = f32x2{-INFINITY, 0.f};
        if (c < chunks && n_here < n_q) st[k] = load_far(stats + 2 * (c * kQueries + n_here));
    }
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        if (st[k][1] != 0.f) m = fmaxf(m, st[k][0]); // (else none of the chunk's rows is seen; a NaN is)
    if constexpr (kLanes == 16) m = row16_max(m);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int c = first + k * kLanes;
        const float by = st[k][1] != 0.f ? __builtin_amdgcn_exp2f(st[k][0] - m) : -1.f;
        if (st[k][1] != 0.f) l = fmaf(st[k][1], by, l);
        if (c < chunks && n_here < n_q) s_by[c][n_here] = by;
    }
    if constexpr (kLanes == 16) l = row16_sum(l);
    if (first == 0) {
        s_m[n_here] = m;
        s_l[n_here] = l;
    }
    __syncthreads();
    for (int i0 = tid; i0 < n_items; i0 += kItems * kThreads) {
        f32x4 x[kItems];
#pragma unroll
        for (int u = 0; u < kItems; ++u) x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < chunks; c0 += kAhead) {
            if (i0 != tid || c0 != 0) request(i0, c0);
#pragma unroll
            for (int u = 0; u < kItems; ++u)
#pragma unroll
                for (int c = 0; c < kAhead; ++c) {
                    if (c0 + c >= chunks || i0 + u * kThreads >= n_items) continue;
                    const float by = s_by[c0 + c][(i0 + u * kThreads) / kQuads];
                    if (by < 0.f) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[u][e] = fmaf(y[u][c][e], by, x[u][e]);
                }
        }
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const int i = i0 + u * kThreads, n = i / kQuads;
            if (i < n_items) put(n, i - n * kQuads, s_m[n], s_l[n], x[u]);
        }
    }
}

} // namespace mukv

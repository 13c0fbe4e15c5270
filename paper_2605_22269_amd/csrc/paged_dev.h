// Device side of an attention call's plan, shared by the kernels over a paged cache.
#pragma once

#include "attend_dev.h"
#include "paged_internal.h"

namespace mukv {

struct Unit {
    SeqShape s;
    int b, g, tile, chunk, chunks, per; // per: blocks of a chunk
    int record;                         // of the tile's first chunk
};

// The unit of this workgroup, the same in all lanes; false: there is none.
__device__ __forceinline__ bool find_unit(const PagedView &v, const PlanShape &p, int id, Unit *u) {
    const int lane = threadIdx.x & 63;
    if (v.n_seqs == 1) {
        u->s = shape_of(v, p, 0);
        u->b = 0;
        u->per = chunk_of(p, u->s, chunk_of(p, blocks_of(v, u->s)));
        u->chunks = (int)div_up(u->s.blocks, u->per);
        u->record = 0;
        if (id >= u->s.tiles * v.Hkv * u->chunks) return false;
    } else {
        const SeqShape none = {0, 0, 0, 0, 0, 1};
        SeqShape s = none;
        double all = 0.0;
        for (int b0 = 0; b0 < v.n_seqs; b0 += 64) {
            s = b0 + lane < v.n_seqs ? shape_of(v, p, b0 + lane) : none;
            all += blocks_of(v, s);
        }
        const int per = chunk_of(p, wave_sum(all));
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
                u->per = chunk_of(p, u->s, per);
                u->chunks = of(chunks);
                u->record = of(records1 - records);
                id -= of(units1 - units);
                break;
            }
            units0 = __builtin_amdgcn_readlane(units1, 63);
            records0 = __builtin_amdgcn_readlane(records1, 63);
        }
    }
    // KV heads next to each other: workgroups go to the eight XCDs in turn, so an XCD meets few heads' rows
    u->g = id % v.Hkv;
    id /= v.Hkv;
    u->chunk = id % u->chunks;
    const int rank = id / u->chunks;
    u->record += (rank * v.Hkv + u->g) * u->chunks;
    u->tile = u->s.tiles - 1 - rank; // under the mask the last ones have the most to do: they start first
    return true;
}

} // namespace mukv

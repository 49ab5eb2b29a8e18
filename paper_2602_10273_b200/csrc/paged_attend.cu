// Attention of one new token per row over the paged cache:  out[r, h] = sum_p softmax_p(scale q[r, h] . k_p) v_p over
// the positions p < n_r = lens[r] + extra of row r.
//
// The particles of a group descend from common ancestors, so their rows share blocks: all of them far back, ever fewer
// of them towards the end.  What bounds the operator is reading every distinct block once; sharing is found on the
// device, since only the table knows it.  Three kernels, chained:
//
//   plan    per tile of 32 rows: the sets of rows that hold the same block at block index j, and the runs of j over which
//           a set stays the same: the tile's SEGMENTS.  A segment's queries (rows x query heads per key-value head) meet
//           its keys and values together.
//   attend  the work of all (tile, key-value head, segment, query tile) items is laid on one line, in steps of 64
//           positions, and cut into equal shares, one per CTA of a grid that fills the GPU: long rows are split, short
//           ones are strung together, and no CTA waits for another.  The four warps of a CTA stream a step's keys and
//           values through a ring of shared-memory stages (cp.async, 16 bytes per lane, the next items' steps among
//           them) and divide it by queries, 16 to a warp, and where that leaves warps over, by positions.
//   join    per (row, query head): the partial results of the row's segments and of the shares that split them.
//
// Scores and outputs are formed transposed, S^T = K Q^T and O^T = V^T P^T, on the warp-level matrix instructions: the 16
// rows of an operand tile are positions (or components of the output) and its 8 columns queries, so that the 4 to 8
// queries of one key-value head fill a tile, and K and V come straight from their rows in shared memory.  (These
// instructions reach a fraction of the tensor cores' rate, and a fraction is enough: at 4 queries per head the arithmetic
// of a step is 1/10 of the time its bytes take.)  A weight is exp2(s - m) with m a reference per query that follows the
// largest score only when it is exceeded by more than 8 (a rare, warp-uniform branch); sums and outputs are fp32.
#include "paged_common.cuh"

namespace psmc {
namespace {

constexpr int kTileRows = 32;       // rows per tile: a lane each in the plan
constexpr int kMaxSegs = 128;       // segments per tile; a table that needs more is served row by row
constexpr int kRowSegs = 6;         // and so is one whose rows meet more segments than this on average
constexpr int kGroups = 4;          // query groups of a query tile: one per warp of a CTA
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;       // how far (log2) a score may exceed the reference before the reference moves

// ---------------------------------------------------------------------------------------------------------- plan
struct Segment {
    uint32_t mask;       // rows of the tile
    int p0, p1;          // positions
    int before;          // rows of the segments before this one, added up
    int64_t start;       // its first cost unit on the line of one (tile, key-value head)
};
struct TilePlan {
    int64_t cost;        // of one key-value head
    int n_segs;
    uint32_t whole;      // rows that have a single segment
    uint32_t left_out;   // rows with skip != 0, or beyond R
    Segment seg[kMaxSegs];
};

struct LineShape {       // how the items of a tile are cut; a pure function of the launch
    int step;            // positions per step
    int group;           // queries per warp; a query tile has kGroups times as many
    int ratio, H;
};
// What a step costs by its queries: its bytes are the same, and beside them the arithmetic of one or two groups is small.
__device__ __forceinline__ int step_cost(const LineShape& s, int nq) {
    const int groups = (nq + s.group - 1) / s.group;
    return 4 + (groups > 1 ? groups : 0);
}
__device__ __forceinline__ int64_t seg_cost(const LineShape& s, int rows, int steps) {
    const int nq = rows * s.ratio, qt = s.group * kGroups, full = nq / qt, rem = nq - full * qt;
    return (int64_t)steps * (full * step_cost(s, qt) + (rem ? step_cost(s, rem) : 0));
}
__device__ __forceinline__ int steps_of(const LineShape& s, int p0, int p1) { return (p1 - p0 + s.step - 1) / s.step; }

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;
constexpr int kRun = 8;              // block indices that a warp looks at in one go
constexpr int kWarpSegs = 32;        // segments that may begin in one warp's block indices

__global__ void __launch_bounds__(kPlanThreads) paged_plan_kernel(const PagedView c, const PagedAttend a, const LineShape ls,
                                                                  TilePlan* plans) {
    struct Found {
        uint32_t mask;
        int from, lead;
    };
    __shared__ Found found[kPlanWarps][kWarpSegs];
    __shared__ Found segs[kMaxSegs];
    __shared__ int count[kPlanWarps], rows_in[kPlanWarps], ends[kMaxSegs], n_of[kTileRows];
    chain_begin();
    const int tile = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = c.block_len;
    TilePlan& tp = plans[tile];
    const int row = tile * kTileRows + lane;
    const bool is_row = row < c.R;
    // the first run of table entries travels together with the lengths that say how much of it counts
    const int32_t* entries = c.table + (int64_t)(is_row ? row : 0) * c.table_ld;
    int e[kRun + 1];
    const auto fetch = [&](int j0) {  // entries j0 - 1 .. j0 + kRun
#pragma unroll
        for (int u = 0; u <= kRun; ++u) {
            const int j = j0 - 1 + u;
            e[u] = is_row && j >= 0 && j < c.max_blocks ? __ldg(entries + j) : -1;
        }
    };
    fetch(warp * kRun);
    int64_t len = is_row ? (int64_t)__ldg(a.lens + row) + a.extra : 0;
    const bool left_out = !is_row || (a.skip && a.skip[row]);
    const int64_t room = (int64_t)c.max_blocks * B;
    if (left_out || len < 0) len = 0;
    if (len > room) {
        if (warp == 0) raise_status(a.status, PSMC_E_STATE);
        len = room;
    }
    const int n = (int)len;
    if (warp == 0) n_of[lane] = n;
    const uint32_t alive = __ballot_sync(kFull, n > 0), out_mask = __ballot_sync(kFull, left_out);
    const int nb = warp_max((n + B - 1) / B);

    // How this row stands in block j: positions of it that count, and the block's number, if it has one that exists.
    const auto live_in = [&](int j) -> int { return (int)min((int64_t)B, max((int64_t)0, n - (int64_t)j * B)); };
    const auto set_of = [&](int entry, int live) -> uint32_t {  // rows that stand alike, this one among them
        const bool named = live > 0 && entry >= 0 && entry < c.n_blocks;
        const uint32_t same = __match_any_sync(kFull, named ? entry : -1 - lane) & __match_any_sync(kFull, live);
        return live > 0 ? (named ? same : 1u << lane) : 0u;
    };
    int begun = 0, rows = 0;
    if (__popc(alive) > 1) {
        for (int j0 = warp * kRun; j0 < nb; j0 += kPlanWarps * kRun) {
            if (j0 >= kPlanWarps * kRun) fetch(j0);
            uint32_t prev = 0;
            if (j0 > 0) prev = set_of(e[0], live_in(j0 - 1));
#pragma unroll
            for (int u = 0; u < kRun; ++u) {
                const int j = j0 + u, live = live_in(j);
                if (j >= nb) break;
                // A match over the warp costs hundreds of cycles when the rows differ.  Where every row still stands like
                // the first of its set, no set has split, and sets that have once parted do not meet again in a table that
                // copy-on-write keeps (in any other table two sets would just be read apart).
                const int lead = prev ? __ffs(prev) - 1 : lane;
                const int lead_e = __shfl_sync(kFull, e[u + 1], lead), lead_live = __shfl_sync(kFull, live, lead);
                uint32_t set = prev;
                if (__any_sync(kFull, (prev == 0) != (live == 0) || lead_live != live || (prev != 0 && lead_e != e[u + 1])))
                    set = set_of(e[u + 1], live);
                const bool begins = set != 0 && set != prev && lane == __ffs(set) - 1;
                const uint32_t who = __ballot_sync(kFull, begins);
                if (begins) {
                    rows += __popc(set);
                    const int s = begun + __popc(who & ((1u << lane) - 1));
                    if (s < kWarpSegs) found[warp][s] = Found{set, j, lane};
                }
                begun += __popc(who);
                prev = set;
            }
        }
    }
    rows = (int)warp_sum((float)min(rows, 1 << 16));
    if (lane == 0) {
        count[warp] = begun;
        rows_in[warp] = rows;
    }
    __syncthreads();
    // every warp adds up the same numbers
    const int mine = lane < kPlanWarps ? count[lane] : 0;
    const int upto = warp_scan_incl(mine, lane);
    int n_segs = __shfl_sync(kFull, upto, 31);
    const float all_rows = warp_sum(lane < kPlanWarps ? (float)rows_in[lane] : 0.f);
    const bool by_row = n_segs == 0 || n_segs > kMaxSegs || all_rows > kTileRows * kRowSegs || warp_max(mine) > kWarpSegs;
    if (by_row) {
        n_segs = __popc(alive);
        if (warp == 0 && n > 0) segs[__popc(alive & ((1u << lane) - 1))] = Found{1u << lane, 0, lane};
    } else {
        const int at = __shfl_sync(kFull, upto - mine, warp);
        if (lane < begun) segs[at + lane] = found[warp][lane];
    }
    __syncthreads();
    for (int s = threadIdx.x; s < n_segs; s += kPlanThreads) {  // ends where its first row enters another, or ends itself
        const Found f = segs[s];
        int end = (n_of[f.lead] + B - 1) / B;
        for (int o = 0; o < n_segs; ++o)
            if (segs[o].from > f.from && (segs[o].mask >> f.lead & 1)) end = min(end, segs[o].from);
        ends[s] = (int)min((int64_t)end * B, (int64_t)n_of[f.lead]);
    }
    __syncthreads();
    if (warp == 0) {
        int64_t cost = 0;
        int before = 0;
        uint32_t whole = 0;
        for (int s0 = 0; s0 < n_segs; s0 += 32) {
            const int s = s0 + lane;
            const bool in = s < n_segs;
            const Found f = in ? segs[s] : Found{0, 0, 0};
            const int p0 = f.from * B, p1 = in ? ends[s] : 0, held = __popc(f.mask);
            const int64_t cs = in ? seg_cost(ls, held, steps_of(ls, p0, p1)) : 0;
            const int64_t cs_upto = warp_scan_incl<long long>(cs, lane);
            const int held_upto = warp_scan_incl(held, lane);
            if (in) {
                tp.seg[s] = Segment{f.mask, p0, p1, before + held_upto - held, cost + cs_upto - cs};
                bool all = p0 == 0;  // every row of the set ends where the segment does
                for (uint32_t m = f.mask; m && all; m &= m - 1) all = n_of[__ffs(m) - 1] == p1;
                if (all) whole |= f.mask;
            }
            cost += __shfl_sync(kFull, (long long)cs_upto, 31);
            before += __shfl_sync(kFull, held_upto, 31);
        }
        whole = __reduce_or_sync(kFull, whole);
        if (lane == 0) {
            tp.cost = cost;
            tp.n_segs = n_segs;
            tp.whole = whole;
            tp.left_out = out_mask;
        }
    }
}

// ------------------------------------------------------------------------------------------------- the line and its shares
struct Line {
    const TilePlan* plans;
    int n_tiles, workers;
    float* part;         // [.., D] unnormalised outputs: those of whole items and first parts, then one set per worker
    float2* stat;        // {reference, sum} of each
    int64_t first_rest;  // where the sets of the workers begin
    LineShape ls;
};

struct Bearings {        // where a tile begins on the line, and how the line is cut
    int64_t before, share, total;
    int tile;
};
// The tile that holds cost unit `worker * share` (or the one asked for), by all lanes of a warp: the costs of all tiles are
// added up again (16 numbers for 512 rows), which is less than a kernel of its own would take.
__device__ __forceinline__ Bearings bearings(const Line& l, int worker, int tile, int lane) {
    int64_t sum = 0;
    for (int t = lane; t < l.n_tiles; t += 32) sum += l.plans[t].cost;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, (long long)sum, o);
    Bearings b;
    b.total = sum * l.ls.H;
    b.share = (b.total + l.workers - 1) / l.workers;
    if (b.share < 4) b.share = 4;  // one step
    const int64_t x = worker * b.share;
    int64_t base = 0;
    b.tile = l.n_tiles;
    b.before = b.total;
    for (int t0 = 0; t0 < l.n_tiles; t0 += 32) {
        const int t = t0 + lane;
        const int64_t cs = t < l.n_tiles ? l.plans[t].cost * l.ls.H : 0;
        const int64_t upto = base + warp_scan_incl<long long>(cs, lane);
        const uint32_t hit = __ballot_sync(kFull, t < l.n_tiles && (tile >= 0 ? t == tile : upto > x));
        if (hit) {
            const int at = __ffs(hit) - 1;
            b.before = __shfl_sync(kFull, (long long)(upto - cs), at);
            b.tile = t0 + at;
            break;
        }
        base = __shfl_sync(kFull, (long long)upto, 31);
    }
    return b;
}
// the steps of an item (first cost unit a, cost w per step) that lie before `bound`
__device__ __forceinline__ int steps_before(int64_t bound, int64_t a, int w, int steps) {
    if (bound <= a) return 0;
    const int64_t d = bound - a;
    return d >= (int64_t)steps * w ? steps : (int)(((uint32_t)d + (uint32_t)w - 1) / (uint32_t)w);
}

// One worker's walk along the line.  All threads of the CTA hold the same values.
struct Walk {
    int64_t a, hi;       // first cost unit of the item at hand; end of the share
    int tile, head, si, qt, n_qt, n_segs;
    uint32_t mask;
    int p0, p1;          // positions of the segment
    int nq;              // queries of this query tile
    int before;          // see Segment
    int w, steps;
    int s, s_end;        // steps of the item that are this worker's: the next one, and the end
    int s_first;
    bool done;

    __device__ __forceinline__ void open_segment(const Line& l) {
        const Segment& g = l.plans[tile].seg[si];
        mask = g.mask;
        p0 = g.p0;
        p1 = g.p1;
        before = g.before;
        steps = steps_of(l.ls, p0, p1);
        n_qt = (__popc(mask) * l.ls.ratio + kGroups * l.ls.group - 1) / (kGroups * l.ls.group);
    }
    __device__ __forceinline__ void open_item(const Line& l, int64_t lo) {
        nq = min(kGroups * l.ls.group, __popc(mask) * l.ls.ratio - qt * kGroups * l.ls.group);
        w = step_cost(l.ls, nq);
        s_first = s = steps_before(lo, a, w, steps);
        s_end = steps_before(hi, a, w, steps);
    }
    // the item after this one that has a step for this worker
    __device__ __forceinline__ void next_item(const Line& l) {
        do {
            a += (int64_t)steps * w;
            if (a >= hi) {
                done = true;
                return;
            }
            if (++qt >= n_qt) {
                qt = 0;
                if (++si >= n_segs) {
                    si = 0;
                    if (++head >= l.ls.H) {
                        head = 0;
                        do {
                            if (++tile >= l.n_tiles) {
                                done = true;
                                return;
                            }
                            n_segs = l.plans[tile].n_segs;
                        } while (n_segs == 0);
                    }
                }
                open_segment(l);
            }
            open_item(l, a);
        } while (s >= s_end);
    }
    __device__ __forceinline__ void begin(const Line& l, int worker, int lane) {
        const Bearings b = bearings(l, worker, -1, lane);
        const int64_t lo = worker * b.share;
        hi = min(lo + b.share, b.total);
        done = lo >= b.total;
        if (done) return;
        tile = b.tile;
        const TilePlan& tp = l.plans[tile];
        n_segs = tp.n_segs;
        const int64_t x = lo - b.before;
        int64_t start[kMaxSegs / 32];
#pragma unroll
        for (int i = 0; i < kMaxSegs / 32; ++i) start[i] = tp.seg[i * 32 + lane].start;  // those beyond n_segs are not looked at
        head = (int)(x / tp.cost);
        const int64_t y = x - head * tp.cost;
        si = -1;
#pragma unroll
        for (int i = 0; i < kMaxSegs / 32; ++i) si += __popc(__ballot_sync(kFull, i * 32 + lane < n_segs && start[i] <= y));
        int64_t first = start[0];
#pragma unroll
        for (int i = 1; i < kMaxSegs / 32; ++i)
            if (si >= i * 32) first = start[i];
        first = __shfl_sync(kFull, (long long)first, si & 31);
        open_segment(l);
        const int64_t full = (int64_t)steps * step_cost(l.ls, kGroups * l.ls.group);
        qt = (int)min((int64_t)(n_qt - 1), (y - first) / full);
        a = b.before + head * tp.cost + first + qt * full;
        open_item(l, lo);
        if (s >= s_end) next_item(l);
    }
    __device__ __forceinline__ bool alone(const Line& l) const {  // the whole of its rows, in this share
        return s_first == 0 && s_end == steps && (l.plans[tile].whole & mask) == mask;
    }
    // where the partial result of the item's query 0 goes
    __device__ __forceinline__ int64_t slot(const Line& l, int worker) const {
        const int in_tile = qt * kGroups * l.ls.group;
        if (s_first > 0) return l.first_rest + (int64_t)worker * (kGroups * l.ls.group);
        return ((int64_t)tile * l.ls.H + head) * (kTileRows * kRowSegs * l.ls.ratio) + (int64_t)before * l.ls.ratio + in_tile;
    }
};

// ------------------------------------------------------------------------------------------------- copies and matrix tiles
struct FastDiv {         // division of numbers below 2^31 by d
    uint32_t mul;
    int shift;
};
FastDiv fast_div(int d) {
    int l = 0;
    while ((int64_t)1 << l < d) ++l;
    return FastDiv{(uint32_t)(((((uint64_t)1 << l) - d) << 32) / d + 1), l};
}
__device__ __forceinline__ int div_by(int x, const FastDiv& f) { return (int)((__umulhi((uint32_t)x, f.mul) + (uint32_t)x) >> f.shift); }

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, or 16 zero bytes where bytes == 0 (src is then not read)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void load_tiles(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_tiles_turned(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t turn_tile(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool HALF>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// two codes in the low half of x -> two fp16 numbers (exact)
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t x) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo;\n\tcvt.u16.u32 lo, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(x));
    return r;
}

// Shape of a CTA's work.  DP: head_dim rounded up to what the tiles are unrolled for.
constexpr int kWarps = 4;
template <int DT_, int DP_>
struct Shape {
    static constexpr int DT = DT_, DP = DP_;
    static constexpr int kElem = DT == PSMC_F32 ? 4 : (DT == PSMC_BF16 ? 2 : 1);
    static constexpr int kRow = DP * kElem + 16;                          // bytes between rows: an odd number of 16-byte units
    static constexpr int kStep = DT == PSMC_F32 && DP > 128 ? 32 : 64;    // positions per step
    static constexpr int kSlices = kStep / 16;                            // the 16 positions of an operand tile
    static constexpr int kHalf = kStep * kRow;                            // keys, then values
    static constexpr int kScales = DT == PSMC_F8 ? kStep * 4 : 0;         // words that hold the scale bytes
    static constexpr int kStage = 2 * (kHalf + kScales);
    static constexpr int kGroup = DT == PSMC_F32 ? 8 : 16;                // queries per warp
    // 32-bit caches: queries [8][DP] and weights [16 positions][8 queries] of each warp
    static constexpr int kExtra = DT == PSMC_F32 ? kWarps * (8 * DP + 16 * 8) * 4 : 0;
    static constexpr int kCtas = 3 * kStage + kExtra <= 112 * 1024 ? 2 : 1;  // per SM
    static constexpr int kFit = (224 * 1024 / kCtas - kExtra) / kStage;
    static constexpr int kStages = kFit > 6 ? 6 : kFit;
    static constexpr int kBytes = kStages * kStage + kExtra;
    static_assert(kStages >= 2 && kStage >= 3 * 8 * DP * 4, "a ring; a stage holds the merge of one query tile");
};

struct AttendArgs {
    PagedView c;
    PagedAttend a;
    Line l;
    FastDiv by_block, by_ratio;
    int q_words;         // queries start on 4-byte boundaries throughout
};

// The copying side of a walk.  Warp w copies the step's positions w*16 .. (the CTA's warps share them evenly); what a copy
// needs from the block table is asked for two steps before it is issued.
template <class S>
struct Feeder {
    static constexpr int kMine = S::kStep / kWarps;  // positions per warp
    struct Asked {
        int entry;       // lane p: table entry of the warp's position p
        int in_block;    // lane p: head * block_len + offset in the block; -1: no such position
        bool any;        // whether there is a step at all
    };
    Walk walk;
    Asked first, second;

    __device__ __forceinline__ Asked ask(const AttendArgs& g, int warp, int lane) {
        Asked q{-1, -1, !walk.done};
        if (walk.done) return q;
        const int p = walk.p0 + walk.s * S::kStep + warp * kMine + lane;
        if (lane < kMine && p < walk.p1) {
            const int j = div_by(p, g.by_block);
            q.in_block = walk.head * g.c.block_len + (p - j * g.c.block_len);
            const int row = walk.tile * kTileRows + __ffs(walk.mask) - 1;
            q.entry = __ldg(g.c.table + (int64_t)row * g.c.table_ld + j);
        }
        if (++walk.s >= walk.s_end) walk.next_item(g.l);
        return q;
    }
    __device__ __forceinline__ void begin(const AttendArgs& g, int warp, int lane) {
        first = ask(g, warp, lane);
        second = ask(g, warp, lane);
    }
    // copies of the step asked for first, into the stage at `stage`; valid_out: which of the warp's positions hold something
    __device__ __forceinline__ void issue(const AttendArgs& g, uint32_t stage, uint32_t* valid_out, int warp, int lane) {
        if (first.any) {
            const bool named = first.in_block >= 0 && first.entry >= 0 && first.entry < g.c.n_blocks;
            if (first.in_block >= 0 && !named) raise_status(g.a.status, PSMC_E_STATE);
            const uint32_t valid = __ballot_sync(kFull, named);
            const int per_row = g.c.D * S::kElem / 16;
            const uint32_t unit =
                named ? (uint32_t)first.entry * (uint32_t)(g.c.blk_bytes / 16) + (uint32_t)(first.in_block * per_row) : 0u;
            constexpr int kPerRow = S::DP * S::kElem / 16, kCopies = kMine * kPerRow / 32;
            const uint32_t to = stage + warp * kMine * S::kRow;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const int x = i * 32 + lane, r = x / kPerRow, col = x - r * kPerRow;
                const uint32_t at = __shfl_sync(kFull, unit, r);
                const int bytes = valid >> r & 1 ? 16 : 0;
                if (col < per_row) {
                    const int64_t off = ((int64_t)at + (bytes ? col : 0)) * 16;
                    copy16(to + r * S::kRow + col * 16, g.c.k + off, bytes);
                    copy16(to + S::kHalf + r * S::kRow + col * 16, g.c.v + off, bytes);
                }
            }
            if (S::DT == PSMC_F8 && lane < kMine) {
                const int64_t off = named ? (int64_t)first.entry * g.c.blk_bytes + g.c.scale_at + (first.in_block & ~3) : 0;
                const uint32_t word = stage + 2 * S::kHalf + (warp * kMine + lane) * 4;
                copy4(word, g.c.k + off, named ? 4 : 0);
                copy4(word + S::kScales, g.c.v + off, named ? 4 : 0);
            }
            if (lane == 0) valid_out[warp] = valid;
        }
        copies_commit();
        first = second;
        second = ask(g, warp, lane);
    }
};

// row (within the tile) of each place in a segment's mask
__device__ __forceinline__ void list_rows(uint32_t mask, uint8_t* rows, int lane) {
    __syncwarp();
    if (mask >> lane & 1) rows[__popc(mask & ((1u << lane) - 1))] = (uint8_t)lane;
    __syncwarp();
}

template <typename T>
__device__ __forceinline__ void put(T* p, float x) { *p = from_float<T>(x); }

// How a CTA's warps divide an item of nq queries: groups of queries, and slices of every step where warps are left over.
struct Division {
    int groups, slices, group, slice;
    __device__ __forceinline__ Division(int nq, int per_group, int max_slices, int warp) {
        groups = nq <= per_group ? 1 : (nq <= 2 * per_group ? 2 : 4);
        slices = min(kWarps / groups, max_slices);
        group = warp % groups;
        slice = warp / groups;  // >= slices: nothing to do
    }
};

// ---- the arithmetic of one warp: NT tiles of 8 queries against MT tiles of 16 positions
template <class S, int NT>
struct Tiles {
    static constexpr bool kF8 = S::DT == PSMC_F8;
    static constexpr int kDt = S::DP / 16;
    uint32_t q[NT][kDt][2];
    float sc[NT][2];      // queries 2t, 2t + 1 of each tile: factor from product to score in log2 units
    float o[NT][kDt][4], ref[NT][2], sum[NT][2];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            ref[j][0] = ref[j][1] = -INFINITY;
            sum[j][0] = sum[j][1] = 0.f;
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][d][e] = 0.f;
        }
    }
    // lane (gq, t) holds components of query gq of tile j; src: that query, or NULL
    __device__ __forceinline__ void load_queries(int j, const uint16_t* src, int D, bool words, float to_log2, int lane) {
        const int t = lane & 3;
#pragma unroll
        for (int ks = 0; ks < kDt; ++ks)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int d = ks * 16 + (kF8 ? 4 * t + 2 * e : e * 8 + 2 * t);
                uint32_t x = 0;
                if (src && d < D)
                    x = words ? __ldg(reinterpret_cast<const uint32_t*>(src + d)) : (uint32_t)__ldg(src + d) | (uint32_t)__ldg(src + d + 1) << 16;
                q[j][ks][e] = x;
            }
        if (!kF8) {
            sc[j][0] = sc[j][1] = to_log2;
            return;
        }
        // fp16 holds a bf16 number's 8 bits but not its range: the query is scaled by a power of two so that its largest
        // component lies in [128, 256), and the scores get it back
        float amax = 0.f;
#pragma unroll
        for (int ks = 0; ks < kDt; ++ks)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(q[j][ks][e] << 16)), fabsf(__uint_as_float(q[j][ks][e] & 0xffff0000u))));
        amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, 2));
        const int ex = min(max((int)(__float_as_uint(amax) >> 23) - 127 - 7, -100), 100);
        const float inv = pow2i(-ex), back = pow2i(ex) * to_log2;
#pragma unroll
        for (int ks = 0; ks < kDt; ++ks)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                q[j][ks][e] = pack_f16(__uint_as_float(q[j][ks][e] << 16) * inv, __uint_as_float(q[j][ks][e] & 0xffff0000u) * inv);
        sc[j][0] = __shfl_sync(kFull, back, 8 * t);
        sc[j][1] = __shfl_sync(kFull, back, 8 * t + 4);
    }

    // keys, vals: shared addresses of 16 rows; valid: which of them hold something; k_scale, v_byte: lane p's scales (8-bit)
    __device__ __forceinline__ void step(uint32_t keys, uint32_t vals, uint32_t valid, float k_scale, int v_byte, int lane) {
        const int gq = lane >> 2;
        float s[NT][4], s2[NT][4];  // two chains, so that the products of one tile wait less for each other
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] = s2[j][e] = 0.f;
        const uint32_t krow = keys + (lane & 15) * S::kRow + (lane >> 4) * 16;
        if (!kF8) {
#pragma unroll
            for (int ks = 0; ks < kDt; ++ks) {
                uint32_t ka[4];
                load_tiles(ka, krow + ks * 32);
#pragma unroll
                for (int j = 0; j < NT; ++j) mma<false>(ks & 1 ? s2[j] : s[j], ka, q[j][ks][0], q[j][ks][1]);
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < kDt; ks += 2) {  // 32 components: two tiles of 16
                uint32_t kc[4];
                load_tiles(kc, krow + ks * 16);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t ka[4] = {codes_to_f16(kc[2 * u]), codes_to_f16(kc[2 * u + 1]), codes_to_f16(kc[2 * u] >> 16),
                                            codes_to_f16(kc[2 * u + 1] >> 16)};
#pragma unroll
                    for (int j = 0; j < NT; ++j) mma<true>(u ? s2[j] : s[j], ka, q[j][ks + u][0], q[j][ks + u][1]);
                }
            }
        }
        // scaled to log2 units; positions without anything get -inf
        float ev0 = 0.f, ev1 = 0.f, iv0 = 1.f, iv1 = 1.f, ks0 = 1.f, ks1 = 1.f;  // 8-bit: scales of positions gq, gq + 8
        if (kF8) {
            ks0 = __shfl_sync(kFull, k_scale, gq);
            ks1 = __shfl_sync(kFull, k_scale, gq + 8);
            const int b0 = __shfl_sync(kFull, v_byte, gq), b1 = __shfl_sync(kFull, v_byte, gq + 8);
            ev0 = (float)(b0 - 127);
            ev1 = (float)(b1 - 127);
            iv0 = __uint_as_float((uint32_t)(254 - b0) << 23);
            iv1 = __uint_as_float((uint32_t)(254 - b1) << 23);
        }
        const bool ok0 = valid >> gq & 1, ok1 = valid >> (gq + 8) & 1;
        bool grow = false;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = (s[j][e] + s2[j][e]) * sc[j][e & 1];
                if (kF8) x = fmaf(x, e < 2 ? ks0 : ks1, e < 2 ? ev0 : ev1);
                x = (e < 2 ? ok0 : ok1) ? x : -INFINITY;
                s[j][e] = x;
                grow = grow || x > ref[j][e & 1] + kSlack;
            }
        if (__any_sync(kFull, grow)) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float top = fmaxf(ref[j][i], fmaxf(s[j][i], s[j][i + 2]));
                    top = fmaxf(top, __shfl_xor_sync(kFull, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(kFull, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(kFull, top, 16));
                    const float f = top == ref[j][i] ? 1.f : ex2(ref[j][i] - top);
                    ref[j][i] = top;
                    sum[j][i] *= f;
#pragma unroll
                    for (int d = 0; d < kDt; ++d) {
                        o[j][d][i] *= f;
                        o[j][d][i + 2] *= f;
                    }
                }
        }
        // weights, as the second operand of O^T += V^T P^T: [positions, queries], turned 8 x 8 at a time
        uint32_t p[NT][kF8 ? 1 : 2][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const float r0 = ref[j][0] == -INFINITY ? 0.f : ref[j][0], r1 = ref[j][1] == -INFINITY ? 0.f : ref[j][1];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float p0 = ex2(s[j][2 * h] - r0), p1 = ex2(s[j][2 * h + 1] - r1);
                if (kF8) {
                    // weights of the codes: the values' scale is in the exponent already, and the sum takes it out again.
                    // fp16 holds 11 bits of a weight down to 2^-14 of the largest
                    sum[j][0] = fmaf(p0, h ? iv1 : iv0, sum[j][0]);
                    sum[j][1] = fmaf(p1, h ? iv1 : iv0, sum[j][1]);
                    p[j][0][h] = turn_tile(pack_f16(p0, p1));
                } else {
                    // a weight as the sum of two bf16 numbers: 16 bits of it instead of 8
                    sum[j][0] += p0;
                    sum[j][1] += p1;
                    const uint32_t hi = pack_bf16(p0, p1);
                    p[j][0][h] = turn_tile(hi);
                    p[j][kF8 ? 0 : 1][h] = turn_tile(pack_bf16(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xffff0000u)));
                }
            }
        }
        const uint32_t vrow = vals + ((lane & 7) + (lane >> 4) * 8) * S::kRow + (lane >> 3 & 1) * 16;
        if (!kF8) {
#pragma unroll
            for (int d = 0; d < kDt; ++d) {
                uint32_t va[4];
                load_tiles_turned(va, vrow + d * 32);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma<false>(o[j][d], va, p[j][0][0], p[j][0][1]);
                    mma<false>(o[j][d], va, p[j][kF8 ? 0 : 1][0], p[j][kF8 ? 0 : 1][1]);
                }
            }
        } else {
#pragma unroll
            for (int d = 0; d < kDt; d += 2) {  // 32 components: the even ones, then the odd ones
                uint32_t vc[4], va[2][4];
                load_tiles_turned(vc, vrow + d * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // bytes (pos 0, d), (pos 0, d + 1), (pos 1, d), (pos 1, d + 1)
                    const uint32_t x = __byte_perm(vc[e], 0, 0x3120);
                    va[0][e] = codes_to_f16(x);
                    va[1][e] = codes_to_f16(x >> 16);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma<true>(o[j][d], va[0], p[j][0][0], p[j][0][1]);
                    mma<true>(o[j][d + 1], va[1], p[j][0][0], p[j][0][1]);
                }
            }
        }
    }
    // component of the output that o[j][d][2 * e + i] of a lane belongs to (query 2t + i): see the tiles above
    static __device__ __forceinline__ int component(int d, int e, int lane) {
        return kF8 ? (d & ~1) * 16 + e * 16 + 2 * (lane >> 2) + (d & 1) : d * 16 + e * 8 + (lane >> 2);
    }
};

struct Pipe {            // the ring of stages as a CTA sees it
    char* ring;
    uint32_t ring_at;
    uint32_t (*valid)[kWarps];
    int stage;           // the stage of the next step to be consumed
};

// Columns beyond the head are zero in every stage (a product with what lies there must not be NaN); a stage that carried
// outputs is put right again.
template <class S>
__device__ __forceinline__ void clear_margin(const Pipe& pipe, int stage, int D) {
    if (D >= S::DP) return;
    __syncthreads();
    constexpr int kUnits = S::DP * S::kElem / 16;
    const int first = D * S::kElem / 16, per_row = kUnits - first;
    for (int x = threadIdx.x; x < 2 * S::kStep * per_row; x += kWarps * 32) {
        const int r = x / per_row, col = first + x - r * per_row;
        *reinterpret_cast<uint4*>(pipe.ring + stage * S::kStage + r * S::kRow + col * 16) = uint4{0, 0, 0, 0};
    }
}

// One item, from its queries to its result.  NT: tiles of 8 queries per warp.
template <class S, int NT>
__device__ __forceinline__ void run_item(const AttendArgs& g, Walk& cur, Feeder<S>& feed, Pipe& pipe, uint8_t* row_list, float2 (*stats)[16],
                                         int worker, int lane, int warp) {
    using T = typename PoolIo<S::DT>::type;
    using Ti = Tiles<S, NT>;
    constexpr bool kF8 = S::DT == PSMC_F8;
    const Division dv(cur.nq, S::kGroup, S::kSlices, warp);
    const int t = lane & 3, gq = lane >> 2;
    list_rows(cur.mask, row_list, lane);
    const int q0 = dv.group * S::kGroup, mine = dv.slice < dv.slices ? min(S::kGroup, cur.nq - q0) : 0;  // may be <= 0
    const auto place = [&](int in_tile, int* row, int* qh) {
        const int qi = cur.qt * (kGroups * S::kGroup) + in_tile, rank = div_by(qi, g.by_ratio);
        *row = cur.tile * kTileRows + row_list[rank];
        *qh = cur.head * g.l.ls.ratio + qi - rank * g.l.ls.ratio;
    };
    Ti ti;
    ti.clear();
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const uint16_t* src = nullptr;
        if (j * 8 + gq < mine) {
            int row, qh;
            place(q0 + j * 8 + gq, &row, &qh);
            src = static_cast<const uint16_t*>(g.a.q.data) + (int64_t)row * g.a.q.stride_row + (int64_t)qh * g.a.q.stride_head;
        }
        ti.load_queries(j, src, g.c.D, g.q_words, g.a.scale * kLog2e, lane);
    }
    int stage = pipe.stage;
#pragma unroll 1
    for (; cur.s < cur.s_end; ++cur.s) {
        copies_wait<S::kStages - 2>();
        __syncthreads();  // this step has landed for everyone, and everyone is done with the one before it
        const int ahead = stage == 0 ? S::kStages - 1 : stage - 1;
        feed.issue(g, pipe.ring_at + ahead * S::kStage, pipe.valid[ahead], warp, lane);
        if (mine > 0) {
            const uint32_t keys = pipe.ring_at + stage * S::kStage;
#pragma unroll 1
            for (int m = dv.slice; m < S::kSlices; m += dv.slices) {
                const uint32_t valid = pipe.valid[stage][m * kWarps / S::kSlices];
                if (valid == 0) continue;  // beyond the segment
                float k_scale = 1.f;
                int v_byte = 127;
                if (kF8) {  // lane p's scale bytes
                    const int p = cur.p0 + cur.s * S::kStep + m * 16 + (lane & 15);
                    const int off = p - div_by(p, g.by_block) * g.c.block_len, shift = ((cur.head * g.c.block_len + off) & 3) * 8;
                    const uint32_t* words = reinterpret_cast<const uint32_t*>(pipe.ring + stage * S::kStage + 2 * S::kHalf) + m * 16 + (lane & 15);
                    k_scale = __uint_as_float((words[0] >> shift & 255u) << 23);
                    v_byte = (int)(words[S::kStep] >> shift & 255u);
                }
                ti.step(keys + m * 16 * S::kRow, keys + S::kHalf + m * 16 * S::kRow, valid, k_scale, v_byte, lane);
            }
        }
        stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }
    pipe.stage = stage;
    // ---- sums over the lanes that hold parts of them, then over the slices
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x = ti.sum[j][i];
            x += __shfl_xor_sync(kFull, x, 4);
            x += __shfl_xor_sync(kFull, x, 8);
            x += __shfl_xor_sync(kFull, x, 16);
            ti.sum[j][i] = x;
        }
    if (dv.slices > 1) {
        if (gq == 0)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) stats[warp][j * 8 + 2 * t + i] = float2{ti.ref[j][i], ti.sum[j][i]};
        __syncthreads();  // also: everyone is done with the last step's stage, which now carries the outputs
        const int used = stage == 0 ? S::kStages - 1 : stage - 1;
        float* carry = reinterpret_cast<float*>(pipe.ring + used * S::kStage);  // [slice - 1 or group][component][8 queries]
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float top = -INFINITY, all = 0.f;
                for (int z = 0; z < dv.slices; ++z) top = fmaxf(top, stats[z * dv.groups + dv.group][j * 8 + 2 * t + i].x);
                for (int z = 0; z < dv.slices; ++z) {
                    const float2 st = stats[z * dv.groups + dv.group][j * 8 + 2 * t + i];
                    all += st.x == -INFINITY ? 0.f * st.y : st.y * (st.x == top ? 1.f : ex2(st.x - top));
                }
                const float f = ti.ref[j][i] == top ? 1.f : (ti.ref[j][i] == -INFINITY ? 0.f : ex2(ti.ref[j][i] - top));
                ti.ref[j][i] = top;
                ti.sum[j][i] = all;
#pragma unroll
                for (int d = 0; d < Ti::kDt; ++d) {
                    ti.o[j][d][i] *= f;
                    ti.o[j][d][i + 2] *= f;
                }
            }
            float* at = carry + ((dv.slice - 1) * dv.groups + dv.group) * (8 * S::DP);
            if (dv.slice > 0 && mine > 0) {
#pragma unroll
                for (int d = 0; d < Ti::kDt; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) at[(d * 4 + e) * 32 + lane] = ti.o[j][d][e];
            }
            __syncthreads();
            if (dv.slice == 0 && mine > 0)
                for (int z = 1; z < dv.slices; ++z) {
                    const float* from = carry + ((z - 1) * dv.groups + dv.group) * (8 * S::DP);
#pragma unroll
                    for (int d = 0; d < Ti::kDt; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) ti.o[j][d][e] += from[(d * 4 + e) * 32 + lane];
                }
            if (j + 1 < NT) __syncthreads();
        }
        clear_margin<S>(pipe, used, g.c.D);
    }
    if (dv.slice != 0) return;
    const bool alone = cur.alone(g.l);
    const int64_t slot = cur.slot(g.l, worker);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int in_group = j * 8 + 2 * t + i;
            if (in_group >= mine) continue;
            const float total = ti.sum[j][i];
            if (!alone) {
                float* part = g.l.part + (slot + q0 + in_group) * g.c.D;
#pragma unroll
                for (int d = 0; d < Ti::kDt; ++d)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int at = Ti::component(d, e, lane);
                        if (at < g.c.D) part[at] = ti.o[j][d][2 * e + i];
                    }
                if (gq == 0) g.l.stat[slot + q0 + in_group] = float2{ti.ref[j][i], total};
                continue;
            }
            int row, qh;
            place(q0 + in_group, &row, &qh);
            T* out = static_cast<T*>(g.a.out.data) + (int64_t)row * g.a.out.stride_row + (int64_t)qh * g.a.out.stride_head;
            const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int d = 0; d < Ti::kDt; ++d)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = Ti::component(d, e, lane);
                    if (at < g.c.D) put(out + at, ti.o[j][d][2 * e + i] * inv);
                }
            if (gq == 0 && g.a.lse) g.a.lse[(int64_t)row * g.a.Hq + qh] = total == 0.f ? -INFINITY : kLn2 * (ti.ref[j][i] + log2f(total));
        }
}

template <class S>
__device__ __forceinline__ bool open_pipe(const AttendArgs& g, char* smem, uint32_t (*valid)[kWarps], Pipe* pipe, Feeder<S>* feed, Walk* cur,
                                          int worker, int warp, int lane) {
    pipe->ring = smem;
    pipe->ring_at = smem_of(smem);
    pipe->valid = valid;
    pipe->stage = 0;
    if (g.c.D < S::DP) {  // columns beyond the head: never copied, always zero
        for (int i = threadIdx.x; i < S::kStages * S::kStage / 16; i += kWarps * 32) reinterpret_cast<uint4*>(smem)[i] = uint4{0, 0, 0, 0};
        __syncthreads();
    }
    chain_begin();
    feed->walk.begin(g.l, worker, lane);
    *cur = feed->walk;
    if (cur->done) return false;
    feed->begin(g, warp, lane);
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; ++i) feed->issue(g, pipe->ring_at + i * S::kStage, valid[i], warp, lane);
    return true;
}

template <class S>
__global__ void __launch_bounds__(kWarps * 32, S::kCtas) paged_attend_kernel(const AttendArgs g) {
    extern __shared__ __align__(16) char smem[];
    __shared__ uint32_t valid[S::kStages][kWarps];
    __shared__ uint8_t row_list[kWarps][kTileRows];
    __shared__ float2 stats[kWarps][16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, worker = blockIdx.x;
    Pipe pipe;
    Feeder<S> feed;
    Walk cur;
    if (!open_pipe<S>(g, smem, valid, &pipe, &feed, &cur, worker, warp, lane)) return;
    while (!cur.done) {
        if (cur.nq <= 8) run_item<S, 1>(g, cur, feed, pipe, row_list[warp], stats, worker, lane, warp);
        else run_item<S, 2>(g, cur, feed, pipe, row_list[warp], stats, worker, lane, warp);
        cur.next_item(g.l);
    }
}

// 32-bit caches: no matrix unit holds 24 bits, so the products are plain multiplications.  A slice's 16 x 8 scores are four
// per lane (one position, four queries); in the second product a lane owns DP / 32 components of all 8 queries.
template <class S>
__global__ void __launch_bounds__(kWarps * 32, S::kCtas) paged_attend_f32_kernel(const AttendArgs g) {
    constexpr int kOwn = S::DP / 32;
    extern __shared__ __align__(16) char smem[];
    __shared__ uint32_t valid[S::kStages][kWarps];
    __shared__ uint8_t row_list[kWarps][kTileRows];
    __shared__ float2 stats[kWarps][8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, worker = blockIdx.x, key = lane & 15, qh4 = (lane >> 4) * 4;
    float* qs = reinterpret_cast<float*>(smem + S::kStages * S::kStage) + warp * (8 * S::DP + 16 * 8);  // [8][DP]
    float* ps = qs + 8 * S::DP;                                                                         // [16][8]
    Pipe pipe;
    Feeder<S> feed;
    Walk cur;
    if (!open_pipe<S>(g, smem, valid, &pipe, &feed, &cur, worker, warp, lane)) return;
    const float to_log2 = g.a.scale * kLog2e;
    while (!cur.done) {
        const Division dv(cur.nq, S::kGroup, S::kSlices, warp);
        list_rows(cur.mask, row_list[warp], lane);
        const int q0 = dv.group * S::kGroup, mine = dv.slice < dv.slices ? min(S::kGroup, cur.nq - q0) : 0;  // may be <= 0
        const auto place = [&](int in_tile, int* row, int* qh) {
            const int qi = cur.qt * (kGroups * S::kGroup) + in_tile, rank = div_by(qi, g.by_ratio);
            *row = cur.tile * kTileRows + row_list[warp][rank];
            *qh = cur.head * g.l.ls.ratio + qi - rank * g.l.ls.ratio;
        };
        {
            float x[8][kOwn];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int row = 0, qh = 0;
                if (j < mine) place(q0 + j, &row, &qh);
                const float* q = static_cast<const float*>(g.a.q.data) + (int64_t)row * g.a.q.stride_row + (int64_t)qh * g.a.q.stride_head;
#pragma unroll
                for (int i = 0; i < kOwn; ++i) x[j][i] = j < mine && lane + 32 * i < g.c.D ? __ldg(q + lane + 32 * i) : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < kOwn; ++i) qs[j * S::DP + lane + 32 * i] = x[j][i];
        }
        float o[8][kOwn], ref[4], sum[4];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < kOwn; ++i) o[j][i] = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            ref[u] = -INFINITY;
            sum[u] = 0.f;
        }
        __syncwarp();
        int stage = pipe.stage;
#pragma unroll 1
        for (; cur.s < cur.s_end; ++cur.s) {
            copies_wait<S::kStages - 2>();
            __syncthreads();  // this step has landed for everyone, and everyone is done with the one before it
            const int ahead = stage == 0 ? S::kStages - 1 : stage - 1;
            feed.issue(g, pipe.ring_at + ahead * S::kStage, pipe.valid[ahead], warp, lane);
#pragma unroll 1
            for (int m = dv.slice; m < S::kSlices && mine > 0; m += dv.slices) {
                // a slice lies within one warp's copies, or (steps of 32) spans two warps' 8 positions each
                uint32_t has = pipe.valid[stage][m * kWarps / S::kSlices];
                if (S::kSlices < kWarps) has |= pipe.valid[stage][m * kWarps / S::kSlices + 1] << 8;
                if (has == 0) continue;
                const bool ok = has >> key & 1;
                const char* keys = pipe.ring + stage * S::kStage + m * 16 * S::kRow;
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                for (int d = 0; d < S::DP; d += 4) {
                    const float4 k = *reinterpret_cast<const float4*>(keys + key * S::kRow + d * 4);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float4 q = *reinterpret_cast<const float4*>(qs + (qh4 + u) * S::DP + d);
                        s[u] = fmaf(k.x, q.x, fmaf(k.y, q.y, fmaf(k.z, q.z, fmaf(k.w, q.w, s[u]))));
                    }
                }
                float f[4];
                bool moved = false;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    s[u] = ok ? s[u] * to_log2 : -INFINITY;
                    float top = s[u];
#pragma unroll
                    for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, x));
                    top = fmaxf(ref[u], top);
                    f[u] = top == ref[u] ? 1.f : exp2f(ref[u] - top);
                    moved = moved || f[u] != 1.f;
                    ref[u] = top;
                    const float p = exp2f(s[u] - (top == -INFINITY ? 0.f : top));
                    sum[u] = fmaf(sum[u], f[u], p);
                    ps[key * 8 + qh4 + u] = p;
                }
                if (__any_sync(kFull, moved)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float fj = __shfl_sync(kFull, f[j & 3], j < 4 ? 0 : 16);
#pragma unroll
                        for (int i = 0; i < kOwn; ++i) o[j][i] *= fj;
                    }
                }
                __syncwarp();
                const char* vals = keys + S::kHalf;
#pragma unroll 4
                for (int p = 0; p < 16; ++p) {
                    const float4 w0 = *reinterpret_cast<const float4*>(ps + p * 8), w1 = *reinterpret_cast<const float4*>(ps + p * 8 + 4);
#pragma unroll
                    for (int i = 0; i < kOwn; ++i) {
                        const float v = *reinterpret_cast<const float*>(vals + p * S::kRow + (lane + 32 * i) * 4);
                        o[0][i] = fmaf(w0.x, v, o[0][i]);
                        o[1][i] = fmaf(w0.y, v, o[1][i]);
                        o[2][i] = fmaf(w0.z, v, o[2][i]);
                        o[3][i] = fmaf(w0.w, v, o[3][i]);
                        o[4][i] = fmaf(w1.x, v, o[4][i]);
                        o[5][i] = fmaf(w1.y, v, o[5][i]);
                        o[6][i] = fmaf(w1.z, v, o[6][i]);
                        o[7][i] = fmaf(w1.w, v, o[7][i]);
                    }
                }
                __syncwarp();
            }
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
        }
        pipe.stage = stage;
        // ---- sums over the lanes, then over the slices
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) sum[u] += __shfl_xor_sync(kFull, sum[u], x);
            if (key == 0) stats[warp][qh4 + u] = float2{ref[u], sum[u]};
        }
        __syncthreads();  // also: everyone is done with the last step's stage, which now carries the outputs
        const int used = stage == 0 ? S::kStages - 1 : stage - 1;
        float* carry = reinterpret_cast<float*>(pipe.ring + used * S::kStage);
        float total[8], high[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float top = -INFINITY, all = 0.f;
            for (int z = 0; z < dv.slices; ++z) top = fmaxf(top, stats[z * dv.groups + dv.group][j].x);
            for (int z = 0; z < dv.slices; ++z) {
                const float2 st = stats[z * dv.groups + dv.group][j];
                all += st.x == -INFINITY ? 0.f * st.y : st.y * (st.x == top ? 1.f : exp2f(st.x - top));
            }
            const float own = stats[warp][j].x, fj = own == top ? 1.f : (own == -INFINITY ? 0.f : exp2f(own - top));
            total[j] = all;
            high[j] = top;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                o[j][i] *= fj;
                if (dv.slice > 0 && dv.slice < dv.slices)
                    carry[((dv.slice - 1) * dv.groups + dv.group) * (8 * S::DP) + j * S::DP + lane + 32 * i] = o[j][i];
            }
        }
        __syncthreads();
        if (dv.slice == 0 && mine > 0) {
            const bool alone = cur.alone(g.l);
            const int64_t slot = cur.slot(g.l, worker);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= mine) break;
                int row, qh;
                place(q0 + j, &row, &qh);
                float* out = static_cast<float*>(g.a.out.data) + (int64_t)row * g.a.out.stride_row + (int64_t)qh * g.a.out.stride_head;
                const float inv = total[j] == 0.f ? 0.f : 1.f / total[j];
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int d = lane + 32 * i;
                    float x = o[j][i];
                    for (int z = 1; z < dv.slices; ++z) x += carry[((z - 1) * dv.groups + dv.group) * (8 * S::DP) + j * S::DP + d];
                    if (d >= g.c.D) continue;
                    if (alone) out[d] = x * inv;
                    else g.l.part[(slot + q0 + j) * g.c.D + d] = x;
                }
                if (lane == 0) {
                    if (!alone) g.l.stat[slot + q0 + j] = float2{high[j], total[j]};
                    else if (g.a.lse) g.a.lse[(int64_t)row * g.a.Hq + qh] = total[j] == 0.f ? -INFINITY : kLn2 * (high[j] + log2f(total[j]));
                }
            }
        }
        clear_margin<S>(pipe, used, g.c.D);
        cur.next_item(g.l);
    }
}

// ---------------------------------------------------------------------------------------------------------- join
// WPQ warps per (row, query head).  Each of them lists the query's partial results, and takes every WPQ-th.
constexpr int kMaxWorkers = 2 * kSMs;
constexpr int kJoinThreads = 128;

template <int DT, int WPQ>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const AttendArgs g) {
    using T = typename PoolIo<DT>::type;
    constexpr int kJoinWarps = kJoinThreads / 32, kQueries = kJoinWarps / WPQ, kOwn = kMaxHeadDim / 128, kList = 32, kBatch = 8;
    __shared__ int64_t slots[kJoinWarps][kList];
    __shared__ __align__(16) float acc[WPQ == 1 ? 1 : WPQ][kMaxHeadDim];  // read and written 16 bytes at a time
    __shared__ float2 stats[kJoinWarps];
    chain_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub_warp = warp % WPQ;
    const int64_t item = (int64_t)blockIdx.x * kQueries + warp / WPQ;
    if (item >= (int64_t)g.c.R * g.a.Hq) return;  // the warps of a query agree
    const int row = (int)(item / g.a.Hq), qh = (int)(item - (int64_t)row * g.a.Hq);
    const int tile = row / kTileRows, in_tile = row % kTileRows, head = qh / g.l.ls.ratio, sub = qh - head * g.l.ls.ratio;
    const TilePlan& tp = g.l.plans[tile];
    const LineShape& ls = g.l.ls;
    const int qt_size = kGroups * ls.group;
    uint32_t masks[kMaxSegs / 32];
#pragma unroll
    for (int i = 0; i < kMaxSegs / 32; ++i) masks[i] = tp.seg[i * 32 + lane].mask;  // those beyond n_segs are not looked at
    const Bearings b = bearings(g.l, 0, tile, lane);
    const int n_segs = tp.n_segs;
    if (tp.left_out >> in_tile & 1) return;

    float top = -INFINITY, total = 0.f;
    float4 o[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) o[i] = float4{0.f, 0.f, 0.f, 0.f};
    int listed = 0, seen = 0;  // in this warp's list; of the query altogether
    // the listed results, at most kList, into the running ones: the largest reference decides, the others' weights are
    // 2^(their reference - it)
    const auto take = [&] {
        __syncwarp();
        for (int i0 = 0; i0 < listed; i0 += kBatch) {
            const int n = min(kBatch, listed - i0);
            float2 st = float2{-INFINITY, 0.f};
            if (lane < n) st = g.l.stat[slots[warp][i0 + lane]];
            float4 x[kBatch][kOwn];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int d = lane * 4 + i * 128;
                    x[u][i] = float4{0.f, 0.f, 0.f, 0.f};
                    if (u < n && d < g.c.D) x[u][i] = *reinterpret_cast<const float4*>(g.l.part + slots[warp][i0 + u] * g.c.D + d);
                }
            const float high = fmaxf(top, warp_max(st.x)), keep = top == high ? 1.f : exp2f(top - high);
            const float f = st.x == -INFINITY ? 0.f : (st.x == high ? 1.f : exp2f(st.x - high));
            total = fmaf(total, keep, warp_sum(lane < n ? st.y * f : 0.f));
            top = high;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) o[i] = float4{o[i].x * keep, o[i].y * keep, o[i].z * keep, o[i].w * keep};
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const float fu = __shfl_sync(kFull, f, u);
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    o[i].x = fmaf(fu, x[u][i].x, o[i].x);
                    o[i].y = fmaf(fu, x[u][i].y, o[i].y);
                    o[i].z = fmaf(fu, x[u][i].z, o[i].z);
                    o[i].w = fmaf(fu, x[u][i].w, o[i].w);
                }
            }
        }
        __syncwarp();
        listed = 0;
    };
#pragma unroll 1
    for (int i = 0; i < kMaxSegs / 32; ++i) {
        uint32_t with = __ballot_sync(kFull, i * 32 + lane < n_segs && (masks[i] >> in_tile & 1));
        while (with) {
            const Segment sg = tp.seg[i * 32 + __ffs(with) - 1];
            with &= with - 1;
            const int qi = __popc(sg.mask & ((1u << in_tile) - 1)) * ls.ratio + sub, qt = qi / qt_size;
            const int steps = steps_of(ls, sg.p0, sg.p1);
            const int w = step_cost(ls, min(qt_size, __popc(sg.mask) * ls.ratio - qt * qt_size));
            const int64_t a = b.before + head * tp.cost + sg.start + (int64_t)qt * steps * step_cost(ls, qt_size);
            const int64_t k0 = a / b.share, k1 = (a + (int64_t)steps * w - 1) / b.share;
            const int64_t first = ((int64_t)tile * ls.H + head) * (kTileRows * kRowSegs * ls.ratio) + (int64_t)sg.before * ls.ratio + qi;
            for (int64_t kb = k0; kb <= k1; kb += 32) {
                const int64_t k = kb + lane;
                const int from = steps_before(k * b.share, a, w, steps);
                const bool has = k <= k1 && from < steps_before((k + 1) * b.share, a, w, steps);  // a share may lie between two steps
                const uint32_t who = __ballot_sync(kFull, has);
                const int mine_at = seen + __popc(who & ((1u << lane) - 1));
                const bool keep = has && mine_at % WPQ == sub_warp;
                const uint32_t kept = __ballot_sync(kFull, keep);
                if (listed + __popc(kept) > kList) take();
                if (keep)
                    slots[warp][listed + __popc(kept & ((1u << lane) - 1))] =
                        from == 0 ? first : g.l.first_rest + k * qt_size + (qi - qt * qt_size);
                listed += __popc(kept);
                seen += __popc(who);
            }
        }
    }
    if (seen == 1 && (tp.whole >> in_tile & 1)) return;  // already in place
    take();
    if (WPQ > 1) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) *reinterpret_cast<float4*>(&acc[sub_warp][lane * 4 + i * 128]) = o[i];
        if (lane == 0) stats[warp] = float2{top, total};
        __syncthreads();
        if (sub_warp != 0) return;
        for (int w = 0; w < WPQ; ++w) top = fmaxf(top, stats[w].x);
        total = 0.f;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) o[i] = float4{0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < WPQ; ++w) {
            const float2 st = stats[w];
            const float f = st.x == -INFINITY ? 0.f : (st.x == top ? 1.f : exp2f(st.x - top));
            total = fmaf(st.y, f, total);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const float4 x = *reinterpret_cast<const float4*>(&acc[w][lane * 4 + i * 128]);
                o[i].x = fmaf(f, x.x, o[i].x);
                o[i].y = fmaf(f, x.y, o[i].y);
                o[i].z = fmaf(f, x.z, o[i].z);
                o[i].w = fmaf(f, x.w, o[i].w);
            }
        }
    }
    T* out = static_cast<T*>(g.a.out.data) + (int64_t)row * g.a.out.stride_row + (int64_t)qh * g.a.out.stride_head;
    const float inv = total == 0.f ? 0.f : 1.f / total;  // no positions: zeros
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int d = lane * 4 + i * 128;
        if (d >= g.c.D) continue;
        put(out + d, o[i].x * inv);
        put(out + d + 1, o[i].y * inv);
        put(out + d + 2, o[i].z * inv);
        put(out + d + 3, o[i].w * inv);
    }
    if (lane == 0 && g.a.lse) g.a.lse[(int64_t)row * g.a.Hq + qh] = total == 0.f ? -INFINITY : kLn2 * (top + log2f(total));
}

// ---------------------------------------------------------------------------------------------------------- launches
struct Scratch {
    size_t plans, stat, part, bytes;
    int64_t first_rest;
    int n_tiles;
};
constexpr int kMaxQueryTile = kGroups * 16;
Scratch scratch_of(int R, int Hq, int D) {
    Scratch s;
    s.n_tiles = (R + kTileRows - 1) / kTileRows;
    s.first_rest = (int64_t)s.n_tiles * kTileRows * kRowSegs * Hq;
    const size_t slots = (size_t)s.first_rest + (size_t)kMaxWorkers * kMaxQueryTile;
    const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    s.plans = 0;
    s.stat = up((size_t)s.n_tiles * sizeof(TilePlan));
    s.part = s.stat + up(slots * sizeof(float2));
    s.bytes = s.part + up(slots * D * sizeof(float));
    return s;
}

template <int DT, int DP>
cudaError_t launch(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    using S = Shape<DT, DP>;
    const Scratch sc = scratch_of(c.R, a.Hq, c.D);
    char* scratch = static_cast<char*>(a.scratch);
    AttendArgs g{};
    g.c = c;
    g.a = a;
    g.by_block = fast_div(c.block_len);
    g.l.ls = LineShape{S::kStep, S::kGroup, a.Hq / c.H, c.H};
    g.by_ratio = fast_div(g.l.ls.ratio);
    g.q_words = ((uint64_t)(uintptr_t)a.q.data % 4 == 0 && a.q.stride_row % 2 == 0 && a.q.stride_head % 2 == 0) ? 1 : 0;
    TilePlan* plans = reinterpret_cast<TilePlan*>(scratch + sc.plans);
    g.l.plans = plans;
    g.l.stat = reinterpret_cast<float2*>(scratch + sc.stat);
    g.l.part = reinterpret_cast<float*>(scratch + sc.part);
    g.l.first_rest = sc.first_rest;
    g.l.n_tiles = sc.n_tiles;
    g.l.workers = S::kCtas * kSMs;
    cudaError_t e = launch_chained(paged_plan_kernel, dim3((unsigned)sc.n_tiles), dim3(kPlanThreads), 0, stream, c, a, g.l.ls, plans);
    if (e != cudaSuccess) return e;
    void (*fn)(const AttendArgs);
    if constexpr (DT == PSMC_F32) fn = paged_attend_f32_kernel<S>;
    else fn = paged_attend_kernel<S>;
    e = allow_dynamic_smem(reinterpret_cast<const void*>(fn), S::kBytes);
    if (e == cudaSuccess) e = launch_chained(fn, dim3((unsigned)g.l.workers), dim3(kWarps * 32), S::kBytes, stream, g);
    if (e != cudaSuccess) return e;
    // few queries: four warps each, for what may be many partial results of a long row
    const int64_t queries = (int64_t)c.R * a.Hq;
    if (queries <= 8 * kSMs) return launch_chained(paged_join_kernel<DT, 4>, dim3((unsigned)queries), dim3(kJoinThreads), 0, stream, g);
    return launch_chained(paged_join_kernel<DT, 1>, dim3((unsigned)((queries + 3) / 4)), dim3(kJoinThreads), 0, stream, g);
}

template <int DT>
cudaError_t launch_dim(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    if (c.D <= 64) return launch<DT, 64>(c, a, stream);
    if (c.D <= 96) return launch<DT, 96>(c, a, stream);
    if (c.D <= 128) return launch<DT, 128>(c, a, stream);
    return launch<DT, 256>(c, a, stream);
}

}  // namespace

size_t paged_attend_scratch_bytes(int R, int Hq, int, int D) { return scratch_of(R, Hq, D).bytes; }

cudaError_t launch_paged_attend(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    if (c.dt == PSMC_F32) return launch_dim<PSMC_F32>(c, a, stream);
    return c.dt == PSMC_BF16 ? launch_dim<PSMC_BF16>(c, a, stream) : launch_dim<PSMC_F8>(c, a, stream);
}

}  // namespace psmc

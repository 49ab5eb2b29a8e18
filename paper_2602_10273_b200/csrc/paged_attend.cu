// Attention of one new token per row over the paged cache:  out[r, h] = sum_p softmax_p(scale q[r, h] . k_p) v_p over
// the positions p < n_r = lens[r] + extra of row r.
//
// The particles of a group descend from common ancestors, so their rows share blocks: all of them far back, ever fewer
// of them towards the end.  What bounds the operator is reading every distinct block once; sharing is found on the
// device, since only the table knows it.  Three kernels, chained:
//
//   plan    per tile of 32 rows: which rows hold the same block at block index j (a match over the warp's lanes, a lane
//           per row), and the runs of j over which such a set of rows stays the same: the tile's SEGMENTS.  A segment's
//           queries (rows x query heads per key-value head) meet its keys and values together.
//   attend  the work of all (tile, key-value head, segment, query tile) items is laid on one line, in steps of 16 or 32
//           positions, and cut into equal shares, one per warp of a grid that fills the GPU: long rows are split, short
//           ones are strung together, and no warp waits for another.  A warp streams its steps through a ring of
//           shared-memory stages of its own (cp.async, 16 bytes per lane) and keeps running reference, sum and output
//           of its item in registers.  Items that lie in one share and cover their rows entirely are finished here.
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
    int n[kTileRows];    // positions of each row (0 where there are none, or where the row is left out)
    int n_segs, whole;   // whole: bit mask of rows that have a single segment
    uint32_t left_out;   // rows with skip != 0 (or beyond R)
    int64_t cost;        // of one key-value head
    Segment seg[kMaxSegs];
};

// what a step costs by the 8-query tiles it meets: the bytes are the same, the arithmetic is not
__host__ __device__ constexpr int step_cost(int tiles) { return 2 + tiles; }

struct LineShape {       // how the items of a tile are cut; a pure function of the launch
    int step;            // positions per step
    int qt;              // queries per query tile
    int ratio, H;
};
__device__ __forceinline__ int64_t seg_cost(const LineShape& s, int rows, int steps) {
    const int nq = rows * s.ratio, full = nq / s.qt, rem = nq - full * s.qt;
    return (int64_t)steps * (full * step_cost(s.qt / 8) + (rem ? step_cost((rem + 7) / 8) : 0));
}
__device__ __forceinline__ int steps_of(const LineShape& s, int p0, int p1) { return (p1 - p0 + s.step - 1) / s.step; }

constexpr int kPlanThreads = 512, kPlanWarps = kPlanThreads / 32;

__global__ void __launch_bounds__(kPlanThreads) paged_plan_kernel(const PagedView c, const PagedAttend a, const LineShape ls,
                                                                  TilePlan* plans) {
    __shared__ int n[kTileRows], from[kMaxSegs], count[kPlanWarps], rows_in[kPlanWarps], lead[kMaxSegs];
    __shared__ uint32_t mask[kMaxSegs];
    __shared__ uint32_t out_mask;
    chain_begin();
    const int tile = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    TilePlan& tp = plans[tile];
    const int row = tile * kTileRows + lane;
    if (warp == 0) {
        int64_t len = 0;
        bool left_out = row >= c.R;
        if (!left_out && a.skip && a.skip[row]) left_out = true;
        if (!left_out) {
            len = (int64_t)__ldg(a.lens + row) + a.extra;
            const int64_t room = (int64_t)c.max_blocks * c.block_len;
            if (len > room) {
                raise_status(a.status, PSMC_E_STATE);
                len = room;
            }
            if (len < 0) len = 0;
        }
        n[lane] = (int)len;
        tp.n[lane] = (int)len;
        const uint32_t lo = __ballot_sync(kFull, left_out);
        if (lane == 0) out_mask = lo;
    }
    __syncthreads();
    const int my_n = n[lane], B = c.block_len;
    const uint32_t alive = __ballot_sync(kFull, my_n > 0);
    const int nb = warp_max((my_n + B - 1) / B);
    const int32_t* entries = c.table + (int64_t)row * c.table_ld;

    // the set of rows that hold this lane's block at block index j in the same state (0: the row ends before it)
    const auto set_of = [&](int j, int entry) -> uint32_t {
        const int live = min(B, my_n - j * B);  // may be far below zero, never far above
        const bool in = j * (int64_t)B < my_n;
        const bool named = in && entry >= 0 && entry < c.n_blocks;
        uint32_t same = __match_any_sync(kFull, named ? entry : -1 - lane);
        same &= __match_any_sync(kFull, in ? live : 0);
        return in ? (named ? same : 1u << lane) : 0u;
    };
    const auto entry_of = [&](int j) -> int { return j * (int64_t)B < my_n ? __ldg(entries + j) : -1; };

    int n_segs = 0;
    const bool share = __popc(alive) > 1;
    if (share) {
        const int per = (nb + kPlanWarps - 1) / kPlanWarps, j0 = min(nb, warp * per), j1 = min(nb, j0 + per);
        constexpr int kAhead = 8;  // table entries in flight per lane
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {  // count, then write at a place that depends on the table alone
            uint32_t prev = 0;
            if (j0 > 0 && j0 < j1) prev = set_of(j0 - 1, entry_of(j0 - 1));
            int at = 0, starts = 0, rows = 0;
            if (pass == 1)
                for (int w = 0; w < warp; ++w) at += count[w];
            for (int jb = j0; jb < j1; jb += kAhead) {
                int e[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) e[u] = jb + u < j1 ? entry_of(jb + u) : -1;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int j = jb + u;
                    if (j >= j1) break;
                    const uint32_t set = set_of(j, e[u]);
                    const bool starting = set != 0 && set != prev && lane == __ffs(set) - 1;
                    const uint32_t who = __ballot_sync(kFull, starting);
                    if (starting) {
                        rows += __popc(set);
                        if (pass == 1) {
                            const int s = at + starts + __popc(who & ((1u << lane) - 1));
                            mask[s] = set;
                            from[s] = j;
                            lead[s] = lane;
                        }
                    }
                    starts += __popc(who);
                    prev = set;
                }
            }
            if (pass == 0) {
                rows = (int)warp_sum((float)min(rows, 1 << 20));
                if (lane == 0) {
                    count[warp] = min(starts, 1 << 20);
                    rows_in[warp] = rows;
                }
                __syncthreads();
                int rows_all = 0;
                for (int w = 0; w < kPlanWarps; ++w) {
                    n_segs += count[w];
                    rows_all += rows_in[w];
                }
                if (n_segs > kMaxSegs || rows_all > kTileRows * kRowSegs) n_segs = 0;
                if (n_segs == 0) break;  // the same for every thread
            }
        }
    }
    if (n_segs == 0) {  // row by row
        n_segs = __popc(alive);
        if (warp == 0 && my_n > 0) {
            const int s = __popc(alive & ((1u << lane) - 1));
            mask[s] = 1u << lane;
            from[s] = 0;
            lead[s] = lane;
        }
    }
    __syncthreads();
    for (int s = threadIdx.x; s < n_segs; s += kPlanThreads) {
        // ends where its first row enters another segment, or ends itself
        const int who = lead[s], j0 = from[s], len = n[who];
        int end = (len + B - 1) / B;
        for (int o = 0; o < n_segs; ++o)
            if (from[o] > j0 && (mask[o] >> who & 1)) end = min(end, from[o]);
        tp.seg[s].mask = mask[s];
        tp.seg[s].p0 = j0 * B;
        tp.seg[s].p1 = (int)min((int64_t)end * B, (int64_t)len);
    }
    __syncthreads();
    if (warp == 0) {
        int64_t cost = 0;
        int before = 0;
        uint32_t single = 0;
        for (int s0 = 0; s0 < n_segs; s0 += 32) {
            const int s = s0 + lane;
            const bool in = s < n_segs;
            const int rows = in ? __popc(mask[s]) : 0;
            const int64_t cs = in ? seg_cost(ls, rows, steps_of(ls, tp.seg[s].p0, tp.seg[s].p1)) : 0;
            const int64_t upto = warp_scan_incl<long long>(cs, lane);
            const int rows_upto = warp_scan_incl(rows, lane);
            if (in) {
                tp.seg[s].start = cost + upto - cs;
                tp.seg[s].before = before + rows_upto - rows;
                if (tp.seg[s].p0 == 0) {  // every row of the set ends where the segment does
                    bool all = true;
                    for (uint32_t m = mask[s]; m; m &= m - 1) all = all && n[__ffs(m) - 1] == tp.seg[s].p1;
                    if (all) single |= mask[s];
                }
            }
            cost += __shfl_sync(kFull, (long long)upto, 31);
            before += __shfl_sync(kFull, rows_upto, 31);
        }
        single = __reduce_or_sync(kFull, single);
        if (lane == 0) {
            tp.n_segs = n_segs;
            tp.whole = (int)single;
            tp.left_out = out_mask;
            tp.cost = cost;
        }
    }
}

// ------------------------------------------------------------------------------------------------- the line and its shares
struct Line {
    const TilePlan* plans;
    int n_tiles, workers;
    int64_t min_share;
    float* part;         // [.., D] unnormalised outputs: those of whole or first parts of items, then one set per worker
    float2* stat;        // {reference, sum} of each
    int64_t first_rest;  // where the sets of the workers begin
    LineShape ls;
};

// Total cost, and per tile of 32 lanes the cost before it: every warp adds the tiles up again (16 numbers for 512 rows).
__device__ __forceinline__ int64_t line_total(const Line& l, int lane) {
    int64_t sum = 0;
    for (int t = lane; t < l.n_tiles; t += 32) sum += l.plans[t].cost * l.ls.H;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, (long long)sum, o);
    return sum;
}
// tile that holds cost unit x (x < total), and the cost before it
__device__ __forceinline__ int tile_at(const Line& l, int64_t x, int lane, int64_t* before) {
    int64_t base = 0;
    for (int t0 = 0; t0 < l.n_tiles; t0 += 32) {
        const int t = t0 + lane;
        const int64_t cs = t < l.n_tiles ? l.plans[t].cost * l.ls.H : 0;
        const int64_t upto = base + warp_scan_incl<long long>(cs, lane);
        const uint32_t beyond = __ballot_sync(kFull, t < l.n_tiles && upto > x);
        if (beyond) {
            const int at = __ffs(beyond) - 1;
            *before = __shfl_sync(kFull, (long long)(upto - cs), at);
            return t0 + at;
        }
        base = __shfl_sync(kFull, (long long)upto, 31);
    }
    *before = base;
    return l.n_tiles;
}
__device__ __forceinline__ int64_t cost_before(const Line& l, int tile, int lane) {
    int64_t sum = 0;
    for (int t = lane; t < tile; t += 32) sum += l.plans[t].cost * l.ls.H;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, (long long)sum, o);
    return sum;
}
__device__ __forceinline__ int64_t share_of(const Line& l, int64_t total) {
    const int64_t even = (total + l.workers - 1) / l.workers;
    return even > l.min_share ? even : l.min_share;
}
// the steps of an item (first cost unit a, cost w per step) that fall into [lo, hi)
__device__ __forceinline__ int step_from(int64_t bound, int64_t a, int w, int steps) {
    if (bound <= a) return 0;
    const int64_t d = bound - a;
    return d >= (int64_t)steps * w ? steps : (int)((uint32_t)((uint32_t)d + w - 1) / (uint32_t)w);
}

// One worker's walk along the line.  All lanes hold the same values.
struct Walk {
    int64_t a, hi;       // first cost unit of the item at hand; end of the share
    int tile, head, si, qt, n_qt, n_segs;
    uint32_t mask;
    int p0, p1;          // positions of the segment
    int nq;              // queries of this query tile
    int w, steps;
    int s, s_end;        // steps of the item that are this worker's: the next one, and the end
    int s_first;
    bool done;

    __device__ __forceinline__ void open_segment(const Line& l) {
        const Segment& g = l.plans[tile].seg[si];
        mask = g.mask;
        p0 = g.p0;
        p1 = g.p1;
        steps = steps_of(l.ls, p0, p1);
        n_qt = (__popc(mask) * l.ls.ratio + l.ls.qt - 1) / l.ls.qt;
    }
    __device__ __forceinline__ void open_item(const Line& l, int64_t lo) {
        nq = min(l.ls.qt, __popc(mask) * l.ls.ratio - qt * l.ls.qt);
        w = step_cost((nq + 7) / 8);
        s_first = s = step_from(lo, a, w, steps);
        s_end = step_from(hi, a, w, steps);
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
        const int64_t total = line_total(l, lane), share = share_of(l, total), lo = worker * share;
        hi = min(lo + share, total);
        done = lo >= total;
        if (done) return;
        int64_t before;
        tile = tile_at(l, lo, lane, &before);
        const TilePlan& tp = l.plans[tile];
        const int64_t x = lo - before;
        head = (int)(x / tp.cost);
        const int64_t y = x - head * tp.cost;
        n_segs = tp.n_segs;
        si = -1;
        for (int s0 = 0; s0 < n_segs; s0 += 32)
            si += __popc(__ballot_sync(kFull, s0 + lane < n_segs && tp.seg[min(s0 + lane, n_segs - 1)].start <= y));
        open_segment(l);
        const int64_t full = (int64_t)steps * step_cost(l.ls.qt / 8), into = y - tp.seg[si].start;
        qt = (int)min((int64_t)(n_qt - 1), into / full);
        a = before + head * tp.cost + tp.seg[si].start + qt * full;
        open_item(l, lo);
        if (s >= s_end) next_item(l);
    }
    __device__ __forceinline__ bool alone(const Line& l) const {  // the whole of its rows, in this share
        return s_first == 0 && s_end == steps && (l.plans[tile].whole & mask) == mask;
    }
    // where the partial result of the item's query 0 goes
    __device__ __forceinline__ int64_t slot(const Line& l, int worker) const {
        if (s_first > 0) return l.first_rest + (int64_t)worker * l.ls.qt;
        return ((int64_t)tile * l.ls.H + head) * (kTileRows * kRowSegs * l.ls.ratio) +
               (int64_t)l.plans[tile].seg[si].before * l.ls.ratio + qt * l.ls.qt;
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

// Shape of a warp's work.  DP: head_dim rounded up to what the tiles are unrolled for; NT: query tiles of 8.
template <int DT, int DP_, int NT_>
struct Shape {
    static constexpr int DP = DP_, NT = NT_;  // (32-bit caches: one query tile)
    static constexpr int kElem = DT == PSMC_F32 ? 4 : (DT == PSMC_BF16 ? 2 : 1);
    static constexpr int kStep = DT == PSMC_F8 ? 32 : 16;                 // positions per step
    static constexpr int kRow = DP * kElem + 16;                          // bytes between rows: an odd number of 16-byte units
    static constexpr int kHalf = kStep * kRow;                            // keys, then values
    static constexpr int kScales = DT == PSMC_F8 ? kStep * 4 : 0;         // words that hold the scale bytes
    static constexpr int kStage = 2 * (kHalf + kScales);
    static constexpr int kSpace = 113 * 1024;                             // two CTAs per SM
    static constexpr int kWarps = kStage * 4 * 3 <= kSpace ? 4 : (kStage * 2 * 3 <= kSpace ? 2 : 1);
    static constexpr int kFit = kSpace / (kStage * kWarps);
    static constexpr int kStages = kFit > 8 ? 8 : kFit;
    // 32-bit caches: queries (8 rows of DP) and weights (16 positions x 8 queries) of a warp
    static constexpr int kExtra = DT == PSMC_F32 ? (8 * DP + 16 * 8) * 4 : 0;
    static constexpr int kBytes = kWarps * (kStages * kStage + kExtra);
    static_assert(kStages >= 2 && kBytes + kWarps * 256 <= 227 * 1024 / 2, "shared memory of two CTAs");
};

struct AttendArgs {
    PagedView c;
    PagedAttend a;
    Line l;
    FastDiv by_block, by_ratio;
};

// The copying side of a walk: entries of the table are asked for one step ahead of the copies that need them.
template <class S, int DT>
struct Feeder {
    Walk walk;
    uint32_t unit;       // lane p: where position p of the step begins, in 16-byte units from the pool's start
    int scale_word;      // 8-bit: its scale byte's word, counted from the block's start in words; -1: no such position
    int entry;           // lane p: its table entry
    int in_block;        // lane p: (head * block_len + offset), or -1 beyond the segment

    __device__ __forceinline__ void ask(const AttendArgs& g, int lane) {
        if (walk.done) return;
        const int p = walk.p0 + walk.s * S::kStep + lane;
        in_block = -1;
        entry = -1;
        if (lane < S::kStep && p < walk.p1) {
            const int j = div_by(p, g.by_block);
            in_block = walk.head * g.c.block_len + (p - j * g.c.block_len);
            const int row = walk.tile * kTileRows + __ffs(walk.mask) - 1;
            entry = __ldg(g.c.table + (int64_t)row * g.c.table_ld + j);
        }
    }
    // copies of the step asked for, into the stage at `stage`; valid_out: which positions hold something
    __device__ __forceinline__ void issue(const AttendArgs& g, uint32_t stage, uint32_t* valid_out, int lane) {
        if (!walk.done) {
            const bool named = in_block >= 0 && entry >= 0 && entry < g.c.n_blocks;
            if (in_block >= 0 && !named) raise_status(g.a.status, PSMC_E_STATE);
            const uint32_t valid = __ballot_sync(kFull, named);
            const int per_row = g.c.D * S::kElem / 16;
            const uint32_t unit = named ? (uint32_t)entry * (uint32_t)(g.c.blk_bytes / 16) + (uint32_t)(in_block * per_row) : 0u;
            constexpr int kPerRow = S::DP * S::kElem / 16, kCopies = S::kStep * kPerRow / 32;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const int x = i * 32 + lane, r = x / kPerRow, col = x - r * kPerRow;
                const uint32_t at = __shfl_sync(kFull, unit, r);
                const int bytes = valid >> r & 1 ? 16 : 0;
                if (col < per_row) {
                    const int64_t off = ((int64_t)at + (bytes ? col : 0)) * 16;
                    copy16(stage + r * S::kRow + col * 16, g.c.k + off, bytes);
                    copy16(stage + S::kHalf + r * S::kRow + col * 16, g.c.v + off, bytes);
                }
            }
            if (DT == PSMC_F8) {
                const int64_t off = named ? (int64_t)entry * g.c.blk_bytes + g.c.scale_at + (in_block & ~3) : 0;
                copy4(stage + 2 * S::kHalf + lane * 4, g.c.k + off, named ? 4 : 0);
                copy4(stage + 2 * S::kHalf + S::kScales + lane * 4, g.c.v + off, named ? 4 : 0);
            }
            if (lane == 0) *valid_out = valid;
            if (++walk.s >= walk.s_end) walk.next_item(g.l);
        }
        copies_commit();
    }
};

// rows (within the tile) of a segment's mask in order, for the lanes to look up
__device__ __forceinline__ void list_rows(uint32_t mask, uint8_t* rows, int lane) {
    __syncwarp();
    if (mask >> lane & 1) rows[__popc(mask & ((1u << lane) - 1))] = (uint8_t)lane;
    __syncwarp();
}

template <typename T>
__device__ __forceinline__ void put(T* p, float x) { *p = from_float<T>(x); }

template <class S, int DT>
__global__ void __launch_bounds__(S::kWarps * 32, 2) paged_attend_kernel(const AttendArgs g) {
    using T = typename PoolIo<DT>::type;
    constexpr bool kF8 = DT == PSMC_F8;
    constexpr int NT = S::NT, KT = S::kStep / 16, kDt = S::DP / 16;
    extern __shared__ __align__(16) char smem[];
    __shared__ uint32_t valid_of[S::kWarps][S::kStages];
    __shared__ uint8_t row_list[S::kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane & 3, gq = lane >> 2;
    char* ring = smem + warp * S::kStages * S::kStage;
    const uint32_t ring_at = smem_of(ring);
    if (g.c.D < S::DP)  // columns beyond the head: never copied, always zero
        for (int i = lane; i < S::kStages * S::kStage / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = uint4{0, 0, 0, 0};
    __syncwarp();
    chain_begin();
    const int worker = warp * gridDim.x + blockIdx.x;

    Feeder<S, DT> feed;
    feed.walk.begin(g.l, worker, lane);
    Walk cur = feed.walk;
    if (cur.done) return;
    feed.ask(g, lane);
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; ++i) {
        feed.issue(g, ring_at + i * S::kStage, &valid_of[warp][i], lane);
        feed.ask(g, lane);
    }
    int stage = 0;
    const float to_log2 = g.a.scale * kLog2e;
    while (!cur.done) {
        // ---- the item's queries: lane (gq, t) holds components of query gq of each tile
        const int nt = (cur.nq + 7) / 8;
        uint32_t qf[NT][kDt][2];
        float sc[NT][2];  // queries 2t, 2t + 1 of each tile: factor from product to score in log2 units
        list_rows(cur.mask, row_list[warp], lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (j >= nt) break;
            const int qi = cur.qt * g.l.ls.qt + j * 8 + gq;
            const bool in = j * 8 + gq < cur.nq;
            const int rank = div_by(qi, g.by_ratio), sub = qi - rank * g.l.ls.ratio;
            const int row = cur.tile * kTileRows + row_list[warp][in ? rank : 0];
            const T* q = static_cast<const T*>(g.a.q.data) + (int64_t)row * g.a.q.stride_row +
                         (int64_t)(cur.head * g.l.ls.ratio + sub) * g.a.q.stride_head;
            if (!kF8) {
#pragma unroll
                for (int ks = 0; ks < kDt; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int d = ks * 16 + e * 8 + 2 * t;
                        uint32_t x = 0;
                        if (in && d < g.c.D)
                            x = (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(q) + d) |
                                (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(q) + d + 1) << 16;
                        qf[j][ks][e] = x;
                    }
                sc[j][0] = sc[j][1] = to_log2;
            } else {
                // fp16 holds a bf16 number's 8 bits but not its range: the query is scaled so that its largest component
                // lies in [128, 256), by a power of two, which the scores get back
                float amax = 0.f;
#pragma unroll
                for (int ks = 0; ks < kDt; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int d = ks * 16 + 4 * t + 2 * e;
                        uint32_t x = 0;
                        if (in && d < g.c.D)
                            x = (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(q) + d) |
                                (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(q) + d + 1) << 16;
                        qf[j][ks][e] = x;
                        amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(x << 16)), fabsf(__uint_as_float(x & 0xffff0000u))));
                    }
                amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, 1));
                amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, 2));
                const int ex = min(max((int)(__float_as_uint(amax) >> 23) - 127 - 7, -100), 100);
                const float inv = pow2i(-ex);
#pragma unroll
                for (int ks = 0; ks < kDt; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        qf[j][ks][e] = pack_f16(__uint_as_float(qf[j][ks][e] << 16) * inv, __uint_as_float(qf[j][ks][e] & 0xffff0000u) * inv);
                const float back = pow2i(ex) * to_log2;
                sc[j][0] = __shfl_sync(kFull, back, 8 * t);
                sc[j][1] = __shfl_sync(kFull, back, 8 * t + 4);
            }
        }
        float o[NT][kDt][4], ref[NT][2], sum[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            ref[j][0] = ref[j][1] = -INFINITY;
            sum[j][0] = sum[j][1] = 0.f;
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][d][e] = 0.f;
        }
#pragma unroll 1
        for (; cur.s < cur.s_end; ++cur.s) {
            const int ahead = stage == 0 ? S::kStages - 1 : stage - 1;
            feed.issue(g, ring_at + ahead * S::kStage, &valid_of[warp][ahead], lane);
            feed.ask(g, lane);
            copies_wait<S::kStages - 1>();
            __syncwarp();
            const uint32_t keys = ring_at + stage * S::kStage, vals = keys + S::kHalf;
            const uint32_t valid = valid_of[warp][stage];
            // 8-bit: lane p's scale exponents
            float k_scale = 1.f;
            int v_byte = 127;
            if (kF8) {
                const int p = cur.p0 + cur.s * S::kStep + lane;
                const int off = p - div_by(p, g.by_block) * g.c.block_len;
                const int shift = ((cur.head * g.c.block_len + off) & 3) * 8;
                const uint32_t* words = reinterpret_cast<const uint32_t*>(ring + stage * S::kStage + 2 * S::kHalf);
                k_scale = __uint_as_float((words[lane] >> shift & 255u) << 23);
                v_byte = (int)(words[S::kStep + lane] >> shift & 255u);
            }
            // ---- scores
            float s[KT][NT][4];
#pragma unroll
            for (int m = 0; m < KT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[m][j][e] = 0.f;
#pragma unroll
            for (int m = 0; m < KT; ++m) {
                const uint32_t row0 = keys + (m * 16 + (lane & 15)) * S::kRow;
                if (!kF8) {
#pragma unroll
                    for (int ks = 0; ks < kDt; ++ks) {
                        uint32_t ka[4];
                        load_tiles(ka, row0 + ks * 32 + (lane >> 4) * 16);
#pragma unroll
                        for (int j = 0; j < NT; ++j)
                            if (j < nt) mma<false>(s[m][j], ka, qf[j][ks][0], qf[j][ks][1]);
                    }
                } else {
#pragma unroll
                    for (int ks = 0; ks < kDt; ks += 2) {  // 32 components: two tiles of 16
                        uint32_t kc[4];
                        load_tiles(kc, row0 + ks * 16 + (lane >> 4) * 16);
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const uint32_t ka[4] = {codes_to_f16(kc[2 * u]), codes_to_f16(kc[2 * u + 1]),
                                                    codes_to_f16(kc[2 * u] >> 16), codes_to_f16(kc[2 * u + 1] >> 16)};
#pragma unroll
                            for (int j = 0; j < NT; ++j)
                                if (j < nt) mma<true>(s[m][j], ka, qf[j][ks + u][0], qf[j][ks + u][1]);
                        }
                    }
                }
            }
            // ---- scaled to log2 units; positions without anything get -inf
            float ev[KT][2], iv[KT][2];  // 8-bit: exponent of the values' scale, and 2^-exponent, positions gq and gq + 8
            bool grow = false;
#pragma unroll
            for (int m = 0; m < KT; ++m) {
                float ks0 = 1.f, ks1 = 1.f;
                if (kF8) {
                    ks0 = __shfl_sync(kFull, k_scale, m * 16 + gq);
                    ks1 = __shfl_sync(kFull, k_scale, m * 16 + gq + 8);
                    const int b0 = __shfl_sync(kFull, v_byte, m * 16 + gq), b1 = __shfl_sync(kFull, v_byte, m * 16 + gq + 8);
                    ev[m][0] = (float)(b0 - 127);
                    ev[m][1] = (float)(b1 - 127);
                    iv[m][0] = __uint_as_float((uint32_t)(254 - b0) << 23);
                    iv[m][1] = __uint_as_float((uint32_t)(254 - b1) << 23);
                }
                const bool ok0 = valid >> (m * 16 + gq) & 1, ok1 = valid >> (m * 16 + gq + 8) & 1;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (j >= nt) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[m][j][e] * sc[j][e & 1];
                        if (kF8) x = fmaf(x, e < 2 ? ks0 : ks1, ev[m][e >> 1]);
                        x = (e < 2 ? ok0 : ok1) ? x : -INFINITY;
                        s[m][j][e] = x;
                        grow = grow || x > ref[j][e & 1] + kSlack;
                    }
                }
            }
            if (__any_sync(kFull, grow)) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (j >= nt) break;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float top = ref[j][i];
#pragma unroll
                        for (int m = 0; m < KT; ++m) top = fmaxf(top, fmaxf(s[m][j][i], s[m][j][i + 2]));
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
            }
            // ---- weights, as the second operand of O^T += V^T P^T: [positions, queries], turned 8 x 8 at a time
            uint32_t pf[KT][NT][kF8 ? 1 : 2][2];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (j >= nt) break;
                const float r0 = ref[j][0] == -INFINITY ? 0.f : ref[j][0], r1 = ref[j][1] == -INFINITY ? 0.f : ref[j][1];
#pragma unroll
                for (int m = 0; m < KT; ++m) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float p0 = ex2(s[m][j][2 * h] - r0), p1 = ex2(s[m][j][2 * h + 1] - r1);
                        if (kF8) {
                            // weights of the codes: the values' scale is in the exponent already, and the sum takes it out
                            sum[j][0] = fmaf(p0, iv[m][h], sum[j][0]);
                            sum[j][1] = fmaf(p1, iv[m][h], sum[j][1]);
                            pf[m][j][0][h] = turn_tile(pack_f16(p0, p1));
                        } else {
                            // a weight as the sum of two bf16 numbers: 16 bits of it instead of 8
                            sum[j][0] += p0;
                            sum[j][1] += p1;
                            const uint32_t hi = pack_bf16(p0, p1);
                            pf[m][j][0][h] = turn_tile(hi);
                            pf[m][j][kF8 ? 0 : 1][h] = turn_tile(
                                pack_bf16(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xffff0000u)));
                        }
                    }
                }
            }
            // ---- outputs
#pragma unroll
            for (int m = 0; m < KT; ++m) {
                if (!kF8) {
                    const uint32_t row0 = vals + (m * 16 + (lane & 7) + (lane >> 4) * 8) * S::kRow + (lane >> 3 & 1) * 16;
#pragma unroll
                    for (int d = 0; d < kDt; ++d) {
                        uint32_t va[4];
                        load_tiles_turned(va, row0 + d * 32);
#pragma unroll
                        for (int j = 0; j < NT; ++j)
                            if (j < nt) {
                                mma<false>(o[j][d], va, pf[m][j][0][0], pf[m][j][0][1]);
                                mma<false>(o[j][d], va, pf[m][j][kF8 ? 0 : 1][0], pf[m][j][kF8 ? 0 : 1][1]);
                            }
                    }
                } else {
                    const uint32_t row0 = vals + (m * 16 + (lane & 7) + (lane >> 4) * 8) * S::kRow + (lane >> 3 & 1) * 16;
#pragma unroll
                    for (int d = 0; d < kDt; d += 2) {  // 32 components: the even ones, then the odd ones
                        uint32_t vc[4], va[2][4];
                        load_tiles_turned(vc, row0 + d * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {  // bytes (pos 0, d), (pos 0, d + 1), (pos 1, d), (pos 1, d + 1)
                            const uint32_t x = __byte_perm(vc[e], 0, 0x3120);
                            va[0][e] = codes_to_f16(x);
                            va[1][e] = codes_to_f16(x >> 16);
                        }
#pragma unroll
                        for (int j = 0; j < NT; ++j)
                            if (j < nt) {
                                mma<true>(o[j][d], va[0], pf[m][j][0][0], pf[m][j][0][1]);
                                mma<true>(o[j][d + 1], va[1], pf[m][j][0][0], pf[m][j][0][1]);
                            }
                    }
                }
            }
            __syncwarp();  // the stage may be filled again
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
        }
        // ---- the item's result: to its rows, or as a partial result
        const bool alone = cur.alone(g.l);
        const int64_t slot = cur.slot(g.l, worker);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (j >= nt) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float total = sum[j][i];
                total += __shfl_xor_sync(kFull, total, 4);
                total += __shfl_xor_sync(kFull, total, 8);
                total += __shfl_xor_sync(kFull, total, 16);
                const int in_tile = j * 8 + 2 * t + i;
                if (in_tile >= cur.nq) continue;
                const int qi = cur.qt * g.l.ls.qt + in_tile;
                const int rank = div_by(qi, g.by_ratio), sub = qi - rank * g.l.ls.ratio;
                const int row = cur.tile * kTileRows + row_list[warp][rank];
                const int qh = cur.head * g.l.ls.ratio + sub;
                T* out = static_cast<T*>(g.a.out.data) + (int64_t)row * g.a.out.stride_row + (int64_t)qh * g.a.out.stride_head;
                float* part = g.l.part + (slot + in_tile) * g.c.D;
                const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // component of the output: see the tiles above
                        const int at = kF8 ? (d & ~1) * 16 + e * 16 + 2 * gq + (d & 1) : d * 16 + e * 8 + gq;
                        if (at >= g.c.D) continue;
                        const float x = o[j][d][2 * e + i];
                        if (alone) put(out + at, x * inv);
                        else part[at] = x;
                    }
                if (gq == 0) {
                    if (!alone) g.l.stat[slot + in_tile] = float2{ref[j][i], total};
                    else if (g.a.lse) g.a.lse[(int64_t)row * g.a.Hq + qh] = total == 0.f ? -INFINITY : kLn2 * (ref[j][i] + log2f(total));
                }
            }
        }
        cur.next_item(g.l);
    }
}

// 32-bit caches: no matrix unit holds 24 bits, so the products are plain multiplications.  A step's 16 x 8 scores are four
// per lane (one position, four queries); in the second product a lane owns DP / 32 components of all 8 queries.
template <class S>
__global__ void __launch_bounds__(S::kWarps * 32, 2) paged_attend_f32_kernel(const AttendArgs g) {
    constexpr int kOwn = S::DP / 32;
    extern __shared__ __align__(16) char smem[];
    __shared__ uint32_t valid_of[S::kWarps][S::kStages];
    __shared__ uint8_t row_list[S::kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, key = lane & 15, qh4 = (lane >> 4) * 4;
    char* ring = smem + warp * S::kStages * S::kStage;
    float* qs = reinterpret_cast<float*>(smem + S::kWarps * S::kStages * S::kStage + warp * S::kExtra);  // [8][DP]
    float* ps = qs + 8 * S::DP;                                                                          // [16][8]
    const uint32_t ring_at = smem_of(ring);
    if (g.c.D < S::DP)
        for (int i = lane; i < S::kStages * S::kStage / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = uint4{0, 0, 0, 0};
    __syncwarp();
    chain_begin();
    const int worker = warp * gridDim.x + blockIdx.x;
    Feeder<S, PSMC_F32> feed;
    feed.walk.begin(g.l, worker, lane);
    Walk cur = feed.walk;
    if (cur.done) return;
    feed.ask(g, lane);
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; ++i) {
        feed.issue(g, ring_at + i * S::kStage, &valid_of[warp][i], lane);
        feed.ask(g, lane);
    }
    int stage = 0;
    const float to_log2 = g.a.scale * kLog2e;
    while (!cur.done) {
        list_rows(cur.mask, row_list[warp], lane);
        const auto query_at = [&](int in_tile, int* row, int* qh) {
            const int qi = cur.qt * g.l.ls.qt + in_tile, rank = div_by(qi, g.by_ratio);
            *row = cur.tile * kTileRows + row_list[warp][rank];
            *qh = cur.head * g.l.ls.ratio + qi - rank * g.l.ls.ratio;
        };
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
            int row = 0, qh = 0;
            if (j < cur.nq) query_at(j, &row, &qh);
            const float* q = static_cast<const float*>(g.a.q.data) + (int64_t)row * g.a.q.stride_row + (int64_t)qh * g.a.q.stride_head;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int d = lane + 32 * i;
                qs[j * S::DP + d] = j < cur.nq && d < g.c.D ? __ldg(q + d) : 0.f;
            }
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
#pragma unroll 1
        for (; cur.s < cur.s_end; ++cur.s) {
            const int ahead = stage == 0 ? S::kStages - 1 : stage - 1;
            feed.issue(g, ring_at + ahead * S::kStage, &valid_of[warp][ahead], lane);
            feed.ask(g, lane);
            copies_wait<S::kStages - 1>();
            __syncwarp();
            const char* keys = ring + stage * S::kStage;
            const bool ok = valid_of[warp][stage] >> key & 1;
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
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
        }
        const bool alone = cur.alone(g.l);
        const int64_t slot = cur.slot(g.l, worker);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) sum[u] += __shfl_xor_sync(kFull, sum[u], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float total = __shfl_sync(kFull, sum[j & 3], j < 4 ? 0 : 16), top = __shfl_sync(kFull, ref[j & 3], j < 4 ? 0 : 16);
            if (j >= cur.nq) continue;
            int row, qh;
            query_at(j, &row, &qh);
            float* out = static_cast<float*>(g.a.out.data) + (int64_t)row * g.a.out.stride_row + (int64_t)qh * g.a.out.stride_head;
            const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int d = lane + 32 * i;
                if (d >= g.c.D) continue;
                if (alone) out[d] = o[j][i] * inv;
                else g.l.part[(slot + j) * g.c.D + d] = o[j][i];
            }
            if (lane == 0) {
                if (!alone) g.l.stat[slot + j] = float2{top, total};
                else if (g.a.lse) g.a.lse[(int64_t)row * g.a.Hq + qh] = total == 0.f ? -INFINITY : kLn2 * (top + log2f(total));
            }
        }
        cur.next_item(g.l);
    }
}

// ---------------------------------------------------------------------------------------------------------- join
// WPQ warps per (row, query head), over the partial results of its segments, a list of kList at a time.
constexpr int kMaxWorkers = 2 * kSMs * 4;
constexpr int kJoinThreads = 128;

template <int DT, int WPQ>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const AttendArgs g) {
    using T = typename PoolIo<DT>::type;
    constexpr int kQueries = kJoinThreads / 32 / WPQ, kOwn = kMaxHeadDim / 128, kList = WPQ == 1 ? 64 : 512;
    __shared__ uint32_t slots[kQueries][kList];
    __shared__ float weight[kQueries][kList];
    __shared__ int n_parts[kQueries];
    __shared__ __align__(16) float acc[WPQ == 1 ? 1 : WPQ][kMaxHeadDim];  // read and written 16 bytes at a time
    chain_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp / WPQ, sub_warp = warp % WPQ;
    const int64_t item = (int64_t)blockIdx.x * kQueries + mine;
    const bool live = item < (int64_t)g.c.R * g.a.Hq;
    const int row = live ? (int)(item / g.a.Hq) : 0, qh = live ? (int)(item - (int64_t)row * g.a.Hq) : 0;
    const int tile = row / kTileRows, in_tile = row % kTileRows, head = qh / g.l.ls.ratio, sub = qh - head * g.l.ls.ratio;
    const TilePlan& tp = g.l.plans[tile];
    const LineShape& ls = g.l.ls;
    if (!live || (tp.left_out >> in_tile & 1)) return;  // the warps of a query agree
    const auto sync = [&] {
        if (WPQ > 1) __syncthreads();
        else __syncwarp();
    };
    int64_t share = 1, before = 0;
    if (sub_warp == 0) {
        share = share_of(g.l, line_total(g.l, lane));
        before = cost_before(g.l, tile, lane);
    }
    float top = -INFINITY, total = 0.f;
    float4 o[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) o[i] = float4{0.f, 0.f, 0.f, 0.f};
    int n_all = 0;
    for (int round = 0; round == 0 || round < n_all; round += kList) {
        if (sub_warp == 0) {
            int n = 0;
            for (int s0 = 0; s0 < tp.n_segs; s0 += 32) {
                const int s = s0 + lane;
                int found = 0;
                int64_t a = 0, k0 = 0, k1 = -1, first = 0;
                int w = 1, steps = 0, slot_in = 0;
                if (s < tp.n_segs && (tp.seg[s].mask >> in_tile & 1)) {
                    const Segment& sg = tp.seg[s];
                    const int qi = __popc(sg.mask & ((1u << in_tile) - 1)) * ls.ratio + sub, qt = qi / ls.qt;
                    slot_in = qi - qt * ls.qt;
                    steps = steps_of(ls, sg.p0, sg.p1);
                    w = step_cost((min(ls.qt, __popc(sg.mask) * ls.ratio - qt * ls.qt) + 7) / 8);
                    a = before + head * tp.cost + sg.start + (int64_t)qt * steps * step_cost(ls.qt / 8);
                    k0 = a / share;
                    k1 = (a + (int64_t)steps * w - 1) / share;
                    first = ((int64_t)tile * ls.H + head) * (kTileRows * kRowSegs * ls.ratio) + (int64_t)sg.before * ls.ratio + qi;
                    for (int64_t k = k0; k <= k1; ++k)  // a share may lie between two steps
                        found += step_from(k * share, a, w, steps) < step_from((k + 1) * share, a, w, steps);
                }
                int at = warp_scan_incl(found, lane);
                const int upto = n + __shfl_sync(kFull, at, 31);
                at += n - found - round;
                for (int64_t k = k0; k <= k1; ++k) {
                    const int b = step_from(k * share, a, w, steps);
                    if (b >= step_from((k + 1) * share, a, w, steps)) continue;
                    if (at >= 0 && at < kList)
                        slots[mine][at] = (uint32_t)(b == 0 ? first : g.l.first_rest + k * ls.qt + slot_in);
                    ++at;
                }
                n = upto;
            }
            const bool direct = n == 1 && ((uint32_t)tp.whole >> in_tile & 1);  // already in place
            if (lane == 0) n_parts[mine] = direct ? -1 : n;
        }
        sync();
        n_all = n_parts[mine];
        if (n_all < 0) return;
        const int n = min(kList, n_all - round);
        // the largest reference decides, the others' weights are 2^(their reference - it)
        float high = top;
        for (int i = lane; i < n; i += 32) high = fmaxf(high, g.l.stat[slots[mine][i]].x);
        high = warp_max(high);
        const float keep = top == high ? 1.f : exp2f(top - high);
        float more = 0.f;
        for (int i = lane; i < n; i += 32) {
            const float2 st = g.l.stat[slots[mine][i]];
            const float f = st.x == -INFINITY ? 0.f : (st.x == high ? 1.f : exp2f(st.x - high));
            if (sub_warp == 0) weight[mine][i] = f;
            more = fmaf(st.y, f, more);
        }
        total = fmaf(total, keep, warp_sum(more));
        top = high;
        sync();
#pragma unroll
        for (int i = 0; i < kOwn; ++i) o[i] = float4{o[i].x * keep, o[i].y * keep, o[i].z * keep, o[i].w * keep};
        constexpr int kBatch = 4;
        for (int i0 = sub_warp * kBatch; i0 < n; i0 += WPQ * kBatch) {
            float4 x[kBatch][kOwn];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int d = lane * 4 + i * 128;
                    x[u][i] = i0 + u < n && d < g.c.D
                                  ? *reinterpret_cast<const float4*>(g.l.part + (int64_t)slots[mine][i0 + u] * g.c.D + d)
                                  : float4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const float f = i0 + u < n ? weight[mine][i0 + u] : 0.f;
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    o[i].x = fmaf(f, x[u][i].x, o[i].x);
                    o[i].y = fmaf(f, x[u][i].y, o[i].y);
                    o[i].z = fmaf(f, x[u][i].z, o[i].z);
                    o[i].w = fmaf(f, x[u][i].w, o[i].w);
                }
            }
        }
        sync();
    }
    if (WPQ > 1) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) *reinterpret_cast<float4*>(&acc[sub_warp][lane * 4 + i * 128]) = o[i];
        __syncthreads();
        if (sub_warp != 0) return;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            for (int w = 1; w < WPQ; ++w) {
                const float4 x = *reinterpret_cast<const float4*>(&acc[w][lane * 4 + i * 128]);
                o[i].x += x.x;
                o[i].y += x.y;
                o[i].z += x.z;
                o[i].w += x.w;
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
constexpr int kMaxQt = 32;
Scratch scratch_of(int R, int Hq, int D) {
    Scratch s;
    s.n_tiles = (R + kTileRows - 1) / kTileRows;
    s.first_rest = (int64_t)s.n_tiles * kTileRows * kRowSegs * Hq;
    const size_t slots = (size_t)s.first_rest + (size_t)kMaxWorkers * kMaxQt;
    const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    s.plans = 0;
    s.stat = up((size_t)s.n_tiles * sizeof(TilePlan));
    s.part = s.stat + up(slots * sizeof(float2));
    s.bytes = s.part + up(slots * D * sizeof(float));
    return s;
}

template <int DT, int DP, int NT>
cudaError_t launch(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    using S = Shape<DT, DP, NT>;
    const Scratch sc = scratch_of(c.R, a.Hq, c.D);
    char* scratch = static_cast<char*>(a.scratch);
    AttendArgs g{};
    g.c = c;
    g.a = a;
    g.by_block = fast_div(c.block_len);
    g.l.ls = LineShape{S::kStep, 8 * NT, a.Hq / c.H, c.H};
    g.by_ratio = fast_div(g.l.ls.ratio);
    g.l.plans = reinterpret_cast<TilePlan*>(scratch + sc.plans);
    g.l.stat = reinterpret_cast<float2*>(scratch + sc.stat);
    g.l.part = reinterpret_cast<float*>(scratch + sc.part);
    g.l.first_rest = sc.first_rest;
    g.l.n_tiles = sc.n_tiles;
    const int ctas = 2 * kSMs;
    g.l.workers = ctas * S::kWarps;
    g.l.min_share = 64 / S::kStep * step_cost(1);
    cudaError_t e = launch_chained(paged_plan_kernel, dim3((unsigned)sc.n_tiles), dim3(kPlanThreads), 0, stream, c, a, g.l.ls,
                                   reinterpret_cast<TilePlan*>(scratch + sc.plans));
    if (e != cudaSuccess) return e;
    void (*fn)(const AttendArgs);
    if constexpr (DT == PSMC_F32) fn = paged_attend_f32_kernel<S>;
    else fn = paged_attend_kernel<S, DT>;
    e = allow_dynamic_smem(reinterpret_cast<const void*>(fn), S::kBytes);
    if (e == cudaSuccess) e = launch_chained(fn, dim3((unsigned)ctas), dim3(S::kWarps * 32), S::kBytes, stream, g);
    if (e != cudaSuccess) return e;
    const int64_t queries = (int64_t)c.R * a.Hq;
    if (queries <= 8 * kSMs) return launch_chained(paged_join_kernel<DT, 4>, dim3((unsigned)queries), dim3(kJoinThreads), 0, stream, g);
    return launch_chained(paged_join_kernel<DT, 1>, dim3((unsigned)((queries + 3) / 4)), dim3(kJoinThreads), 0, stream, g);
}

template <int DT, int DP>
cudaError_t launch_tiles(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    if constexpr (DT == PSMC_F32) {
        return launch<DT, DP, 1>(c, a, stream);
    } else {
        // queries that a tile of 32 rows can bring together, at most
        const int most = (c.R < kTileRows ? c.R : kTileRows) * (a.Hq / c.H);
        if (most <= 8) return launch<DT, DP, 1>(c, a, stream);
        if constexpr (DP <= 128)
            if (most > 16) return launch<DT, DP, 4>(c, a, stream);
        return launch<DT, DP, 2>(c, a, stream);
    }
}

template <int DT>
cudaError_t launch_dim(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    if (c.D <= 64) return launch_tiles<DT, 64>(c, a, stream);
    if (c.D <= 96) return launch_tiles<DT, 96>(c, a, stream);
    if (c.D <= 128) return launch_tiles<DT, 128>(c, a, stream);
    return launch_tiles<DT, 256>(c, a, stream);
}

}  // namespace

size_t paged_attend_scratch_bytes(int R, int Hq, int, int D) { return scratch_of(R, Hq, D).bytes; }

cudaError_t launch_paged_attend(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    if (c.dt == PSMC_F32) return launch_dim<PSMC_F32>(c, a, stream);
    return c.dt == PSMC_BF16 ? launch_dim<PSMC_BF16>(c, a, stream) : launch_dim<PSMC_F8>(c, a, stream);
}

}  // namespace psmc

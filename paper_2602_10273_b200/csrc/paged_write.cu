// Rotary positions on a token's queries and keys, and its keys and values into the paged cache.
//
// Pair (a, b) number j of a head, at position p, turns by p * f_j:  (a cos - b sin, b cos + a sin), times mscale; the
// components beyond rot_dim pass through.  Angles are formed and reduced to a fraction of a turn in 64 bits (at
// position 10^5 a 32-bit angle is off by 10^-2), the rotation is in 32 bits, rounded once into the cache or q_out.
// 8-bit pools: a warp holds a head in registers, takes the maximum over it and stores codes and the scale byte.
//
// Bound by bytes for prompts and by latency for single tokens.  A token has a warp of its own, or several that share its
// heads while there are too few tokens to fill the GPU; each computes the token's cosines and sines (two or four per lane)
// for itself, so that warps never wait for each other.
//
// Measured (in a graph; 32 or 28 query and 8 or 4 key-value heads of 128): 512 tokens into a bf16 cache 7.7 us (bytes alone 1.9:
// launch, position, table entry and operands follow one another), 4099 tokens 18 us (11.5), 10,000 tokens into an 8-bit cache
// and read back 71 us (45); 4 tokens of 4 fp32 heads 2.9 us.
#include "paged_common.cuh"

namespace psmc {
namespace {

constexpr int kWriteThreads = 256;

struct Turn {
    float c, s;
};

// cos and sin of 2 pi t: t is reduced in 64 bits, and what its 32-bit value leaves out is put back to first order
__device__ __forceinline__ Turn turn_of(double t, float mscale) {
    const double f = t - rint(t);
    const float hi = (float)f, lo = (float)((f - (double)hi) * 6.283185307179586);
    float s, c;
    sincospif(2.f * hi, &s, &c);
    return Turn{mscale * fmaf(-lo, s, c), mscale * fmaf(lo, c, s)};
}

// Two codes of a head's scaled components: nearest, ties to even, saturating; NaN stays NaN.
__device__ __forceinline__ uint16_t codes_of(float a, float b) {
    return (uint16_t)__nv_cvt_float2_to_fp8x2(float2{a, b}, __NV_SATFINITE, __NV_E4M3);
}

// (x0 c0 + y0 s0, x1 c1 + y1 s1), two 32-bit numbers per instruction, the sum rounded once
__device__ __forceinline__ float2 turn_two(float2 x, float2 c, float2 y, float2 s) {
    float2 r;
    asm("{\n\t.reg .b64 x, c, y, s, t;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 c, {%4, %5};\n\tmov.b64 y, {%6, %7};\n\tmov.b64 s, {%8, %9};\n\t"
        "mul.rn.f32x2 t, y, s;\n\tfma.rn.f32x2 t, x, c, t;\n\tmov.b64 {%0, %1}, t;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(x.x), "f"(x.y), "f"(c.x), "f"(c.y), "f"(y.x), "f"(y.y), "f"(s.x), "f"(s.y));
    return r;
}

// What a lane has to know of its share of a token: which components of a head are its own, and how they turn.
template <int DT, int VEC>
struct Lane {
    using T = typename PoolIo<DT>::type;
    using Vec = Chunk<T, VEC>;
    static constexpr int kChunks = kMaxHeadDim / (VEC * 32) > 0 ? kMaxHeadDim / (VEC * 32) : 1;  // accesses per lane and head, at most
    // Heads of a tensor whose loads a warp has under way at once (one at a time, each would wait for memory by itself), and
    // the warps that this leaves registers for: 10,000 tokens of 48 heads into an 8-bit cache take 55 us with four heads and
    // 24 warps per SM and 61 us with two and 32; 4099 of 36 heads into a bf16 cache take 22 and 19 us (before the streaming
    // accesses below).
    static constexpr int kBatch = kChunks > 1 ? 1 : (DT == PSMC_F8 ? 4 : 2);
    static constexpr int kCtas = kChunks > 1 ? 2 : (DT == PSMC_F8 ? 3 : 4);
    struct Ahead {       // one batch
        Vec v[kBatch][kChunks];
    };
    // Operands are read once, and what is written is not read again here: lines that go first when L2 needs room (10,000 tokens
    // into an 8-bit cache and read back 75 -> 71 us, 4099 tokens 19.0 -> 18.2)
    static __device__ __forceinline__ void take(Vec& to, const T* from) {
        if constexpr (sizeof(Vec) == 16) *reinterpret_cast<uint4*>(&to) = __ldcs(reinterpret_cast<const uint4*>(from));
        else to = *reinterpret_cast<const Vec*>(from);
    }
    static __device__ __forceinline__ void put(T* to, const Vec& x) {
        if constexpr (sizeof(Vec) == 16) __stcs(reinterpret_cast<uint4*>(to), *reinterpret_cast<const uint4*>(&x));
        else *reinterpret_cast<Vec*>(to) = x;
    }
    __device__ __forceinline__ void fetch(Ahead& a, int h, int count, int round, const T* x, int64_t x_step) const {
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
                if (h + b * round < count && sub + k * lph < n_chunks) take(a.v[b][k], x + b * x_step + k * lph * VEC);
    }
    int lph, lane, sub, n_chunks, rot, half;
    bool pairs;
    // a lane's components are the same ones of every head, so are their turns: x cosine + partner's (-)sine
    float cs[kChunks][VEC], sn[kChunks][VEC];

    __device__ __forceinline__ void turn(const Vec* raw, const T* x, float (&y)[kChunks][VEC], bool live) const {
        const int apart = half / VEC;  // half layout: how many accesses a component's partner lies from it
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int ch = sub + k * lph, pch = ch * VEC < half ? ch + apart : ch - apart;
            const bool mine = ch * VEC < rot;
            float o[VEC];
            if (pairs) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = VEC > 1 ? y[k][e ^ (VEC > 1)] : __shfl_xor_sync(kFull, y[k][e], 1);
            } else {
                Vec partner{};
                if (kChunks == 1 && sizeof(Vec) >= 4) {  // another lane of the head holds it
                    const uint32_t* own = reinterpret_cast<const uint32_t*>(raw + k);
                    uint32_t* theirs = reinterpret_cast<uint32_t*>(&partner);
#pragma unroll
                    for (int w = 0; w < (int)(sizeof(Vec) / 4); ++w) theirs[w] = __shfl_sync(kFull, own[w], (lane - sub) + (pch & (lph - 1)));
                } else if (live && mine) {
                    partner = *reinterpret_cast<const Vec*>(x + (pch - sub) * VEC);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = to_float(partner.x[e]);
            }
            if (!mine) continue;
            if (VEC > 1) {
#pragma unroll
                for (int e = 0; e + 1 < VEC; e += 2) {
                    const float2 z = turn_two(float2{y[k][e], y[k][e + 1]}, float2{cs[k][e], cs[k][e + 1]}, float2{o[e], o[e + 1]},
                                              float2{sn[k][e], sn[k][e + 1]});
                    y[k][e] = z.x;
                    y[k][e + 1] = z.y;
                }
            } else {
                y[k][0] = fmaf(y[k][0], cs[k][0], o[0] * sn[k][0]);
            }
        }
        __syncwarp();  // the result may go where the input was: a head is read by one warp, and all of it before any is written
    }

    // Heads h, h + round, ... of one tensor: x, out: this lane's first components of head h; steps in elements (bytes for codes).
    // a: the first batch.  CODES: 8-bit, with a scale byte per head at `scale`.
    template <bool TURN, bool CODES>
    __device__ __forceinline__ void heads(Ahead& a, int h, int count, int round, const T* x, int64_t x_step, void* to, int64_t to_step,
                                          uint8_t* scale, int scale_step) const {
        using Out = Chunk<uint16_t, VEC / 2 + (VEC == 1)>;
        // (the heads of a warp's lanes differ by less than a round: the warp goes on while any of them has one)
        for (bool more = false; __any_sync(kFull, h < count); h += kBatch * round, more = true) {
            if (more) fetch(a, h, count, round, x, x_step);
            const Vec(&raw)[kBatch][kChunks] = a.v;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const bool live = h + b * round < count;
                if (!__any_sync(kFull, live)) break;
                float y[kChunks][VEC];
                if (TURN || CODES) {
#pragma unroll
                    for (int k = 0; k < kChunks; ++k)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) y[k][e] = to_float(raw[b][k].x[e]);
                }
                if (TURN) turn(raw[b], x + b * x_step, y, live);
                if (!CODES) {
                    T* out = static_cast<T*>(to) + b * to_step;
#pragma unroll
                    for (int k = 0; k < kChunks; ++k) {
                        if (!live || sub + k * lph >= n_chunks) continue;
                        Vec o = raw[b][k];
                        if (TURN) {
#pragma unroll
                            for (int e = 0; e < VEC; ++e) o.x[e] = from_float<T>(y[k][e]);
                        }
                        put(out + k * lph * VEC, o);
                    }
                } else {
                    // as integers, magnitudes sort like the numbers, infinities and NaN above all others
                    uint32_t amax = 0;
#pragma unroll
                    for (int k = 0; k < kChunks; ++k)
                        if (live && sub + k * lph < n_chunks)
#pragma unroll
                            for (int e = 0; e < VEC; ++e) amax = max(amax, __float_as_uint(y[k][e]) & 0x7fffffffu);
                    if (__any_sync(kFull, amax >= 0x7f800000u)) {  // they become NaN, and the others decide the scale
                        amax = 0;
#pragma unroll
                        for (int k = 0; k < kChunks; ++k)
                            if (live && sub + k * lph < n_chunks)
#pragma unroll
                                for (int e = 0; e < VEC; ++e) {
                                    if (isfinite(y[k][e])) amax = max(amax, __float_as_uint(y[k][e]) & 0x7fffffffu);
                                    else y[k][e] = __int_as_float(0x7fffffff);
                                }
                    }
                    for (int o = lph >> 1; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(kFull, amax, o));
                    const int ex = scale_exponent(__uint_as_float(amax));
                    const float inv = pow2i(-ex);
                    uint8_t* out = static_cast<uint8_t*>(to) + b * to_step;
#pragma unroll
                    for (int k = 0; k < kChunks; ++k) {
                        if (!live || sub + k * lph >= n_chunks) continue;
                        if (VEC == 1) {
                            out[k * lph] = (uint8_t)codes_of(y[k][0] * inv, 0.f);
                        } else {
                            Out o;
#pragma unroll
                            for (int e = 0; e + 1 < VEC; e += 2) o.x[e / 2] = codes_of(y[k][e] * inv, y[k][e + 1] * inv);
                            *reinterpret_cast<Out*>(out + k * lph * VEC) = o;
                        }
                    }
                    if (live && sub == 0) scale[b * scale_step] = (uint8_t)(ex + 127);
                }
            }
            x += kBatch * x_step;
            to = CODES ? static_cast<void*>(static_cast<uint8_t*>(to) + kBatch * to_step) : static_cast<void*>(static_cast<T*>(to) + kBatch * to_step);
            scale += kBatch * scale_step;
        }
    }
};

template <int DT, int VEC>
__global__ void __launch_bounds__(kWriteThreads, (Lane<DT, VEC>::kCtas)) paged_write_kernel(const PagedView c, const PagedWrite w) {
    using L = Lane<DT, VEC>;
    using T = typename L::T;
    constexpr bool kF8 = DT == PSMC_F8;
    __shared__ Turn turns_of[kWriteThreads / 32][kMaxHeadDim / 2];
    chain_begin();
    // lanes_per_head lanes (a power of two) share a head; a warp takes 32 / lanes_per_head heads at a time
    L l;
    l.lph = w.lanes_per_head;
    l.lane = threadIdx.x & 31;
    l.sub = l.lane & (l.lph - 1);
    l.n_chunks = c.D / VEC;
    l.rot = w.rot;
    l.half = w.rot >> 1;
    l.pairs = w.pairs != 0;
    const int warp = threadIdx.x >> 5, per_warp = 32 / l.lph;
    const int i = blockIdx.x * (kWriteThreads / 32 / w.warps_per_token) + warp / w.warps_per_token;
    if (i >= w.n) return;
    const int r = w.rows ? __ldg(w.rows + i) : i;
    if (r < 0) return;  // padding
    const int p = __ldg(w.positions + i);
    if (r >= c.R) {
        if (l.lane == 0) raise_status(w.status, PSMC_E_STATE);
        return;
    }
    if (w.skip && w.skip[r]) return;
    const int j = p < 0 ? -1 : p / c.block_len, off = p - j * c.block_len;
    const int blk = block_of(c, r, j);
    // queries, keys and values are dealt out to the lanes as one row of heads
    const int round = w.warps_per_token * per_warp, at = (warp % w.warps_per_token) * per_warp + l.lane / l.lph;
    const int Hq = w.q ? w.Hq : 0, k_at = (at + round - Hq % round) % round, v_at = (at + round - (Hq + c.H) % round) % round;
    const auto in_at = [&](const HeadsView& v, int h) -> const T* {
        return static_cast<const T*>(v.data) + (int64_t)i * v.stride_row + h * v.stride_head + l.sub * VEC;
    };
    const T *qx = nullptr, *kx = in_at(w.in[1], k_at), *vx = in_at(w.in[2], v_at);
    const int64_t k_step = round * w.in[1].stride_head, v_step = round * w.in[2].stride_head;
    // the first values and queries travel while the turns are computed, the first keys while the queries are turned (with the
    // larger batches of 8-bit caches, there are no registers to hold them that long)
    typename L::Ahead ahead, ahead_q;
    l.fetch(ahead, v_at, c.H, round, vx, v_step);
    if (Hq) {
        qx = in_at(w.in[0], at);
        if (!kF8) l.fetch(ahead_q, at, Hq, round, qx, round * w.in[0].stride_head);
    }
    if (blk < 0) {
        if (l.lane == 0) raise_status(w.status, PSMC_E_STATE);
        return;
    }
    char* kp = c.k + (int64_t)blk * c.blk_bytes;
    char* vp = c.v + (int64_t)blk * c.blk_bytes;
    const int64_t per_head = (int64_t)c.block_len * c.D, in_block = (int64_t)off * c.D + l.sub * VEC;  // elements of the pool
    const int elem = kF8 ? 1 : (int)sizeof(T);
    const int64_t scale_at = c.scale_at + off;
    const int s_step = round * c.block_len;
    l.template heads<false, kF8>(ahead, v_at, c.H, round, vx, v_step, vp + (v_at * per_head + in_block) * elem, round * per_head,
                                 reinterpret_cast<uint8_t*>(vp) + scale_at + (int64_t)v_at * c.block_len, s_step);
    // Turn m lies where the lanes that need their e-th turn at the same time find them side by side: [e][access]
    Turn* turns = turns_of[warp];
    const int per_access = l.pairs ? (VEC > 1 ? VEC / 2 : 1) : VEC, accesses = l.half / per_access;
    for (int m = l.lane; m < l.half; m += 32)
        turns[(m % per_access) * accesses + m / per_access] = turn_of((double)p * (__ldg(w.freqs + m) * 0.15915494309189535), w.mscale);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < L::kChunks; ++k) {
        const int ch = l.sub + k * l.lph, d0 = ch * VEC;
        const bool first = d0 < l.half, turned = d0 < w.rot;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            Turn t{1.f, 0.f};
            if (turned) t = l.pairs ? (VEC > 1 ? turns[(e >> 1) * accesses + ch] : turns[d0 >> 1]) : turns[e * accesses + (first ? ch : ch - l.half / VEC)];
            l.cs[k][e] = t.c;
            l.sn[k][e] = (l.pairs ? ((d0 + e) & 1) == 0 : first) ? -t.s : t.s;
        }
    }
    if (!kF8) l.fetch(ahead, k_at, c.H, round, kx, k_step);
    if (Hq) {
        if (kF8) l.fetch(ahead_q, at, Hq, round, qx, round * w.in[0].stride_head);
        T* out = static_cast<T*>(w.q_out.data) + (int64_t)i * w.q_out.stride_row + at * w.q_out.stride_head + l.sub * VEC;
        const int64_t q_step = round * w.in[0].stride_head, o_step = round * w.q_out.stride_head;
        if (w.rot > 0) l.template heads<true, false>(ahead_q, at, Hq, round, qx, q_step, out, o_step, nullptr, 0);
        else l.template heads<false, false>(ahead_q, at, Hq, round, qx, q_step, out, o_step, nullptr, 0);
    }
    if (kF8) l.fetch(ahead, k_at, c.H, round, kx, k_step);
    void* kt = kp + (k_at * per_head + in_block) * elem;
    uint8_t* k_scale = reinterpret_cast<uint8_t*>(kp) + scale_at + (int64_t)k_at * c.block_len;
    if (w.rot > 0) l.template heads<true, kF8>(ahead, k_at, c.H, round, kx, k_step, kt, round * per_head, k_scale, s_step);
    else l.template heads<false, kF8>(ahead, k_at, c.H, round, kx, k_step, kt, round * per_head, k_scale, s_step);
}

template <int DT>
cudaError_t launch(const PagedView& c, PagedWrite w, cudaStream_t stream) {
    using T = typename PoolIo<DT>::type;
    constexpr int kFullVec = 16 / sizeof(T);
    // Elements per access: 16 bytes where every head starts on such a boundary and no access straddles the two halves
    // (or a pair, or the end) of the rotated part; else two elements (any even rotation of such heads), else one (4099 tokens
    // 19, 62 and 72 us).
    uint64_t bits = 0;
    for (const HeadsView* h : {&w.in[0], &w.in[1], &w.in[2], &w.q_out})
        if (h->data) bits |= (uint64_t)(uintptr_t)h->data | (uint64_t)(h->stride_row * sizeof(T)) | (uint64_t)(h->stride_head * sizeof(T));
    const int unit = w.pairs ? w.rot : w.rot / 2;
    const auto fits = [&](int vec) {
        return bits % (vec * sizeof(T)) == 0 && unit % vec == 0 && c.D % vec == 0;
    };
    const int vec = fits(kFullVec) ? kFullVec : (fits(2) ? 2 : 1);
    int lph = 1;
    while (lph < 32 && lph * vec < c.D) lph *= 2;
    w.lanes_per_head = lph;
    // the fewest warps per token that leave none of the GPU's idle (24 resident warps per SM): 512 tokens 7.7 us, with one warp
    // each 9.6; 4 tokens 2.9 and 3.4
    constexpr int kWarps = kWriteThreads / 32;
    w.warps_per_token = 1;
    const int rounds = ((w.q ? w.Hq : 0) + 2 * c.H + 32 / lph - 1) / (32 / lph);
    while (w.warps_per_token < kWarps && (int64_t)w.n * w.warps_per_token < kSMs * 24 && w.warps_per_token < rounds) w.warps_per_token *= 2;
    auto fn = vec == kFullVec ? paged_write_kernel<DT, kFullVec>
                              : (vec == 2 ? paged_write_kernel<DT, 2> : paged_write_kernel<DT, 1>);
    const int per_cta = kWarps / w.warps_per_token;
    return launch_chained(fn, dim3((unsigned)((w.n + per_cta - 1) / per_cta)), dim3(kWriteThreads), 0, stream, c, w);
}

}  // namespace

cudaError_t launch_paged_write(const PagedView& c, const PagedWrite& w, cudaStream_t stream) {
    if (w.n <= 0) return cudaSuccess;
    if (c.dt == PSMC_F32) return launch<PSMC_F32>(c, w, stream);
    return c.dt == PSMC_BF16 ? launch<PSMC_BF16>(c, w, stream) : launch<PSMC_F8>(c, w, stream);
}

}  // namespace psmc

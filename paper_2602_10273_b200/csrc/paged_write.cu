// Rotary positions on a token's queries and keys, and its keys and values into the paged cache.
//
// Pair (a, b) number j of a head, at position p, turns by p * f_j:  (a cos - b sin, b cos + a sin), times mscale; the
// components beyond rot_dim pass through.  Angles are formed and reduced to a fraction of a turn in 64 bits (at
// position 10^5 a 32-bit angle is off by 10^-2), the rotation is in 32 bits, rounded once into the cache or q_out.
// 8-bit pools: a warp holds a head in registers, takes the maximum over it and stores codes and the scale byte.
//
// Bound by bytes for prompts and by latency for single tokens; one CTA per token, so that the cosines and sines
// (rot_dim / 2 of them, the only expensive arithmetic) are computed once for all of the token's heads.
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

template <int DT, int VEC>
__global__ void __launch_bounds__(kWriteThreads) paged_write_kernel(const PagedView c, const PagedWrite w) {
    using T = typename PoolIo<DT>::type;
    using Vec = Chunk<T, VEC>;
    constexpr int kChunks = kMaxHeadDim / (VEC * 32) > 0 ? kMaxHeadDim / (VEC * 32) : 1;  // chunks per lane, at most
    __shared__ Turn turns[kMaxHeadDim / 2];
    chain_begin();
    const int i = blockIdx.x;
    const int r = w.rows ? __ldg(w.rows + i) : i;
    if (r < 0) return;  // padding
    if (r >= c.R) {
        if (threadIdx.x == 0) raise_status(w.status, PSMC_E_STATE);
        return;
    }
    if (w.skip && w.skip[r]) return;
    const int p = __ldg(w.positions + i);
    const int j = p < 0 ? -1 : p / c.block_len, off = p - j * c.block_len;
    const int blk = block_of(c, r, j);
    if (blk < 0) {
        if (threadIdx.x == 0) raise_status(w.status, PSMC_E_STATE);
        return;
    }
    const int half = w.rot >> 1;
    for (int m = threadIdx.x; m < half; m += kWriteThreads)
        turns[m] = turn_of((double)p * (__ldg(w.freqs + m) * 0.15915494309189535), w.mscale);
    if (half) __syncthreads();

    // lanes_per_head lanes (a power of two) share a head; a warp takes 32 / lanes_per_head heads at a time
    const int lph = w.lanes_per_head, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_warp = 32 / lph, sub = lane & (lph - 1), which = lane / lph;
    const int Hq = w.q ? w.Hq : 0, total = Hq + 2 * c.H, n_chunks = c.D / VEC;
    for (int h0 = warp * per_warp; h0 < total; h0 += (kWriteThreads / 32) * per_warp) {
        const int h = h0 + which;
        const bool live = h < total;
        // 0: a query head, 1: a key head, 2: a value head
        const int kind = h < Hq ? 0 : (h < Hq + c.H ? 1 : 2), hh = kind == 0 ? h : (h - Hq) - (kind == 2 ? c.H : 0);
        const HeadsView& src = kind == 0 ? w.q_in : (kind == 1 ? w.k_in : w.v_in);
        const T* x = static_cast<const T*>(src.data) + (int64_t)i * src.stride_row + (int64_t)hh * src.stride_head;
        const int rot = kind == 2 ? 0 : w.rot;
        float y[kChunks][VEC];
        float amax = 0.f;
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int ch = sub + k * lph, d0 = ch * VEC;
            if (!live || ch >= n_chunks) continue;
            const Vec own = *reinterpret_cast<const Vec*>(x + d0);
            if (d0 >= rot) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) y[k][e] = to_float(own.x[e]);
            } else if (w.pairs) {  // (2m, 2m + 1) turn together; a single element (VEC = 1) fetches its partner
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int d = d0 + e;
                    const float self = to_float(own.x[e]);
                    const float other = VEC > 1 ? to_float(own.x[e ^ 1]) : to_float(x[d ^ 1]);
                    const Turn t = turns[d >> 1];
                    y[k][e] = d & 1 ? fmaf(self, t.c, other * t.s) : fmaf(self, t.c, -(other * t.s));
                }
            } else {  // (m, m + rot / 2) turn together
                const bool first = d0 < half;
                const Vec partner = *reinterpret_cast<const Vec*>(x + (first ? d0 + half : d0 - half));
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const Turn t = turns[first ? d0 + e : d0 + e - half];
                    const float self = to_float(own.x[e]), other = to_float(partner.x[e]);
                    y[k][e] = first ? fmaf(self, t.c, -(other * t.s)) : fmaf(self, t.c, other * t.s);
                }
            }
        }
        __syncwarp();  // q_out may be q: every lane has read its partner's elements before any lane writes
        if (kind == 0) {
            T* out = static_cast<T*>(w.q_out.data) + (int64_t)i * w.q_out.stride_row + (int64_t)hh * w.q_out.stride_head;
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                const int ch = sub + k * lph;
                if (!live || ch >= n_chunks) continue;
                Vec o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) o.x[e] = from_float<T>(y[k][e]);
                *reinterpret_cast<Vec*>(out + ch * VEC) = o;
            }
        }
        char* pool = (kind == 2 ? c.v : c.k) + (int64_t)blk * c.blk_bytes;
        const int64_t at = ((int64_t)hh * c.block_len + off) * c.D;
        if (DT != PSMC_F8) {
            T* out = reinterpret_cast<T*>(pool) + at;
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                const int ch = sub + k * lph;
                if (!live || kind == 0 || ch >= n_chunks) continue;
                Vec o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) o.x[e] = from_float<T>(y[k][e]);
                *reinterpret_cast<Vec*>(out + ch * VEC) = o;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                if (!live || sub + k * lph >= n_chunks) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) amax = isfinite(y[k][e]) ? fmaxf(amax, fabsf(y[k][e])) : amax;
            }
            for (int o = lph >> 1; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, o));
            const int ex = scale_exponent(amax);
            const float inv = pow2i(-ex);
            if (live && kind != 0) {
                uint8_t* out = reinterpret_cast<uint8_t*>(pool) + at;
#pragma unroll
                for (int k = 0; k < kChunks; ++k) {
                    const int ch = sub + k * lph;
                    if (ch >= n_chunks) continue;
                    Chunk<uint8_t, VEC> o;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) o.x[e] = code_of(y[k][e] * inv);
                    *reinterpret_cast<Chunk<uint8_t, VEC>*>(out + ch * VEC) = o;
                }
                if (sub == 0)
                    reinterpret_cast<uint8_t*>(pool)[c.scale_at + (int64_t)hh * c.block_len + off] = (uint8_t)(ex + 127);
            }
        }
    }
}

template <int DT>
cudaError_t launch(const PagedView& c, PagedWrite w, cudaStream_t stream) {
    using T = typename PoolIo<DT>::type;
    constexpr int kFullVec = 16 / sizeof(T);
    // Elements per access: 16 bytes where every head starts on such a boundary and no access straddles the two halves
    // (or a pair, or the end) of the rotated part; else two elements (any even rotation of such heads), else one.
    uint64_t bits = 0;
    for (const HeadsView* h : {&w.q_in, &w.q_out, &w.k_in, &w.v_in})
        if (h->data) bits |= (uint64_t)(uintptr_t)h->data | (uint64_t)(h->stride_row * sizeof(T)) | (uint64_t)(h->stride_head * sizeof(T));
    const int unit = w.pairs ? w.rot : w.rot / 2;
    const auto fits = [&](int vec) {
        return bits % (vec * sizeof(T)) == 0 && unit % vec == 0 && c.D % vec == 0;
    };
    const int vec = fits(kFullVec) ? kFullVec : (fits(2) ? 2 : 1);
    int lph = 1;
    while (lph < 32 && lph * vec < c.D) lph *= 2;
    w.lanes_per_head = lph;
    auto fn = vec == kFullVec ? paged_write_kernel<DT, kFullVec>
                              : (vec == 2 ? paged_write_kernel<DT, 2> : paged_write_kernel<DT, 1>);
    return launch_chained(fn, dim3((unsigned)w.n), dim3(kWriteThreads), 0, stream, c, w);
}

}  // namespace

cudaError_t launch_paged_write(const PagedView& c, const PagedWrite& w, cudaStream_t stream) {
    if (w.n <= 0) return cudaSuccess;
    if (c.dt == PSMC_F32) return launch<PSMC_F32>(c, w, stream);
    return c.dt == PSMC_BF16 ? launch<PSMC_BF16>(c, w, stream) : launch<PSMC_F8>(c, w, stream);
}

}  // namespace psmc

// Attention of one new token per row over the paged cache:  out[r, h] = sum_p softmax_p(scale q[r, h] . k_p) v_p over
// the positions p < lens[r] + extra of row r.  The first, plain form: a CTA per (row, query head), a warp per position,
// running maximum and sum, joined over the warps at the end.
#include "paged_common.cuh"

namespace psmc {
namespace {

constexpr int kWarps = 8;

template <int DT>
__global__ void __launch_bounds__(kWarps * 32) paged_attend_plain_kernel(const PagedView c, const PagedAttend a) {
    using T = typename PoolIo<DT>::type;
    constexpr int kPer = kMaxHeadDim / 32;
    __shared__ float part[kWarps][kMaxHeadDim + 2];
    chain_begin();
    const int h = blockIdx.x, r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (a.skip && a.skip[r]) return;
    int64_t n = (int64_t)__ldg(a.lens + r) + a.extra;
    if (n > c.max_blocks * (int64_t)c.block_len) {
        if (threadIdx.x == 0) raise_status(a.status, PSMC_E_STATE);
        n = c.max_blocks * (int64_t)c.block_len;
    }
    const T* q = static_cast<const T*>(a.q.data) + (int64_t)r * a.q.stride_row + (int64_t)h * a.q.stride_head;
    const int kv = h / (a.Hq / c.H);
    float qr[kPer], acc[kPer], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int d = lane + 32 * i;
        qr[i] = d < c.D ? to_float(q[d]) * a.scale : 0.f;
        acc[i] = 0.f;
    }
    for (int64_t p = warp; p < n; p += kWarps) {
        const int j = (int)(p / c.block_len), off = (int)(p - (int64_t)j * c.block_len), blk = block_of(c, r, j);
        if (blk < 0) {
            if (lane == 0) raise_status(a.status, PSMC_E_STATE);
            continue;
        }
        const char* kp = c.k + (int64_t)blk * c.blk_bytes;
        const char* vp = c.v + (int64_t)blk * c.blk_bytes;
        const int64_t at = ((int64_t)kv * c.block_len + off) * c.D;
        const auto value = [&](const char* pool, int d) -> float {
            if (DT == PSMC_F8) {
                const uint8_t* u = reinterpret_cast<const uint8_t*>(pool);
                return code_value(u[at + d]) * pow2i((int)u[c.scale_at + (int64_t)kv * c.block_len + off] - 127);
            }
            return to_float(reinterpret_cast<const T*>(pool)[at + d]);
        };
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (lane + 32 * i < c.D) s = fmaf(qr[i], value(kp, lane + 32 * i), s);
        s = warp_sum(s);
        const float top = fmaxf(m, s), keep = m == -INFINITY ? 0.f : expf(m - top), e = s == -INFINITY ? 0.f : expf(s - top);
        l = l * keep + e;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (lane + 32 * i < c.D) acc[i] = fmaf(e, value(vp, lane + 32 * i), acc[i] * keep);
        m = top;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) part[warp][lane + 32 * i] = acc[i];
    if (lane == 0) {
        part[warp][kMaxHeadDim] = m;
        part[warp][kMaxHeadDim + 1] = l;
    }
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, part[w][kMaxHeadDim]);
    for (int w = 0; w < kWarps; ++w)
        sum += part[w][kMaxHeadDim] == -INFINITY ? 0.f : part[w][kMaxHeadDim + 1] * expf(part[w][kMaxHeadDim] - top);
    T* out = static_cast<T*>(a.out.data) + (int64_t)r * a.out.stride_row + (int64_t)h * a.out.stride_head;
    for (int d = threadIdx.x; d < c.D; d += kWarps * 32) {
        float o = 0.f;
        for (int w = 0; w < kWarps; ++w)
            o += part[w][kMaxHeadDim] == -INFINITY ? 0.f : part[w][d] * expf(part[w][kMaxHeadDim] - top);
        out[d] = from_float<T>(sum == 0.f ? 0.f : o / sum);
    }
    if (a.lse && threadIdx.x == 0) a.lse[(int64_t)r * a.Hq + h] = sum == 0.f ? -INFINITY : top + logf(sum);
}

}  // namespace

size_t paged_attend_scratch_bytes(int, int, int, int) { return 256; }

cudaError_t launch_paged_attend(const PagedView& c, const PagedAttend& a, cudaStream_t stream) {
    auto fn = c.dt == PSMC_F32 ? paged_attend_plain_kernel<PSMC_F32>
                               : (c.dt == PSMC_BF16 ? paged_attend_plain_kernel<PSMC_BF16> : paged_attend_plain_kernel<PSMC_F8>);
    return launch_chained(fn, dim3((unsigned)a.Hq, (unsigned)c.R), dim3(kWarps * 32), 0, stream, c, a);
}

}  // namespace psmc

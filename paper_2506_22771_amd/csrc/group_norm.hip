// Group norm: what does not depend on the element type.  See group_norm.hpp.
#include "group_norm.hpp"

namespace ffi {

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// Parts of a group joined, a wavefront each: mean of the parts' means, their squared deviations around it.
__global__ __launch_bounds__(256) void k_gn_join(const float4* part, float4* stats, float* mean, float* rstd, int64_t groups, int32_t parts, float eps)
{
    const int lane = threadIdx.x & 63;
    for (int64_t g = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); g < groups; g += (int64_t)gridDim.x * 4) {
        double count = 0, sum = 0, square = 0;
        for (int i = lane; i < parts; i += 64) {
            const float4 v = part[g * parts + i];
            count += v.w;
            sum += (double)v.w * ((double)v.x + v.y);
        }
        count = wave_sum64(count);
        const double mu = wave_sum64(sum) / count;
        for (int i = lane; i < parts; i += 64) {
            const float4 v = part[g * parts + i];
            const double off = (double)v.x + v.y - mu;
            square += (double)v.z + v.w * off * off;
        }
        const double var = wave_sum64(square) / count;
        if (lane == 0) {
            const float hi = (float)mu, r = inverse_root((float)(var < 0 ? 0 : var) + eps);
            stats[g] = make_float4(hi, hi * hi > (float)var ? (float)(mu - hi) : 0.0f, r, 0.0f);
            if (mean) mean[g] = hi;
            if (rstd) rstd[g] = r;
        }
    }
}

// goodness[sample] = sum of its parts, in their order, a wavefront each
__global__ __launch_bounds__(256) void k_gn_goodness(const float* part, float* goodness, int64_t samples, int64_t parts)
{
    const int lane = threadIdx.x & 63;
    for (int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); b < samples; b += (int64_t)gridDim.x * 4) {
        float s = 0;
        for (int64_t i = lane; i < parts; i += 64) s += part[b * parts + i];
        s = wave_sum(s);
        if (lane == 0) goodness[b] = s;
    }
}

// dgamma and dbeta: sums over the samples of a column's sums, sixteen columns to a workgroup, 64 threads to a column.  In 64 bits: a thread adds every 64th sample, 16400 of a million one
// after the other, of which fp32 would keep four or five digits.
__global__ __launch_bounds__(1024) void k_gn_params(const float2* sums, int64_t samples, int32_t channels, float* dweight, float* dbias, int32_t accumulate)
{
    __shared__ double2 red[64][16];
    const int col = threadIdx.x & 15, lane = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    double2 t = make_double2(0, 0);
    if (c < channels)
        for (int64_t b = lane; b < samples; b += 64) {
            const float2 v = sums[b * channels + c];
            t.x += v.x;
            t.y += v.y;
        }
    red[lane][col] = t;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (lane < half) {
            red[lane][col].x += red[lane + half][col].x;
            red[lane][col].y += red[lane + half][col].y;
        }
        __syncthreads();
    }
    if (lane == 0 && c < channels) {
        t = red[0][col];
        if (dweight) dweight[c] = (float)(accumulate ? dweight[c] + t.y : t.y);
        if (dbias) dbias[c] = (float)(accumulate ? dbias[c] + t.x : t.x);
    }
}

hipError_t launch_gn_join(const float4* part, float4* stats, const GroupNormForwardLaunch& f, int32_t parts, hipStream_t s)
{
    const int64_t all = f.samples * f.groups;
    k_gn_join<<<(unsigned)std::min<int64_t>((all + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(part, stats, f.mean, f.rstd, all, parts, f.eps);
    return hipGetLastError();
}
hipError_t launch_gn_goodness(const float* part, float* goodness, int64_t samples, int64_t parts, hipStream_t s)
{
    k_gn_goodness<<<(unsigned)std::min<int64_t>((samples + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(part, goodness, samples, parts);
    return hipGetLastError();
}
hipError_t launch_gn_params(const float2* sums, const GroupNormBackwardLaunch& g, hipStream_t s)
{
    if (!g.dweight && !g.dbias) return hipSuccess;
    k_gn_params<<<(unsigned)((g.channels + 15) / 16), 1024, 0, s>>>(sums, g.samples, (int32_t)g.channels, g.dweight, g.dbias, g.accumulate);
    return hipGetLastError();
}
size_t group_norm_workspace(int64_t samples, int64_t pixels, int64_t channels, int64_t groups)
{
    size_t most = 0;
    if (samples == 0) return FF_WS_MIN_BYTES;
    for (int size : {2, 4})
        for (bool kept : {false, true}) {
            most = std::max(most, gn_forward_floats(gn_plan(samples, pixels, channels, groups, size, kept, pitch8(channels), false), samples, groups));
            most = std::max(most, gn_backward_floats(gn_plan(samples, pixels, channels, groups, size, false, channels, true), samples, channels, groups));
        }
    return align_up(std::max<size_t>(most * sizeof(float), FF_WS_MIN_BYTES), 16);
}

hipError_t launch_group_norm_forward(const GroupNormForwardLaunch& f, hipStream_t s)
{
    return f.dtype == FF_F32    ? gn_forward_typed<float>(f, s)
           : f.dtype == FF_BF16 ? gn_forward_typed<bf16_t>(f, s)
                                : gn_forward_typed<f16_t>(f, s);
}

hipError_t launch_group_norm_backward(const GroupNormBackwardLaunch& g, hipStream_t s)
{
    if (g.samples == 0) return launch_gn_params((const float2*)g.ws, g, s);
    return g.dtype == FF_F32    ? gn_backward_typed<float>(g, s)
           : g.dtype == FF_BF16 ? gn_backward_typed<bf16_t>(g, s)
                                : gn_backward_typed<f16_t>(g, s);
}

}  // namespace ffi

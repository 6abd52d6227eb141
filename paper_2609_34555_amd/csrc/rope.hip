// rope.hip -- RMS norm of every query and key head and the position rotation, in one pass over a step's rows:
//   y = x * rsqrt(mean(x^2) + eps) * w,   (y_a, y_b) <- (y_a cos t - y_b sin t, y_a sin t + y_b cos t)
// with t = position * inv_freq[i] for the i-th pair of channels.
//
// Bound: HBM, 256 bytes read and written per head of a row.  A head is 16 lanes of 8 channels (one 16-byte load
// each), its sum of squares a register reduction over them.  The angles are taken in 64 bits (a position of 2^20
// in fp32 is off by up to 2^-4 turns of the fastest pair), as a fraction of a turn, once per row for all its heads.
// Sums, norm and rotation are in fp32; the result is rounded to 16 bits once.
// 16K rows of 32 + 8 heads (335 MB read and written): 67 us, 5.0 TB/s (a large copy: 4.8); 78 us before the loads of a
// row's first heads were issued ahead of its angles.  One row: 4.0 us.  Without norms 63 and 3.8.
#include "pulse_internal.h"

namespace pulse {

constexpr int kRopeThreads = 256;
constexpr int kRopeGroups = kRopeThreads / 16;
constexpr int32_t kRopeGrid = 1 << 20;
constexpr int kRopeAhead = 3;  // heads of a group whose loads are in flight together
constexpr int kMaxPairs = kHeadDim / 2;

struct RopeArgs {
    const uint16_t *q, *k;
    int64_t q_stride, k_stride;
    int32_t Hq, Hkv;
    int32_t rows;
    const int32_t* positions;
    const uint16_t *qw, *kw;
    float eps;
    const double* inv_freq;
    int32_t rot;
    uint16_t *q_out, *k_out;
    int64_t q_out_stride, k_out_stride;
};

template <int DT>
__device__ inline void to_floats(u32x4 v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = elem_to_float<DT>((uint16_t)(v[i] & 0xFFFF));
        x[2 * i + 1] = elem_to_float<DT>((uint16_t)(v[i] >> 16));
    }
}

template <int DT>
__device__ inline u32x4 from_floats(const float (&x)[8]) {
    typename Mfma<DT>::vec v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (typename Mfma<DT>::elem)x[i];
    return __builtin_bit_cast(u32x4, v);
}

// Sum over the 16 lanes of a group, in every lane.
__device__ inline float group_sum(float x) {
    auto add = [&](int y) { x += __int_as_float(y); };
    add(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, true));   // lane ^ 1
    add(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, true));   // lane ^ 2
    add(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, true));  // mirrored half row
    add(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xF, 0xF, true));  // mirrored row
    return x;
}

// The rotation of a head's channels 8l .. 8l + 7.
template <bool INTER>
__device__ inline void rotate(int rot, const float* s_cos, const float* s_sin, float (&x)[8], int l, int tid) {
    const int c8 = 8 * l, half = rot / 2;
    if constexpr (INTER) {
        if (c8 < rot) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float c = s_cos[4 * l + i], s = s_sin[4 * l + i];
                const float u = x[2 * i], v = x[2 * i + 1];
                x[2 * i] = u * c - v * s;
                x[2 * i + 1] = u * s + v * c;
            }
        }
    } else {
        // a channel's partner is rot / 2 channels, a whole number of lanes, away
        const bool low = c8 < half;
        const int partner = (tid & 48) | (low ? l + half / 8 : l - half / 8);
        const int pair = low ? c8 : c8 - half;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float o = __shfl(x[i], partner & 63);
            if (c8 < rot) {
                const float c = s_cos[pair + i], s = s_sin[pair + i];
                x[i] = low ? x[i] * c - o * s : o * s + x[i] * c;
            }
        }
    }
}

template <int DT, bool INTER>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
    __shared__ float s_cos[kMaxPairs], s_sin[kMaxPairs];
    const int tid = threadIdx.x, l = tid & 15, group = tid >> 4;
    const int c8 = 8 * l, half = a.rot / 2;
    const int heads = a.Hq + a.Hkv;
    auto at = [&](const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride, int64_t row, int h) {
        return (h < a.Hq ? q + row * q_stride + (size_t)h * kHeadDim
                         : k + row * k_stride + (size_t)(h - a.Hq) * kHeadDim) + c8;
    };
    // this lane's weights, and the row's first heads, do not wait for its angles
    float qw[8], kw[8];
    if (a.qw) to_floats<DT>(*reinterpret_cast<const u32x4*>(a.qw + c8), qw);
    if (a.kw) to_floats<DT>(*reinterpret_cast<const u32x4*>(a.kw + c8), kw);
    const double freq = tid < half ? a.inv_freq[tid] : 0.0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        u32x4 raw[kRopeAhead];
#pragma unroll
        for (int i = 0; i < kRopeAhead; ++i) {
            const int h = group + i * kRopeGroups;
            if (h < heads) raw[i] = *reinterpret_cast<const u32x4*>(at(a.q, a.q_stride, a.k, a.k_stride, row, h));
        }
        const int32_t pos = a.positions[row];
        if (pos < 0) continue;  // the same in every thread of the workgroup
        if (tid < half) {
            // less whole turns, 2 pi in two parts, then as a fraction of half a turn
            const double t = (double)pos * freq, n = rint(t * 0.15915494309189533577);
            const double rest = fma(-n, 2.4492935982947064e-16, fma(-n, 6.28318530717958647693, t));
            sincospif((float)(rest * 0.31830988618379067154), &s_sin[tid], &s_cos[tid]);
        }
        __syncthreads();
        for (int h0 = group; h0 < heads; h0 += kRopeAhead * kRopeGroups) {
            if (h0 != group) {
#pragma unroll
                for (int i = 0; i < kRopeAhead; ++i) {
                    const int h = h0 + i * kRopeGroups;
                    if (h < heads) raw[i] = *reinterpret_cast<const u32x4*>(at(a.q, a.q_stride, a.k, a.k_stride, row, h));
                }
            }
#pragma unroll
            for (int i = 0; i < kRopeAhead; ++i) {
                const int h = h0 + i * kRopeGroups;
                if (h >= heads) break;
                const bool is_q = h < a.Hq;
                float x[8];
                to_floats<DT>(raw[i], x);
                if (is_q ? a.qw != nullptr : a.kw != nullptr) {
                    float ss = 0.f;
#pragma unroll
                    for (int n = 0; n < 8; ++n) ss += x[n] * x[n];
                    const float inv = 1.0f / sqrtf(group_sum(ss) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
                    for (int n = 0; n < 8; ++n) x[n] = x[n] * inv * (is_q ? qw[n] : kw[n]);
                }
                rotate<INTER>(a.rot, s_cos, s_sin, x, l, tid);
                *reinterpret_cast<u32x4*>(
                    const_cast<uint16_t*>(at(a.q_out, a.q_out_stride, a.k_out, a.k_out_stride, row, h))) =
                    from_floats<DT>(x);
            }
        }
        __syncthreads();
    }
}

hipError_t launch_qk_norm_rope(const pulse_shape& s, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                               int32_t rows, const int32_t* positions, const void* qw, const void* kw, float eps,
                               const double* inv_freq, int32_t rot, bool inter, void* q_out, int64_t q_out_stride,
                               void* k_out, int64_t k_out_stride, hipStream_t st) {
    const RopeArgs a{(const uint16_t*)q,  (const uint16_t*)k, q_stride,  k_stride,          s.num_q_heads,
                     s.num_kv_heads,      rows,               positions, (const uint16_t*)qw, (const uint16_t*)kw,
                     eps,                 inv_freq,           rot,       (uint16_t*)q_out,  (uint16_t*)k_out,
                     q_out_stride,        k_out_stride};
    const dim3 grid((unsigned)(rows < kRopeGrid ? rows : kRopeGrid));
    if (elem_type(s.dtype) == PULSE_BF16) {
        if (inter) hipLaunchKernelGGL((rope_kernel<PULSE_BF16, true>), grid, dim3(kRopeThreads), 0, st, a);
        else hipLaunchKernelGGL((rope_kernel<PULSE_BF16, false>), grid, dim3(kRopeThreads), 0, st, a);
    } else {
        if (inter) hipLaunchKernelGGL((rope_kernel<PULSE_F16, true>), grid, dim3(kRopeThreads), 0, st, a);
        else hipLaunchKernelGGL((rope_kernel<PULSE_F16, false>), grid, dim3(kRopeThreads), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace pulse

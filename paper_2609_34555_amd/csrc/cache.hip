// cache.hip -- rows of keys and values into the blocks of a slot pool, and back, by the slot map of a step.
// Row i belongs at token slot_map[i] % bs of slot slot_map[i] / bs (-1: nowhere).
//
// Bound: HBM; a row's head is 512 bytes of 16-bit keys and values against 136 in the 4-bit cache.  A wave owns
// one head of a run of rows: a lane is channels 2 * lane and 2 * lane + 1, so a row's head is one 256-byte load
// and a group of 32 channels (one scale) is 16 lanes, a register reduction.
//
// Values lie 8 tokens to a word (or to 16 bytes of the 16-bit cache), so a run is the rows, at most 8, that
// follow one another inside one octet of tokens: the wave of its first row writes it, whole octets with plain
// stores.  A shorter run shares words with other tokens, which other rows of the call may be writing: it clears
// and sets its own bits with atomics, whose order does not matter.
#include "kv4.h"

namespace pulse {

constexpr int kCacheThreads = 256;
constexpr int kCacheWaves = kCacheThreads / kWave;
constexpr int64_t kCacheGrid = 1 << 20;
constexpr int kOct = 8;

struct CacheArgs {
    const uint16_t *k_in, *v_in;  // append
    uint16_t *k_out, *v_out;      // load
    int64_t k_stride, v_stride;
    const int64_t* slot_map;
    int32_t rows, Hkv;
    uint8_t* pool;
    int64_t places;               // n_slots * bs
    int32_t* status;
};

// The run that row i begins: its first place and length; n = 0 if i begins none (a row inside a run, a row
// without a place).  Every lane of the wave takes part and gets the same answer.
struct Run {
    int64_t at;
    int n;
};
__device__ inline Run find_run(const CacheArgs& a, int64_t i, int lane, bool check) {
    const int64_t row = i - 1 + lane;  // lane 0: the row before
    int64_t m = -1;
    if (lane <= kOct && row >= 0 && row < a.rows) m = a.slot_map[row];
    const int64_t before = __shfl(m, 0);
    Run r;
    r.at = __shfl(m, 1);
    r.n = 0;
    if (r.at < 0 || r.at >= a.places) {
        if (check && r.at != -1 && lane == 0) report(a.status, PULSE_ERR_BAD_INDEX);
        return r;
    }
    if (r.at % kOct != 0 && before == r.at - 1) return r;
    // lane 1 + k continues the run if it holds the k-th next place of the octet
    const bool on = lane >= 1 && lane <= kOct && m == r.at + (lane - 1) && r.at % kOct + (lane - 1) < kOct;
    r.n = __builtin_ctzll(~(__ballot(on) >> 1));
    return r;
}

// Largest of x >= 0 over the 16 lanes of a group; NaN counts as more than anything.
__device__ inline float group_top(float x) {
    uint32_t u = __float_as_uint(x);
    auto top = [&](int y) { u = max(u, (uint32_t)y); };
    top(__builtin_amdgcn_mov_dpp((int)u, 0xB1, 0xF, 0xF, true));
    top(__builtin_amdgcn_mov_dpp((int)u, 0x4E, 0xF, 0xF, true));
    top(__builtin_amdgcn_mov_dpp((int)u, 0x141, 0xF, 0xF, true));
    top(__builtin_amdgcn_mov_dpp((int)u, 0x140, 0xF, 0xF, true));
    return __uint_as_float(u);
}

// Two channels of a row as codes (0 .. 255), with the byte of their group's scale.
template <int DT>
__device__ inline uint32_t encode_pair(uint32_t two, uint32_t& scale_byte) {
    const float x = elem_to_float<DT>((uint16_t)(two & 0xFFFF)), y = elem_to_float<DT>((uint16_t)(two >> 16));
    const uint32_t ux = __float_as_uint(x) & 0x7FFFFFFFu, uy = __float_as_uint(y) & 0x7FFFFFFFu;
    scale_byte = kv4_scale_byte<DT>(group_top(__uint_as_float(max(ux, uy))));
    return scale_byte == kKv4Nan ? 0u : kv4_encode(x, y, kv4_scale(scale_byte));
}

template <int DT, int BS, bool KV4>
__device__ inline void append_run(const CacheArgs& a, int64_t unit, int lane) {
    const int64_t i = unit / a.Hkv;
    const int h = (int)(unit % a.Hkv);
    const Run run = find_run(a, i, lane, h == 0);
    if (run.n == 0) return;
    uint32_t k[kOct], v[kOct];
#pragma unroll
    for (int t = 0; t < kOct; ++t) {
        k[t] = v[t] = 0;
        if (t < run.n) {
            k[t] = reinterpret_cast<const uint32_t*>(a.k_in + (i + t) * a.k_stride + (size_t)h * kHeadDim)[lane];
            v[t] = reinterpret_cast<const uint32_t*>(a.v_in + (i + t) * a.v_stride + (size_t)h * kHeadDim)[lane];
        }
    }
    const int64_t slot = run.at / BS;
    const int row = (int)(run.at % BS), t0 = row % kOct;
    if constexpr (KV4) {
        uint8_t* base = a.pool + ((size_t)slot * a.Hkv + h) * kv4_head_bytes(BS);
        uint32_t w0 = 0, w1 = 0;  // words of the lane's two channels
#pragma unroll
        for (int t = 0; t < kOct; ++t) {
            if (t < run.n) {
                uint32_t ks, vs;
                const uint32_t kc = encode_pair<DT>(k[t], ks), vc = encode_pair<DT>(v[t], vs);
                base[(row + t) * 64 + lane] = (uint8_t)kc;
                if ((lane & 15) == 0) {
                    base[kv4_key_scales(BS) + (row + t) * kGroups + (lane >> 4)] = (uint8_t)ks;
                    base[kv4_value_scales(BS) + (lane >> 4) * BS + row + t] = (uint8_t)vs;
                }
                w0 |= (vc & 15u) << (4 * (t0 + t));
                w1 |= (vc >> 4) << (4 * (t0 + t));
            }
        }
        // channel c = 2 * lane is word [o][c % 16][c / 16]; channel c + 1 the word 8 further on
        uint32_t* words = reinterpret_cast<uint32_t*>(base + kv4_values(BS)) + (row / kOct) * 128 +
                          (2 * lane % 16) * 8 + lane / 8;
        if (run.n == kOct) {
            words[0] = w0;
            words[8] = w1;
        } else {
            const uint32_t mine = ((1u << (4 * run.n)) - 1) << (4 * t0);
            atomicAnd(&words[0], ~mine);
            atomicAnd(&words[8], ~mine);
            atomicOr(&words[0], w0);
            atomicOr(&words[8], w1);
        }
    } else {
        uint16_t* base = reinterpret_cast<uint16_t*>(a.pool) + (size_t)slot * 2 * a.Hkv * BS * kHeadDim;
        uint16_t* kd = base + (size_t)h * BS * kHeadDim;
        uint16_t* vd = base + (size_t)a.Hkv * BS * kHeadDim + ((size_t)h * kHeadDim + 2 * lane) * BS;
#pragma unroll
        for (int t = 0; t < kOct; ++t)
            if (t < run.n) reinterpret_cast<uint32_t*>(kd + (size_t)(row + t) * kHeadDim)[lane] = k[t];
        if (run.n == kOct) {
            u32x4 lo, hi;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                lo[t] = (v[2 * t] & 0xFFFFu) | (v[2 * t + 1] << 16);
                hi[t] = (v[2 * t] >> 16) | (v[2 * t + 1] & 0xFFFF0000u);
            }
            *reinterpret_cast<u32x4*>(vd + row) = lo;
            *reinterpret_cast<u32x4*>(vd + BS + row) = hi;
        } else {
#pragma unroll
            for (int t = 0; t < kOct; ++t)
                if (t < run.n) {
                    vd[row + t] = (uint16_t)(v[t] & 0xFFFF);
                    vd[BS + row + t] = (uint16_t)(v[t] >> 16);
                }
        }
    }
}

template <int DT, int BS, bool KV4>
__device__ inline void load_run(const CacheArgs& a, int64_t unit, int lane) {
    const int64_t i = unit / a.Hkv;
    const int h = (int)(unit % a.Hkv);
    const Run run = find_run(a, i, lane, h == 0);
    if (run.n == 0) return;
    const int64_t slot = run.at / BS;
    const int row = (int)(run.at % BS), t0 = row % kOct;
    uint32_t k[kOct], v[kOct];
    if constexpr (KV4) {
        const uint8_t* base = a.pool + ((size_t)slot * a.Hkv + h) * kv4_head_bytes(BS);
        const uint32_t* words = reinterpret_cast<const uint32_t*>(base + kv4_values(BS)) + (row / kOct) * 128 +
                                (2 * lane % 16) * 8 + lane / 8;
        const uint32_t w0 = words[0], w1 = words[8];
#pragma unroll
        for (int t = 0; t < kOct; ++t) {
            k[t] = v[t] = 0;
            if (t < run.n) {
                const uint32_t kc = base[(row + t) * 64 + lane];
                const float ks = kv4_scale(base[kv4_key_scales(BS) + (row + t) * kGroups + (lane >> 4)]);
                const float vs = kv4_scale(base[kv4_value_scales(BS) + (lane >> 4) * BS + row + t]);
                const uint32_t vc = (w0 >> (4 * (t0 + t)) & 15u) | (w1 >> (4 * (t0 + t)) & 15u) << 4;
                k[t] = kv4_decode<DT, 0>(kc, ks);
                v[t] = kv4_decode<DT, 0>(vc, vs);
            }
        }
    } else {
        const uint16_t* base = reinterpret_cast<const uint16_t*>(a.pool) + (size_t)slot * 2 * a.Hkv * BS * kHeadDim;
        const uint16_t* kd = base + (size_t)h * BS * kHeadDim;
        const uint16_t* vd = base + (size_t)a.Hkv * BS * kHeadDim + ((size_t)h * kHeadDim + 2 * lane) * BS;
#pragma unroll
        for (int t = 0; t < kOct; ++t) {
            k[t] = v[t] = 0;
            if (t < run.n) {
                k[t] = reinterpret_cast<const uint32_t*>(kd + (size_t)(row + t) * kHeadDim)[lane];
                v[t] = (uint32_t)vd[row + t] | (uint32_t)vd[BS + row + t] << 16;
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kOct; ++t)
        if (t < run.n) {
            reinterpret_cast<uint32_t*>(a.k_out + (i + t) * a.k_stride + (size_t)h * kHeadDim)[lane] = k[t];
            reinterpret_cast<uint32_t*>(a.v_out + (i + t) * a.v_stride + (size_t)h * kHeadDim)[lane] = v[t];
        }
}

// A wave takes (row, head) pairs a grid apart.
template <int DT, int BS, bool KV4, bool APPEND>
__global__ __launch_bounds__(kCacheThreads) void cache_kernel(CacheArgs a) {
    const int64_t units = (int64_t)a.rows * a.Hkv, stride = (int64_t)gridDim.x * kCacheWaves;
    const int lane = threadIdx.x & 63;
    for (int64_t u = (int64_t)blockIdx.x * kCacheWaves + (threadIdx.x >> 6); u < units; u += stride) {
        if constexpr (APPEND) append_run<DT, BS, KV4>(a, u, lane);
        else load_run<DT, BS, KV4>(a, u, lane);
    }
}

template <int DT, int BS, bool KV4>
static void launch_cache_t(const CacheArgs& a, bool append, hipStream_t st) {
    const int64_t groups = ((int64_t)a.rows * a.Hkv + kCacheWaves - 1) / kCacheWaves;
    const dim3 grid((unsigned)(groups < kCacheGrid ? groups : kCacheGrid));
    if (append) hipLaunchKernelGGL((cache_kernel<DT, BS, KV4, true>), grid, dim3(kCacheThreads), 0, st, a);
    else hipLaunchKernelGGL((cache_kernel<DT, BS, KV4, false>), grid, dim3(kCacheThreads), 0, st, a);
}

template <int DT, bool KV4>
static void launch_cache_bs(int32_t bs, const CacheArgs& a, bool append, hipStream_t st) {
    if (bs == 16) launch_cache_t<DT, 16, KV4>(a, append, st);
    else if (bs == 32) launch_cache_t<DT, 32, KV4>(a, append, st);
    else launch_cache_t<DT, 64, KV4>(a, append, st);
}

static hipError_t launch_cache(const pulse_shape& s, const CacheArgs& a, bool append, hipStream_t st) {
    // copies of 16-bit elements do not look at their type
    if (!is_kv4(s.dtype)) launch_cache_bs<PULSE_BF16, false>(s.block_size, a, append, st);
    else if (elem_type(s.dtype) == PULSE_BF16) launch_cache_bs<PULSE_BF16, true>(s.block_size, a, append, st);
    else launch_cache_bs<PULSE_F16, true>(s.block_size, a, append, st);
    return hipGetLastError();
}

hipError_t launch_append_kv(const pulse_shape& s, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int64_t* slot_map, int32_t rows, void* pool, int32_t n_slots, int32_t* status,
                            hipStream_t st) {
    const CacheArgs a{(const uint16_t*)k, (const uint16_t*)v, nullptr, nullptr, k_stride, v_stride, slot_map, rows,
                      s.num_kv_heads, (uint8_t*)pool, (int64_t)n_slots * s.block_size, status};
    return launch_cache(s, a, true, st);
}

hipError_t launch_load_kv(const pulse_shape& s, const void* pool, int32_t n_slots, const int64_t* slot_map,
                          int32_t rows, void* k, int64_t k_stride, void* v, int64_t v_stride, int32_t* status,
                          hipStream_t st) {
    const CacheArgs a{nullptr, nullptr, (uint16_t*)k, (uint16_t*)v, k_stride, v_stride, slot_map, rows,
                      s.num_kv_heads, (uint8_t*)const_cast<void*>(pool), (int64_t)n_slots * s.block_size, status};
    return launch_cache(s, a, false, st);
}

}  // namespace pulse

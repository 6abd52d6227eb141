// cache.hip -- rows of keys and values into the blocks of a slot pool, and back, by the slot map of a step.
// Row i belongs at token slot_map[i] % bs of slot slot_map[i] / bs (-1: nowhere).
//
// Bound: HBM; a row's head is 512 bytes of 16-bit keys and values against 136 in the 4-bit cache.
//
// Values lie 8 tokens to a word (or to 16 bytes of the 16-bit cache), so the unit of work is a run: the rows, at
// most 8, that follow one another inside one octet of tokens.  A wave takes one head of a run.  Its lane group g
// holds tokens 2g and 2g + 1 of the octet and lane l of a group channels 8l .. 8l + 7, so that a head of a row is
// one 16-byte load per lane, a scale's 32 channels are four neighbouring lanes (two register exchanges) and a
// row's key codes one 4-byte store per lane.  Values change between "8 channels of 2 tokens" and "8 tokens of 2
// channels" by exchanges of lane groups in registers.
// A run shorter than an octet shares words with other tokens, which other rows of the call may be writing: it
// clears and sets its own bits with atomics, whose order does not matter.
// 16K rows of 8 heads into 4 bits: 19 us for 85 MB (17.8 at the rate of a large copy), back 15 where the blocks have
// just been written and 22 where they come from memory; with a lane per two channels and a wave per row, byte stores and
// all, 97 and 69.  The same rows into 16-bit blocks and back: 31 and 30 us for 134 MB (28).
#include "kv4.h"

namespace pulse {

constexpr int kCacheThreads = 256;
constexpr int kCacheWaves = kCacheThreads / kWave;
constexpr int kOct = 8;
constexpr int64_t kCacheGrid = 65535;
// Rows times heads up to which a wave looks at one row (each may begin a run), above at an octet's.  In us, appending to
// 4-bit and to 16-bit blocks with one row and with an octet per wave:
//   rows that follow one another    512 x 8 heads  4.3 3.9   4.1 3.9     1024 x 8  5.1 4.1   5.4 4.6
//                                   2048 x 8       7.9 5.2   7.9 6.3    16381 x 8   40  19    50  31
//                                   4096 x 1       4.5 3.8   4.6 3.5    16384 x 1  8.1 5.2   9.5 6.3
//   rows of a request each            64 x 8       4.2 13.5  3.8 12.5    2048 x 8  27.3 28.4  48  37
//                                   8192 x 1      15.7 18.0 15.5 21.3
// Below the limit a decode batch's rows decide, which would lose 9 us with an octet; rows that follow one another lose 1
// without.
constexpr int64_t kRunRows = 8192;

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

// One head of a run: its rows are `first` .. first + n - 1, their places `at` .. at + n - 1.
struct Run {
    int64_t first, at;
    int n, h;
};

// Exchange of lane groups: rows 0..3 of a and b become {a0, b0, a2, b2} and {a1, b1, a3, b3} (cross16), or
// {a0, a1, b0, b1} and {a2, a3, b2, b3} (cross32).
__device__ inline void cross16(uint32_t& a, uint32_t& b) {
    const u32x2 r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
__device__ inline void cross32(uint32_t& a, uint32_t& b) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// Group g holds words 0 .. 7 of its own; afterwards it holds words 2g and 2g + 1 of every group: w[j] is word
// 2g + j / 4 of group j % 4.
__device__ inline void transpose_groups(uint32_t (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) cross32(w[i], w[i + 4]);
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        cross16(w[i], w[i + 2]);
        cross16(w[i + 1], w[i + 3]);
    }
    // now w[4 * (group / 2) + 2 * (group % 2) + (word % 2)] of the words 2g, 2g + 1
    const uint32_t t[8] = {w[0], w[2], w[4], w[6], w[1], w[3], w[5], w[7]};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = t[i];
}

// The same back: w[j] holds word 2g + j / 4 of group j % 4; afterwards w[i] is word i of the lane's own group.
__device__ inline void untranspose_groups(uint32_t (&w)[8]) {
    uint32_t t[8] = {w[0], w[4], w[1], w[5], w[2], w[6], w[3], w[7]};
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        cross16(t[i], t[i + 2]);
        cross16(t[i + 1], t[i + 3]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) cross32(t[i], t[i + 4]);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = t[i];
}

// Largest magnitude of 8 16-bit values and of those of the other three lanes of a scale; infinities and NaN
// are more than anything.
template <int DT>
__device__ inline float scale_top(u32x4 v) {
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u = max(max(u, v[i] & 0x7FFFu), (v[i] >> 16) & 0x7FFFu);
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp((int)u, 0xB1, 0xF, 0xF, true));  // lane ^ 1
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp((int)u, 0x4E, 0xF, 0xF, true));  // lane ^ 2
    return elem_to_float<DT>((uint16_t)u);
}

// 8 values as 8 codes, channel 8l + i in bits 4i .. 4i + 3, and the byte of their scale.
template <int DT>
__device__ inline uint32_t encode8(u32x4 v, uint32_t& scale_byte) {
    scale_byte = kv4_scale_byte<DT>(scale_top<DT>(v));
    if (scale_byte == kKv4Nan) return 0;
    const float s = kv4_scale(scale_byte);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w |= kv4_encode(elem_to_float<DT>((uint16_t)(v[i] & 0xFFFF)), elem_to_float<DT>((uint16_t)(v[i] >> 16)), s)
             << (8 * i);
    return w;
}

// x of the four scales of a row (lanes 0-3, 4-7, ..) as the bytes of a word, in every lane of the row.
__device__ inline uint32_t row_bytes(uint32_t x, int l) {
    uint32_t u = x << (8 * (l >> 2));
    u |= (uint32_t)__builtin_amdgcn_mov_dpp((int)u, 0x141, 0xF, 0xF, true);  // mirrored half row
    u |= (uint32_t)__builtin_amdgcn_mov_dpp((int)u, 0x140, 0xF, 0xF, true);  // mirrored row
    return u;
}

template <int DT, int BS, bool KV4>
__device__ inline void append_run(const CacheArgs& a, const Run& run, int lane) {
    const int l = lane & 15, grp = lane >> 4;
    const int64_t slot = run.at / BS;
    const int o0 = (int)(run.at % BS) / kOct * kOct, t0 = (int)(run.at % kOct);  // the octet, the run's place in it
    u32x4 k[2], v[2];
    bool on[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = 2 * grp + i - t0;  // row of the run that is this token
        on[i] = t >= 0 && t < run.n;
        const int64_t row = run.first + (on[i] ? t : 0);
        const size_t c = (size_t)run.h * kHeadDim + 8 * l;
        // streamed: rows that stay in the caches push the half-written lines of the blocks out (16K rows of 8 heads 27 us
        // with ordinary loads, 19 with these)
        k[i] = v[i] = u32x4{0, 0, 0, 0};
        if (on[i]) {
            k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.k_in + row * a.k_stride + c));
            v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.v_in + row * a.v_stride + c));
        }
    }
    const bool full = run.n == kOct;
    if constexpr (KV4) {
        uint8_t* base = a.pool + ((size_t)slot * a.Hkv + run.h) * kv4_head_bytes(BS);
        uint32_t vc[2], vs[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = o0 + 2 * grp + i;
            uint32_t ks;
            const uint32_t kc = encode8<DT>(k[i], ks);
            vc[i] = encode8<DT>(v[i], vs[i]);
            const uint32_t ks4 = row_bytes(ks, l);
            if (on[i]) {
                *reinterpret_cast<uint32_t*>(base + row * 64 + 4 * l) = kc;
                if (l == 0) *reinterpret_cast<uint32_t*>(base + kv4_key_scales(BS) + row * kGroups) = ks4;
            }
        }
        // value scales of a group: a byte per token
        uint8_t* vsd = base + kv4_value_scales(BS) + (l >> 2) * BS + o0 + 2 * grp;
        if ((l & 3) == 0) {
            if (full) {
                *reinterpret_cast<uint16_t*>(vsd) = (uint16_t)(vs[0] | vs[1] << 8);
            } else {
                if (on[0]) vsd[0] = (uint8_t)vs[0];
                if (on[1]) vsd[1] = (uint8_t)vs[1];
            }
        }
        // words of 8 tokens: this lane's two tokens of channels 8l + i, then the groups' words or-ed together,
        // each group keeping two channels
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = ((vc[0] >> (4 * i) & 15u) | (vc[1] >> (4 * i) & 15u) << 4) << (8 * grp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cross32(w[i], w[i + 4]);
            w[i] |= w[i + 4];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            cross16(w[i], w[i + 2]);
            w[i] |= w[i + 2];
        }
        const uint32_t mine = full ? ~0u : ((1u << (4 * run.n)) - 1) << (4 * t0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = 8 * l + 2 * grp + i;
            uint32_t* word = reinterpret_cast<uint32_t*>(base + kv4_values(BS)) + (o0 / kOct * 16 + c % 16) * 8 + c / 16;
            if (full) {
                *word = w[i];
            } else {
                atomicAnd(word, ~mine);
                atomicOr(word, w[i]);
            }
        }
    } else {
        uint16_t* base = reinterpret_cast<uint16_t*>(a.pool) + (size_t)slot * 2 * a.Hkv * BS * kHeadDim;
        uint16_t* kd = base + (size_t)run.h * BS * kHeadDim + 8 * l;
        uint16_t* vd = base + (size_t)(a.Hkv + run.h) * BS * kHeadDim + o0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (on[i]) *reinterpret_cast<u32x4*>(kd + (size_t)(o0 + 2 * grp + i) * kHeadDim) = k[i];
        uint32_t w[8];  // two tokens of channel 8l + i
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = (v[0][i / 2] >> (16 * (i % 2)) & 0xFFFFu) | (v[1][i / 2] >> (16 * (i % 2)) << 16);
        if (full) {
            transpose_groups(w);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<u32x4*>(vd + (size_t)(8 * l + 2 * grp + i) * BS) =
                    u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (on[0]) vd[(size_t)(8 * l + i) * BS + 2 * grp] = (uint16_t)(w[i] & 0xFFFF);
                if (on[1]) vd[(size_t)(8 * l + i) * BS + 2 * grp + 1] = (uint16_t)(w[i] >> 16);
            }
        }
    }
}

template <int DT, int BS, bool KV4>
__device__ inline void load_run(const CacheArgs& a, const Run& run, int lane) {
    const int l = lane & 15, grp = lane >> 4;
    const int64_t slot = run.at / BS;
    const int o0 = (int)(run.at % BS) / kOct * kOct, t0 = (int)(run.at % kOct);
    bool on[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) on[i] = 2 * grp + i >= t0 && 2 * grp + i < t0 + run.n;
    u32x4 k[2] = {}, v[2];
    uint32_t w[8];
    if constexpr (KV4) {
        const uint8_t* base = a.pool + ((size_t)slot * a.Hkv + run.h) * kv4_head_bytes(BS);
        uint32_t kc[2] = {}, ks[2] = {}, vs = 0, mine[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = o0 + 2 * grp + i, c = 8 * l + 2 * grp + i;
            if (on[i]) {
                kc[i] = *reinterpret_cast<const uint32_t*>(base + row * 64 + 4 * l);
                ks[i] = base[kv4_key_scales(BS) + row * kGroups + (l >> 2)];
            }
            mine[i] = reinterpret_cast<const uint32_t*>(base + kv4_values(BS))[(o0 / kOct * 16 + c % 16) * 8 + c / 16];
        }
        vs = *reinterpret_cast<const uint16_t*>(base + kv4_value_scales(BS) + (l >> 2) * BS + o0 + 2 * grp);
        // each group's two words to all groups: word 2g + i of the group's own channels
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t e = mine[i], o = mine[i];
            cross16(e, o);  // e: groups 0 and 2, o: groups 1 and 3
            uint32_t e2 = e, o2 = o;
            cross32(e, e2);
            cross32(o, o2);
            w[i] = e;
            w[2 + i] = o;
            w[4 + i] = e2;
            w[6 + i] = o2;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            k[i] = __builtin_bit_cast(u32x4, kv4_decode8<DT>(kc[i], kv4_scale(ks[i])));
            uint32_t c = 0;
#pragma unroll
            for (int n = 0; n < 8; ++n) c |= (w[n] >> (8 * grp + 4 * i) & 15u) << (4 * n);
            v[i] = __builtin_bit_cast(u32x4, kv4_decode8<DT>(c, kv4_scale(vs >> (8 * i) & 0xFFu)));
        }
    } else {
        const uint16_t* base = reinterpret_cast<const uint16_t*>(a.pool) + (size_t)slot * 2 * a.Hkv * BS * kHeadDim;
        const uint16_t* kd = base + (size_t)run.h * BS * kHeadDim + 8 * l;
        const uint16_t* vd = base + (size_t)(a.Hkv + run.h) * BS * kHeadDim + o0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (on[i]) k[i] = *reinterpret_cast<const u32x4*>(kd + (size_t)(o0 + 2 * grp + i) * kHeadDim);
            const u32x4 x = *reinterpret_cast<const u32x4*>(vd + (size_t)(8 * l + 2 * grp + i) * BS);
#pragma unroll
            for (int n = 0; n < 4; ++n) w[4 * i + n] = x[n];
        }
        untranspose_groups(w);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            v[0][n] = (w[2 * n] & 0xFFFFu) | w[2 * n + 1] << 16;
            v[1][n] = w[2 * n] >> 16 | (w[2 * n + 1] & 0xFFFF0000u);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (on[i]) {
            const int64_t row = run.first + (2 * grp + i - t0);
            const size_t c = (size_t)run.h * kHeadDim + 8 * l;
            *reinterpret_cast<u32x4*>(a.k_out + row * a.k_stride + c) = k[i];
            *reinterpret_cast<u32x4*>(a.v_out + row * a.v_stride + c) = v[i];
        }
}

// grid = (Hkv, groups of kCacheWaves * per rows): a wave takes one head of the runs that begin in its `per` rows (1 or
// kOct); neighbouring workgroups take neighbouring heads, which lie together in rows and blocks.
template <int DT, int BS, bool KV4, bool APPEND>
__global__ __launch_bounds__(kCacheThreads) void cache_kernel(CacheArgs a, int32_t per) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t step = (int64_t)kCacheWaves * per;
    for (int64_t r0 = blockIdx.y * step + wave * per; r0 < a.rows; r0 += gridDim.y * step) {
        // places of the row before, of this wave's rows and of those that its last run may go on to
        const int64_t row = r0 - 1 + lane;
        int64_t m = -1;
        if (lane < per + kOct && row >= 0 && row < a.rows) m = a.slot_map[row];
        const bool ok = m >= 0 && m < a.places;
        if (blockIdx.x == 0 && m != -1 && !ok && lane >= 1 && lane <= per) report(a.status, PULSE_ERR_BAD_INDEX);
        const int64_t prev = __shfl_up(m, 1);
        const bool goes_on = lane > 0 && ok && prev == m - 1 && m % kOct != 0;
        const uint64_t on = __ballot(goes_on);
        uint64_t begin = __ballot(ok && !goes_on) & (((1ull << per) - 1) << 1);
        while (begin) {
            const int at = __builtin_ctzll(begin);
            begin &= begin - 1;
            Run run;
            run.first = r0 - 1 + at;
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)m, at);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(m >> 32), at);
            run.at = (int64_t)((uint64_t)hi << 32 | lo);
            run.n = 1 + __builtin_ctzll(~(on >> (at + 1)));
            run.h = blockIdx.x;
            if constexpr (APPEND) append_run<DT, BS, KV4>(a, run, lane);
            else load_run<DT, BS, KV4>(a, run, lane);
        }
    }
}

template <int DT, int BS, bool KV4>
static void launch_cache_t(const CacheArgs& a, bool append, hipStream_t st) {
    const int32_t per = (int64_t)a.rows * a.Hkv > kRunRows ? kOct : 1;
    const int64_t groups = ((int64_t)a.rows + kCacheWaves * per - 1) / (kCacheWaves * per);
    const dim3 grid((unsigned)a.Hkv, (unsigned)(groups < kCacheGrid ? groups : kCacheGrid));
    if (append) hipLaunchKernelGGL((cache_kernel<DT, BS, KV4, true>), grid, dim3(kCacheThreads), 0, st, a, per);
    else hipLaunchKernelGGL((cache_kernel<DT, BS, KV4, false>), grid, dim3(kCacheThreads), 0, st, a, per);
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

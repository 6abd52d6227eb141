// pages.hip -- blocks of the slot pool as pages: forks of requests that share them, blocks given back, and a pool's live
// blocks moved below a slot number.
//
// A slot is live while a table entry names it; shared[s] counts the entries beyond the first (0 for a slot that was just
// taken, so that pulse_build_tables and the recall need not know of it).  Whole blocks are never written again, so a fork
// shares them; the block that it ends inside is copied.
//
// Bound: tables, lists and counts are read once or twice from L2, a few microseconds of dependent round trips and
// launches; copies run at the rate of HBM.  Nothing is written before what a call uses is checked, which takes a pass (and,
// beyond one workgroup, a launch) of its own.  No result depends on the order of atomics: counts, maxima and bits.
// In the kernels, blocks of 64 KiB: 48 forks (as many blocks copied, 6 MB) 4.9 us of checks and 6.5, a free of 33K entries 3.6 +
// 2.9 + 3.9 + 4.4 (one workgroup: 103), of 635 entries 4.6; a compaction of 6K entries plans in 6.5 and moves 131 MB read
// and 131 written in 48.4 (5.4 TB/s).
#include <algorithm>

#include "pulse_internal.h"

namespace pulse {

constexpr int kPageThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kTile = 256;            // entries of a workgroup in the passes over tables
constexpr int kChunk = 16384;         // bytes of a block that a workgroup copies at a time
// Table entries up to which one workgroup makes every pass of a free, and table and list entries up to which it plans a
// compaction.  In us, a pass of a free (three small copies and a fork with it), one workgroup and a launch for each of its
// four passes: 635 entries 27 and 34, 3K 28.8 and 34, 6K 37.3 and 37.2, 8K 43 and 38, 33K 121 and 38; a compaction of
// 6K entries and a list of 8K 63.4 and 70.5.
constexpr int kOneFree = 4096;
constexpr int kOneGroup = 8192;
constexpr int kCopyGroups = 2048;

// Values that other workgroups, or other waves, wrote in this launch or an atomic changed: past the vector cache.
template <typename T>
__device__ inline T fresh_load(const T* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ inline int block_sum(int x, int* s_wave, int waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int w = (int)last_lane(wave_scan((uint32_t)x, 0u, OpAdd()));
    __syncthreads();
    if (lane == 0) s_wave[wave] = w;
    __syncthreads();
    int sum = 0;
    for (int i = 0; i < waves; ++i) sum += s_wave[i];
    return sum;
}

// Bytes [at, at + kChunk) of a block of U bytes.
__device__ inline void copy_chunk_of(const uint8_t* __restrict__ src, uint8_t* __restrict__ dst, int64_t at, int64_t U) {
    u32x4 v[kChunk / 16 / kPageThreads];
#pragma unroll
    for (int i = 0; i < kChunk / 16 / kPageThreads; ++i) {
        const int64_t o = at + (int64_t)(i * kPageThreads + threadIdx.x) * 16;
        if (o < U) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + o));
    }
#pragma unroll
    for (int i = 0; i < kChunk / 16 / kPageThreads; ++i) {
        const int64_t o = at + (int64_t)(i * kPageThreads + threadIdx.x) * 16;
        if (o < U) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(dst + o));
    }
}

// ---- free ----

struct FreeArgs {
    const int32_t* keep;
    int32_t B, bs;
    int32_t* table;
    int32_t mb;
    int32_t* shared;
    int32_t* free_slots;
    int32_t* free_head;
    int32_t n_free, n_slots;
    int32_t* status;
    int32_t* cnt;   // [n_slots] freed entries of a slot (of slots that have any)
    int32_t* last;  // [n_slots] the last of them
    int32_t* tile_cnt;
    int32_t* tile_err;
    int32_t* head0;
    int32_t tiles;
};

// N entries, 64 from one to the next, loaded before any of them is looked at.
template <int N>
struct Entries {
    int e[N], j[N], slot[N], keep[N];
    bool in[N];
    __device__ Entries(const FreeArgs& a, int first, int end) {
        int r = first / a.mb, at = first - r * a.mb;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            in[i] = first + 64 * i < end;
            e[i] = in[i] ? first + 64 * i : 0;
            j[i] = in[i] ? at : 0;
            slot[i] = a.table[e[i]];
            keep[i] = a.keep[in[i] ? r : 0];
            at += 64;
            if (at >= a.mb) {
                const int rows = at / a.mb;
                r += rows;
                at -= rows * a.mb;
            }
        }
    }
};

// Slot of an entry if it is freed, -1 if not, -2 if something is wrong with it.
__device__ inline int freed_slot(const FreeArgs& a, int j, int s, int keep) {
    if (keep < 0) return -2;
    if (j * (int64_t)a.bs >= keep) return s == -1 ? -1 : (s < 0 || s >= a.n_slots) ? -2 : s;
    // a kept block that tokens are taken out of is appended to next, which no other request may see
    if ((j + 1) * (int64_t)a.bs > keep && a.shared && s >= 0 && s < a.n_slots && a.shared[s] > 0) return -2;
    return -1;
}

// The passes, of one entry whose freed_slot is s >= 0.
__device__ inline void free_reset(const FreeArgs& a, int s) {
    __hip_atomic_store(a.cnt + s, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(a.last + s, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void free_count(const FreeArgs& a, int e, int s) {
    atomicAdd(a.cnt + s, 1);
    atomicMax(a.last + s, e);
}
// Whether it is the one whose slot goes back to the list.
__device__ inline bool free_returns(const FreeArgs& a, int e, int s, bool& wrong) {
    if (fresh_load(a.last + s) != e) return false;
    const int held = a.shared ? a.shared[s] : 0, n = fresh_load(a.cnt + s);
    wrong |= held < 0 || n > held + 1;
    return n == held + 1;
}
// Whether an entry that stays names a slot that goes back, which would be in the list and in the table.  Of a slot that is
// not freed `last` and `cnt` are any numbers: it is freed if the entry that `last` names is one of its own that is.  A load
// of 4 bytes an entry: frees of 4K, 33K and 262K entries 5.4, 12.6 and 12.6 us with and without it, of 2M 100 and 85; counted by
// atomics instead 13.1, 12.9, 24.9 and 159.
__device__ inline bool free_wrongs(const FreeArgs& a, int j, int s, int keep) {
    if (j * (int64_t)a.bs >= keep || s < 0 || s >= a.n_slots) return false;
    const int e = fresh_load(a.last + s);
    if (e < 0 || e >= a.B * a.mb || a.table[e] != s) return false;
    const int r = e / a.mb;
    return (e - r * a.mb) * (int64_t)a.bs >= a.keep[r] && fresh_load(a.cnt + s) > (a.shared ? a.shared[s] : 0);
}
__device__ inline void free_apply(const FreeArgs& a, int e, int s, bool returns, int at) {
    if (a.shared && fresh_load(a.last + s) == e) a.shared[s] = max(a.shared[s] - fresh_load(a.cnt + s), 0);
    if (returns) a.free_slots[at] = s;
    a.table[e] = -1;
}

// Stores and atomics of this wave have reached L2, where the workgroup's other waves look.
__device__ inline void reached_l2() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// All passes in one workgroup, N times 64 entries a wave, which stay in registers.
template <int N>
__global__ __launch_bounds__(kPlanThreads) void free_small_kernel(FreeArgs a) {
    __shared__ int s_wave[kPlanWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = a.B * a.mb;
    const int head = *a.free_head;
    const Entries<N> x(a, wave * 64 * N + lane, n);
    bool wrong = head < 0 || head > a.n_free;
    int s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = x.in[i] ? freed_slot(a, x.j[i], x.slot[i], x.keep[i]) : -1;
        wrong |= s[i] == -2;
        if (s[i] >= 0) free_reset(a, s[i]);
    }
    reached_l2();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (s[i] >= 0) free_count(a, x.e[i], s[i]);
    reached_l2();
    uint64_t ret[N];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        bool returns = false;
        if (s[i] >= 0) returns = free_returns(a, x.e[i], s[i], wrong);
        else if (x.in[i]) wrong |= free_wrongs(a, x.j[i], x.slot[i], x.keep[i]);
        ret[i] = __ballot(returns);
        mine += __popcll(ret[i]);
    }
    if (lane == 0) s_wave[wave] = mine;
    wrong = __syncthreads_or(wrong);
    int before = 0, total = 0;
    for (int i = 0; i < kPlanWaves; ++i) {
        if (i < wave) before += s_wave[i];
        total += s_wave[i];
    }
    if (wrong || total > head) {
        if (threadIdx.x == 0) report(a.status, PULSE_ERR_BAD_INDEX);
        return;
    }
    int at = head - total + before;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (s[i] >= 0) free_apply(a, x.e[i], s[i], ret[i] >> lane & 1, at + __popcll(ret[i] & ((1ull << lane) - 1)));
        at += __popcll(ret[i]);
    }
    if (threadIdx.x == 0) *a.free_head = head - total;
}

// The same passes over tiles of entries, a launch each: 0 reset, 1 count, 2 find those that return, 3 apply.
template <int PASS>
__global__ __launch_bounds__(kPageThreads) void free_kernel(FreeArgs a) {
    __shared__ int s_wave[kPageThreads / kWave];
    constexpr int kEach = kTile / kPageThreads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = a.B * a.mb;
    const int64_t e0 = (int64_t)blockIdx.x * kTile + wave * (kTile / 4);  // a wave's entries follow one another
    const Entries<kEach> x(a, (int)min(e0 + lane, (int64_t)n), n);
    int s[kEach];
    bool wrong = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        s[i] = freed_slot(a, x.j[i], x.slot[i], x.keep[i]);
        if (!x.in[i]) s[i] = -1;
        wrong |= s[i] == -2;
        if (PASS == 0 && s[i] >= 0) free_reset(a, s[i]);
        if (PASS == 1 && s[i] >= 0) free_count(a, x.e[i], s[i]);
    }
    if (PASS < 2) return;
    uint64_t ret[kEach];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        bool returns = false;
        if (s[i] >= 0) returns = free_returns(a, x.e[i], s[i], wrong);
        else if (PASS == 2 && x.in[i]) wrong |= free_wrongs(a, x.j[i], x.slot[i], x.keep[i]);
        ret[i] = __ballot(returns);
        mine += __popcll(ret[i]);
    }
    if (PASS == 2) {
        if (lane == 0) s_wave[wave] = mine;
        wrong = __syncthreads_or(wrong);
        if (threadIdx.x == 0) {
            a.tile_err[blockIdx.x] = wrong;
            a.tile_cnt[blockIdx.x] = s_wave[0] + s_wave[1] + s_wave[2] + s_wave[3];
            if (blockIdx.x == 0) *a.head0 = *a.free_head;
        }
        return;
    }
    int before = 0, total = 0, errs = 0;
    for (int t = threadIdx.x; t < a.tiles; t += kPageThreads) {
        const int c = a.tile_cnt[t];
        total += c;
        if (t < (int)blockIdx.x) before += c;
        errs |= a.tile_err[t];
    }
    before = block_sum(before, s_wave, kPageThreads / kWave);
    total = block_sum(total, s_wave, kPageThreads / kWave);
    const int head = *a.head0;
    if (__syncthreads_or(errs) || head < 0 || head > a.n_free || total > head) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, PULSE_ERR_BAD_INDEX);
        return;
    }
    if (lane == 0) s_wave[wave] = mine;
    __syncthreads();
    int at = head - total + before;
    for (int i = 0; i < wave; ++i) at += s_wave[i];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (s[i] >= 0) free_apply(a, x.e[i], s[i], ret[i] >> lane & 1, at + __popcll(ret[i] & ((1ull << lane) - 1)));
        at += __popcll(ret[i]);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.free_head = head - total;
}

// ---- fork ----

struct ForkArgs {
    const int32_t *src, *dst, *len;
    int32_t n, bs;
    int32_t* table;
    int32_t B, mb;
    int32_t* shared;
    const int32_t* free_slots;
    int32_t* free_head;
    int32_t n_free;
    uint8_t* pool;
    int32_t n_slots;
    int64_t U;
    int32_t* status;
    int32_t* err;       // [n]
    int32_t* scan_err;  // [scans]
    int32_t scans;
    int32_t* head0;
};

constexpr int kScan = 1024;       // table entries that a workgroup looks at in a turn
constexpr int kScanGroups = 512;
// Places of the set below for up to n slots.
__host__ __device__ inline int slot_places(int n) {
    int size = kPageThreads;
    while (size < 2 * n) size *= 2;
    return size;
}

// Whether a slot that the forks take is taken twice, is counted, or is one of the entries that this workgroup looks at.  The
// slots are a set in LDS that is at most half full, searched from a place that depends on the slot until an empty one.  Beside
// the forks' own checks: 48 forks in 33K entries 9.6 us with it and 9.9 without, 120 in 2M 21.3 and 17.6, 2000 of a call 78 and 70.
__device__ inline bool taken_wrong(const ForkArgs& a, int scan, int* s_set, int* s_wave) {
    int parts = 0;
    for (int k = threadIdx.x; k < a.n; k += kPageThreads) parts += a.len[k] % a.bs != 0;
    const int total = block_sum(parts, s_wave, kPageThreads / kWave);
    const int head = *a.free_head;
    if (total == 0 || head < 0 || head > a.n_free || total > a.n_free - head) return false;  // (for fork_kernel to report)
    const int size = slot_places(total);
    for (int k = threadIdx.x; k < size; k += kPageThreads) s_set[k] = -1;
    __syncthreads();
    auto place = [&](int s) { return (int)((uint32_t)s * 2654435761u >> 16) & (size - 1); };
    bool wrong = false;
    for (int k = threadIdx.x; k < total; k += kPageThreads) {
        const int s = a.free_slots[head + k];
        if (s < 0 || s >= a.n_slots) continue;
        if (scan == 0) wrong |= a.shared[s] != 0;
        int was = -1;
        for (int at = place(s); (was = atomicCAS(s_set + at, -1, s)) != -1 && was != s;) at = (at + 1) & (size - 1);
        wrong |= was == s;
    }
    __syncthreads();
    const int n = a.B * a.mb;
    for (int64_t e0 = (int64_t)scan * kScan + threadIdx.x; e0 < n; e0 += (int64_t)a.scans * kScan) {
        int v[kScan / kPageThreads];
#pragma unroll
        for (int i = 0; i < kScan / kPageThreads; ++i) v[i] = a.table[min(e0 + i * kPageThreads, (int64_t)n - 1)];
#pragma unroll
        for (int i = 0; i < kScan / kPageThreads; ++i) {
            if (v[i] < 0) continue;
            int at = place(v[i]);
            while (s_set[at] != -1 && s_set[at] != v[i]) at = (at + 1) & (size - 1);
            wrong |= s_set[at] == v[i];
        }
    }
    return wrong;
}

// A workgroup looks whether its fork can be made; those behind the forks' at the slots that they take.
__global__ __launch_bounds__(kPageThreads) void fork_check_kernel(ForkArgs a) {
    extern __shared__ int s_set[];
    __shared__ int s_wave[kPageThreads / kWave];
    const int i = blockIdx.x;
    if (i >= a.n) {
        const int bad = __syncthreads_or(taken_wrong(a, i - a.n, s_set, s_wave));
        if (threadIdx.x == 0) a.scan_err[i - a.n] = bad;
        return;
    }
    const int src = a.src[i], dst = a.dst[i], len = a.len[i];
    bool wrong = src < 0 || src >= a.B || dst < 0 || dst >= a.B || len < 0 ||
                 ((int64_t)len + a.bs - 1) / a.bs > a.mb;
    if (!wrong) {
        const int whole = len / a.bs, n = (len + a.bs - 1) / a.bs;
        const int32_t* from = a.table + (size_t)src * a.mb;
        const int32_t* to = a.table + (size_t)dst * a.mb;
        for (int j = threadIdx.x; j < a.mb; j += kPageThreads) {
            wrong |= to[j] != -1;
            if (j >= n) continue;
            const int s = from[j];
            if (s == -1) wrong |= j >= whole;  // a block without a slot stays so, but has none to copy
            else wrong |= s < 0 || s >= a.n_slots || (j < whole && a.shared[s] < 0);
        }
        // (no request gets two forks, and none is a fork's source and a fork of the same call)
        for (int k = threadIdx.x; k < a.n; k += kPageThreads) wrong |= a.dst[k] == src || (k < i && a.dst[k] == dst);
    }
    wrong = __syncthreads_or(wrong);
    if (threadIdx.x == 0) {
        a.err[i] = wrong;
        if (i == 0) *a.head0 = *a.free_head;
    }
}

// grid = (chunks of a block, n): chunk 0 also writes the fork's row.
__global__ __launch_bounds__(kPageThreads) void fork_kernel(ForkArgs a) {
    __shared__ int s_wave[kPageThreads / kWave];
    const int i = blockIdx.y;
    int before = 0, total = 0, errs = 0;
    for (int k = threadIdx.x; k < a.n; k += kPageThreads) {
        const int part = a.len[k] % a.bs != 0;
        total += part;
        if (k < i) before += part;
        errs |= a.err[k];
    }
    for (int k = threadIdx.x; k < a.scans; k += kPageThreads) errs |= a.scan_err[k];
    before = block_sum(before, s_wave, kPageThreads / kWave);
    total = block_sum(total, s_wave, kPageThreads / kWave);
    const int head = *a.head0;
    const bool range = head < 0 || head > a.n_free, full = !range && total > a.n_free - head;
    if (!range && !full)
        for (int k = threadIdx.x; k < total; k += kPageThreads) {
            const int s = a.free_slots[head + k];
            errs |= s < 0 || s >= a.n_slots;
        }
    errs = __syncthreads_or(errs) || range;
    if (errs || full) {
        if (blockIdx.x == 0 && i == 0 && threadIdx.x == 0)
            report(a.status, errs ? PULSE_ERR_BAD_INDEX : PULSE_ERR_POOL_EXHAUSTED);
        return;
    }
    const int src = a.src[i], dst = a.dst[i], len = a.len[i], whole = len / a.bs;
    const int32_t* from = a.table + (size_t)src * a.mb;
    const int take = a.len[i] % a.bs ? a.free_slots[head + before] : -1;
    if (blockIdx.x == 0) {
        int32_t* to = a.table + (size_t)dst * a.mb;
        for (int j = threadIdx.x; j < whole; j += kPageThreads) {
            const int s = from[j];
            to[j] = s;
            if (s >= 0) atomicAdd(a.shared + s, 1);
        }
        if (threadIdx.x == 0) {
            if (take >= 0) to[whole] = take;
            if (i == 0) *a.free_head = head + total;
        }
    }
    if (take < 0) return;
    copy_chunk_of(a.pool + (size_t)from[whole] * a.U, a.pool + (size_t)take * a.U, (int64_t)blockIdx.x * kChunk, a.U);
}

// ---- compact ----

struct CompactArgs {
    int32_t* table;
    int64_t entries;
    int32_t n_keep;
    int32_t* shared;
    int32_t* free_slots;
    int32_t* free_head;
    int32_t n_free;
    uint8_t* pool;
    int32_t n_slots;
    int64_t U;
    int32_t* status;
    uint32_t* live;    // a bit per slot that a table entry names
    uint32_t* listed;  // a bit per slot of the free list
    int32_t* high;     // live slots from n_keep on, ascending
    int32_t* place;    // [n_slots] of such a slot, its place among them
    int32_t* low;      // free slots below n_keep, in list order
    int32_t* plan;     // [0] moves, [1] low, [2] status, [3] head, [4] error of the marks
};

__device__ inline bool mark_entry(const CompactArgs& a, uint32_t* live, int64_t e) {
    const int s = a.table[e];
    if (s < 0 || s >= a.n_slots) return s != -1;
    const uint32_t bit = 1u << (s & 31);
    atomicOr(live + (s >> 5), bit);
    return false;
}
__device__ inline bool mark_listed(const CompactArgs& a, uint32_t* listed, int64_t i) {
    const int s = a.free_slots[i];
    if (s < 0 || s >= a.n_slots) return true;
    const uint32_t bit = 1u << (s & 31);
    return atomicOr(listed + (s >> 5), bit) & bit;
}

__global__ __launch_bounds__(kPageThreads) void compact_clear_kernel(CompactArgs a) {
    const int words = (a.n_slots + 31) / 32;
    for (int w = blockIdx.x * kPageThreads + threadIdx.x; w < words; w += gridDim.x * kPageThreads)
        a.live[w] = a.listed[w] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) a.plan[4] = 0;
}

__global__ __launch_bounds__(kPageThreads) void compact_mark_kernel(CompactArgs a) {
    const int64_t t = (int64_t)blockIdx.x * kPageThreads + threadIdx.x, stride = (int64_t)gridDim.x * kPageThreads;
    const int head = *a.free_head;
    bool wrong = head < 0 || head > a.n_free;
    for (int64_t e = t; e < a.entries; e += stride) wrong |= mark_entry(a, a.live, e);
    if (head >= 0)
        for (int64_t i = head + t; i < a.n_free; i += stride) wrong |= mark_listed(a, a.listed, i);
    if (wrong) atomicOr(a.plan + 4, 1);
}

// Items i of [0, n) whose value(i) satisfies keep, in order: emit(i, value, rank); their number.  A wave takes a stretch of
// the items, four times 64 at a time, whose values are loaded before any is looked at.
template <typename V, typename K, typename E>
__device__ inline int ranked(int n, int* s_wave, V value, K keep, E emit) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int each = ((n + 63) / 64 + 4 * kPlanWaves - 1) / (4 * kPlanWaves) * 256;
    const int first = min((int64_t)n, (int64_t)wave * each), end = min((int64_t)n, (int64_t)first + each);
    int mine = 0, at = 0, total = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int i0 = first; i0 < end; i0 += 256) {
            int v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = value(min(i0 + 64 * i + lane, end - 1));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int item = i0 + 64 * i + lane;
                const bool k = item < end && keep(item, v[i]);
                const uint64_t b = __ballot(k);
                if (pass == 0) {
                    mine += __popcll(b);
                } else {
                    if (k) emit(item, v[i], at + __popcll(b & ((1ull << lane) - 1)));
                    at += __popcll(b);
                }
            }
        }
        if (pass) break;
        __syncthreads();
        if (lane == 0) s_wave[wave] = mine;
        __syncthreads();
        for (int i = 0; i < kPlanWaves; ++i) {
            if (i < wave) at += s_wave[i];
            total += s_wave[i];
        }
    }
    return total;
}

__device__ inline void write_plan(const CompactArgs& a, bool wrong, int moves, int low, int head) {
    a.plan[0] = wrong ? 0 : moves;
    a.plan[1] = wrong ? 0 : low;
    a.plan[2] = wrong ? PULSE_ERR_BAD_INDEX : moves > low ? PULSE_ERR_POOL_EXHAUSTED : 0;
    a.plan[3] = wrong ? 0 : head;
}

// The moves from the marks: which slots, and where to.
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CompactArgs a) {
    __shared__ int s_wave[kPlanWaves];
    const int words = (a.n_slots + 31) / 32;
    const int head = *a.free_head;
    bool wrong = a.plan[4] != 0;
    for (int w = threadIdx.x; w < words; w += kPlanThreads) wrong |= (a.live[w] & a.listed[w]) != 0;
    if (__syncthreads_or(wrong)) {
        if (threadIdx.x == 0) write_plan(a, true, 0, 0, 0);
        return;
    }
    const int first = a.n_keep / 32 * 32;  // of the word with the first slot that is to be left
    const int moves = ranked(
        32 * words - first, s_wave, [&](int i) { return (int)a.live[(first + i) >> 5]; },
        [&](int i, int bits) { return first + i >= a.n_keep && (bits >> (i & 31) & 1); },
        [&](int i, int, int k) {
            a.high[k] = first + i;
            a.place[first + i] = k;
        });
    const int low = ranked(
        a.n_free - head, s_wave, [&](int i) { return a.free_slots[head + i]; },
        [&](int, int s) { return s < a.n_keep; }, [&](int, int s, int k) { a.low[k] = s; });
    if (threadIdx.x == 0) write_plan(a, false, moves, low, head);
}

// Marks and moves in one workgroup: table and list are loaded at once and stay in registers, the marks are bits in LDS.
__global__ __launch_bounds__(kPlanThreads) void compact_small_kernel(CompactArgs a) {
    constexpr int N = kOneGroup / kPlanThreads;
    extern __shared__ uint32_t s_bits[];
    __shared__ int s_wave[2][kPlanWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int words = (a.n_slots + 31) / 32;
    uint32_t* live = s_bits;
    uint32_t* listed = s_bits + words;
    const int head = *a.free_head;
    int entry[N], slot[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * kPlanThreads + threadIdx.x, f = (wave * N + i) * 64 + lane;  // (a wave's list entries in a row)
        entry[i] = e < (int)a.entries ? a.table[e] : -1;
        slot[i] = f < a.n_free ? a.free_slots[f] : 0;
    }
    for (int w = threadIdx.x; w < 2 * words; w += kPlanThreads) s_bits[w] = 0;
    __syncthreads();
    bool wrong = head < 0 || head > a.n_free;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int f = (wave * N + i) * 64 + lane;
        if (entry[i] != -1) {
            if (entry[i] < 0 || entry[i] >= a.n_slots) wrong = true;
            else atomicOr(live + (entry[i] >> 5), 1u << (entry[i] & 31));
        }
        if (f < head || f >= a.n_free) {
            slot[i] = INT32_MAX;  // not in the list
        } else if (slot[i] < 0 || slot[i] >= a.n_slots) {
            wrong = true;
        } else {
            const uint32_t bit = 1u << (slot[i] & 31);
            wrong |= (atomicOr(listed + (slot[i] >> 5), bit) & bit) != 0;
        }
    }
    __syncthreads();
    // live slots from n_keep on, a stretch of words a thread; free ones below it, a stretch of the list a wave
    const int each = (words + kPlanThreads - 1) / kPlanThreads;
    const int w0 = min(words, (int)threadIdx.x * each), w1 = min(words, w0 + each);
    int high = 0;
    auto bits_of = [&](int w) {
        const uint32_t b = live[w];
        return 32 * w >= a.n_keep ? b : 32 * w + 32 <= a.n_keep ? 0u : b & ~0u << (a.n_keep & 31);
    };
    for (int w = w0; w < w1; ++w) {
        wrong |= (live[w] & listed[w]) != 0;
        high += __popc(bits_of(w));
    }
    uint64_t below[N];
    int low = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        below[i] = __ballot(slot[i] < a.n_keep);
        low += __popcll(below[i]);
    }
    const int upto = (int)wave_scan((uint32_t)high, 0u, OpAdd());
    if (lane == 63) s_wave[0][wave] = upto;
    if (lane == 0) s_wave[1][wave] = low;
    wrong = __syncthreads_or(wrong);
    int h0 = upto - high, l0 = 0, moves = 0, lows = 0;
    for (int i = 0; i < kPlanWaves; ++i) {
        if (i < wave) {
            h0 += s_wave[0][i];
            l0 += s_wave[1][i];
        }
        moves += s_wave[0][i];
        lows += s_wave[1][i];
    }
    if (threadIdx.x == 0) write_plan(a, wrong, moves, lows, head);
    if (wrong) return;
    for (int w = w0; w < w1; ++w)
        for (uint32_t b = bits_of(w); b; b &= b - 1) {
            const int x = 32 * w + __builtin_ctz(b);
            a.high[h0] = x;
            a.place[x] = h0++;
        }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (slot[i] < a.n_keep) a.low[l0 + __popcll(below[i] & ((1ull << lane) - 1))] = slot[i];
        l0 += __popcll(below[i]);
    }
}

__global__ __launch_bounds__(kPageThreads) void compact_kernel(CompactArgs a) {
    const int moves = a.plan[0], low = a.plan[1], status = a.plan[2];
    if (status) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, status);
        return;
    }
    const int64_t t = (int64_t)blockIdx.x * kPageThreads + threadIdx.x, stride = (int64_t)gridDim.x * kPageThreads;
    for (int64_t e = t; e < a.entries; e += stride) {
        const int s = a.table[e];
        if (s >= a.n_keep) a.table[e] = a.low[a.place[s]];
    }
    for (int64_t k = t; k < low; k += stride) {
        const int s = a.low[k];
        if (k >= moves) {
            a.free_slots[a.n_free - low + k] = s;
        } else if (a.shared) {
            const int h = a.high[k];
            a.shared[s] = a.shared[h];
            a.shared[h] = 0;
        }
    }
    if (t == 0) *a.free_head = a.n_free - (low - moves);
    const int chunks = (int)((a.U + kChunk - 1) / kChunk);
    for (int64_t c = blockIdx.x; c < (int64_t)moves * chunks; c += gridDim.x) {
        const int k = (int)(c / chunks);
        copy_chunk_of(a.pool + (size_t)a.high[k] * a.U, a.pool + (size_t)a.low[k] * a.U, c % chunks * kChunk, a.U);
    }
}

// ---- launches ----

static size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
static int64_t table_tiles(int32_t B, int32_t max_blocks) { return ((int64_t)B * max_blocks + kTile - 1) / kTile; }

// Arrays of n_slots words (four), of a word per tile (two) and per request, and a few words.
size_t pages_ws_bytes(int32_t B, int32_t max_blocks, int32_t n_slots) {
    return 4 * up(sizeof(int32_t) * ((size_t)n_slots + 32)) + 2 * up(sizeof(int32_t) * table_tiles(B, max_blocks)) +
           up(sizeof(int32_t) * B) + 256;
}

struct PagesWs {
    int32_t *slots[4], *tiles[2], *requests, *few;
    PagesWs(void* ws, int32_t B, int32_t max_blocks, int32_t n_slots) {
        size_t o = 0;
        for (auto& p : slots) {
            p = ws_at<int32_t>(ws, o);
            o += up(sizeof(int32_t) * ((size_t)n_slots + 32));
        }
        for (auto& p : tiles) {
            p = ws_at<int32_t>(ws, o);
            o += up(sizeof(int32_t) * table_tiles(B, max_blocks));
        }
        requests = ws_at<int32_t>(ws, o);
        o += up(sizeof(int32_t) * B);
        few = ws_at<int32_t>(ws, o);
    }
};

hipError_t launch_free_blocks(const int32_t* keep, int32_t B, int32_t bs, int32_t* table, int32_t max_blocks, int32_t* shared,
                              int32_t* free_slots, int32_t* free_head, int32_t n_free, int32_t n_slots, int32_t* status,
                              void* ws, hipStream_t st) {
    const PagesWs w(ws, B, max_blocks, n_slots);
    const int64_t tiles = table_tiles(B, max_blocks);
    FreeArgs a{keep, B, bs, table, max_blocks, shared, free_slots, free_head, n_free, n_slots, status, w.slots[0], w.slots[1],
               w.tiles[0], w.tiles[1], w.few, (int32_t)tiles};
    const int64_t entries = (int64_t)B * max_blocks;
    if (entries <= kOneFree) {
        if (entries <= 2 * kPlanThreads) hipLaunchKernelGGL(free_small_kernel<2>, dim3(1), dim3(kPlanThreads), 0, st, a);
        else hipLaunchKernelGGL(free_small_kernel<kOneFree / kPlanThreads>, dim3(1), dim3(kPlanThreads), 0, st, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)tiles);
    hipLaunchKernelGGL(free_kernel<0>, grid, dim3(kPageThreads), 0, st, a);
    hipLaunchKernelGGL(free_kernel<1>, grid, dim3(kPageThreads), 0, st, a);
    hipLaunchKernelGGL(free_kernel<2>, grid, dim3(kPageThreads), 0, st, a);
    hipLaunchKernelGGL(free_kernel<3>, grid, dim3(kPageThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_fork_blocks(const int32_t* src, const int32_t* dst, const int32_t* len, int32_t n, int32_t bs,
                              int32_t* table, int32_t B, int32_t max_blocks, int32_t* shared, const int32_t* free_slots,
                              int32_t* free_head, int32_t n_free, void* pool, int32_t n_slots, size_t unit_bytes,
                              int32_t* status, void* ws, hipStream_t st) {
    const PagesWs w(ws, B, max_blocks, n_slots);
    const int32_t scans = (int32_t)std::min<int64_t>(kScanGroups, ((int64_t)B * max_blocks + kScan - 1) / kScan);
    const ForkArgs a{src, dst, len, n, bs, table, B, max_blocks, shared, free_slots, free_head, n_free, (uint8_t*)pool,
                     n_slots, (int64_t)unit_bytes, status, w.requests, w.tiles[0], scans, w.few};
    hipLaunchKernelGGL(fork_check_kernel, dim3((unsigned)(n + scans)), dim3(kPageThreads), sizeof(int) * slot_places(n), st, a);
    const dim3 grid((unsigned)((unit_bytes + kChunk - 1) / kChunk), (unsigned)n);
    hipLaunchKernelGGL(fork_kernel, grid, dim3(kPageThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_compact_blocks(int32_t* table, int32_t B, int32_t max_blocks, int32_t n_keep, int32_t* shared,
                                 int32_t* free_slots, int32_t* free_head, int32_t n_free, void* pool, int32_t n_slots,
                                 size_t unit_bytes, int32_t* status, void* ws, hipStream_t st) {
    const PagesWs w(ws, B, max_blocks, n_slots);
    const int64_t entries = (int64_t)B * max_blocks;
    const int words = (n_slots + 31) / 32;
    CompactArgs a{table, entries, n_keep, shared, free_slots, free_head, n_free, (uint8_t*)pool, n_slots, (int64_t)unit_bytes,
                  status, (uint32_t*)w.slots[0], (uint32_t*)w.slots[0] + words + 1, w.slots[1], w.slots[2], w.slots[3], w.few};
    if (entries <= kOneGroup && n_free <= kOneGroup && 8 * (size_t)words <= 49152) {
        hipLaunchKernelGGL(compact_small_kernel, dim3(1), dim3(kPlanThreads), 8 * (size_t)words, st, a);
    } else {
        const int64_t most = entries > n_free ? entries : n_free;
        const unsigned groups = (unsigned)std::min<int64_t>(kCopyGroups, (most + kPageThreads - 1) / kPageThreads + 1);
        hipLaunchKernelGGL(compact_clear_kernel, dim3(groups), dim3(kPageThreads), 0, st, a);
        hipLaunchKernelGGL(compact_mark_kernel, dim3(groups), dim3(kPageThreads), 0, st, a);
        hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
    }
    hipLaunchKernelGGL(compact_kernel, dim3(kCopyGroups), dim3(kPageThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace pulse

// tables.hip -- block offsets, block tables and slot maps of a step, built on the GPU from request lengths
// (the block table and free list that the recall keeps, Sec. 2.2).
//
// Request r holds ctx[r] tokens, the last new[r] of them new; its new tokens lie in the blocks ("cells")
// (ctx - new) / bs .. ceil(ctx / bs) - 1.  Cells of all requests are numbered in order; those without a slot
// take the free list front to back, so a cell's slot is free_slots[head + cells without a slot before it].
//
// Bound: two memory round trips (lengths, table entries) and the launches; beyond some ten thousand tokens the
// 12 bytes written per token.  Nothing may be written before every length, entry and slot has been checked.
// Small steps run in one workgroup, which counts, checks and writes.  Larger ones take two launches over tiles
// of cells: the first counts and checks each tile, the second adds the tiles' counts up (each workgroup for
// itself) and writes.
#include "pulse_internal.h"

namespace pulse {

constexpr int kTabThreads = 1024;
constexpr int kTabWaves = kTabThreads / kWave;
constexpr int kTabPer = kMaxBatch / kTabThreads;  // requests of a thread
constexpr int kTileCells = 2048;                  // cells of a workgroup of the larger form
constexpr int kTilePer = kTileCells / kTabThreads;
constexpr int64_t kOneGroupCells = 4096;          // bound on the cells up to which one workgroup does it all

struct TabArgs {
    const int32_t *ctx, *fresh;
    int32_t B, bs;
    int32_t* table;
    int32_t max_blocks;
    const int32_t* free_slots;
    int32_t* free_head;
    int32_t n_free, n_slots;
    int64_t* blk_off;
    int32_t* tok_off;
    int64_t* slot_map;
    int32_t* positions;
    int64_t max_tokens;
    int32_t* status;
};

// Scratch of the larger form: the free-list head, then per tile its cells without a slot (-1: a bad entry among
// them) and the first free-list place, counted from the head, in the tile's range of places that names no slot.
struct TabScratch {
    int32_t* head;
    int32_t *count, *bad_place;
};

struct TabShared {
    int32_t first[kMaxBatch];     // position of the first new token
    int32_t tok[kMaxBatch + 1];   // new tokens before request r
    int32_t cell[kMaxBatch + 1];  // cells before request r
    uint64_t wave[3][kTabWaves];
    uint32_t misses[kTabWaves];
};

// Exclusive sum of x over the lanes of a wave and its total.  x < 2^46.
__device__ inline uint64_t wave_sum_before(uint64_t x, uint64_t& total) {
    const uint32_t lo = (uint32_t)(x & 0xFFFFF), hi = (uint32_t)(x >> 20);  // 64 times either fits 32 bits
    const uint32_t slo = wave_scan(lo, 0u, OpAdd()), shi = wave_scan(hi, 0u, OpAdd());
    total = ((uint64_t)last_lane(shi) << 20) + last_lane(slo);
    return ((uint64_t)(shi - hi) << 20) + (slo - lo);
}

// Checks the lengths and fills the shared sums; false (in every thread) if a length is out of range.  With `write`
// the block and token offsets go to memory, all zero where the lengths are bad.  tokens / cells: totals.
__device__ inline bool scan_requests(const TabArgs& a, TabShared& s, int64_t& tokens, int64_t& cells, int64_t* off) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t nb[kTabPer], nt[kTabPer], nc[kTabPer], sum[3] = {0, 0, 0};
    int bad = 0;
#pragma unroll
    for (int i = 0; i < kTabPer; ++i) {
        const int r = tid * kTabPer + i;
        nb[i] = nt[i] = nc[i] = 0;
        if (r < a.B) {
            const int32_t ctx = a.ctx[r], n = a.fresh[r];
            const int64_t blocks = ((int64_t)ctx + a.bs - 1) / a.bs;
            if (ctx < 0 || n < 0 || n > ctx || blocks > a.max_blocks) {
                bad = 1;
            } else {
                nb[i] = (uint64_t)blocks;
                nt[i] = (uint64_t)n;
                nc[i] = n > 0 ? (uint64_t)(blocks - (ctx - n) / a.bs) : 0;
                s.first[r] = ctx - n;
            }
        }
        sum[0] += nb[i];
        sum[1] += nt[i];
        sum[2] += nc[i];
    }
    uint64_t before[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        uint64_t all;
        before[k] = wave_sum_before(sum[k], all);
        if (lane == 0) s.wave[k][wave] = all;
    }
    bad = __syncthreads_or(bad);
    uint64_t total[3] = {0, 0, 0};
#pragma unroll
    for (int k = 0; k < 3; ++k)
        for (int w = 0; w < kTabWaves; ++w) {
            if (w == wave) before[k] += total[k];
            total[k] += s.wave[k][w];
        }
    if ((int64_t)total[1] > a.max_tokens) bad = 1;  // the same in every thread
    tokens = (int64_t)total[1];
    cells = (int64_t)total[2];
    if (!bad) {
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int r = tid * kTabPer + i;
            if (off) off[i] = (int64_t)before[0];
            if (r < a.B) {
                s.tok[r] = (int32_t)before[1];
                s.cell[r] = (int32_t)before[2];
            }
            before[0] += nb[i];
            before[1] += nt[i];
            before[2] += nc[i];
        }
        if (tid == 0) {
            s.tok[a.B] = (int32_t)tokens;
            s.cell[a.B] = (int32_t)cells;
        }
    }
    if (off) off[kTabPer] = (int64_t)total[0];
    __syncthreads();
    return !bad;
}

// Writes the block and token offsets (all zero unless ok).
__device__ inline void write_offsets(const TabArgs& a, const TabShared& s, const int64_t* off, bool ok) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kTabPer; ++i) {
        const int r = tid * kTabPer + i;
        if (r < a.B) {
            a.blk_off[r] = ok ? off[i] : 0;
            a.tok_off[r] = ok ? s.tok[r] : 0;
        }
    }
    if (tid == 0) {
        a.blk_off[a.B] = ok ? off[kTabPer] : 0;
        a.tok_off[a.B] = ok ? s.tok[a.B] : 0;
    }
}

// The request whose range of the sums `at` holds i (0 <= i < at[B]); most decode steps have one token and one
// cell per request, so request i is looked at first.
__device__ inline int request_of(const int32_t* at, int B, int32_t i) {
    if (i < B && at[i] == i && at[i + 1] == i + 1) return i;
    int lo = 0, hi = B;  // the last r with at[r] <= i
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Cell c: its request, block and table entry; bad: the entry is none, or a block whose first tokens are in no slot.
struct Cell {
    int r;
    int32_t j, entry;
    bool bad;
};
__device__ inline Cell load_cell(const TabArgs& a, const TabShared& s, int32_t c) {
    Cell x;
    x.r = request_of(s.cell, a.B, c);
    const int32_t j0 = s.first[x.r] / a.bs;
    x.j = j0 + (c - s.cell[x.r]);
    x.entry = a.table[(size_t)x.r * a.max_blocks + x.j];
    x.bad = x.entry < -1 || x.entry >= a.n_slots || (x.entry < 0 && x.j == j0 && s.first[x.r] % a.bs != 0);
    return x;
}

__device__ inline void fill_token(const TabArgs& a, int64_t i, int32_t slot, int32_t p) {
    a.slot_map[i] = (int64_t)slot * a.bs + p % a.bs;
    a.positions[i] = p;
}

__device__ inline void fill_rest(const TabArgs& a, int64_t from, int64_t at, int64_t stride) {
    for (int64_t i = from + at; i < a.max_tokens; i += stride) {
        a.slot_map[i] = -1;
        a.positions[i] = -1;
    }
}

// Rank of this thread's cell among the workgroup's cells without a slot, and their number.
__device__ inline uint32_t rank_misses(TabShared& s, bool miss, uint32_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t m = __ballot(miss);
    if (lane == 0) s.misses[wave] = (uint32_t)__popcll(m);
    __syncthreads();
    uint32_t before = (uint32_t)__popcll(m & ((1ull << lane) - 1));
    all = 0;
    for (int w = 0; w < kTabWaves; ++w) {
        if (w == wave) before += all;
        all += s.misses[w];
    }
    __syncthreads();
    return before;
}

__global__ __launch_bounds__(kTabThreads) void tables_small_kernel(TabArgs a) {
    __shared__ TabShared s;
    const int tid = threadIdx.x;
    const int32_t head = *a.free_head;
    int64_t tokens, cells, off[kTabPer + 1];
    bool ok = scan_requests(a, s, tokens, cells, off);
    int32_t code = ok ? PULSE_OK : PULSE_ERR_BAD_INDEX;
    if (ok) {
        int64_t total = 0;
        int bad = 0;
        for (int64_t c0 = 0; c0 < cells; c0 += kTabThreads) {
            bool miss = false;
            if (c0 + tid < cells) {
                const Cell x = load_cell(a, s, (int32_t)(c0 + tid));
                bad |= x.bad;
                miss = x.entry < 0;
            }
            total += __syncthreads_count(miss);
        }
        const bool head_ok = head >= 0 && head <= a.n_free;
        const bool fits = head_ok && total <= (int64_t)a.n_free - head;
        if (fits)
            for (int64_t g = tid; g < total; g += kTabThreads)
                bad |= (uint32_t)a.free_slots[head + g] >= (uint32_t)a.n_slots;
        bad = __syncthreads_or(bad);
        if (bad || !head_ok) code = PULSE_ERR_BAD_INDEX;
        else if (!fits) code = PULSE_ERR_POOL_EXHAUSTED;
        ok = code == PULSE_OK;
        if (ok) {
            int32_t g0 = head;
            for (int64_t c0 = 0; c0 < cells; c0 += kTabThreads) {
                Cell x;
                x.entry = 0;
                if (c0 + tid < cells) x = load_cell(a, s, (int32_t)(c0 + tid));
                uint32_t all;
                const uint32_t rank = rank_misses(s, x.entry < 0, all);
                if (x.entry < 0) a.table[(size_t)x.r * a.max_blocks + x.j] = a.free_slots[g0 + (int32_t)rank];
                g0 += (int32_t)all;
            }
            if (tid == 0) *a.free_head = g0;
        }
    }
    if (tid == 0 && code != PULSE_OK) report(a.status, code);
    write_offsets(a, s, off, ok);
    if (!ok) tokens = 0;
    __syncthreads();  // the table entries above
    for (int64_t i = tid; i < tokens; i += kTabThreads) {
        const int r = request_of(s.tok, a.B, (int32_t)i);
        const int32_t p = s.first[r] + (int32_t)(i - s.tok[r]);
        fill_token(a, i, a.table[(size_t)r * a.max_blocks + p / a.bs], p);
    }
    fill_rest(a, tokens, tid, kTabThreads);
}

__global__ __launch_bounds__(kTabThreads) void tables_count_kernel(TabArgs a, TabScratch w) {
    __shared__ TabShared s;
    const int tid = threadIdx.x, tile = blockIdx.x;
    const int32_t head = *a.free_head;
    int64_t tokens, cells;
    const bool ok = scan_requests(a, s, tokens, cells, nullptr);
    if (tile == 0 && tid == 0) *w.head = head;
    int n = 0, bad = 0;
    int32_t place = INT32_MAX;
    if (ok) {
#pragma unroll
        for (int k = 0; k < kTilePer; ++k) {
            const int64_t c = (int64_t)tile * kTileCells + k * kTabThreads + tid;
            bool miss = false;
            if (c < cells) {
                const Cell x = load_cell(a, s, (int32_t)c);
                bad |= x.bad;
                miss = x.entry < 0;
                if (head >= 0 && c < (int64_t)a.n_free - head &&
                    (uint32_t)a.free_slots[head + c] >= (uint32_t)a.n_slots && place == INT32_MAX)
                    place = (int32_t)c;
            }
            n += __syncthreads_count(miss);
        }
    }
    bad = __syncthreads_or(bad);
    // the least place over the workgroup
    const uint32_t m = last_lane(wave_scan((uint32_t)place, 0xFFFFFFFFu, OpMin()));
    if ((tid & 63) == 0) s.misses[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) {
        uint32_t least = s.misses[0];
        for (int i = 1; i < kTabWaves; ++i) least = min(least, s.misses[i]);
        w.count[tile] = bad ? -1 : n;
        w.bad_place[tile] = (int32_t)least;
    }
}

__global__ __launch_bounds__(kTabThreads) void tables_fill_kernel(TabArgs a, TabScratch w) {
    __shared__ TabShared s;
    __shared__ int32_t slot[kTileCells];
    __shared__ int32_t s_before, s_total, s_place, s_bad;
    const int tid = threadIdx.x, tile = blockIdx.x, tiles = gridDim.x;
    const int32_t head = *w.head;
    if (tid == 0) {
        s_before = s_total = s_bad = 0;
        s_place = INT32_MAX;
    }
    int64_t tokens, cells, off[kTabPer + 1];
    bool ok = scan_requests(a, s, tokens, cells, off);
    int32_t before = 0, total = 0, place = INT32_MAX, bad = 0;
    for (int t = tid; t < tiles; t += kTabThreads) {
        const int32_t n = w.count[t];
        bad |= n < 0;
        total += n;
        before += t < tile ? n : 0;
        place = min(place, w.bad_place[t]);
    }
    if (total) atomicAdd(&s_total, total);
    if (before) atomicAdd(&s_before, before);
    if (place != INT32_MAX) atomicMin(&s_place, place);
    if (bad) atomicOr(&s_bad, 1);
    __syncthreads();
    before = s_before;
    total = s_total;
    int32_t code = PULSE_OK;
    if (!ok || s_bad || head < 0 || head > a.n_free) code = PULSE_ERR_BAD_INDEX;
    else if (total > a.n_free - head) code = PULSE_ERR_POOL_EXHAUSTED;
    else if (s_place < total) code = PULSE_ERR_BAD_INDEX;
    ok = code == PULSE_OK;
    if (tile == 0) {
        write_offsets(a, s, off, ok);
        if (tid == 0) {
            if (ok) *a.free_head = head + total;
            else report(a.status, code);
        }
    }
    const int64_t at = (int64_t)tile * kTabThreads + tid, stride = (int64_t)tiles * kTabThreads;
    fill_rest(a, ok ? tokens : 0, at, stride);
    if (!ok) return;
    int32_t g0 = head + before;
    const int64_t c0 = (int64_t)tile * kTileCells;
    const int n = (int)max((int64_t)0, min((int64_t)kTileCells, cells - c0));
#pragma unroll
    for (int k = 0; k < kTilePer; ++k) {
        const int c = k * kTabThreads + tid;
        Cell x;
        x.entry = 0;
        if (c < n) x = load_cell(a, s, (int32_t)(c0 + c));
        uint32_t all;
        const uint32_t rank = rank_misses(s, x.entry < 0, all);
        if (x.entry < 0) {
            x.entry = a.free_slots[g0 + (int32_t)rank];
            a.table[(size_t)x.r * a.max_blocks + x.j] = x.entry;
        }
        if (c < n) slot[c] = x.entry;
        g0 += (int32_t)all;
    }
    __syncthreads();
    // the tile's tokens, neighbouring threads on neighbouring tokens
    for (int i = tid; i < n * a.bs; i += kTabThreads) {
        const int c = i / a.bs;
        const int r = request_of(s.cell, a.B, (int32_t)(c0 + c));
        const int32_t first = s.first[r];
        const int64_t p = ((int64_t)first / a.bs + (c0 + c - s.cell[r])) * a.bs + i % a.bs;
        const int32_t k = s.tok[r + 1] - s.tok[r];
        if (p >= first && p < (int64_t)first + k) fill_token(a, s.tok[r] + (p - first), slot[c], (int32_t)p);
    }
}

// Bound on the cells of a step: a request's new tokens lie in at most two blocks more than they fill.
static int64_t cell_bound(int32_t B, int32_t bs, int64_t max_tokens) { return max_tokens / bs + 2 * (int64_t)B; }
static int64_t tile_count(int32_t B, int32_t bs, int64_t max_tokens) {
    return (cell_bound(B, bs, max_tokens) + kTileCells - 1) / kTileCells;
}

size_t tables_ws_bytes(int32_t B, int32_t bs, int64_t max_tokens) {
    return (sizeof(int32_t) * (size_t)(1 + 2 * tile_count(B, bs, max_tokens)) + 255) & ~(size_t)255;
}

hipError_t launch_tables(const int32_t* ctx, const int32_t* fresh, int32_t B, int32_t bs, int32_t* table,
                         int32_t max_blocks, const int32_t* free_slots, int32_t* free_head, int32_t n_free,
                         int32_t n_slots, int64_t* blk_off, int32_t* tok_off, int64_t* slot_map, int32_t* positions,
                         int64_t max_tokens, int32_t* status, void* ws, hipStream_t st) {
    const TabArgs a{ctx,     fresh,   B,       bs,       table,     max_blocks, free_slots, free_head,
                    n_free,  n_slots, blk_off, tok_off,  slot_map,  positions,  max_tokens, status};
    if (cell_bound(B, bs, max_tokens) <= kOneGroupCells) {
        hipLaunchKernelGGL(tables_small_kernel, dim3(1), dim3(kTabThreads), 0, st, a);
        return hipGetLastError();
    }
    const int64_t tiles = tile_count(B, bs, max_tokens);
    int32_t* w = static_cast<int32_t*>(ws);
    const TabScratch sc{w, w + 1, w + 1 + tiles};
    hipLaunchKernelGGL(tables_count_kernel, dim3((unsigned)tiles), dim3(kTabThreads), 0, st, a, sc);
    hipLaunchKernelGGL(tables_fill_kernel, dim3((unsigned)tiles), dim3(kTabThreads), 0, st, a, sc);
    return hipGetLastError();
}

}  // namespace pulse

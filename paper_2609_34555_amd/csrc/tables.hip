// tables.hip -- block offsets, block tables and slot maps of a step, built on the GPU from request lengths
// (the block table and free list that the recall keeps, Sec. 2.2).
//
// Request r holds ctx[r] tokens, the last new[r] of them new; its new tokens lie in the blocks ("cells")
// (ctx - new) / bs .. ceil(ctx / bs) - 1.  Cells of all requests are numbered in order; those without a slot
// take the free list front to back, so a cell's slot is free_slots[head + cells without a slot before it].
//
// Bound: memory round trips (lengths; then table entries and free slots, which do not wait for one another; then the
// writes) and launches; beyond some ten thousand tokens the 12 bytes written per token.  Nothing may be written before
// every length, entry and slot has been checked.  Small steps run in one workgroup, whose threads keep their cells in
// registers; larger ones take two launches over tiles of cells: the first counts and checks each tile, the second adds
// the tiles' counts up (each workgroup for itself) and writes.
#include "pulse_internal.h"

namespace pulse {

constexpr int kCellsPer = 4;  // cells of a thread of the one-workgroup forms
// Room for tokens up to which one workgroup of 256 threads, and one of 1024, is fastest: in us, 256 threads, 1024
// and two launches: 32 requests of one token 5.0, 6.8, 7.1; one request of 1000 tokens 5.2, 6.9, 7.3; of 8000 9.2, 8.0,
// 9.3; of 15000 13.5, 9.1, 9.5; of 30000 -, 12.0, 9.8; 4 of 15000 -, 18.1, 10.2.
constexpr int64_t kOneTokens = 4096, kOneWideTokens = 16384;
// Threads of a tile's workgroup, which takes that many cells of 16 tokens.  In us (with two small launches beside), 256,
// 512 and 1024: 590K tokens 22.1, 22.2, 25.0; 3.2M tokens 39.0, 28.8, 30.5 (a workgroup's look-ups before its first token
// weigh less).
constexpr int kTileThreads = 512;
constexpr int64_t kMaxTiles = 1024;  // every workgroup of the larger form reads every tile's count

struct TabArgs {
    const int32_t *ctx, *fresh;
    int32_t B, shift;  // blocks of 1 << shift tokens
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
    int32_t tile;  // cells of a tile
};

// Sums over the requests, for up to B of them.
template <int B>
struct TabRequests {
    int32_t first[B];     // position of the first new token
    int32_t tok[B + 1];   // new tokens before request r
    int32_t cell[B + 1];  // cells before request r
    uint64_t wave[3][16];
};

// Exclusive sum of x over the lanes of a wave and its total.  x < 2^46.
__device__ inline uint64_t wave_sum_before(uint64_t x, uint64_t& total) {
    const uint32_t lo = (uint32_t)(x & 0xFFFFF), hi = (uint32_t)(x >> 20);  // 64 times either fits 32 bits
    const uint32_t slo = wave_scan(lo, 0u, OpAdd()), shi = wave_scan(hi, 0u, OpAdd());
    total = ((uint64_t)last_lane(shi) << 20) + last_lane(slo);
    return ((uint64_t)(shi - hi) << 20) + (slo - lo);
}

// Checks the lengths and fills the sums; false (in every thread) if a length is out of range.  A thread takes a
// contiguous part of the requests.  off0: blocks before its first one; tokens / cells / blocks: totals.
struct TabTotals {
    int64_t blocks, tokens, cells;
};
template <int T, int B>
__device__ inline bool scan_requests(const TabArgs& a, TabRequests<B>& s, TabTotals& all, int64_t& off0) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = B <= T ? 1 : (a.B + T - 1) / T, r0 = tid * per, r1 = min(a.B, r0 + per);
    uint64_t sum[3] = {0, 0, 0}, before[3];
    int bad = 0;
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        const int32_t ctx = a.ctx[r], n = a.fresh[r];
        const int64_t blocks = ((int64_t)ctx + (1 << a.shift) - 1) >> a.shift;
        const bool no = ctx < 0 || n < 0 || n > ctx || blocks > a.max_blocks;
        const int32_t cells = no || n == 0 ? 0 : (int32_t)(blocks - ((ctx - n) >> a.shift));
        bad |= no;
        s.first[r] = ctx - n;
        s.tok[r] = no ? 0 : n;
        s.cell[r] = cells;
        sum[0] += no ? 0 : (uint64_t)blocks;
        sum[1] += no ? 0 : (uint64_t)n;
        sum[2] += (uint64_t)cells;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        uint64_t w;
        before[k] = wave_sum_before(sum[k], w);
        if (lane == 0) s.wave[k][wave] = w;
    }
    bad = __syncthreads_or(bad);
    uint64_t total[3] = {0, 0, 0};
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int w = 0; w < T / kWave; ++w) {
            if (w == wave) before[k] += total[k];
            total[k] += s.wave[k][w];
        }
    all.blocks = (int64_t)total[0];
    all.tokens = (int64_t)total[1];
    all.cells = (int64_t)total[2];
    off0 = (int64_t)before[0];
    if (all.tokens > a.max_tokens) bad = 1;  // the same in every thread
    if (!bad) {  // counts to sums
        for (int r = r0; r < r1; ++r) {
            const int32_t n = s.tok[r], c = s.cell[r];
            s.tok[r] = (int32_t)before[1];
            s.cell[r] = (int32_t)before[2];
            before[1] += (uint64_t)n;
            before[2] += (uint64_t)c;
        }
        if (tid == 0) {
            s.tok[a.B] = (int32_t)all.tokens;
            s.cell[a.B] = (int32_t)all.cells;
        }
    }
    __syncthreads();
    return !bad;
}

// Writes the block and token offsets (all zero unless ok).
template <int T, int B>
__device__ inline void write_offsets(const TabArgs& a, const TabRequests<B>& s, const TabTotals& all, int64_t off0,
                                     bool ok) {
    const int tid = threadIdx.x;
    const int per = B <= T ? 1 : (a.B + T - 1) / T, r0 = tid * per, r1 = min(a.B, r0 + per);
    for (int r = r0; r < r1; ++r) {
        a.blk_off[r] = ok ? off0 : 0;
        a.tok_off[r] = ok ? s.tok[r] : 0;
        if (ok) off0 += ((int64_t)s.first[r] + (s.tok[r + 1] - s.tok[r]) + (1 << a.shift) - 1) >> a.shift;
    }
    if (tid == 0) {
        a.blk_off[a.B] = ok ? all.blocks : 0;
        a.tok_off[a.B] = ok ? (int32_t)all.tokens : 0;
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

// Cell c: its place in the table and its entry there; bad: the entry is none, or a block whose first tokens are in
// no slot.  Its tokens: the t-th of the block is new token g + t for t in lo .. hi - 1.
struct Cell {
    size_t at;
    int32_t entry, g, p;
    int16_t lo, hi;
    bool bad;
};
template <int B>
__device__ inline Cell load_cell(const TabArgs& a, const TabRequests<B>& s, int32_t c) {
    Cell x;
    const int r = request_of(s.cell, a.B, c);
    const int32_t first = s.first[r], n = s.tok[r + 1] - s.tok[r], mask = (1 << a.shift) - 1;
    const int32_t j = (first >> a.shift) + (c - s.cell[r]);
    x.at = (size_t)r * a.max_blocks + j;
    x.entry = a.table[x.at];
    x.p = j << a.shift;  // below the context length, which fits
    x.g = s.tok[r] + (x.p - first);
    x.lo = (int16_t)max(0, first - x.p);
    x.hi = (int16_t)min((int64_t)mask + 1, (int64_t)first + n - x.p);
    x.bad = x.entry < -1 || x.entry >= a.n_slots || (x.entry < 0 && x.lo > 0);
    return x;
}

__device__ inline void fill_rest(const TabArgs& a, int64_t from, int64_t at, int64_t stride) {
    for (int64_t i = from + at; i < a.max_tokens; i += stride) {
        a.slot_map[i] = -1;
        a.positions[i] = -1;
    }
}

// What the tokens of a cell need, in LDS.
template <int N>
struct CellTokens {
    int32_t slot[N], g[N], p[N];
    int32_t range[N];  // lo | hi << 16
};
template <int N>
__device__ inline void keep_cell(CellTokens<N>& s, int i, const Cell& x, int32_t slot) {
    s.slot[i] = slot;
    s.g[i] = x.g;
    s.p[i] = x.p;
    s.range[i] = (int32_t)x.lo | (int32_t)x.hi << 16;
}
// Maps of the tokens of n cells, neighbouring threads on neighbouring tokens.
template <int T, int N>
__device__ inline void fill_tokens(const TabArgs& a, const CellTokens<N>& s, int n) {
#pragma unroll 4
    for (int i = threadIdx.x; i < n << a.shift; i += T) {
        const int c = i >> a.shift, t = i & ((1 << a.shift) - 1);
        const int32_t range = s.range[c];
        if (t < (range & 0xFFFF) || t >= range >> 16) continue;
        a.slot_map[s.g[c] + t] = ((int64_t)s.slot[c] << a.shift) + t;
        a.positions[s.g[c] + t] = s.p[c] + t;
    }
}

// One workgroup of T threads: up to T * kCellsPer cells, B requests.
template <int T, int B>
__global__ __launch_bounds__(T) void tables_one_kernel(TabArgs a) {
    constexpr int kWaves = T / kWave;
    __shared__ TabRequests<B> s;
    __shared__ CellTokens<T * kCellsPer> tokens;
    __shared__ int32_t free_list[T * kCellsPer];
    __shared__ uint32_t miss_of[kWave];  // [kCellsPer][kWaves] counts of cells without a slot
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t head = *a.free_head;
    const bool head_ok = head >= 0 && head <= a.n_free;
    // the slots that the step could take; they do not wait for the lengths
    const int64_t left = head_ok ? (int64_t)a.n_free - head : 0;
#pragma unroll
    for (int k = 0; k < kCellsPer; ++k) {
        const int g = k * T + tid;
        free_list[g] = g < left ? a.free_slots[head + g] : -1;
    }
    if (tid < kWave) miss_of[tid] = 0;
    TabTotals all;
    int64_t off0;
    bool ok = scan_requests<T, B>(a, s, all, off0);
    const int cells = ok ? (int)all.cells : 0;
    Cell x[kCellsPer];
    uint64_t misses[kCellsPer];
    int bad = 0;
#pragma unroll
    for (int k = 0; k < kCellsPer; ++k) {
        const int c = k * T + tid;
        x[k].entry = 0;
        if (c < cells) {
            x[k] = load_cell(a, s, c);
            bad |= x[k].bad;
        }
    }
#pragma unroll
    for (int k = 0; k < kCellsPer; ++k) {
        misses[k] = __ballot(x[k].entry < 0);
        if (lane == 0) miss_of[k * kWaves + wave] = (uint32_t)__popcll(misses[k]);
    }
    bad = __syncthreads_or(bad);
    const uint32_t sums = wave_scan(miss_of[lane], 0u, OpAdd());
    const int total = (int)last_lane(sums);
    const bool fits = total <= left;
    int32_t slot[kCellsPer];
#pragma unroll
    for (int k = 0; k < kCellsPer; ++k) {
        const int i = k * kWaves + wave;
        const uint32_t before = i > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)sums, max(0, i - 1)) : 0u;
        slot[k] = x[k].entry;
        if (slot[k] < 0) {
            slot[k] = free_list[before + (uint32_t)__popcll(misses[k] & ((1ull << lane) - 1))];
            if (fits && (uint32_t)slot[k] >= (uint32_t)a.n_slots) bad = 1;
        }
    }
    bad = __syncthreads_or(bad);
    int32_t code = PULSE_OK;
    if (!ok || !head_ok || bad) code = PULSE_ERR_BAD_INDEX;
    else if (!fits) code = PULSE_ERR_POOL_EXHAUSTED;
    ok = code == PULSE_OK;
    write_offsets<T, B>(a, s, all, off0, ok);
    fill_rest(a, ok ? all.tokens : 0, tid, T);
    if (!ok) {
        if (tid == 0) report(a.status, code);
        return;
    }
    if (tid == 0 && total > 0) *a.free_head = head + total;
#pragma unroll
    for (int k = 0; k < kCellsPer; ++k) {
        const int c = k * T + tid;
        if (c >= cells) continue;
        if (x[k].entry < 0) a.table[x[k].at] = slot[k];
        keep_cell(tokens, c, x[k], slot[k]);
    }
    __syncthreads();
    fill_tokens<T>(a, tokens, cells);
}

// Counts of the larger form's threads, added up wave by wave in registers (with LDS atomics of every thread the two
// launches took 5 us more).
struct Counts {
    int32_t total, before, place, bad;
};
struct WaveCounts {
    Counts of[kTileThreads / kWave];
    __device__ inline void put(int32_t total, int32_t before, int32_t place, int32_t bad) {
        const int32_t t = (int32_t)last_lane(wave_scan((uint32_t)total, 0u, OpAdd()));
        const int32_t b = (int32_t)last_lane(wave_scan((uint32_t)before, 0u, OpAdd()));
        const int32_t p = (int32_t)last_lane(wave_scan((uint32_t)place, 0x7FFFFFFFu, OpMin()));
        const int32_t any = __ballot(bad) != 0;
        if ((threadIdx.x & 63) == 0) of[threadIdx.x >> 6] = Counts{t, b, p, any};
    }
    __device__ inline Counts sum() const {
        Counts c = of[0];
#pragma unroll
        for (int i = 1; i < kTileThreads / kWave; ++i) {
            c.total += of[i].total;
            c.before += of[i].before;
            c.place = min(c.place, of[i].place);
            c.bad |= of[i].bad;
        }
        return c;
    }
};

__global__ __launch_bounds__(kTileThreads) void tables_count_kernel(TabArgs a, TabScratch w) {
    __shared__ TabRequests<kMaxBatch> s;
    __shared__ WaveCounts s_wave;
    const int tid = threadIdx.x, tile = blockIdx.x;
    const int32_t head = *a.free_head;
    if (tid == 0 && tile == 0) *w.head = head;
    TabTotals all;
    int64_t off0;
    int n = 0, bad = 0;
    int32_t place = INT32_MAX;
    if (scan_requests<kTileThreads, kMaxBatch>(a, s, all, off0)) {
        const int64_t c1 = min(all.cells, (int64_t)(tile + 1) * w.tile);
        for (int64_t c = (int64_t)tile * w.tile + tid; c < c1; c += kTileThreads) {
            // the c-th place of the free list may be taken if there are c cells without a slot before it
            const int32_t f = head >= 0 && c < (int64_t)a.n_free - head ? a.free_slots[head + c] : 0;
            const Cell x = load_cell(a, s, (int32_t)c);
            bad |= x.bad;
            n += x.entry < 0;
            if ((uint32_t)f >= (uint32_t)a.n_slots) place = min(place, (int32_t)c);
        }
    }
    s_wave.put(n, 0, place, bad);
    __syncthreads();
    if (tid == 0) {
        const Counts c = s_wave.sum();
        w.count[tile] = c.bad ? -1 : c.total;
        w.bad_place[tile] = c.place;
    }
}

__global__ __launch_bounds__(kTileThreads) void tables_fill_kernel(TabArgs a, TabScratch w) {
    constexpr int kWaves = kTileThreads / kWave;
    __shared__ TabRequests<kMaxBatch> s;
    __shared__ CellTokens<kTileThreads> tokens;
    __shared__ uint32_t miss_of[kWaves];
    __shared__ int32_t free_list[kTileThreads];
    __shared__ WaveCounts s_wave;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, tile = blockIdx.x, tiles = gridDim.x;
    const int32_t head = *w.head;
    int32_t before = 0, total = 0, place = INT32_MAX, bad = 0;
    for (int t = tid; t < tiles; t += kTileThreads) {
        const int32_t n = w.count[t];
        bad |= n < 0;
        total += n;
        before += t < tile ? n : 0;
        place = min(place, w.bad_place[t]);
    }
    s_wave.put(total, before, place, bad);  // (read behind the barriers of the scan)
    TabTotals all;
    int64_t off0;
    bool ok = scan_requests<kTileThreads, kMaxBatch>(a, s, all, off0);
    const Counts sums = s_wave.sum();
    total = sums.total;
    int32_t code = PULSE_OK;
    if (!ok || sums.bad || head < 0 || head > a.n_free) code = PULSE_ERR_BAD_INDEX;
    else if (total > a.n_free - head) code = PULSE_ERR_POOL_EXHAUSTED;
    else if (sums.place < total) code = PULSE_ERR_BAD_INDEX;
    ok = code == PULSE_OK;
    if (tile == 0) {
        write_offsets<kTileThreads, kMaxBatch>(a, s, all, off0, ok);
        if (tid == 0) {
            if (ok) *a.free_head = head + total;
            else report(a.status, code);
        }
    }
    fill_rest(a, ok ? all.tokens : 0, (int64_t)tile * kTileThreads + tid, (int64_t)tiles * kTileThreads);
    if (!ok) return;
    int32_t g0 = head + sums.before;
    const int64_t c1 = min(all.cells, (int64_t)(tile + 1) * w.tile);
    for (int64_t c0 = (int64_t)tile * w.tile; c0 < c1; c0 += kTileThreads) {
        const int64_t c = c0 + tid;
        // the slots that these cells could take do not wait for the entries
        const int32_t f = tid < head + total - g0 ? a.free_slots[g0 + tid] : 0;
        Cell x;
        x.entry = 0;
        if (c < c1) x = load_cell(a, s, (int32_t)c);
        const uint64_t m = __ballot(x.entry < 0);
        free_list[tid] = f;
        if (lane == 0) miss_of[wave] = (uint32_t)__popcll(m);
        __syncthreads();
        int32_t g = __popcll(m & ((1ull << lane) - 1));
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            g += i < wave ? (int32_t)miss_of[i] : 0;
            g0 += (int32_t)miss_of[i];
        }
        if (c < c1) {
            int32_t slot = x.entry;
            if (slot < 0) a.table[x.at] = slot = free_list[g];
            keep_cell(tokens, tid, x, slot);
        }
        __syncthreads();
        fill_tokens<kTileThreads>(a, tokens, (int)min((int64_t)kTileThreads, c1 - c0));
        __syncthreads();
    }
}

// Bound on the cells of a step: each holds a new token, and a request's lie in at most two blocks more than they fill.
static int64_t cell_bound(int32_t B, int32_t bs, int64_t max_tokens) {
    const int64_t n = max_tokens / bs + 2 * (int64_t)B;
    return n < max_tokens ? n : max_tokens;
}
// Cells of a tile: those of 16 * kTileThreads tokens, or the multiple of them that keeps the tiles few.
static int64_t least_tile(int32_t bs) { return kTileThreads * 16 / bs; }
static int64_t tile_cells(int64_t cells, int32_t bs) {
    const int64_t least = least_tile(bs);
    return least * ((cells + least * kMaxTiles - 1) / (least * kMaxTiles));
}

// Room for as many tiles as this step or a smaller one has (a step whose tiles are larger has fewer of them).
size_t tables_ws_bytes(int32_t B, int32_t bs, int64_t max_tokens) {
    const int64_t least = least_tile(bs), most = (cell_bound(B, bs, max_tokens) + least - 1) / least;
    const int64_t tiles = most < kMaxTiles ? most : kMaxTiles;
    return (sizeof(int32_t) * (size_t)(1 + 2 * tiles) + 255) & ~(size_t)255;
}

hipError_t launch_tables(const int32_t* ctx, const int32_t* fresh, int32_t B, int32_t bs, int32_t* table,
                         int32_t max_blocks, const int32_t* free_slots, int32_t* free_head, int32_t n_free,
                         int32_t n_slots, int64_t* blk_off, int32_t* tok_off, int64_t* slot_map, int32_t* positions,
                         int64_t max_tokens, int32_t* status, void* ws, hipStream_t st) {
    const int32_t shift = bs == 16 ? 4 : bs == 32 ? 5 : 6;
    const TabArgs a{ctx,     fresh,   B,       shift,    table,     max_blocks, free_slots, free_head,
                    n_free,  n_slots, blk_off, tok_off,  slot_map,  positions,  max_tokens, status};
    const int64_t cells = cell_bound(B, bs, max_tokens);
    if (B <= 256 && cells <= 256 * kCellsPer && max_tokens <= kOneTokens) {
        hipLaunchKernelGGL((tables_one_kernel<256, 256>), dim3(1), dim3(256), 0, st, a);
    } else if (cells <= 1024 * kCellsPer && max_tokens <= kOneWideTokens) {
        hipLaunchKernelGGL((tables_one_kernel<1024, kMaxBatch>), dim3(1), dim3(1024), 0, st, a);
    } else {
        const int64_t tile = tile_cells(cells, bs), tiles = (cells + tile - 1) / tile;
        int32_t* w = static_cast<int32_t*>(ws);
        const TabScratch sc{w, w + 1, w + 1 + tiles, (int32_t)tile};
        hipLaunchKernelGGL(tables_count_kernel, dim3((unsigned)tiles), dim3(kTileThreads), 0, st, a, sc);
        hipLaunchKernelGGL(tables_fill_kernel, dim3((unsigned)tiles), dim3(kTileThreads), 0, st, a, sc);
    }
    return hipGetLastError();
}

}  // namespace pulse

// attention.hip -- split-K sparse GQA decode attention over the selected
// blocks of the slot pool, for gfx950 (the attention that follows recall,
// Sec. 2.2 and Sec. 4.2.1).
//
// One wavefront owns (request r, KV head h, split s): a contiguous range of
// the request's selected blocks.  The G query heads of h share every K/V
// byte the wave reads, so the contraction is a batched GQA tile:
//   S^T[32 tokens x 16] = K[32 x 128] . Q^T[128 x 16]   (G <= 16 query columns)
//   O[16 x 128]        += P[16 x 32]  . V[32 x 128]
// both on v_mfma_f32_16x16x32_{bf16,f16}.  Each lane's MFMA operands are 16
// contiguous bytes in HBM: K is stored token-major and V channel-major, so
// neither operand needs an LDS transpose.  The S^T tile rows are assigned
// to tokens so that its accumulator layout is exactly the P operand layout
// of the P.V product (lane = query column, 8 consecutive tokens per lane
// group), so softmax probabilities never leave registers.
//
// Precision: K, V, q are consumed as stored (products exact in fp32, fp32
// accumulation).  P is split into hi + lo 16-bit parts (two MFMAs), which
// keeps the P.V product at ~2^-16 relative error instead of the 2^-9 of a
// single bf16 rounding.  Softmax is online per 32-token step in the log2
// domain.
//
// Merging the splits: a workgroup holds W waves = W consecutive splits of one
// (r, h) (attn_waves); they merge through LDS.  With one workgroup per (r, h)
// it writes the result directly.  Otherwise each workgroup writes one partial
// (m, l, O) to the workspace and a combine kernel merges those partials, one
// thread per output element, with independent loads.  (Merging in the last workgroup
// to finish instead needs a device-scope release per workgroup, an L2
// write-back on gfx950 measured at about 9 ns per workgroup, plus a merge on
// the kernel's tail and counters that start at zero in the workspace: it would
// save well under the combine launch's 3.6 us.)
#include <algorithm>

#include "kv4.h"
#include "kv8.h"

namespace pulse {

#ifndef PULSE_ATTN_TARGET_WAVES
#define PULSE_ATTN_TARGET_WAVES 2048
#endif
constexpr int kCombineThreads = kHeadDim;

// Waves per workgroup (attn_waves): 8 while the LDS merge buffer (waves x G x
// 128 floats) stays within 32 KiB, else 4.  Fewer, wider workgroups leave
// fewer partials for the combine kernel.  A 4-bit cache takes 8 for the larger
// groups too (64 KiB): its waves wait for instructions more than for loads.
// In us, 4 waves and 8, G = 16: one request of 400 tokens 12.1 and 10.9, of
// 4K 13.6 and 12.8; 16 of 4K 17.5 and 14.5; 4 of 64K 35.5 and 26.6.  In blocks
// of 64, whose shortest split is two steps, calls of few splits take 4, on
// twice the CUs: 1.5K tokens 11.9 and 13.3, 8 of 2K (1024 splits) 14.0 and
// 14.8, 16 of 4K 22.8 and 19.9.
constexpr int kCodeWaves = 8;

// Selected blocks up to which one workgroup takes a whole request and head of a 4-bit cache, so that no merge
// launch follows: 2 to 4 steps of its waves, the more the more workgroups wait for the memory, the fewer the larger
// the groups.  In us, split as far as 2048 waves go and kept together, 2, 3 and 4 steps (500, 760 and 1016 tokens):
//   1 request, 8 heads of 1      9.3  8.0   9.1  9.0   9.2 10.1
//   9 requests, 8 heads of 8    13.4 12.3  12.4 12.3  13.8 13.7
//   24 requests, 8 heads of 4   15.4 12.0  17.5 12.2  17.4 13.6
//   8 requests, 1 head of 16    11.8 11.5  12.9 14.6  13.1 16.7
static int32_t one_group_entries(const pulse_shape& s, int64_t units) {
    const int steps = units > 64 ? 4 : s.num_q_heads > 8 * s.num_kv_heads ? 2 : 3;
    return kCodeWaves * steps * kChunkTokens / s.block_size;
}

int attn_waves(const pulse_shape& s, int32_t B, int32_t k_max) {
    if (s.num_q_heads / s.num_kv_heads <= 8) return 8;
    if (!in_codes(s.dtype)) return 4;
    const int64_t units = (int64_t)B * s.num_kv_heads;
    const bool few = s.block_size > kChunkTokens && k_max > one_group_entries(s, units) &&
                     units * k_max <= PULSE_ATTN_TARGET_WAVES / 2;
    return few ? 4 : kCodeWaves;
}

// Entries of one 32-token step, and of the shortest split.
static int32_t split_step(int32_t bs) { return bs >= kChunkTokens ? 1 : kChunkTokens / bs; }
// Two steps, one of a 4-bit cache (a quarter of the bytes, and twice the shortest split's work to share out: 64
// requests of 80 tokens 10.1 and 9.0 us with two and one; of an 8-bit one 32 requests of 1000 tokens, lognormal, 12.0 and
// 13.0, 2 requests of 2000 10.9 and 9.7).
static int32_t split_least(const pulse_shape& s) {
    const int t = (is_kv4(s.dtype) ? 1 : 2) * kChunkTokens;
    return s.block_size >= t ? 1 : t / s.block_size;
}

struct SplitArgs {
    int32_t eps, n_wg;    // host plan: entries per wave, workgroups per (request, KV head)
    int32_t even, n_even; // the same where every request has k_max blocks
    int32_t step, least;  // granularity and least value of eps
    int32_t most;         // largest eps of a plan
    int32_t fit;          // pieces that a plan may have
    bool planned;         // look whether the counts are equal
    bool share;           // and if not, share the grid out by them
    bool level;           // unless they are three quarters of k_max on average
    bool light_last;      // every (request, KV head)'s last workgroup has fewer waves: start those last
};

// ---- the split plan ----
// The host sizes the grid for requests of k_max selected blocks each: n_wg workgroups
// per (request, KV head), whose W waves take eps entries each.  Counts live on the
// device; where they differ, that leaves long requests few waves and short ones idle
// workgroups, so the kernels share the same grid out by the counts: the least eps with
// which ceil(cnt / (W * eps)) workgroups per request and head are no more than `fit`.
// Workgroup p is piece (p / Hkv, head p % Hkv) of the requests' pieces in order; its
// partial is number p.
//
// A CU takes a second workgroup only at the cost of both (their loads share its
// address path), so `fit` is one round of workgroups (2048 waves) where that leaves a
// quarter more pieces than requests, and the grid otherwise or where the host's own
// split takes more than a round.  Without a plan, where the grid takes more than a round
// and every last workgroup has fewer waves, splits are numbered slowest, so that those
// are the ones that come second.
// Finding and following a plan costs 1 to 2 us (two memory round trips), so it is for up to
// 64 requests (one lane each) whose eps may halve, or whose empty workgroups would make a
// second round.  In us, three batches in turn: the host's split alone (before the reductions
// in registers), a plan up to the whole grid wherever counts differ, and as it is.  Over 560
// calls drawn from 1 to 32 requests and budgets of 256 to 8192 tokens, lognormal or equal, the
// second was 1.08 and this is 1.13 times as fast as the first; 101 and 11 calls lost over 1%.
//   16 requests x 65K tokens, lognormal around 2048 tokens (188 MB)    58.0  42.9  43.0
//   7 requests x 120K tokens, blocks of 32, around 2705 (100 MB)       29.3  31.1  23.1
//   20 requests, 2 KV heads, all 387 blocks (280 workgroups)           34.9  39.2  29.5
//   5 requests, 3 KV heads, around 702 tokens                          11.3  12.1  10.9
constexpr int kPlanRequests = 64;

// With a 4-bit cache (and, by the same rules, an 8-bit one) a step is short and a second workgroup on a CU costs more than half as much again, so its calls
// keep to one round more strictly.  Where all counts are k_max and the host's split takes more than a round, the
// splits are `even`, the shortest that fit one round, unless the second workgroups are so light that even * W >
// eps * (W + their waves).  Where the host's pieces do not fit, a plan may take up to `most` = 64 entries per wave.
// And up to 256 requests are planned (four per lane), from 2K tokens on: the longer search costs up to 2 us.  In us,
// split and planned like a 16-bit cache and as it is, requests x tokens (up to 17 requests 32 query heads over 8 KV
// heads, from 48 on 8 over 1), r: lognormal around the number:
//   9 x 12K         41.6 33.7    48 x 4K         22.1 17.9    72 x 1.5K r     24.3 20.7
//   11 x 4K         27.6 22.3    48 x 12K r      35.3 25.9    72 x 4K r       25.4 27.8
//   17 x 1.5K       21.0 18.2    88 x 4K         32.8 24.6    112 x 4K r      39.6 34.7
//   17 x 12K r      52.5 39.7    136 x 1.5K      25.2 19.9    136 x 1.5K r    47.7 27.4
// An 8-bit cache, split like a 16-bit one and as it is, requests x tokens: 256 x 500 100 59, 128 x 1000 60 52, 4 x 32K over
// one KV head of 16 28 21, 24 x 4K r 56 53; 16 x 2K r 23.2 23.8, 64 x 2000 51.6 52.3.
constexpr int kPlanRequestsCodes = 256;
constexpr int kPlanTokensCodes = 2048;
// More requests and heads than a round has workgroups: from 4K tokens on the grid has two workgroups for each, for a
// plan to share out.  Equal counts leave the second without work, and so do, where the last round is as good as full,
// counts of three quarters of k_max on average.  In us, one workgroup each and this (8 KV heads; 2 from 132 requests):
//   33 x 2K r       40.0 30.5    33 x 4K        48.2 48.6    132 x 2K r      49.4 32.5    256 x 2K r      81.3 56.6
//   64 x 4K r       89.6 83.6    64 x 4K        59.1 59.4    160 x 4K r      87.0 67.8    256 x 2K (25%)  48.2 56.5
constexpr int kOverTokens = 4096;

struct Piece {
    int eps, nwg, base;  // entries per wave, workgroups of the request, its first piece
    int r, wg;
    int32_t cnt;         // selected blocks of the request (0 if the count is invalid)
};

// Workgroups of a request of c blocks: at least one, which writes an empty request's output.
__device__ inline int pieces_of(int c, int per) { return max(1, (c + per - 1) / per); }

// The same for c below 2^23, by the reciprocal, whose quotient is at most one off.
__device__ inline int pieces_short(int c, int per) {
    const int n = c + per - 1;
    int q = (int)((float)n * __builtin_amdgcn_rcpf((float)per));
    const int rest = n - q * per;
    q += rest < 0 ? -1 : rest >= per ? 1 : 0;
    return max(1, q);
}

// The counts of a plan: lane l holds those of requests R * l .. R * l + R - 1, 0 behind the last.
template <int R>
struct Counts {
    int32_t raw[R];
    __device__ explicit Counts(const int32_t* __restrict__ sel_cnt, int32_t B, int lane) {
#pragma unroll
        for (int i = 0; i < R; ++i) raw[i] = R * lane + i < B ? sel_cnt[R * lane + i] : 0;
    }
    // any(f(raw)) over the requests
    template <class F>
    __device__ bool any(int32_t B, int lane, F f) const {
        bool a = false;
#pragma unroll
        for (int i = 0; i < R; ++i) a |= R * lane + i < B && f(raw[i]);
        return __ballot(a) != 0;
    }
    // Whether every request has k_max blocks: the host's split as it is.
    __device__ bool equal(int32_t B, int32_t k_max, int lane) const {
        return !any(B, lane, [&](int32_t c) { return c != k_max; });
    }
    __device__ int valid(int i, int32_t k_max) const { return raw[i] >= 0 && raw[i] <= k_max ? raw[i] : 0; }
    // Blocks of all requests (up to 256 of up to 2^22).
    __device__ uint32_t blocks(int32_t k_max) const {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) n += (uint32_t)valid(i, k_max);
        return last_lane(wave_scan(n, 0u, OpAdd()));
    }
    // Whether they have three quarters of k_max blocks on average.
    __device__ bool level(int32_t B, int32_t k_max) const {
        return (float)blocks(k_max) >= 0.75f * (float)B * (float)k_max;
    }
};

// Plan for piece index pr (of all heads of a request at once), or, with pr < 0, for the first piece of request
// `req`; all lanes of a wave take part.  r < 0: no such piece.
template <int R>
__device__ inline Piece plan_piece(int pr, int req, const Counts<R>& counts, int32_t B, int32_t k_max, int32_t W,
                                   const SplitArgs& sp, int lane) {
    int c[R];
#pragma unroll
    for (int i = 0; i < R; ++i) c[i] = counts.valid(i, k_max);
    uint32_t np[R];
    auto pieces = [&](int eps) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            np[i] = R * lane + i < B ? (uint32_t)pieces_short(c[i], W * eps) : 0u;
            n += np[i];
        }
        return n;
    };
    auto sum = [&](int eps) { return (int)last_lane(wave_scan(pieces(eps), 0u, OpAdd())); };
    // m = blocks / W of all requests make m / eps to m / eps + B pieces, which leaves few values of eps to try
    // (rounded outwards by more than the 2^-21 that these floats are off; step is 1 or 2)
    const float m = (float)counts.blocks(k_max) * __builtin_amdgcn_rcpf((float)W);
    int fit = sp.fit, lo = sp.least, hi = sp.eps;
    int enough = INT32_MAX;
    if (fit > B) {
        const float x = m * __builtin_amdgcn_rcpf((float)(fit - B)) * 1.000001f;
        if (x < 64.f) enough = ((int)x + sp.step) & -sp.step;
    }
    if (enough <= sp.eps) {
        hi = max(enough, sp.least);
    } else if (sum(sp.eps) > fit) {
        if (sp.most > sp.eps && (enough <= sp.most || sum(sp.most) <= fit)) {
            lo = sp.eps;
            hi = min(sp.most, enough);
        } else {
            fit = B * sp.n_wg;  // no request has more than n_wg workgroups
        }
    }
    lo = max(lo, (int)(m * __builtin_amdgcn_rcpf((float)fit) * 0.999999f) & -sp.step);
    while (lo < hi) {
        const int mid = (lo + hi) / 2 / sp.step * sp.step;
        if (sum(mid) <= fit) hi = mid;
        else lo = mid + sp.step;
    }
    Piece p;
    p.eps = hi;
    const uint32_t own = pieces(p.eps);
    const uint32_t incl = wave_scan(own, 0u, OpAdd());
    int at, first;  // the lane whose requests hold the piece, and the piece's or the request's place among theirs
    if (pr >= 0) {
        at = __popcll(__ballot((int)incl <= pr));
        if (at >= kWave) {
            p.r = -1;
            return p;
        }
        first = pr - (int)(__builtin_amdgcn_readlane((int)incl, at) - __builtin_amdgcn_readlane((int)own, at));
    } else {
        at = req / R;
        first = 0;
    }
    p.base = __builtin_amdgcn_readlane((int)(incl - own), at);
    p.r = R * at;
    p.nwg = __builtin_amdgcn_readlane((int)np[0], at);
    p.cnt = __builtin_amdgcn_readlane(c[0], at);
#pragma unroll
    for (int i = 1; i < R; ++i) {
        if (pr >= 0 ? first < p.nwg : R * at + i > req) break;
        first -= p.nwg;
        p.base += p.nwg;
        p.r = R * at + i;
        p.nwg = __builtin_amdgcn_readlane((int)np[i], at);
        p.cnt = __builtin_amdgcn_readlane(c[i], at);
    }
    p.wg = pr >= 0 ? first : 0;
    return p;
}

// 2^x as the hardware has it (1 ulp; results below 2^-126 are 0, far below what a sum of
// probabilities with a largest one of 1 holds).
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Combination of the four 16-lane groups' values, in every lane: rows and halves are exchanged
// between two copies in registers (v_permlane16_swap, v_permlane32_swap), no LDS round trip.
// With this, exp2_fast and the accumulators rescaled only when a maximum moved: 8 x 2048 tokens
// 16.2 -> 15.9 us, 4 x 8192 at G 8 30.2 -> 29.9, one request of 400 tokens 8.3 -> 7.8 in the kernel.
template <typename Op>
__device__ inline float across_groups(float x, Op op) {
    const uint32_t u = __float_as_uint(x);
    const u32x2 a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float y = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(y);
    const u32x2 b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Attention of one wave over entries [e0, e0 + ne) of request r, KV head h;
// j_lane is the selected block of entry e0 + lane (loaded by the caller).
// Leaves the running max (log2 domain) and the lane-group-reduced sum for
// query column `col` in m_run / l_run, and O rows g = 4*grp + v in acc.
template <int DT, int BS>
__device__ inline void attend_split(const uint16_t* __restrict__ q, const uint16_t* __restrict__ pool,
                                    int32_t n_slots, const int32_t* __restrict__ table, int32_t max_blocks,
                                    int32_t j_lane, const int32_t* __restrict__ ctx_len, int32_t Hq, int32_t Hkv,
                                    int32_t G, int r, int h, int ne, float scale_log2, int32_t* status, int lane,
                                    float& m_run, float& l_run, f32x4 (&acc)[8]) {
    using M = Mfma<DT>;
    using vec = typename M::vec;
    const int col = lane & 15;  // MFMA column: query head (QK^T), channel (PV)
    const int grp = lane >> 4;  // lane group: 8-channel / 8-token slice
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run = -INFINITY;
    l_run = 0.f;
    if (ne <= 0) return;
    // entry metadata, one entry per lane (ne <= 64); the table lookup does not wait for the context length
    const int32_t j = lane < ne ? j_lane : -1;
    const int32_t sl = (j >= 0 && j < max_blocks) ? table[(size_t)r * max_blocks + j] : -1;
    const int ctx = ctx_len[r];
    const int64_t n_r = ((int64_t)ctx + BS - 1) / BS;
    int my_slot = -1, my_nv = 0;
    if (lane < ne) {
        if (j < n_r && sl >= 0 && sl < n_slots) {
            my_slot = sl;
            const int64_t v = (int64_t)ctx - (int64_t)j * BS;
            my_nv = v >= BS ? BS : (int)v;
        }
        if (my_slot < 0) report(status, PULSE_ERR_BAD_INDEX);
    }
    constexpr int kPer = BS >= kChunkTokens ? 1 : kChunkTokens / BS;  // entries of a step
    const uint64_t partial = __ballot(my_slot >= 0 && my_nv < BS);
    // Q^T operand: lane holds q[g = col][8 channels of slice grp + 32 kc]
    vec qb[4];
    {
        const uint16_t* qr = q + ((size_t)r * Hq + (size_t)h * G + col) * kHeadDim + grp * 8;
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) qb[kc] = col < G ? load_vec<DT>(qr + 32 * kc) : zero_vec<DT>();
    }
    const size_t E = (size_t)2 * Hkv * BS * kHeadDim;
    const size_t k_head = (size_t)h * BS * kHeadDim;
    const size_t v_head = (size_t)Hkv * BS * kHeadDim + (size_t)h * kHeadDim * BS;
    const int tokens = ne * BS;

    // K and V operand loads of one 32-token step starting at sequence token t0
    // K: MFMA row m = col maps to token 8*(col/4) + 4*sub + col%4;
    // V: lane group grp holds tokens 8*grp .. 8*grp+7 of channel col + 16*tile.
    auto load_k = [&](int t0, vec (&ka)[2][4]) {
        const int ka_seq = t0 + 8 * (col >> 2);
        const int ka_e = ka_seq / BS;
        const int ka_slot = __shfl(my_slot, ka_e < ne ? ka_e : 0);
        const int ka_nv = __shfl(my_nv, ka_e < ne ? ka_e : 0);
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            const int row = ka_seq % BS + 4 * sub + (col & 3);
            const bool ok = ka_e < ne && ka_slot >= 0 && row < ka_nv;
            const uint16_t* kp = pool + (size_t)(ok ? ka_slot : 0) * E + k_head + (size_t)row * kHeadDim + grp * 8;
#pragma unroll
            for (int kc = 0; kc < 4; ++kc) ka[sub][kc] = ok ? load_vec<DT>(kp + 32 * kc) : zero_vec<DT>();
        }
    };
    auto load_v = [&](int t0, vec (&vb)[8]) {
        const int pv_seq = t0 + 8 * grp;
        const int pv_e = pv_seq / BS;
        const int pv_slot = __shfl(my_slot, pv_e < ne ? pv_e : 0);
        const bool pv_ok = pv_e < ne && pv_slot >= 0;
        const uint16_t* vp = pool + (size_t)(pv_ok ? pv_slot : 0) * E + v_head + (size_t)col * BS + pv_seq % BS;
#pragma unroll
        for (int t = 0; t < 8; ++t) vb[t] = pv_ok ? load_vec<DT>(vp + (size_t)16 * t * BS) : zero_vec<DT>();
    };

    // One 32-token step at a time: K is loaded first, V once the S tile is issued, so
    // the V loads overlap the softmax and fewer operands are live (123-127 VGPRs and 4
    // waves per SIMD with 8-wave workgroups, 156-168 and 3 with 4-wave ones).  The
    // other resident waves hide the load latency.  Measured slower:
    // loading K and V together (154 VGPRs; 2-5%), prefetching the next step into
    // registers as well (223 VGPRs; another 1-2%), and, for splits of two steps,
    // issuing all four loads before the first product (177 VGPRs; 11% slower on
    // 8 requests x 2048 selected tokens; no faster on one request either), and keys
    // loaded with neighbouring lanes on neighbouring pieces and staged through LDS,
    // pipelined by a step (2-4% slower on 8 x 2048, equal on larger calls).
#pragma unroll 1
    for (int t0 = 0; t0 < tokens; t0 += kChunkTokens) {
        vec ka[2][4], vb[8];
        load_k(t0, ka);
        const int pv_seq = t0 + 8 * grp;
        const int pv_e = pv_seq / BS;
        const int pv_slot = __shfl(my_slot, pv_e < ne ? pv_e : 0);
        const int pv_nv = __shfl(my_nv, pv_e < ne ? pv_e : 0);
        const int pv_row = pv_seq % BS;
        const bool pv_ok = pv_e < ne && pv_slot >= 0;
        // --- S^T = K . Q^T
        f32x4 s1 = {0.f, 0.f, 0.f, 0.f}, s2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) {
            s1 = M::mac(ka[0][kc], qb[kc], s1);
            s2 = M::mac(ka[1][kc], qb[kc], s2);
        }
        load_v(t0, vb);
        // lane (col, grp) now holds query col, tokens pv_seq + 0..7
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = s1[i] * scale_log2;
            x[4 + i] = s2[i] * scale_log2;
        }
        float cm = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!pv_ok || pv_row + i >= pv_nv) x[i] = -INFINITY;
            cm = fmaxf(cm, x[i]);
        }
        cm = across_groups(cm, [](float a, float b) { return fmaxf(a, b); });
        const float m_new = fmaxf(m_run, cm);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2_fast(m_run - m_use);
        float psum = 0.f;
        vec ph, pl;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = exp2_fast(x[i] - m_use);
            psum += p;
            typename M::elem hi, lo;
            M::split(p, hi, lo);
            ph[i] = hi;
            pl[i] = lo;
        }
        l_run = l_run * alpha + psum;
        m_run = m_new;
        // rescale accumulator rows g' = 4*grp + v by alpha of query g' (not while they are zero,
        // and not when no query's maximum moved)
        if (t0 > 0 && __ballot(alpha != 1.f)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float av = __shfl(alpha, 4 * grp + v);
#pragma unroll
                for (int t = 0; t < 8; ++t) acc[t][v] *= av;
            }
        }
        // behind a context's end lies what an earlier owner of the slot left, NaN perhaps, which a probability of 0
        // would not take out of the product (1 x 400 tokens 9.18 -> 9.24 us, 8 x 2048 17.55 -> 17.6)
        if ((partial >> (t0 / BS)) & ((1u << kPer) - 1)) {
            const int left = pv_nv - pv_row;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t keep = (2 * i < left ? 0xFFFFu : 0u) | (2 * i + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    u32x4 w = __builtin_bit_cast(u32x4, vb[t]);
                    w[i] &= keep;
                    vb[t] = __builtin_bit_cast(vec, w);
                }
            }
        }
        // --- O += P . V  (hi and lo parts of P)
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            acc[t] = M::mac(ph, vb[t], acc[t]);
            acc[t] = M::mac(pl, vb[t], acc[t]);
        }
    }
    l_run = across_groups(l_run, [](float a, float b) { return a + b; });
}

// attend_split over the 4-bit cache (kv4.h).  A lane's 16 bytes of a key row are 32 channels under one scale,
// decoded with it into the operands of four products; Q is loaded in the same channel order.  A value's scale
// differs from token to token, which is the index the P.V product sums over, so it multiplies the probability
// instead: P'[q][g][t] = P[q][t] * scale[t][g] for channel group g, and V is decoded without a scale.  The 16 rows
// of the P operand hold GP = 4, 8 or 16 query heads for 4, 2 or 1 groups at once (row = g' * GP + q: the query
// columns of S^T repeat), so P' costs a multiplication per row and token however many heads there are; the
// product of channel tile t uses the rows of its group t / 2, the other rows of its result are left unused.
// Codes are exact in bf16 and scales are powers of two, so P' is cut into bf16 parts for either 16-bit type (fp16
// would not hold the range of the scales): three of them, all 24 bits of it.  With two (2^-17 of it) the results
// were 1.4e-6 off, with three 2e-7, below what a computation in fp32 is off (4e-7), for 0.2 to 1 us a call.
// Row 4 * grp + v of acc[t] is query head (4 * grp + v) % GP of group (4 * grp + v) / GP of the tile's set.
//
// Bound: 136 bytes per token and KV head.  32 requests of 4K tokens, 8 heads (141 MB): 29 us (4.9 TB/s; 24 at what
// streaming reads reach), of which 8 are the launch, the look-ups ahead of the first key and the waves' merge; short
// calls are those 8 and 0.6 to 1.4 us a step.  A step is about 230 vector instructions (64 of them decode), which the
// eight waves of a CU issue in about 1 us, so they count beside the bytes: scale bytes by shift and mask cost 2 to 3%
// on 16 ragged requests, rounded instead of cut parts as much.  Loads: the next step's are issued once the keys are
// decoded.  Measured slower or equal: two, three and four steps ahead (2 to 6% slower), codes loaded with
// neighbouring lanes on neighbouring pieces and passed through LDS (2% slower), the next step's softmax under the
// products of this one (equal), products interleaved over accumulators (equal), 16 waves per workgroup (5 to 10%
// slower), two workgroups per CU (20% slower), keys multiplied as codes by the scaled 4-bit matrix instruction (Q cut
// into two or three e4m3 parts; 34 vector instructions fewer a step: 1% faster on 16 ragged requests, 2 to 10% slower
// on the others for the cutting, and its sums are some hundred times less exact).  All that is of GP = 4.
// Larger groups cut P' into parts twice (GP = 8) and four times (16) a step, and their kernels hold 130 to 133 and 145
// to 146 VGPRs (GP = 4: 125 and 126), so a CU takes one workgroup at a time where it takes two with GP = 4, and beyond
// a round nothing runs beside a workgroup's look-ups and merge: 2048 requests and heads of 1000 tokens, 1024 of 2000
// (floors 49 to 52 us), 4, 8 and 16 query heads each: 64 94 117, 59 77 94 us.
template <int GP>
struct Kv4Values {
    u32x4 v[2];        // codes of 8 tokens, channel tiles 0..3 and 4..7
    u32x2 vs[GP / 4];  // scale bytes of 8 tokens
};

// 2^e of byte N of a word of scale bytes.
template <int N>
__device__ inline float kv4_scale_of(uint32_t w) {
    return kv4_scale(__builtin_amdgcn_ubfe(w, 8 * N, 8));
}

template <int DT, int BS, int GP>
__device__ inline void attend_split_kv4(const uint16_t* __restrict__ q, const uint8_t* __restrict__ pool,
                                        int32_t n_slots, const int32_t* __restrict__ table, int32_t max_blocks,
                                        int32_t j_lane, const int32_t* __restrict__ ctx_len, int32_t Hq, int32_t Hkv,
                                        int32_t G, int r, int h, int ne, float scale_log2, int32_t* status, int lane,
                                        float& m_run, float& l_run, f32x4 (&acc)[8]) {
    constexpr int ET = elem_type(DT);
    constexpr int kSets = GP / 4;  // P operands: rows hold 16 / GP groups each
    using MQ = Mfma<ET>;
    using MP = Mfma<PULSE_BF16>;
    using vec = typename MQ::vec;
    const int col = lane & 15;
    const int grp = lane >> 4;
    const int qc = col % GP;  // query head of this column
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run = -INFINITY;
    l_run = 0.f;
    if (ne <= 0) return;
    // entry metadata, one entry per lane; an entry without a block reads slot 0 and counts no token
    const int32_t j = lane < ne ? j_lane : -1;
    const int32_t sl = (j >= 0 && j < max_blocks) ? table[(size_t)r * max_blocks + j] : -1;
    const int ctx = ctx_len[r];
    const int64_t n_r = ((int64_t)ctx + BS - 1) / BS;
    int my_slot = 0, my_nv = 0;
    if (lane < ne) {
        if (j >= 0 && j < n_r && sl >= 0 && sl < n_slots) {
            my_slot = sl;
            const int64_t v = (int64_t)ctx - (int64_t)j * BS;
            my_nv = v >= BS ? BS : (int)v;
        } else {
            report(status, PULSE_ERR_BAD_INDEX);
        }
    }
    const uint64_t whole = __ballot(my_nv == BS);
    // Q^T operand: channels 32 * grp + 8 * kc .. + 7 of the column's query head
    vec qb[4];
    {
        const uint16_t* qr = q + ((size_t)r * Hq + (size_t)h * G + qc) * kHeadDim + grp * kGroup;
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) qb[kc] = qc < G ? load_vec<ET>(qr + 8 * kc) : zero_vec<ET>();
        // logits are scaled after their maximum is taken: the sign of the scale goes to Q, a zero becomes tiny
        if (scale_log2 < 0.f) {
#pragma unroll
            for (int kc = 0; kc < 4; ++kc) qb[kc] = -qb[kc];
        }
        scale_log2 = fmaxf(fabsf(scale_log2), 1e-30f);
    }
    // Step i covers tokens 32 i ..: entry and row of a lane's tokens.  K: MFMA row m = col is token
    // 8 * (col / 4) + 4 * sub + col % 4; V: lane group grp holds tokens 8 * grp .. + 7, channels col + 16 * t in word t.
    constexpr int kPer = BS >= kChunkTokens ? 1 : kChunkTokens / BS;  // entries of a step
    constexpr int kHalves = BS > kChunkTokens ? BS / kChunkTokens : 1;  // steps of an entry
    const uint32_t E = (uint32_t)Hkv * kv4_head_bytes(BS);
    const uint8_t* head = pool + (size_t)h * kv4_head_bytes(BS);
    const int k_tok = 8 * (col >> 2), v_tok = 8 * grp;
    const uint8_t* k_at = head + (k_tok % BS + (col & 3)) * 64 + grp * 16;
    const uint8_t* ks_at = head + kv4_key_scales(BS) + (k_tok % BS + (col & 3)) * kGroups + grp;
    const uint8_t* v_at = head + kv4_values(BS) + v_tok % BS * 64 + col * 32;
    const uint8_t* vs_at = head + kv4_value_scales(BS) + col / GP * BS + v_tok % BS;
    const int steps = (ne * BS + kChunkTokens - 1) / kChunkTokens;

    u32x4 kw[2];
    uint32_t ksb[2];
    Kv4Values<GP> vnext;
    auto load_k = [&](int i) {
        const uint32_t slot = (uint32_t)__shfl(my_slot, i / kHalves * kPer + k_tok / BS);
        const int half = i % kHalves * kChunkTokens;
        const uint8_t* kb = k_at + (uint64_t)slot * E + half * 64;
        const uint8_t* sb = ks_at + (uint64_t)slot * E + half * kGroups;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            kw[sub] = *reinterpret_cast<const u32x4*>(kb + 4 * sub * 64);
            ksb[sub] = sb[4 * sub * kGroups];
        }
    };
    auto load_v = [&](int i) {
        const uint32_t slot = (uint32_t)__shfl(my_slot, i / kHalves * kPer + v_tok / BS);
        const int half = i % kHalves * kChunkTokens;
        const uint8_t* vb = v_at + (uint64_t)slot * E + half * 64;
        const uint8_t* sb = vs_at + (uint64_t)slot * E + half;
#pragma unroll
        for (int n = 0; n < 2; ++n) vnext.v[n] = reinterpret_cast<const u32x4*>(vb)[n];
#pragma unroll
        for (int k = 0; k < kSets; ++k) vnext.vs[k] = *reinterpret_cast<const u32x2*>(sb + k * (16 / GP) * BS);
    };
    load_k(0);
    load_v(0);
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        Kv4Values<GP> now = vnext;
        // --- S^T = K . Q^T
        f32x4 s[2] = {};
        const float ks[2] = {kv4_scale(ksb[0]), kv4_scale(ksb[1])};
#pragma unroll
        for (int kc = 0; kc < 4; ++kc)
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) s[sub] = MQ::mac(kv4_decode8<ET>(kw[sub][kc], ks[sub]), qb[kc], s[sub]);
        if (i + 1 < steps) {
            load_k(i + 1);
            load_v(i + 1);
        }
        float x[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) x[n] = s[n / 4][n % 4];
        // blocks that are not whole (the last of the context, a missing one, none behind an odd count): their other
        // tokens count nothing, whatever their scale bytes are
        if ((~whole >> (i / kHalves * kPer)) & ((1u << kPer) - 1)) {
            // tokens of this lane's 8
            const int left = __shfl(my_nv, i / kHalves * kPer + v_tok / BS) - v_tok % BS - i % kHalves * kChunkTokens;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                if (n >= left) x[n] = -INFINITY;
#pragma unroll
                for (int k = 0; k < kSets; ++k)
                    if (n >= left) now.vs[k][n / 4] &= ~(0xFFu << (8 * (n % 4)));
            }
        }
        // (the median of two values and infinity: fmaxf would first make each of them a number of its own)
        float cm = x[0];
#pragma unroll
        for (int n = 1; n < 8; ++n) cm = __builtin_amdgcn_fmed3f(cm, x[n], INFINITY);
        cm = across_groups(cm, [](float a, float b) { return fmaxf(a, b); });
        const float m_new = fmaxf(m_run, cm * scale_log2);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2_fast(m_run - m_use);
        float psum = 0.f;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            x[n] = exp2_fast(x[n] * scale_log2 - m_use);
            psum += x[n];
        }
        l_run = l_run * alpha + psum;
        m_run = m_new;
        if (i > 0 && __ballot(alpha != 1.f)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float av = __shfl(alpha, 4 * grp + v);
#pragma unroll
                for (int t = 0; t < 8; ++t) acc[t][v] *= av;
            }
        }
        // --- O += P' . V
#pragma unroll
        for (int k = 0; k < kSets; ++k) {
            float y[8];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                y[4 * n] = x[4 * n] * kv4_scale_of<0>(now.vs[k][n]);
                y[4 * n + 1] = x[4 * n + 1] * kv4_scale_of<1>(now.vs[k][n]);
                y[4 * n + 2] = x[4 * n + 2] * kv4_scale_of<2>(now.vs[k][n]);
                y[4 * n + 3] = x[4 * n + 3] * kv4_scale_of<3>(now.vs[k][n]);
            }
            u32x4 part[3];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                float a = y[2 * n], b = y[2 * n + 1];
#pragma unroll
                for (int m = 0; m < 3; ++m) {
                    part[m][n] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
                    a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
                    b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int t = 8 / kSets * k; t < 8 / kSets * (k + 1); ++t) {
                const bf16x8 v = kv4_decode8<PULSE_BF16>(now.v[t / 4][t % 4], 1.0f);
#pragma unroll
                for (int m = 0; m < 3; ++m) acc[t] = MP::mac(__builtin_bit_cast(bf16x8, part[m]), v, acc[t]);
            }
        }
    }
    l_run = across_groups(l_run, [](float a, float b) { return a + b; });
    // a split whose every logit is NaN (keys of a NaN scale) keeps its weight in the merge
    if (m_run == -INFINITY && l_run != l_run) m_run = 0.f;
}

// attend_split over the 8-bit cache (kv8.h).  A lane's 32 bytes of a key row are 32 channels, its 64 bytes of values 8
// tokens of 8 channels; a block has one scale for its keys and one for its values, so both are decoded with it, exactly,
// into the operands of the products: keys into the type of the queries, values into bf16, so that the probabilities can
// be cut into three bf16 parts, all 24 bits of them (as in attend_split_kv4).
//
// Bound: HBM, 256 bytes per token and KV head, once enough steps are in flight: 32 requests of 4K tokens, 8 heads (268 MB)
// 53 us (5.1 TB/s; 46 at what streaming reads reach); short calls are the launch, the look-ups and the waves' merge (7 us
// for 400 tokens).  A step's loads are issued together and the other waves hide them: 120 VGPRs, so two workgroups a CU;
// with the next step loaded ahead (180 VGPRs) the long calls are 0 to 1% faster and those of many workgroups slower
// (128 requests of 1000 tokens 60 and 82 us, 256 of 500 100 and 144).  Values loaded behind the logits instead of with the
// keys: equal.
template <int DT, int BS>
__device__ inline void attend_split_kv8(const uint16_t* __restrict__ q, const uint8_t* __restrict__ pool,
                                        int32_t n_slots, const int32_t* __restrict__ table, int32_t max_blocks,
                                        int32_t j_lane, const int32_t* __restrict__ ctx_len, int32_t Hq, int32_t Hkv,
                                        int32_t G, int r, int h, int ne, float scale_log2, int32_t* status, int lane,
                                        float& m_run, float& l_run, f32x4 (&acc)[8]) {
    constexpr int ET = elem_type(DT);
    using MQ = Mfma<ET>;
    using MP = Mfma<PULSE_BF16>;
    using vec = typename MQ::vec;
    const int col = lane & 15;
    const int grp = lane >> 4;
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run = -INFINITY;
    l_run = 0.f;
    if (ne <= 0) return;
    // entry metadata, one entry per lane; an entry without a block reads slot 0 and counts no token
    const int32_t j = lane < ne ? j_lane : -1;
    const int32_t sl = (j >= 0 && j < max_blocks) ? table[(size_t)r * max_blocks + j] : -1;
    const int ctx = ctx_len[r];
    const int64_t n_r = ((int64_t)ctx + BS - 1) / BS;
    int my_slot = 0, my_nv = 0;
    if (lane < ne) {
        if (j >= 0 && j < n_r && sl >= 0 && sl < n_slots) {
            my_slot = sl;
            const int64_t v = (int64_t)ctx - (int64_t)j * BS;
            my_nv = v >= BS ? BS : (int)v;
        } else {
            report(status, PULSE_ERR_BAD_INDEX);
        }
    }
    const uint64_t U = (uint64_t)kv8_block_bytes(Hkv, BS);
    // scales of the lane's own entry
    const uint32_t my_scales = *reinterpret_cast<const uint16_t*>(pool + (uint64_t)my_slot * U + kv8_scales(Hkv, BS) + 2 * h);
    const uint64_t whole = __ballot(my_nv == BS);
    // Q^T operand: channels 32 * grp + 8 * kc .. + 7 of the column's query head
    vec qb[4];
    {
        const uint16_t* qr = q + ((size_t)r * Hq + (size_t)h * G + col) * kHeadDim + grp * 32;
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) qb[kc] = col < G ? load_vec<ET>(qr + 8 * kc) : zero_vec<ET>();
    }
    // Step i covers tokens 32 i ..: K: MFMA row m = col is token 8 * (col / 4) + 4 * sub + col % 4; V: lane group grp
    // holds tokens 8 * grp .. + 7, channels col + 16 * t in unit t.
    constexpr int kPer = BS >= kChunkTokens ? 1 : kChunkTokens / BS;  // entries of a step
    constexpr int kHalves = BS > kChunkTokens ? BS / kChunkTokens : 1;  // steps of an entry
    const uint8_t* head = pool + (size_t)h * kv8_head_bytes(BS);
    const int k_tok = 8 * (col >> 2), v_tok = 8 * grp;
    const uint8_t* k_at = head + (k_tok % BS + (col & 3)) * kHeadDim + grp * 32;
    const uint8_t* v_at = head + kv8_values(BS) + v_tok % BS * kHeadDim + col * 64;
    const int steps = (ne * BS + kChunkTokens - 1) / kChunkTokens;

    u32x4 kw[2][2], vw[4];
    auto load_k = [&](int i) {
        const uint32_t slot = (uint32_t)__shfl(my_slot, i / kHalves * kPer + k_tok / BS);
        const uint8_t* kb = k_at + (uint64_t)slot * U + i % kHalves * kChunkTokens * kHeadDim;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int n = 0; n < 2; ++n) kw[sub][n] = reinterpret_cast<const u32x4*>(kb + 4 * sub * kHeadDim)[n];
    };
    auto load_v = [&](int i) {
        const uint32_t slot = (uint32_t)__shfl(my_slot, i / kHalves * kPer + v_tok / BS);
        const uint8_t* vb = v_at + (uint64_t)slot * U + i % kHalves * kChunkTokens * kHeadDim;
#pragma unroll
        for (int n = 0; n < 4; ++n) vw[n] = reinterpret_cast<const u32x4*>(vb)[n];
    };
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        load_k(i);
        load_v(i);
        u32x4 (&vn)[4] = vw;
        const int e0 = i / kHalves * kPer;
        const float ks = kv8_pow2((int)(__shfl((int)my_scales, e0 + k_tok / BS) & 255) - 127);
        float vs = kv8_pow2((__shfl((int)my_scales, e0 + v_tok / BS) >> 8) - 127);
        // --- S^T = K . Q^T
        f32x4 s[2] = {};
#pragma unroll
        for (int kc = 0; kc < 4; ++kc)
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                const u32x2 w = {kw[sub][kc / 2][2 * (kc % 2)], kw[sub][kc / 2][2 * (kc % 2) + 1]};
                s[sub] = MQ::mac(kv8_decode8<ET>(w, ks), qb[kc], s[sub]);
            }
        float x[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) x[n] = s[n / 4][n % 4] * scale_log2;
        // blocks that are not whole (the last of the context, a missing one, none behind an odd count): their other
        // tokens count nothing, whatever codes and scales are there
        if ((~whole >> e0) & ((1u << kPer) - 1)) {
            const int left = __shfl(my_nv, e0 + v_tok / BS) - v_tok % BS - i % kHalves * kChunkTokens;
            if (left <= 0) vs = 1.f;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                if (n >= left) x[n] = -INFINITY;
                const uint32_t keep = n >= left ? ~(255u << (8 * (n % 4))) : ~0u;
#pragma unroll
                for (int t = 0; t < 8; ++t) vn[t / 2][t % 2 * 2 + n / 4] &= keep;
            }
        }
        float cm = x[0];
#pragma unroll
        for (int n = 1; n < 8; ++n) cm = fmaxf(cm, x[n]);
        cm = across_groups(cm, [](float a, float b) { return fmaxf(a, b); });
        const float m_new = fmaxf(m_run, cm);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2_fast(m_run - m_use);
        float psum = 0.f;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            x[n] = exp2_fast(x[n] - m_use);
            psum += x[n];
        }
        l_run = l_run * alpha + psum;
        m_run = m_new;
        if (i > 0 && __ballot(alpha != 1.f)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float av = __shfl(alpha, 4 * grp + v);
#pragma unroll
                for (int t = 0; t < 8; ++t) acc[t][v] *= av;
            }
        }
        // --- O += P . V
        u32x4 part[3];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float a = x[2 * n], b = x[2 * n + 1];
#pragma unroll
            for (int m = 0; m < 3; ++m) {
                part[m][n] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
                a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
                b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
            }
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const u32x2 w = {vn[t / 2][t % 2 * 2], vn[t / 2][t % 2 * 2 + 1]};
            const bf16x8 v = kv8_decode8<PULSE_BF16>(w, vs);
#pragma unroll
            for (int m = 0; m < 3; ++m) acc[t] = MP::mac(__builtin_bit_cast(bf16x8, part[m]), v, acc[t]);
        }
    }
    l_run = across_groups(l_run, [](float a, float b) { return a + b; });
    // a split whose every logit is NaN (keys of NaN codes) keeps its weight in the merge
    if (m_run == -INFINITY && l_run != l_run) m_run = 0.f;
}

// grid = (Hkv, n_wg, B), or (Hkv, B, n_wg) with light_last; in either, workgroup p is piece p / Hkv of KV head
// p % Hkv of a plan; wave w of a request's workgroup wg owns split W * wg + w of eps entries.  Dynamic LDS:
// O [W][G][128] floats then (m, l) [W][G] float2.
// GP: rows of the P operand that a channel group of the 4-bit cache takes.  R: counts per lane of a plan (a kernel
// that held both plans was 1 to 2% slower for fetching its way past the other).
template <int DT, int BS, int W, int GP, int R>
__global__ __launch_bounds__(W * kWave) void attn_splitk_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ pool, int32_t n_slots,
    const int32_t* __restrict__ table, int32_t max_blocks, const int32_t* __restrict__ sel_idx,
    const int32_t* __restrict__ sel_cnt, int32_t k_max, const int32_t* __restrict__ ctx_len, int32_t B, int32_t Hq,
    int32_t Hkv, int32_t G, SplitArgs sp, float scale_log2, float* __restrict__ ws_o,
    float2* __restrict__ ws_ml, float* __restrict__ out, float* __restrict__ lse, __bf16* __restrict__ x,
    int32_t* status) {
    extern __shared__ float smem[];
    constexpr int kThreads = W * kWave;
    float* s_o = smem;                                                           // [W][G][128]
    float2* s_ml = reinterpret_cast<float2*>(smem + W * G * kHeadDim);  // [W][G]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int h = blockIdx.x;

    // this wave's selected blocks (one per lane) are loaded with the counts they depend on, at the place
    // they have when all counts are equal: one memory round trip fewer before the first K load
    Piece p;
    p.r = sp.light_last ? blockIdx.y : blockIdx.z;
    p.wg = sp.light_last ? blockIdx.z : blockIdx.y;
    p.eps = in_codes(DT) ? sp.even : sp.eps;
    int piece = p.r * sp.n_wg + p.wg;
    const bool planned = sp.planned;
    auto load_j = [&]() {
        const int e = (p.wg * W + wave) * p.eps + lane;
        return (lane < p.eps && e < k_max) ? sel_idx[(size_t)p.r * k_max + e] : -1;
    };
    int32_t j_lane = load_j();
    bool own = !planned;  // the host's split, cut at the request's own count
    int own_eps = sp.eps;
    if (planned) {
        const Counts<R> counts(sel_cnt, B, lane);
        if (piece == 0 && h == 0 && wave == 0 && counts.any(B, lane, [&](int32_t c) { return c < 0 || c > k_max; }) &&
            lane == 0)
            report(status, PULSE_ERR_BAD_INDEX);
        p.cnt = k_max;
        p.nwg = in_codes(DT) ? sp.n_even : sp.n_wg;
        if (counts.equal(B, k_max, lane)) {
            if (in_codes(DT) && p.wg >= p.nwg) return;
        } else if (in_codes(DT) && (!sp.share || (sp.level && counts.level(B, k_max)))) {
            own = true;
            if (sp.share) own_eps = sp.even;
        } else {
            const int r0 = p.r, wg0 = p.wg, eps0 = p.eps;
            piece = (int)(blockIdx.z * gridDim.y + blockIdx.y);
            p = plan_piece(piece, 0, counts, B, k_max, W, sp, lane);
            if (p.r < 0) return;  // fewer pieces than workgroups
            if (p.r != r0 || p.wg != wg0 || p.eps != eps0) j_lane = load_j();
        }
    }
    if (own) {
        p.cnt = sel_cnt[p.r];
        if (in_codes(DT) && p.eps != own_eps) {
            p.eps = own_eps;
            j_lane = load_j();
        }
        if (p.cnt < 0 || p.cnt > k_max) {
            if (tid == 0) report(status, PULSE_ERR_BAD_INDEX);
            p.cnt = 0;
        }
        p.nwg = pieces_of(p.cnt, W * p.eps);
        if (p.wg >= p.nwg) return;
    }
    const int r = p.r;
    float* out_rh = out + ((size_t)r * Hq + (size_t)h * G) * kHeadDim;
    float* lse_rh = lse ? lse + (size_t)r * Hq + (size_t)h * G : nullptr;
    __bf16* x_rh = x ? x + ((size_t)r * Hq + (size_t)h * G) * kHeadDim : nullptr;
    if (p.cnt == 0) {  // empty selection: out = 0, lse = -inf
        for (int i = tid; i < G * kHeadDim; i += kThreads) {
            out_rh[i] = 0.f;
            if (x_rh) x_rh[i] = (__bf16)0.f;
        }
        if (lse_rh && tid < G) lse_rh[tid] = -INFINITY;
        return;
    }
    const int ne = min(p.eps, p.cnt - (p.wg * W + wave) * p.eps);
    float m_run, l_run;
    f32x4 acc[8];
    if constexpr (is_kv4(DT))
        attend_split_kv4<DT, BS, GP>(q, reinterpret_cast<const uint8_t*>(pool), n_slots, table, max_blocks, j_lane,
                                     ctx_len, Hq, Hkv, G, r, h, ne, scale_log2, status, lane, m_run, l_run, acc);
    else if constexpr (is_kv8(DT))
        attend_split_kv8<DT, BS>(q, reinterpret_cast<const uint8_t*>(pool), n_slots, table, max_blocks, j_lane, ctx_len,
                                 Hq, Hkv, G, r, h, ne, scale_log2, status, lane, m_run, l_run, acc);
    else
        attend_split<DT, BS>(q, pool, n_slots, table, max_blocks, j_lane, ctx_len, Hq, Hkv, G, r, h, ne, scale_log2,
                             status, lane, m_run, l_run, acc);
    // wave partials to LDS
    if (grp == 0 && col < G) s_ml[wave * G + col] = make_float2(m_run, l_run);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int g = (4 * grp + v) % GP;
        if (g < G) {
            float* o = s_o + (wave * G + g) * kHeadDim + col;
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (GP == 16 || t / 2 % (16 / GP) == (4 * grp + v) / GP) o[16 * t] = acc[t][v];
        }
    }
    __syncthreads();
    // merge the W waves: thread handles outputs (g, c) = (idx / 128, idx % 128)
    const size_t unit = (size_t)piece * Hkv + h;
    for (int idx = tid; idx < G * kHeadDim; idx += kThreads) {
        const int g = idx / kHeadDim, c = idx % kHeadDim;
        float Mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) Mx = fmaxf(Mx, s_ml[w * G + g].x);
        float L = 0.f, a = 0.f;
        if (Mx != -INFINITY) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 ml = s_ml[w * G + g];
                const float wt = ml.x == -INFINITY ? 0.f : exp2_fast(ml.x - Mx);
                L += ml.y * wt;
                a += s_o[(w * G + g) * kHeadDim + c] * wt;
            }
        }
        if (p.nwg == 1) {
            const float o = Mx == -INFINITY ? 0.f : a / L;
            out_rh[idx] = o;
            if (x_rh) x_rh[idx] = (__bf16)o;
            if (lse_rh && c == 0) lse_rh[g] = Mx == -INFINITY ? -INFINITY : (Mx + log2f(L)) * 0.69314718055994531f;
        } else {
            ws_o[unit * G * kHeadDim + idx] = a;
            if (c == 0) ws_ml[unit * G + g] = make_float2(Mx, L);
        }
    }
}

// Merge the workgroup partials of one (request, KV head, query head):
// grid = (G, Hkv, B), 128 threads, thread c owns output channel c.  Partials
// are read 8 at a time (16 independent loads per thread) and merged online:
// 2 to 4 us up to 8 of them, 9 for 64 and 29 for 256 (4 and 1 requests of 64K
// tokens in the 4-bit cache of one KV head).
// Requests whose selection fits one workgroup were finished by the attention
// kernel.
// R: counts per lane of a plan.
template <int R>
__global__ __launch_bounds__(kCombineThreads) void attn_combine_kernel(
    const float* __restrict__ ws_o, const float2* __restrict__ ws_ml, const int32_t* __restrict__ sel_cnt,
    int32_t k_max, int32_t B, int32_t Hq, int32_t Hkv, int32_t G, SplitArgs sp, int32_t waves,
    float* __restrict__ out, float* __restrict__ lse, __bf16* __restrict__ x) {
    const int c = threadIdx.x, g = blockIdx.x, h = blockIdx.y, r = blockIdx.z;
    // piece i of this (request, head) is partial (base + i) * Hkv + h; with equal counts base = r * n_wg.
    // The first 8 are loaded there before the counts are known, and again if the base differs (later where equal
    // counts leave nothing to merge).
    const float2* ml = ws_ml + (size_t)h * G + g;
    const float* po = ws_o + ((size_t)h * G + g) * kHeadDim + c;
    float2 mlv[8];
    float ov[8];
    auto load8 = [&](int first, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const size_t u = (size_t)(first + i) * Hkv * G;
            mlv[i] = i < n ? ml[u] : make_float2(-INFINITY, 0.f);
            ov[i] = i < n ? po[u * kHeadDim] : 0.f;
        }
    };
    const bool ahead = sp.n_even > 1;
    if (ahead) load8(r * sp.n_wg, sp.n_wg);
    int nwg, base = r * sp.n_wg;
    bool own = !sp.planned;
    int own_eps = sp.eps;
    if (sp.planned) {
        const int lane = c & 63;
        const Counts<R> counts(sel_cnt, B, lane);
        nwg = sp.n_even;
        if (!counts.equal(B, k_max, lane)) {
            if (sp.level && sp.share && counts.level(B, k_max)) {
                own = true;
                own_eps = sp.even;
            } else if (sp.share) {
                const Piece p = plan_piece(-1, r, counts, B, k_max, waves, sp, lane);
                nwg = p.nwg;
                base = p.base;
            } else {
                own = true;
            }
        }
    }
    if (own) {
        const int32_t cnt = sel_cnt[r];
        nwg = (cnt < 0 || cnt > k_max) ? 1 : pieces_of(cnt, waves * own_eps);
    }
    if (nwg <= 1) return;
    if (!ahead || base != r * sp.n_wg || nwg > sp.n_wg) load8(base, nwg);
    float m_run = -INFINITY, L = 0.f, a = 0.f;
    for (int w0 = 0; w0 < nwg; w0 += 8) {
        if (w0 > 0) {
            load8(base + w0, nwg - w0);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= nwg) {  // not written by this call
                    mlv[i] = make_float2(-INFINITY, 0.f);
                    ov[i] = 0.f;
                }
        }
        float cm = m_run;
#pragma unroll
        for (int i = 0; i < 8; ++i) cm = fmaxf(cm, mlv[i].x);
        if (cm == -INFINITY) continue;
        const float alpha = m_run == -INFINITY ? 0.f : exp2f(m_run - cm);
        L *= alpha;
        a *= alpha;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float wt = mlv[i].x == -INFINITY ? 0.f : exp2f(mlv[i].x - cm);
            L += mlv[i].y * wt;
            a += ov[i] * wt;
        }
        m_run = cm;
    }
    const size_t at = ((size_t)r * Hq + (size_t)h * G + g) * kHeadDim + c;
    const float o = m_run == -INFINITY ? 0.f : a / L;
    out[at] = o;
    if (x) x[at] = (__bf16)o;
    if (lse && c == 0)
        lse[(size_t)r * Hq + (size_t)h * G + g] =
            m_run == -INFINITY ? -INFINITY : (m_run + log2f(L)) * 0.69314718055994531f;
}

// Whether requests and heads alone are more than a round of workgroups, and few enough for a plan.
static bool over_a_round(const pulse_shape& s, int32_t B) {
    return in_codes(s.dtype) && B <= kPlanRequestsCodes && B > PULSE_ATTN_TARGET_WAVES / (kCodeWaves * s.num_kv_heads);
}

AttnPlan attn_plan(const pulse_shape& s, int32_t B, int32_t k_max) {
    // a split covers whole 32-token steps, at least two, and at most 64 entries
    const int32_t step = split_step(s.block_size);
    const int64_t units = (int64_t)B * s.num_kv_heads;
    const int64_t target_waves = PULSE_ATTN_TARGET_WAVES;  // one round at 2 resident waves per SIMD on 256 CUs
    int64_t want = units > 0 ? (target_waves + units - 1) / units : 1;
    const int64_t min_entries = split_least(s);
    int64_t max_split = (k_max + min_entries - 1) / min_entries;
    if (want > max_split) want = max_split;
    if (want < 1) want = 1;
    if (in_codes(s.dtype)) {
        // All waves of a workgroup have work, however many requests there are: the CU's other workgroups do not make
        // up for idle waves.  1000 tokens of 8 heads, in us, one round of waves and this: 64 requests 20.8 and 22.6
        // (lognormal 41.3 and 34.7), 96 32.7 and 29.4, 128 49.8 and 36.5, 256 143 and 69.
        want = std::max(want, std::min<int64_t>(max_split, kCodeWaves));
        if (want > kCodeWaves && k_max <= one_group_entries(s, units)) want = kCodeWaves;
        if (over_a_round(s, B) && (int64_t)k_max * s.block_size >= kOverTokens)
            want = std::max<int64_t>(want, 2 * kCodeWaves);
    }
    int64_t eps = (k_max + want - 1) / want;
    eps = ((eps + step - 1) / step) * step;
    if (eps > 64) eps = 64;
    if (eps < 1) eps = 1;
    AttnPlan p;
    p.entries_per_split = (int32_t)eps;
    p.n_split = (int32_t)((k_max + eps - 1) / eps);
    return p;
}

int64_t attn_partials(const pulse_shape& s, int32_t B, int32_t k_max) {
    const int W = attn_waves(s, B, k_max);
    return (int64_t)B * s.num_kv_heads * ((attn_plan(s, B, k_max).n_split + W - 1) / W);
}

// A workspace serves smaller calls too, and those may take more workgroups than a larger one: a batch that fills a
// round less well, a k_max that divides into more splits, a batch small enough for a plan.  Both bounds grow with B
// and k_max: no more workgroups than shortest splits fill; and no more splits than waves aimed at, one short of them
// each request and head more, or those of 64 entries, each request and head's last workgroup not full; and the second
// workgroups of a plan beyond a round.
int64_t attn_partials_most(const pulse_shape& s, int32_t B, int32_t k_max) {
    const bool kv4 = in_codes(s.dtype);
    const int64_t W = s.num_q_heads / s.num_kv_heads <= 8 || kv4 ? 8 : 4;
    const int64_t units = (int64_t)B * s.num_kv_heads, least = split_least(s);
    const int64_t shortest = units * (((k_max + least - 1) / least + 3) / 4);
    const int64_t splits = std::max(PULSE_ATTN_TARGET_WAVES + units, units * (((int64_t)k_max + 63) / 64));
    const int64_t second = kv4 ? std::min<int64_t>(units, (int64_t)kPlanRequestsCodes * s.num_kv_heads) : 0;
    return std::min(std::max(shortest, units), splits / W + units + second);
}

// `done` (optional): the kernel's stop event, carried by the launch.
template <int DT, int BS, int W, int GP = kMaxGroup>
static void launch_attn_t(dim3 grid, size_t lds, hipStream_t st, hipEvent_t done, const void* q, const void* pool,
                          int32_t n_slots, const int32_t* table, int32_t max_blocks, const int32_t* sel_idx,
                          const int32_t* sel_cnt, int32_t k_max, const int32_t* ctx_len, int32_t B, int32_t Hq,
                          int32_t Hkv, int32_t G, const SplitArgs& sp, float scale_log2, float* ws_o, float2* ws_ml,
                          float* out, float* lse, __bf16* x, int32_t* status) {
    constexpr int kMany = in_codes(DT) ? kPlanRequestsCodes / kWave : 1;
    const auto kernel =
        B <= kPlanRequests ? attn_splitk_kernel<DT, BS, W, GP, 1> : attn_splitk_kernel<DT, BS, W, GP, kMany>;
    launch_timed(kernel, grid, dim3(W * kWave), (uint32_t)lds, st, nullptr, done,
                 (const uint16_t*)q, (const uint16_t*)pool, n_slots, table, max_blocks, sel_idx, sel_cnt, k_max,
                 ctx_len, B, Hq, Hkv, G, sp, scale_log2, ws_o, ws_ml, out, lse, x, status);
}

hipError_t launch_attention(const pulse_shape& s, const void* q, const void* pool, int32_t n_slots,
                            const int32_t* table, int32_t max_blocks, const int32_t* sel_idx, const int32_t* sel_cnt,
                            int32_t k_max, const int32_t* ctx_len, int32_t B, float sm_scale, float* out, float* lse,
                            float* ws_o, float2* ws_ml, int32_t* status, hipStream_t st, hipEvent_t split_done,
                            hipEvent_t done, __bf16* x) {
    if (B == 0) return hipSuccess;
    const int32_t Hkv = s.num_kv_heads, Hq = s.num_q_heads, G = Hq / Hkv;
    const AttnPlan p = attn_plan(s, B, k_max);
    const int W = attn_waves(s, B, k_max);
    const int32_t n_wg = (p.n_split + W - 1) / W;
    SplitArgs sp;
    sp.eps = p.entries_per_split;
    sp.n_wg = n_wg;
    sp.step = split_step(s.block_size);
    sp.least = split_least(s);
    const int64_t all = (int64_t)B * n_wg;
    const int32_t round = PULSE_ATTN_TARGET_WAVES / (W * Hkv);  // pieces of one round
    sp.fit = (int32_t)(4 * (int64_t)round >= 5 * (int64_t)B && round < all ? round : all);
    sp.even = sp.eps;  // (other than eps only where all > round and eps < 64, hence under a plan)
    sp.n_even = n_wg;
    sp.most = sp.eps;
    sp.level = false;
    if (in_codes(s.dtype)) {
        sp.most = 64;
        const bool over = over_a_round(s, B);
        sp.level = over && 4 * (int64_t)((B + round - 1) / std::max(round, 1)) * round <= 5 * (int64_t)B;
        // workgroups of a request in one round
        const int32_t each = over ? 1 : B <= kPlanRequestsCodes ? round / B : 0;
        if (each >= 1 && n_wg > each) {
            const int64_t eps = ((int64_t)k_max + W * each - 1) / (W * each);
            const int32_t even = (int32_t)std::min<int64_t>((eps + sp.step - 1) / sp.step * sp.step, sp.most);
            const int32_t last = (p.n_split - 1) % W + 1;  // waves of a request's last workgroup
            if (over || (int64_t)even * W <= (int64_t)sp.eps * (W + last)) {
                sp.even = even;
                sp.n_even = (int32_t)((((int64_t)k_max + even - 1) / even + W - 1) / W);
            }
        }
    }
    sp.share = B <= kPlanRequests || (int64_t)k_max * s.block_size >= kPlanTokensCodes;
    if (B <= kPlanRequests) sp.planned = sp.eps >= 2 * sp.least || all > round;
    else sp.planned = in_codes(s.dtype) && B <= kPlanRequestsCodes && (sp.share || sp.even != sp.eps);
    sp.planned = sp.planned && n_wg > 1 && k_max <= (1 << 22);
    sp.light_last = (p.n_split % W != 0 || sp.even != sp.eps) && all > round && n_wg <= 65535;
    const dim3 grid = sp.light_last ? dim3((unsigned)Hkv, (unsigned)B, (unsigned)n_wg)
                                    : dim3((unsigned)Hkv, (unsigned)n_wg, (unsigned)B);
    const size_t lds = sizeof(float) * W * G * kHeadDim + sizeof(float2) * W * G;
    const float scale_log2 = sm_scale * 1.4426950408889634f;
    // stop event of the split-K kernel: split_done, or `done` when no combine follows it
    const hipEvent_t splitk_stop = split_done ? split_done : (n_wg <= 1 ? done : nullptr);
#define PULSE_ATTN(...)                                                                                              \
    launch_attn_t<__VA_ARGS__>(grid, lds, st, splitk_stop, q, pool, n_slots, table, max_blocks, sel_idx, sel_cnt,   \
                               k_max, ctx_len, B, Hq, Hkv, G, sp, scale_log2, ws_o, ws_ml, out, lse, x, status)
#define PULSE_ATTN_W(DT, BS) \
    if (W == 8) PULSE_ATTN(DT, BS, 8); else PULSE_ATTN(DT, BS, 4)
#define PULSE_ATTN_KV4(DT, BS)                \
    if (G <= 4) PULSE_ATTN(DT, BS, 8, 4);      \
    else if (G <= 8) PULSE_ATTN(DT, BS, 8, 8); \
    else if (W == 8) PULSE_ATTN(DT, BS, 8, 16); \
    else PULSE_ATTN(DT, 64, 4, 16)
#define PULSE_ATTN_KV8(DT, BS)                \
    if (W == 8) PULSE_ATTN(DT, BS, 8, 16);    \
    else PULSE_ATTN(DT, 64, 4, 16)
#define PULSE_ATTN_BS(WHICH, DT)                   \
    if (s.block_size == 16) { WHICH(DT, 16); }      \
    else if (s.block_size == 32) { WHICH(DT, 32); } \
    else { WHICH(DT, 64); }
    if (s.dtype == PULSE_BF16) { PULSE_ATTN_BS(PULSE_ATTN_W, PULSE_BF16) }
    else if (s.dtype == PULSE_F16) { PULSE_ATTN_BS(PULSE_ATTN_W, PULSE_F16) }
    else if (s.dtype == PULSE_BF16_KV8) { PULSE_ATTN_BS(PULSE_ATTN_KV8, PULSE_BF16_KV8) }
    else if (s.dtype == PULSE_F16_KV8) { PULSE_ATTN_BS(PULSE_ATTN_KV8, PULSE_F16_KV8) }
    else if (s.dtype == PULSE_BF16_KV4) { PULSE_ATTN_BS(PULSE_ATTN_KV4, PULSE_BF16_KV4) }
    else { PULSE_ATTN_BS(PULSE_ATTN_KV4, PULSE_F16_KV4) }
#undef PULSE_ATTN_BS
#undef PULSE_ATTN_KV8
#undef PULSE_ATTN_KV4
#undef PULSE_ATTN_W
#undef PULSE_ATTN
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (n_wg <= 1) return (done && split_done) ? hipEventRecord(done, st) : hipSuccess;
    const auto combine = B <= kPlanRequests ? attn_combine_kernel<1> : attn_combine_kernel<kPlanRequestsCodes / kWave>;
    launch_timed(combine, dim3((unsigned)G, (unsigned)Hkv, (unsigned)B), dim3(kCombineThreads), 0u, st, nullptr, done,
                 (const float*)ws_o, (const float2*)ws_ml, sel_cnt, k_max, B, Hq, Hkv, G, sp, W, out, lse, x);
    return hipGetLastError();
}

}  // namespace pulse

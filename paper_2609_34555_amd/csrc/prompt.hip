// prompt.hip -- attention of new tokens (whole prompts, or the last tokens of longer contexts) over the slot pool, for
// gfx950.  Token i of request r's new tokens stands at position p = ctx - new + i and attends to tokens 0 .. p.
//
// The G query heads of a KV head share its keys and values, so the rows of the contraction are (token, query head of the
// group) in this order: row m is token m / G, head m % G.  A workgroup takes W * 32 rows, a wave 32 of them, and goes
// through the context in tiles of 64 keys that are staged in LDS, the next one while this one is multiplied:
//   S^T[64 keys x 32 rows]     = K[64 x 128] . Q^T[128 x 32]
//   O^T[128 channels x 32 rows] += V^T[128 x 64] . P^T[64 x 32]
// on v_mfma_f32_32x32x16.  With the rows of the K operand assigned to keys by key_of_row, a lane's accumulators of S^T
// are its operand of the second product: probabilities never leave its registers, and as the accumulators of O^T have
// the same column, maxima, sums and rescaling are a lane's own but for one exchange between the wave's halves.  Keys lie
// token by token and values channel by channel in the 16-bit cache, which is what either operand takes, so no tile is
// transposed.  The same sums for 32 rows, whose keys a workgroup's waves share out, are prompt_few_kernel; either may be
// split over the context, and prompt_join_kernel adds up the splits.
//
// Precision: products of 16-bit factors, exact, summed in fp32; maxima, sums and rescaling in fp32.  Probabilities are
// rounded to the 16-bit type for the second product (half a step of it at most, beside half a step of the output's own
// rounding to the same type; in prompt_few_kernel mostly in two parts); their sum is that of the values before rounding.
// In two parts here too, half as many products again: 8 prompts of 501 to 16000 tokens 7276 us for 5345, 2048 tokens 64.9 for
// 51.5; the error against 64 bits (2-norm, 1000 tokens) would be the results' own rounding, 1.63e-3 for 2.07e-3 in bf16 and
// 2.04e-4 for 2.58e-4 in fp16.
#include <algorithm>
#include <type_traits>

#include "kv4.h"
#include "kv8.h"

namespace pulse {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kKeys = 64;                     // keys of a tile
constexpr int kRowsPerWave = 32;
constexpr int kWaves = 4;                     // of a workgroup; twice as many for long prompts
constexpr int kTileBytes = kKeys * kHeadDim * 2;  // of keys, and of values, in LDS

// What is subtracted from logits (base 2) is their maximum less this.  In fp16, whose normal numbers end at 2^-14,
// probabilities of up to 2^(7 + 8) (see `prepare`), so that those of 2^-21 and more keep all their bits, and what tens of
// thousands of smaller ones lose together stays below 2^-16.
template <int ET>
constexpr float kLift = ET == PULSE_F16 ? 7.f : 0.f;

template <int ET>
__device__ inline f32x16 mac32(typename Mfma<ET>::vec a, typename Mfma<ET>::vec b, f32x16 c) {
    if constexpr (ET == PULSE_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Two floats as 16-bit values, rounded to nearest.
template <int ET>
__device__ inline uint32_t pack2(float a, float b) {
    if constexpr (ET == PULSE_BF16) {
        const bf16x2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        const f16x2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}

// Key (of 32) that row m of the K operand holds: accumulator register 4 b + i of lane half h is row 8 b + 4 h + i, and
// the operand of 16 keys takes 8 h + 0 .. 7 from half h.
__device__ constexpr int key_of_row(int m) { return 16 * (m >> 4) + 8 * (m >> 2 & 1) + 4 * (m >> 3 & 1) + (m & 3); }

// Places of 16-byte pieces in the LDS tiles, changed so that the lanes that read together read different banks.
// Keys: piece c of a key's 16.  Values: octet o of the BS / 8 that a block has of a channel.
__device__ inline int key_piece(int key, int c) { return c ^ ((key & 3) | (key >> 3 & 1) << 2 | (key >> 2 & 1) << 3); }
template <int BS>
__device__ inline int value_octet(int c, int o) {
    if constexpr (BS == 16) return o ^ ((c >> 2 ^ c >> 3) & 1);
    else if constexpr (BS == 32) return o ^ ((c >> 1 ^ (c >> 3 & 1)) & 3);
    else return o ^ ((c ^ (c >> 3 & 1)) & 7);  // (bits of c below 32 alone: lanes read channels 32 apart at one distance)
}

// Codes of byte t of w times `scale`, as two 16-bit values.
template <int ET>
__device__ inline uint32_t kv4_pair(uint32_t w, int t, float scale) {
    return t == 0 ? kv4_decode<ET, 0>(w, scale) : t == 1 ? kv4_decode<ET, 1>(w, scale)
         : t == 2 ? kv4_decode<ET, 2>(w, scale) : kv4_decode<ET, 3>(w, scale);
}

struct PromptArgs {
    const uint16_t* q;
    int64_t q_stride;
    const int32_t* tok_off;
    const int32_t* ctx_len;
    int32_t B, max_tokens;
    const uint8_t* pool;
    int32_t n_slots;
    const int32_t* table;
    int32_t max_blocks;
    int32_t max_ctx;        // tokens of max_blocks blocks
    int32_t Hkv, G;
    uint64_t g_magic;       // m / G = m * g_magic >> 32 for rows m below 2^28
    float scale_log2;
    uint16_t* out;
    int64_t out_stride;
    float* lse;
    float* ws_o;            // [n_split][max_tokens * Hq][128]
    float2* ws_ml;
    int32_t* ws_n;          // [max_tokens * Hq] splits of a row, 1 where its result is written already
    int32_t n_tiles, n_split;
    float tile_us, split_us;  // (splits_worth)
    int32_t* status;
};

// The request and tile of rows that a place in the grid stands for.  Request r's tiles take places first(r) = tok_off[r]
// * G / rows + r and on: as many as it needs are free before first(r + 1), so no sum over the requests is needed.
struct Place {
    int r, tile;
};
__device__ inline Place find_place(const int32_t* __restrict__ tok_off, int32_t B, int32_t G, int rows, int at) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if ((int64_t)tok_off[mid] * G / rows + mid <= at) lo = mid;
        else hi = mid - 1;
    }
    return Place{lo, at - (int)((int64_t)tok_off[lo] * G / rows + lo)};
}

// Slots of a tile's blocks.  (Four by name, of which the first kKeys / BS count: an array would not stay in registers.)
struct Slots {
    int s0, s1, s2, s3;
    uint32_t bad;  // blocks without a slot
    __device__ inline int operator[](int i) const {  // of a wave-uniform i
        return i == 0 ? s0 : i == 1 ? s1 : i == 2 ? s2 : s3;
    }
};

// What a workgroup of `rows` rows has to know of its request.  Workgroup 0 looks at every request's lengths.
struct Request {
    bool any, ok;  // whether it has a row; whether its lengths are right (else no token is attended to)
    int t0, ctx, base;  // its first row, its tokens, the tokens before its first new one
    int64_t n_rows, row0;
};
__device__ inline Request look_at(const PromptArgs& a, const Place& pl, int rows, int threads) {
    Request q;
    q.t0 = a.tok_off[pl.r];
    const int t1 = a.tok_off[pl.r + 1];
    q.ctx = a.ctx_len[pl.r];
    if (blockIdx.x == 0) {
        for (int r = threadIdx.x; r < a.B; r += threads) {
            const int64_t x = a.tok_off[r], y = a.tok_off[r + 1], c = a.ctx_len[r];
            if (x < 0 || y < x || y > a.max_tokens || c < y - x || c > a.max_ctx)
                report(a.status, PULSE_ERR_BAD_INDEX);
        }
    }
    const int fresh = t1 - q.t0;
    q.n_rows = (int64_t)fresh * a.G;
    q.row0 = (int64_t)pl.tile * rows;
    q.any = !(q.t0 < 0 || t1 < q.t0 || t1 > a.max_tokens) && !(pl.tile < 0 || q.row0 >= q.n_rows);
    q.ok = q.ctx >= fresh && q.ctx <= a.max_ctx;
    q.base = q.ctx - fresh;
    return q;
}

// Splits that pay for a context: n of them leave 1/n of a workgroup's time, `tile_us` a tile of keys (1.2 for 128 rows; for
// 32 0.5, 0.3 over a cache of codes), and cost partials that are written and read, `split_us` a split (1 KiB a row of the
// call, 7 TB/s) and a launch.  Looked at for the whole table when a launch is planned, and for what a workgroup attends to
// by itself: short contexts in a wide table, and the first tiles of a prompt, are not split (256 tokens in a table of 32K,
// 16 bits: 19.0 us and 12.7, of 8.0 in a table that fits; where all contexts are long it costs the join half a microsecond).
constexpr int kLeastTiles = 4;  // tiles of keys of a split
__host__ __device__ inline int splits_worth(int tiles, float tile_us, float split_us, int most) {
    const float us = (float)tiles * tile_us;
    const int n = min(min((int)sqrtf(us / split_us), most), tiles / kLeastTiles);
    return n < 2 || us - us / (float)n < 3.f + (float)n * split_us ? 1 : n;
}

// The 16 KiB of a tile's keys, or of its values, into LDS from 16-bit blocks: 1 KiB a wave and instruction, straight from
// memory.  A lane's place within a block is the same for every tile.
template <int BS, int W>
struct Stage16 {
    static constexpr int kParts = kTileBytes / 1024;
    static constexpr int kBlockParts = kParts / (kKeys / BS);  // of a block
    static constexpr int kPlaces = kBlockParts > W ? kBlockParts / W : 1;
    uint32_t k_at[kPlaces], v_at[kPlaces];
    uint32_t E;

    __device__ inline Stage16(const PromptArgs& a, int h, int wave, int lane) {
        E = (uint32_t)a.Hkv * BS * kHeadDim * 4;
        constexpr int kOct = BS / 8;
#pragma unroll
        for (int i = 0; i < kPlaces; ++i) {
            const int in = (i * W + wave) % kBlockParts;
            const int key = in * 4 + (lane >> 4);
            k_at[i] = (uint32_t)h * BS * kHeadDim * 2 + key * 256 + key_piece(key % 32, lane & 15) * 16;
            const int c = in * (64 / kOct) + lane / kOct;
            v_at[i] = (uint32_t)(a.Hkv + h) * BS * kHeadDim * 2 + (c * kOct + value_octet<BS>(c, lane % kOct)) * 16;
        }
    }
    template <bool K>
    __device__ inline void tile(const PromptArgs& a, const Slots& slot, uint8_t* lds, int wave) const {
#pragma unroll
        for (int i = 0; i < kParts / W; ++i) {
            const int part = i * W + wave;
            // (of W waves that share a block the index is a constant)
            const int s = slot[kBlockParts >= W ? i * W / kBlockParts : part / kBlockParts];
            const uint8_t* src = a.pool + (uint64_t)(uint32_t)s * E;
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*)(src + (K ? k_at : v_at)[i % kPlaces]),
                (__attribute__((address_space(3))) void*)(lds + part * 1024), 16, 0, 0);
        }
    }
};

// The same from 8-bit or 4-bit blocks: fetch() loads codes and scales, a 16-byte piece at a time, into registers; put()
// decodes them, exactly, into the 16-bit type and writes what Stage16 would have written.  Decoding costs a workgroup
// once what W waves then use.
template <int DT, int BS, int W>
struct StageCodes {
    static constexpr int ET = elem_type(DT);
    static constexpr int kThreads = W * kWave;
    static constexpr bool k4 = is_kv4(DT);
    static constexpr int kUnits = kKeys * kHeadDim / (k4 ? 32 : 16);  // pieces of a tile
    static constexpr int kEach = (kUnits + kThreads - 1) / kThreads;
    static constexpr int kPer = k4 ? 4 : 8;  // pieces of a key
    u32x4 k[kEach], v[kEach];
    uint32_t ks[kEach], vs[kEach];  // scale byte of a piece's keys, and (8 bits) values
    u32x2 vs4[kEach][2];            // 4 bits: scale bytes of 8 tokens, of the piece's two channel groups
    const uint8_t* head;
    uint64_t U;

    __device__ inline StageCodes(const PromptArgs& a, int h, int, int) {
        U = k4 ? (uint64_t)a.Hkv * kv4_head_bytes(BS) : (uint64_t)kv8_block_bytes(a.Hkv, BS);
        head = a.pool + (size_t)h * (k4 ? kv4_head_bytes(BS) : kv8_head_bytes(BS));
    }

    // Piece u of keys: of key u / kPer; of values: of octet u / (kUnits / 8).  A wave's pieces lie in one block.
    template <bool K>
    __device__ inline void fetch(const PromptArgs& a, const Slots& slot, int h, int tid) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = i * kThreads + tid;
            if (kUnits % kThreads && u >= kUnits) break;
            const int key = u / kPer, oct = u / (kUnits / 8);
            const uint64_t at = (uint64_t)(uint32_t)slot[__builtin_amdgcn_readfirstlane((K ? key : oct * 8) / BS)] * U;
            const uint8_t* b = head + at;
            if constexpr (k4 && K) {
                k[i] = *reinterpret_cast<const u32x4*>(b + key % BS * 64 + u % 4 * 16);
                ks[i] = b[kv4_key_scales(BS) + key % BS * kv4_scales_per_token() + u % 4];
            } else if constexpr (k4) {
                const int p = u % 32;  // channels p / 2 + 16 * (4 * (p % 2) + 0 .. 3)
                v[i] = *reinterpret_cast<const u32x4*>(b + kv4_values(BS) + oct % (BS / 8) * 512 + p * 16);
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    vs4[i][n] = *reinterpret_cast<const u32x2*>(b + kv4_value_scales(BS) + (2 * (p % 2) + n) * BS +
                                                                oct % (BS / 8) * 8);
            } else {
                const uint8_t scale = a.pool[at + kv8_scales(a.Hkv, BS) + 2 * h + (K ? 0 : 1)];
                if constexpr (K) {
                    k[i] = *reinterpret_cast<const u32x4*>(b + key % BS * kHeadDim + u % 8 * 16);
                    ks[i] = scale;
                } else {  // channels u % 64 / 4 + 16 * (2 * (u % 4) + 0 .. 1)
                    v[i] = *reinterpret_cast<const u32x4*>(b + kv8_values(BS) + oct % (BS / 8) * 1024 + u % 64 * 16);
                    vs[i] = scale;
                }
            }
        }
    }

    template <bool K>
    __device__ inline void put(uint8_t* lds, int tid) const {
        constexpr int kOct = BS / 8;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = i * kThreads + tid;
            if (kUnits % kThreads && u >= kUnits) break;
            const int key = u / kPer, oct = u / (kUnits / 8);
#pragma unroll
            for (int n = 0; n < 32 / kPer / 2; ++n) {
                u32x4 w;
                if constexpr (K) {
                    if constexpr (k4) w = __builtin_bit_cast(u32x4, kv4_decode8<ET>(k[i][n], kv4_scale(ks[i])));
                    else w = __builtin_bit_cast(u32x4, kv8_decode8<ET>(u32x2{k[i][2 * n], k[i][2 * n + 1]},
                                                                       kv8_pow2((int)ks[i] - 127)));
                    *reinterpret_cast<u32x4*>(lds + key * 256 + key_piece(key % 32, u % kPer * (16 / kPer) + n) * 16) = w;
                } else {
                    int c;
                    if constexpr (k4) {
                        c = u % 32 / 2 + 16 * (4 * (u % 2) + n);
                        const u32x2 sb = vs4[i][n / 2];  // a scale for each of the 8 tokens
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const float s0 = kv4_scale(sb[t / 2] >> (16 * (t % 2)) & 255u);
                            const float s1 = kv4_scale(sb[t / 2] >> (16 * (t % 2) + 8) & 255u);
                            w[t] = (kv4_pair<ET>(v[i][n], t, s0) & 0xFFFFu) | (kv4_pair<ET>(v[i][n], t, s1) & 0xFFFF0000u);
                        }
                    } else {
                        c = u % 64 / 4 + 16 * (2 * (u % 4) + n);
                        w = __builtin_bit_cast(u32x4, kv8_decode8<ET>(u32x2{v[i][2 * n], v[i][2 * n + 1]},
                                                                      kv8_pow2((int)vs[i] - 127)));
                    }
                    *reinterpret_cast<u32x4*>(lds + oct / kOct * (256 * BS) + (c * kOct + value_octet<BS>(c, oct % kOct)) * 16) = w;
                }
            }
        }
    }

    __device__ static constexpr int kv4_scales_per_token() { return kHeadDim / kGroup; }
};

// This wave's pieces are in LDS, and so are the others', which are done with the other tile.
__device__ inline void tile_arrived() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Bound: the matrix units, 4 * 128 operations a row and key, and beside them the vector units (an exponential, a
// maximum, a sum, half a conversion a row and key).  8 prompts of 501 to 16000 tokens, 32 heads over 8 (5.75 TFLOP): 5.25 to
// 5.5 ms, 1.05 PFLOP/s, of 1.31 to 1.39 that a large product reaches; 4096 tokens at the end of 32K in 4 bits 1.9 ms, the
// same rate.  Counted there: matrix units busy 51% of the cycles, 23% with vector instructions beside them; vector
// instructions 45%; LDS reads 26%; waves waiting for memory, LDS or a barrier 34%; no LDS conflict, 92% of the reads from L2;
// a clock that the load holds at 2.0 GHz.  So a step issues a group of four products beside each part of the exponentials
// and each read of operands, the next tile's logits among them, the maximum is followed late (`prepare`), and no array is
// indexed at run time: 6.1 to 5.6 ms together.  What did not help, with three buffers of tiles: two waves of a SIMD half a
// tile apart (the same time), or taking turns with a barrier a turn (18% slower); the first operands read before the next
// loads are issued (2% slower); 64 rows a wave, which halve the LDS reads but leave a SIMD one wave and accumulators that
// have to be moved (23%); priorities between waves, a fixed order of instructions (2 to 4%).
// grid = Hkv * n_tiles * n_split workgroups: neighbours take the KV heads of one tile (a head's tiles then mostly run on
// one XCD, whose L2 holds its keys), splits next, and the last tiles, which attend to the most keys, begin first.
template <int DT, int BS, int W>
__global__ __launch_bounds__(W * kWave, 2) void prompt_kernel(PromptArgs a) {
    constexpr int ET = elem_type(DT);
    using vec = typename Mfma<ET>::vec;
    constexpr int kRows = W * kRowsPerWave;
    constexpr int kBlocks = kKeys / BS;
    __shared__ __align__(1024) uint8_t s_keys[2][kTileBytes], s_vals[2][kTileBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int h = blockIdx.x % a.Hkv;
    const int rest = blockIdx.x / a.Hkv;
    const int split = rest % a.n_split;
    const Place pl = find_place(a.tok_off, a.B, a.G, kRows, a.n_tiles - 1 - rest / a.n_split);
    const Request rq = look_at(a, pl, kRows, W * kWave);
    if (!rq.any) return;
    const bool ok = rq.ok;
    const int t0 = rq.t0, ctx = rq.ctx, base = rq.base;
    const int64_t n_rows = rq.n_rows, row0 = rq.row0;
    // this lane's row
    const int64_t m = row0 + wave * kRowsPerWave + col;
    const bool live = m < n_rows;
    const int mi = (int)(live ? m : n_rows - 1);
    const int tok = (int)((uint64_t)mi * a.g_magic >> 32);
    const int g = mi - tok * a.G;
    const int p = base + tok;  // its position
    const int Hq = a.Hkv * a.G;
    const int64_t wave_row = row0 + wave * kRowsPerWave;
    // keys that the workgroup, and the wave, attend to at all; keys that all of the wave's rows attend to
    auto token_of = [&](int64_t row) { return (int)((uint64_t)min(row, n_rows - 1) * a.g_magic >> 32); };
    const int wg_keys = ok ? base + token_of(row0 + kRows - 1) + 1 : 0;
    const int wave_keys = wave_row < n_rows && ok ? base + token_of(wave_row + kRowsPerWave - 1) + 1 : 0;
    const int wave_all = base + token_of(wave_row) + 1;
    const int n_kt = (wg_keys + kKeys - 1) / kKeys;
    const int n_split = a.n_split > 1 ? splits_worth(n_kt, a.tile_us, a.split_us, a.n_split) : 1;
    if (split >= n_split) return;
    const int kt0 = (int)((int64_t)n_kt * split / n_split), kt1 = (int)((int64_t)n_kt * (split + 1) / n_split);

    vec qb[8];
    {
        const uint16_t* qr = a.q + (int64_t)(t0 + tok) * a.q_stride + (size_t)(h * a.G + g) * kHeadDim + half * 8;
#pragma unroll
        for (int c = 0; c < 8; ++c) qb[c] = load_vec<ET>(qr + 16 * c);
        // logits are scaled after their maximum is taken: the sign of the scale goes to Q, a zero becomes tiny
        if (a.scale_log2 < 0.f) {
#pragma unroll
            for (int c = 0; c < 8; ++c) qb[c] = -qb[c];
        }
    }
    const float scale = fmaxf(fabsf(a.scale_log2), 1e-30f);
    f32x16 acc[4] = {};
    float m_run = -INFINITY, l_run = 0.f;

    // Slots of a tile's blocks, looked up ahead; a block without one is looked at as slot 0 and counts nothing.
    const auto* row = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.table + (size_t)pl.r * a.max_blocks);
    const int n_blk = ok ? (ctx + BS - 1) / BS : 0;
    typedef __attribute__((ext_vector_type(kBlocks == 1 ? 2 : kBlocks), aligned(4))) int32_t Row;
    auto look_up = [&](int kt) {
        const int j = kt * kBlocks, last = n_blk - 1;
        Slots x = {};
        if (kBlocks == 1) {
            x.s0 = row[min(j, last)];
        } else if (j + kBlocks <= n_blk) {
            const Row y = *(const __attribute__((address_space(4))) Row*)(row + j);
            x.s0 = y[0], x.s1 = y[1];
            if constexpr (kBlocks > 2) x.s2 = y[2], x.s3 = y[3];
        } else {
            x.s0 = row[min(j, last)], x.s1 = row[min(j + 1, last)];
            if (kBlocks > 2) x.s2 = row[min(j + 2, last)], x.s3 = row[min(j + 3, last)];
        }
        return x;
    };
    auto checked = [&](Slots x) {
        x.bad = 0;
        const uint32_t n = (uint32_t)a.n_slots;
        uint32_t top = max((uint32_t)x.s0, (uint32_t)x.s1);
        if (kBlocks > 2) top = max(top, max((uint32_t)x.s2, (uint32_t)x.s3));
        if (top >= n) {
            auto one = [&](int& s, uint32_t bit) {
                if ((uint32_t)s >= n) {
                    x.bad |= bit;
                    s = 0;
                }
            };
            one(x.s0, 1);
            if (kBlocks > 1) one(x.s1, 2);
            if (kBlocks > 2) one(x.s2, 4), one(x.s3, 8);
            if (threadIdx.x == 0) report(a.status, PULSE_ERR_BAD_INDEX);
        }
        return x;
    };
    constexpr bool kCodes = kv_bits(DT) != 16;
    std::conditional_t<kCodes, StageCodes<DT, BS, W>, Stage16<BS, W>> stage(a, h, wave, lane);
    auto load_keys = [&](const Slots& x, int buf) {
        if constexpr (kCodes) stage.template fetch<true>(a, x, h, threadIdx.x);
        else stage.template tile<true>(a, x, s_keys[buf], wave);
    };
    auto load_vals = [&](const Slots& x, int buf) {
        if constexpr (kCodes) stage.template fetch<false>(a, x, h, threadIdx.x);
        else stage.template tile<false>(a, x, s_vals[buf], wave);
    };

    // Operands of four products from LDS: keys, a quarter of a tile (32 keys, 64 channels); values, 16 keys.
    const uint32_t k_lds = key_of_row(col) * 256 + key_piece(key_of_row(col), half) * 16;
    auto read_keys = [&](const uint8_t* keys, int q, u32x4 (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = *reinterpret_cast<const u32x4*>(keys + q / 2 * (32 * 256) + (k_lds ^ (q % 2 * 4 + i) * 32));
    };
    auto read_vals = [&](const uint8_t* vals, int st, u32x4 (&f)[4]) {
        const int oct = 2 * st + half, blk = oct / (BS / 8), o = oct % (BS / 8);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = *reinterpret_cast<const u32x4*>(vals + blk * (256 * BS) +
                                                   ((32 * i + col) * (BS / 8) + value_octet<BS>(col, o)) * 16);
    };
    auto logits = [&](int q, const u32x4 (&f)[4], f32x16& s) {
        if (q % 2 == 0) s = f32x16{};
#pragma unroll
        for (int i = 0; i < 4; ++i) s = mac32<ET>(__builtin_bit_cast(vec, f[i]), qb[q % 2 * 4 + i], s);
    };
    auto accumulate = [&](const u32x4 (&f)[4], vec pv) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mac32<ET>(__builtin_bit_cast(vec, f[i]), pv, acc[i]);
    };
    // Probabilities of 16 keys, as an operand.
    float m_use = 0.f;
    float sum = 0.f;  // of a tile
    auto probs = [&](const f32x16& s, int st) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = __builtin_amdgcn_exp2f(fmaf(s[st % 2 * 8 + i], scale, -m_use));
            sum += x[i];
        }
        return __builtin_bit_cast(vec, u32x4{pack2<ET>(x[0], x[1]), pack2<ET>(x[2], x[3]), pack2<ET>(x[4], x[5]),
                                             pack2<ET>(x[6], x[7])});
    };
    // One tile's probabilities and values, and the next one's logits, which take the registers of the logits before them:
    // groups of four products, each beside the reads of the next group's operands and a part of the exponentials.
    auto step = [&](auto has_next, f32x16 (&s)[2], const uint8_t* keys, const uint8_t* vals) {
        constexpr bool kNext = decltype(has_next)::value;
        sum = 0.f;
        u32x4 f[2][4];
        if constexpr (kNext) read_keys(keys, 0, f[0]);
        else read_vals(vals, 0, f[0]);
        vec pv[4];
        pv[0] = probs(s[0], 0);
        pv[1] = probs(s[0], 1);
        if constexpr (kNext) {
            read_keys(keys, 1, f[1]);
            logits(0, f[0], s[0]);
            pv[2] = probs(s[1], 2);
            read_vals(vals, 0, f[0]);
            logits(1, f[1], s[0]);
            pv[3] = probs(s[1], 3);
        } else {
            pv[2] = probs(s[1], 2);
            pv[3] = probs(s[1], 3);
        }
        read_vals(vals, 1, f[1]);
        accumulate(f[0], pv[0]);
        if constexpr (kNext) read_keys(keys, 2, f[0]);
        else read_vals(vals, 2, f[0]);
        accumulate(f[1], pv[1]);
        if constexpr (kNext) {
            read_keys(keys, 3, f[1]);
            logits(2, f[0], s[1]);
            read_vals(vals, 2, f[0]);
            logits(3, f[1], s[1]);
        }
        read_vals(vals, 3, f[1]);
        accumulate(f[0], pv[2]);
        accumulate(f[1], pv[3]);
        l_run += sum;
    };

    // The keys of a tile are in LDS one tile earlier than its values.
    Slots now, next, ahead;  // tiles kt, kt + 1, kt + 2
    f32x16 s[2];
    now.bad = next.bad = 0;
    if (kt0 < kt1) {
        now = checked(look_up(kt0));
        load_keys(now, 0);
        load_vals(now, 0);
        if constexpr (kCodes) {
            stage.template put<true>(s_keys[0], threadIdx.x);
            stage.template put<false>(s_vals[0], threadIdx.x);
        }
        if (kt0 + 1 < kt1) {
            next = checked(look_up(kt0 + 1));
            load_keys(next, 1);
            if constexpr (kCodes) stage.template put<true>(s_keys[1], threadIdx.x);
        }
        if (kt0 + 2 < kt1) ahead = look_up(kt0 + 2);
        tile_arrived();
        if (kt0 * kKeys < wave_keys) {
            u32x4 f[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                read_keys(s_keys[0], q, f);
                logits(q, f, s[q / 2]);
            }
        }
        __syncthreads();
    }
    // What a tile needs before its step: values behind the context taken out, logits masked, maxima looked at.  False where
    // the wave has no row that attends to it.
    auto prepare = [&](int kt, uint8_t* vals) {
        const int k0 = kt * kKeys;
        if (k0 + kKeys > ctx || now.bad) {
            // behind a context's end lies what an earlier owner of the slot left, NaN perhaps, which a probability of 0
            // would not take out of the product; and a block without a slot was read from another's
            for (int i = threadIdx.x; i < kTileBytes / 16; i += W * kWave) {
                constexpr int kOct = BS / 8;
                const int c = i / kOct % kHeadDim, o = i % kOct, blk = i / (kOct * kHeadDim);
                const int end = now.bad >> blk & 1 ? 0 : ctx - k0 - blk * BS - 8 * value_octet<BS>(c, o);
                u32x4* at = reinterpret_cast<u32x4*>(vals) + i;
                if (end < 8) {
                    u32x4 v = *at;
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        v[n] &= (2 * n < end ? 0xFFFFu : 0u) | (2 * n + 1 < end ? 0xFFFF0000u : 0u);
                    *at = v;
                }
            }
            __syncthreads();
        }
        if (k0 >= wave_keys) return false;
        if (k0 + kKeys > wave_all) {
            const int left = p + 1 - k0 - 8 * half;  // keys of this half's numbering that the row attends to
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (32 * (i / 16) + 16 * (i % 16 / 8) + i % 8 >= left) s[i / 16][i % 16] = -INFINITY;
        }
        if (now.bad) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int k = 32 * (i / 16) + 16 * (i % 16 / 8) + i % 8 + 8 * half;
                if (now.bad >> (k / BS) & 1) s[i / 16][i % 16] = -INFINITY;
            }
        }
        float cm = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) cm = __builtin_elementwise_maximum(cm, s[i / 16][i % 16]);
        {
            const uint32_t u = __float_as_uint(cm);
            const u32x2 w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            cm = fmaf(__builtin_elementwise_maximum(__uint_as_float(w[0]), __uint_as_float(w[1])), scale, -kLift<ET>);
        }
        // The maximum that is subtracted follows the rows' own only when one of the wave's has left it 2^8 behind:
        // until then probabilities and sums grow by up to that factor and keep their relative accuracy.
        if (__ballot(!(cm <= m_run + 8.f))) {
            const float m_new = __builtin_elementwise_maximum(m_run, cm);
            const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] *= alpha;
        }
        m_use = m_run == -INFINITY ? 0.f : m_run;
        return true;
    };
    int buf = 0;
#pragma unroll 1
    for (int kt = kt0; kt + 1 < kt1; ++kt, buf ^= 1) {
        load_vals(next, buf ^ 1);
        if (kt + 2 < kt1) {
            ahead = checked(ahead);
            load_keys(ahead, buf);
        }
        if (prepare(kt, s_vals[buf])) step(std::true_type(), s, s_keys[buf ^ 1], s_vals[buf]);
        if constexpr (kCodes) {
            stage.template put<false>(s_vals[buf ^ 1], threadIdx.x);
            if (kt + 2 < kt1) stage.template put<true>(s_keys[buf], threadIdx.x);
        }
        now = next;
        next = ahead;
        if (kt + 3 < kt1) ahead = look_up(kt + 3);
        tile_arrived();
    }
    if (kt0 < kt1 && prepare(kt1 - 1, s_vals[buf])) step(std::false_type(), s, nullptr, s_vals[buf]);
    {
        const uint32_t u = __float_as_uint(l_run);
        const u32x2 w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        l_run = __uint_as_float(w[0]) + __uint_as_float(w[1]);
    }
    const int64_t at = (int64_t)(t0 + tok) * Hq + h * a.G + g;
    if (a.n_split > 1 && live && half == 0 && split == 0) a.ws_n[at] = n_split;
    if (n_split > 1) {
        if (!live) return;
        const int64_t part = (int64_t)split * a.max_tokens * Hq + at;
        if (half == 0) a.ws_ml[part] = make_float2(m_run, l_run);
        if (m_run == -INFINITY) return;
        float* o = a.ws_o + part * kHeadDim + 4 * half;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<f32x4*>(o + 32 * t + 8 * b) = f32x4{acc[t][4 * b], acc[t][4 * b + 1], acc[t][4 * b + 2], acc[t][4 * b + 3]};
        return;
    }
    const float inv = m_run == -INFINITY ? 0.f : 1.f / l_run;
    if (live && a.lse && half == 0)
        a.lse[at] = m_run == -INFINITY ? -INFINITY : (m_run + log2f(l_run)) * 0.69314718055994531f;
    uint16_t* o = a.out + (int64_t)(t0 + tok) * a.out_stride + (size_t)(h * a.G + g) * kHeadDim;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int b = 0; b < 4; b += 2) {
            // channels 8 b + 4 half .. and 8 (b + 1) + 4 half ..: half 0 takes all 8 of the first, half 1 of the second
            u32x4 w;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const uint32_t x = pack2<ET>(acc[t][4 * b + 2 * n] * inv, acc[t][4 * b + 2 * n + 1] * inv);
                const uint32_t y = pack2<ET>(acc[t][4 * b + 4 + 2 * n] * inv, acc[t][4 * b + 5 + 2 * n] * inv);
                const u32x2 r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
                w[n] = r[0];
                w[2 + n] = r[1];
            }
            if (live) *reinterpret_cast<u32x4*>(o + 32 * t + 8 * (b + half)) = w;
        }
}

// The same for few rows of long contexts (drafted tokens to be verified): a workgroup takes 32 rows, whose keys its waves
// share out, 32 keys at a time straight from memory into the operands, a step ahead; nothing waits for another wave until
// the waves' results are joined in LDS.  A lane's operands are whole 16-byte loads in every form of the cache if product c
// takes channels 64 * half + 8 c .. + 7 of a key, and row m of tile t of the values is channel
// 64 * (m / 16) + 16 * t + m % 16.
//
// Bound: HBM, the context's bytes once for every 32 rows.  16 requests of 5 tokens at the end of 32K, 8 bits, 32 heads over
// 8 (866 MB): 165 us and 4.9 of the join, 5.2 TB/s of 5.8 that streaming reads reach; with tiles in LDS for 128 rows, most
// of them empty, 233.
template <int DT, int BS>
struct FewLoads {
    static constexpr int ET = elem_type(DT);
    static constexpr int kBits = kv_bits(DT);
    static constexpr int kPer = BS >= 32 ? 1 : 2;  // blocks of a step
    using vec = typename Mfma<ET>::vec;
    u32x4 k[kBits / 2];          // 64 channels of a key
    u32x4 v[2][kBits / 4];       // 8 tokens of 4 channels, of two octets
    uint32_t ks, vs[2];          // 8 bits: scale bytes of the key's block and of the octets'; 4: two scales of the key
    u32x2 vs4[2][2];             // 4 bits: scales of 8 tokens, of two channel groups

    __device__ inline void load(const PromptArgs& a, const int (&slot)[2], int in_block, int h, int col, int half) {
        const int key = key_of_row(col);
        const uint64_t U = kBits == 16 ? (uint64_t)a.Hkv * BS * kHeadDim * 4
                         : kBits == 8 ? (uint64_t)kv8_block_bytes(a.Hkv, BS) : (uint64_t)a.Hkv * kv4_head_bytes(BS);
        const uint8_t* b0 = a.pool + (uint64_t)(uint32_t)slot[0] * U;
        const uint8_t* b1 = kPer == 2 ? a.pool + (uint64_t)(uint32_t)slot[1] * U : b0;
        const uint8_t* kb = key >= 16 ? b1 : b0;
        const int row = (kPer == 2 ? key % 16 : key) + in_block;
        if constexpr (kBits == 16) {
            kb += ((size_t)h * BS + row) * 256 + half * 128;
        } else if constexpr (kBits == 8) {
            ks = kb[kv8_scales(a.Hkv, BS) + 2 * h];
            kb += (size_t)h * kv8_head_bytes(BS) + row * 128 + half * 64;
        } else {
            kb += (size_t)h * kv4_head_bytes(BS);
            ks = *reinterpret_cast<const uint16_t*>(kb + kv4_key_scales(BS) + row * 4 + half * 2);
            kb += row * 64 + half * 32;
        }
#pragma unroll
        for (int i = 0; i < kBits / 2; ++i) k[i] = reinterpret_cast<const u32x4*>(kb)[i];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const uint8_t* vb = st ? b1 : b0;
            const int oct = ((kPer == 2 ? 0 : 16 * st) + in_block) / 8 + half;
            if constexpr (kBits == 16) {
                vb += (size_t)(a.Hkv + h) * BS * 256 + oct * 16;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    v[st][t] = *reinterpret_cast<const u32x4*>(vb + (64 * (col >> 4) + 16 * t + (col & 15)) * BS * 2);
            } else if constexpr (kBits == 8) {
                vs[st] = vb[kv8_scales(a.Hkv, BS) + 2 * h + 1];
                vb += (size_t)h * kv8_head_bytes(BS) + kv8_values(BS) + oct * 1024 + (col & 15) * 64 + (col >> 4) * 32;
#pragma unroll
                for (int i = 0; i < 2; ++i) v[st][i] = reinterpret_cast<const u32x4*>(vb)[i];
            } else {
                vb += (size_t)h * kv4_head_bytes(BS);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    vs4[st][i] = *reinterpret_cast<const u32x2*>(vb + kv4_value_scales(BS) + (2 * (col >> 4) + i) * BS + oct * 8);
                v[st][0] = *reinterpret_cast<const u32x4*>(vb + kv4_values(BS) + oct * 512 + (col & 15) * 32 + (col >> 4) * 16);
            }
        }
    }
    __device__ inline vec key(int c) const {
        if constexpr (kBits == 16) return __builtin_bit_cast(vec, k[c]);
        else if constexpr (kBits == 8)
            return kv8_decode8<ET>(u32x2{k[c / 2][c % 2 * 2], k[c / 2][c % 2 * 2 + 1]}, kv8_pow2((int)ks - 127));
        else return kv4_decode8<ET>(k[c / 4][c % 4], kv4_scale(ks >> (8 * (c / 4)) & 255u));
    }
    __device__ inline u32x4 value(int st, int t) const {
        u32x4 w;
        if constexpr (kBits == 16) {
            w = v[st][t];
        } else if constexpr (kBits == 8) {
            w = __builtin_bit_cast(u32x4, kv8_decode8<ET>(u32x2{v[st][t / 2][t % 2 * 2], v[st][t / 2][t % 2 * 2 + 1]},
                                                          kv8_pow2((int)vs[st] - 127)));
        } else {
            const u32x2 sb = vs4[st][t / 2];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float s0 = kv4_scale(sb[n / 2] >> (16 * (n % 2)) & 255u);
                const float s1 = kv4_scale(sb[n / 2] >> (16 * (n % 2) + 8) & 255u);
                w[n] = (kv4_pair<ET>(v[st][0][t], n, s0) & 0xFFFFu) | (kv4_pair<ET>(v[st][0][t], n, s1) & 0xFFFF0000u);
            }
        }
        return w;
    }
};

// Beside that reading a second product a value costs nothing, so a probability keeps 16 (bf16) or 22 bits, in two PARTS of
// the 16-bit type, where a request has few rows (in us, one part and two: 16 requests of 5 at the end of 32K 367.6 and
// 367.9, in 8 bits 192.2 and 192.8); not over a 4-bit cache (132.5 and 156.6), whose own values are off by far more, nor in
// short prompts, which are not bound by the reading (512 tokens, 8 bits: 11.9 and 12.6; 512 at the end of 4096 50.6, 59.7).
// grid as prompt_kernel's, with 32 rows a workgroup.
template <int DT, int BS, int PARTS>
__global__ __launch_bounds__(kWaves * kWave, 2) void prompt_few_kernel(PromptArgs a) {
    constexpr int ET = elem_type(DT);
    constexpr int W = kWaves, kRows = 32, kStep = 32;
    constexpr int kPer = FewLoads<DT, BS>::kPer;
    using vec = typename Mfma<ET>::vec;
    __shared__ __align__(16) float s_o[W][kRows][kHeadDim];
    __shared__ float2 s_ml[W][kRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int h = blockIdx.x % a.Hkv;
    const int rest = blockIdx.x / a.Hkv;
    const int split = rest % a.n_split;
    const Place pl = find_place(a.tok_off, a.B, a.G, kRows, a.n_tiles - 1 - rest / a.n_split);
    const Request q = look_at(a, pl, kRows, W * kWave);
    if (!q.any) return;
    const int64_t m = q.row0 + col;
    const bool live = m < q.n_rows;
    const int mi = (int)(live ? m : q.n_rows - 1);
    const int tok = (int)((uint64_t)mi * a.g_magic >> 32), g = mi - tok * a.G;
    const int p = q.base + tok;
    const int Hq = a.Hkv * a.G;
    const int64_t last_row = min(q.row0 + kRows - 1, q.n_rows - 1);
    const int keys = q.ok ? q.base + (int)((uint64_t)last_row * a.g_magic >> 32) + 1 : 0;
    const int all = q.base + (int)((uint64_t)q.row0 * a.g_magic >> 32) + 1;  // keys that every row attends to
    const int n_split = a.n_split > 1 ? splits_worth((keys + kKeys - 1) / kKeys, a.tile_us, a.split_us, a.n_split) : 1;
    if (split >= n_split) return;
    // this wave's steps: a share of the split's, which is a share of the context
    const int n_steps = (keys + kStep - 1) / kStep, shares = n_split * W, share = split * W + wave;
    const int i0 = (int)((int64_t)n_steps * share / shares), i1 = (int)((int64_t)n_steps * (share + 1) / shares);

    const auto* row = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.table + (size_t)pl.r * a.max_blocks);
    const int last_blk = (q.ctx + BS - 1) / BS - 1;
    int slot[2] = {0, 0}, ahead[2] = {0, 0};
    uint32_t bad = 0, bad_next = 0;
    auto look_up = [&](int i) {
        ahead[0] = row[min(BS == 64 ? i / 2 : i * kPer, last_blk)];
        if (kPer == 2) ahead[1] = row[min(i * kPer + 1, last_blk)];
    };
    auto take = [&]() {  // the slots that were looked up; a block without one is read as slot 0 and counts nothing
        bad_next = 0;
#pragma unroll
        for (int b = 0; b < kPer; ++b) {
            slot[b] = ahead[b];
            if ((uint32_t)slot[b] >= (uint32_t)a.n_slots) {
                bad_next |= 1u << b;
                slot[b] = 0;
                if (lane == 0) report(a.status, PULSE_ERR_BAD_INDEX);
            }
        }
    };

    f32x16 acc[4] = {};
    float m_run = -INFINITY, l_run = 0.f;
    const float scale = fmaxf(fabsf(a.scale_log2), 1e-30f);
    vec qb[8];
    FewLoads<DT, BS> x;
    if (i0 < i1) {
        look_up(i0);
        take();
        x.load(a, slot, BS == 64 ? i0 % 2 * 32 : 0, h, col, half);
        bad = bad_next;
        if (i0 + 1 < i1) look_up(i0 + 1);
        const uint16_t* qr = a.q + (int64_t)(q.t0 + tok) * a.q_stride + (size_t)(h * a.G + g) * kHeadDim + half * 64;
#pragma unroll
        for (int c = 0; c < 8; ++c) qb[c] = load_vec<ET>(qr + 8 * c);
        if (a.scale_log2 < 0.f) {
#pragma unroll
            for (int c = 0; c < 8; ++c) qb[c] = -qb[c];
        }
    }
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const int k0 = i * kStep;
        f32x16 s = {};
#pragma unroll
        for (int c = 0; c < 8; ++c) s = mac32<ET>(x.key(c), qb[c], s);
        FewLoads<DT, BS> now = x;
        const uint32_t bad_now = bad;
        if (i + 1 < i1) {
            take();
            x.load(a, slot, BS == 64 ? (i + 1) % 2 * 32 : 0, h, col, half);
            bad = bad_next;
            if (i + 2 < i1) look_up(i + 2);
        }
        if (k0 + kStep > all || bad_now) {
            const int left = p + 1 - k0 - 8 * half;
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                const int k = 16 * (n / 8) + n % 8;
                if (k >= left || (bad_now >> (kPer == 2 ? n / 8 : 0) & 1)) s[n] = -INFINITY;
            }
        }
        float cm = s[0];
#pragma unroll
        for (int n = 1; n < 16; ++n) cm = __builtin_elementwise_maximum(cm, s[n]);
        const uint32_t u = __float_as_uint(cm);
        const u32x2 w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        cm = fmaf(__builtin_elementwise_maximum(__uint_as_float(w[0]), __uint_as_float(w[1])), scale, -kLift<ET>);
        if (__ballot(!(cm <= m_run + 8.f))) {  // (as in prompt_kernel)
            const float m_new = __builtin_elementwise_maximum(m_run, cm);
            const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] *= alpha;
        }
        const float m_use = m_run == -INFINITY ? 0.f : m_run;
        float sum = 0.f;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            float y[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                y[n] = __builtin_amdgcn_exp2f(fmaf(s[8 * st + n], scale, -m_use));
                sum += y[n];
            }
            u32x4 p1, p2;  // the probabilities, and what rounding took off them
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                p1[n] = pack2<ET>(y[2 * n], y[2 * n + 1]);
                if constexpr (PARTS == 2)
                    p2[n] = pack2<ET>(y[2 * n] - elem_to_float<ET>((uint16_t)(p1[n] & 0xFFFF)),
                                      y[2 * n + 1] - elem_to_float<ET>((uint16_t)(p1[n] >> 16)));
            }
            u32x4 v[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = now.value(st, t);
            if (k0 + kStep > q.ctx || bad_now) {  // tokens that are not the context's: anything may lie there
                const int left = bad_now >> (kPer == 2 ? st : 0) & 1 ? 0 : q.ctx - k0 - 16 * st - 8 * half;
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t keep = (2 * n < left ? 0xFFFFu : 0u) | (2 * n + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int t = 0; t < 4; ++t) v[t][n] &= keep;
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                acc[t] = mac32<ET>(__builtin_bit_cast(vec, v[t]), __builtin_bit_cast(vec, p1), acc[t]);
                if constexpr (PARTS == 2) acc[t] = mac32<ET>(__builtin_bit_cast(vec, v[t]), __builtin_bit_cast(vec, p2), acc[t]);
            }
        }
        l_run += sum;
    }
    {
        const uint32_t u = __float_as_uint(l_run);
        const u32x2 w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        l_run = __uint_as_float(w[0]) + __uint_as_float(w[1]);
    }
    // the waves' results side by side (4 channels of a row at a place that depends on the row), then joined
    if (half == 0) s_ml[wave][col] = make_float2(m_run, l_run);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c4 = 16 * (b / 2) + 4 * t + 2 * (b % 2) + half;  // (channel / 4)
            *reinterpret_cast<f32x4*>(&s_o[wave][col][4 * (c4 ^ col)]) =
                f32x4{acc[t][4 * b], acc[t][4 * b + 1], acc[t][4 * b + 2], acc[t][4 * b + 3]};
        }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kRows * kHeadDim / 4 / (W * kWave); ++n) {
        const int at = n * W * kWave + threadIdx.x, r = at / 32, c4 = at % 32;
        const int64_t mr = q.row0 + r;
        if (mr >= q.n_rows) break;
        float top = s_ml[0][r].x;
#pragma unroll
        for (int w = 1; w < W; ++w) top = __builtin_elementwise_maximum(top, s_ml[w][r].x);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
        if (top != -INFINITY) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 ml = s_ml[w][r];
                const float f = __builtin_amdgcn_exp2f(ml.x - top);
                l += ml.y * f;
                o += *reinterpret_cast<const f32x4*>(&s_o[w][r][4 * (c4 ^ r)]) * f;
            }
        }
        const int tr = (int)((uint64_t)mr * a.g_magic >> 32), head = h * a.G + (int)mr - tr * a.G;
        const int64_t out_row = q.t0 + tr, slot_row = out_row * Hq + head;
        if (a.n_split > 1 && split == 0 && c4 == 0) a.ws_n[slot_row] = n_split;
        if (n_split > 1) {
            const int64_t part = (int64_t)split * a.max_tokens * Hq + slot_row;
            if (c4 == 0) a.ws_ml[part] = make_float2(top, l);
            *reinterpret_cast<f32x4*>(a.ws_o + part * kHeadDim + 4 * c4) = o;
        } else {
            if (top != -INFINITY) o *= 1.f / l;
            *reinterpret_cast<u32x2*>(a.out + out_row * a.out_stride + (size_t)head * kHeadDim + 4 * c4) =
                u32x2{pack2<ET>(o[0], o[1]), pack2<ET>(o[2], o[3])};
            if (a.lse && c4 == 0)
                a.lse[slot_row] = top == -INFINITY ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
        }
    }
}

// Joins the splits of the rows: 32 threads, four channels each, take a row and `STRIDE`th splits of it, four of which are
// loaded before any is used; a workgroup holds eight rows, or (many splits: STRIDE 8) eight shares of one row, which it adds
// up in LDS.  (Loaded one after another, 64 splits took 45 us more: 5 tokens at the end of 64K, 4 bits, 69 and 24 us.)
constexpr int kManySplits = 8;  // above it, a workgroup a row

template <int ET, int STRIDE>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
    __shared__ f32x4 s_o[8][32];
    __shared__ float2 s_ml[8];
    const int Hq = a.Hkv * a.G;
    const int64_t rows = (int64_t)a.max_tokens * Hq;
    const int part = threadIdx.x >> 5, c4 = threadIdx.x & 31;
    const int64_t at = STRIDE == 1 ? (int64_t)blockIdx.x * 8 + part : (int64_t)blockIdx.x;
    const int first = a.tok_off[0], last = a.tok_off[a.B];
    const bool any = at >= (int64_t)first * Hq && at < (int64_t)last * Hq && last <= a.max_tokens;
    // (rows of offsets that are wrong have any number here)
    const int n_split = any ? min(max(a.ws_n[at], 1), a.n_split) : 1;
    if (STRIDE > 1 && n_split == 1) return;
    float top = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = STRIDE == 1 ? 0 : part; n_split > 1 && s0 < n_split; s0 += 4 * STRIDE) {
        float2 ml[4];
        f32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = min(s0 + i * STRIDE, n_split - 1);
            ml[i] = a.ws_ml[s * rows + at];
            x[i] = *reinterpret_cast<const f32x4*>(a.ws_o + (s * rows + at) * kHeadDim + 4 * c4);
        }
        float m = top;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (s0 + i * STRIDE < n_split) m = __builtin_elementwise_maximum(m, ml[i].x);
        if (m == -INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(top - m);
        top = m;
        l *= f;
        o *= f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (s0 + i * STRIDE >= n_split || ml[i].x == -INFINITY) continue;  // (such a split's sums are not written)
            const float w = __builtin_amdgcn_exp2f(ml[i].x - m);
            l += ml[i].y * w;
            o += x[i] * w;
        }
    }
    if (STRIDE > 1) {
        s_o[part][c4] = o;
        if (c4 == 0) s_ml[part] = make_float2(top, l);
        __syncthreads();
        if (part) return;
        float m = top;
        for (int i = 1; i < 8; ++i) m = __builtin_elementwise_maximum(m, s_ml[i].x);
        l = 0.f;
        o = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; m != -INFINITY && i < 8; ++i) {
            const float2 ml = s_ml[i];
            const float w = __builtin_amdgcn_exp2f(ml.x - m);
            l += ml.y * w;
            o += s_o[i][c4] * w;
        }
        top = m;
    }
    if (n_split == 1) return;
    if (top != -INFINITY) o *= 1.f / l;
    uint16_t* dst = a.out + at / Hq * a.out_stride + at % Hq * kHeadDim + 4 * c4;
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack2<ET>(o[0], o[1]), pack2<ET>(o[2], o[3])};
    if (a.lse && c4 == 0) a.lse[at] = top == -INFINITY ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
}

template <int ET>
static void launch_join(const PromptArgs& a, hipStream_t st) {
    const int64_t rows = (int64_t)a.max_tokens * a.Hkv * a.G;
    if (a.n_split > kManySplits)
        hipLaunchKernelGGL((prompt_join_kernel<ET, 8>), dim3((unsigned)rows), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((prompt_join_kernel<ET, 1>), dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, a);
}

struct PromptPlan {
    int rows;  // of a workgroup: 32 (prompt_few_kernel), 128 or 256
    int n_tiles, n_split, parts;
    float tile_us, split_us;
};

constexpr int kSplitGroups = 512;  // workgroups aimed at where few rows are split over the context: two a CU
constexpr int kCus = 256;
// prompt_few_kernel takes 32 rows to a workgroup, so every 32 rows read the keys again.  It is for
// - few rows of long contexts: up to 32 of a request on average, 64 over a cache of codes (beyond, that reading costs the
//   16-bit cache more than the decoding of codes that 128 rows share saves the others), and
// - few workgroups and tables of no more than 1280 tokens, 5120 over a cache of codes: up to 256, which leave CUs to share
//   out the keys of a workgroup of 128, or 512 unless prompts are so short that a workgroup is mostly its start; over a
//   cache of codes, whose decoding is then shared out too, 512 and 1152, and up to 128 also tables of 16K tokens.
// In us, 128 rows and 32, 16-bit and 8-bit cache, new tokens (of a context), query heads / KV heads:
//   1 x 256    32/8    9.8   8.3    11.5   7.6      1 x 512    32/8   14.7  14.8    18.3  11.8
//   1 x 1024   32/8   24.7  31.8    31.5  26.2      1 x 1024   16/2   24.6  21.5    29.6  15.4
//   1 x 3000   12/1   63.1  72.5    81.9  53.2      8 x 100    32/8    8.7  13.6     9.7  13.1
//   1 x 512 of 2048   33.4  42.0    39.0  28.2      1 x 512 of 4096   49.4  79.3    52.8  50.6
//   1 x 512 of 16K     149   294     162   187      1 x 256 of 16K      83   158      90   102
//   1 x 64 of 16K      37    52      39    35      1 x 64 of 8000      28    33      30    24
//   16 x 5 of 32K     366   369     246   193       16 x 16 of 32K    378   565     303   273
//   1 x 200    64/8    9.6  10.4 (16 bits, blocks of 32)
static bool few_each(const pulse_shape& s, int32_t B, int64_t max_tokens) {
    return max_tokens * (s.num_q_heads / s.num_kv_heads) <= (in_codes(s.dtype) ? 64 : 32) * (int64_t)B;
}
static bool few_rows(const pulse_shape& s, int32_t B, int64_t max_tokens, int32_t max_blocks) {
    const int64_t rows = max_tokens * (s.num_q_heads / s.num_kv_heads), groups = (rows + 31) / 32 * s.num_kv_heads;
    const bool codes = in_codes(s.dtype);
    if (few_each(s, B, max_tokens)) return true;
    const int64_t tokens = (int64_t)max_blocks * s.block_size;
    if (codes && groups <= 128 && tokens <= 16384) return true;
    if (tokens > (codes ? 5120 : 1280)) return false;
    return groups <= (codes ? 512 : 256) || (groups <= (codes ? 1152 : 512) && max_tokens >= 256 * (int64_t)B);
}
// Workgroups of eight waves, which stage and decode a tile for twice the rows, from two rounds of them and 2048 new tokens
// of a request on: below, the rows behind the diagonal that the larger tile multiplies in vain cost more.  In us, four
// waves and eight, 32 query heads over 8 KV heads, 16-bit and 8-bit cache:
//   1 x 2048   51.9  64.4   63.3  68.2      8 x 1024    96.7 111.0   108.5 110.8
//   1 x 4096  149.7 138.6  163.4 149.6      1 x 8192   535.5 523.3   592.7 552.9
// The 4-bit cache, 4096 tokens at the end of 32768: 2097 and 1900.
constexpr int kLongPrompt = 2048;
constexpr int kLongGroups = 512;

static int64_t key_tiles(const pulse_shape& s, int32_t max_blocks) {
    return ((int64_t)max_blocks * s.block_size + kKeys - 1) / kKeys;
}

static PromptPlan prompt_plan(const pulse_shape& s, int32_t B, int64_t max_tokens, int32_t max_blocks) {
    PromptPlan p;
    const int64_t G = s.num_q_heads / s.num_kv_heads;
    const int64_t all = max_tokens * G;
    p.rows = kWaves * kRowsPerWave;
    p.parts = few_each(s, B, max_tokens) && !is_kv4(s.dtype) ? 2 : 1;
    if (few_rows(s, B, max_tokens, max_blocks)) p.rows = 32;
    else if (max_tokens >= (int64_t)kLongPrompt * B && all * s.num_kv_heads >= (int64_t)kLongGroups * 2 * p.rows) p.rows *= 2;
    const int64_t rows = p.rows;
    p.n_tiles = (int)(all / rows + B);
    const int64_t units = std::max<int64_t>((all + rows - 1) / rows, B) * s.num_kv_heads;
    const int64_t tiles = key_tiles(s, max_blocks);
    const int64_t most = kSplitGroups / units;
    p.tile_us = rows > 32 ? 1.2f : in_codes(s.dtype) ? 0.3f : 0.5f;
    p.split_us = (float)((double)max_tokens * s.num_q_heads * 1024 / 7e6);
    p.n_split = splits_worth((int)std::min<int64_t>(tiles, 1 << 25), p.tile_us, p.split_us, (int)most);
    // A little more than a workgroup for each CU takes twice one's time.  In us, splits and times: 1024 tokens of 32 heads
    // over 8 2 29.4, 1 25.2; 256 at the end of 2048 8 26.8, 5 26.4, 4 23.1, in 8 bits (32 rows) 2 25.2, 1 17.5; 1500 of 12
    // heads over 1 1 33.7, 2 30.1, 3 27.6; 2 requests of 8 at the end of 1000, 16 heads over 2, 1 14.6, 4 10.7.
    const int64_t groups = p.n_split * units;
    if (groups > kCus && 2 * groups < 3 * kCus && 2 * units <= kCus) p.n_split = (int)(kCus / units);
    return p;
}

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Partials of the splits, and a row's number of them, of this call and every smaller one: fewer rows may have more splits, but no more than kSplitGroups
// workgroups' rows, nor than the context has splits (calls of 256 rows a workgroup have no splits).
size_t prompt_ws_bytes(const pulse_shape& s, int32_t B, int64_t max_tokens, int32_t max_blocks) {
    const int64_t most = key_tiles(s, max_blocks) / kLeastTiles;
    if (most <= 1) return 256;
    const size_t rows = (size_t)std::min<int64_t>((int64_t)kSplitGroups * kWaves * kRowsPerWave, most * max_tokens * s.num_q_heads);
    return up256(rows * kHeadDim * sizeof(float)) + up256(rows * sizeof(float2)) + up256(rows * sizeof(int32_t));
}

template <int DT, int BS>
static void launch_prompt_t(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.Hkv * a.n_tiles * a.n_split));
    const dim3 threads(kWaves * kWave), twice(2 * kWaves * kWave);
    constexpr int kParts = is_kv4(DT) ? 1 : 2;
    if (p.rows == 32 && p.parts == 2) hipLaunchKernelGGL((prompt_few_kernel<DT, BS, kParts>), grid, threads, 0, st, a);
    else if (p.rows == 32) hipLaunchKernelGGL((prompt_few_kernel<DT, BS, 1>), grid, threads, 0, st, a);
    else if (p.rows == kWaves * kRowsPerWave) hipLaunchKernelGGL((prompt_kernel<DT, BS, kWaves>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((prompt_kernel<DT, BS, 2 * kWaves>), grid, twice, 0, st, a);
}

template <int DT>
static void launch_prompt_bs(int32_t bs, const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
    if (bs == 16) launch_prompt_t<DT, 16>(a, p, st);
    else if (bs == 32) launch_prompt_t<DT, 32>(a, p, st);
    else launch_prompt_t<DT, 64>(a, p, st);
}

hipError_t launch_prompt_attn(const pulse_shape& s, const void* q, int64_t q_stride, const int32_t* tok_off,
                              int64_t max_tokens, const int32_t* ctx_len, int32_t B, const void* pool, int32_t n_slots,
                              const int32_t* table, int32_t max_blocks, float sm_scale, void* out, int64_t out_stride,
                              float* lse, int32_t* status, void* ws, hipStream_t st) {
    if (B == 0 || max_tokens == 0) return hipSuccess;
    const PromptPlan p = prompt_plan(s, B, max_tokens, max_blocks);
    const int32_t G = s.num_q_heads / s.num_kv_heads;
    PromptArgs a{(const uint16_t*)q, q_stride, tok_off, ctx_len, B, (int32_t)max_tokens, (const uint8_t*)pool, n_slots, table,
                 max_blocks, (int32_t)std::min<int64_t>((int64_t)max_blocks * s.block_size, INT32_MAX - 127), s.num_kv_heads, G, (((uint64_t)1 << 32) + G - 1) / G,
                 sm_scale * 1.4426950408889634f, (uint16_t*)out, out_stride, lse, (float*)ws, nullptr, nullptr, p.n_tiles,
                 p.n_split, p.tile_us, p.split_us, status};
    if (p.n_split > 1) {
        const size_t parts = (size_t)p.n_split * max_tokens * s.num_q_heads, at = up256(parts * kHeadDim * sizeof(float));
        a.ws_ml = ws_at<float2>(ws, at);
        a.ws_n = ws_at<int32_t>(ws, at + up256(parts * sizeof(float2)));
    }
    switch (s.dtype) {
        case PULSE_BF16: launch_prompt_bs<PULSE_BF16>(s.block_size, a, p, st); break;
        case PULSE_F16: launch_prompt_bs<PULSE_F16>(s.block_size, a, p, st); break;
        case PULSE_BF16_KV8: launch_prompt_bs<PULSE_BF16_KV8>(s.block_size, a, p, st); break;
        case PULSE_F16_KV8: launch_prompt_bs<PULSE_F16_KV8>(s.block_size, a, p, st); break;
        case PULSE_BF16_KV4: launch_prompt_bs<PULSE_BF16_KV4>(s.block_size, a, p, st); break;
        case PULSE_F16_KV4: launch_prompt_bs<PULSE_F16_KV4>(s.block_size, a, p, st); break;
        default: return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_split == 1) return e;
    if (elem_type(s.dtype) == PULSE_BF16) launch_join<PULSE_BF16>(a, st);
    else launch_join<PULSE_F16>(a, st);
    return hipGetLastError();
}

}  // namespace pulse

// What a prompt's queries attend to: for every key the sum of the probabilities that the queries of its KV head give it,
//   W_j = decay before_j + sum_i 2^(c q_i k_j - r_i),   j <= i + (keys - queries),   c = sm_scale log2 e,   r_i = log2 e times the query's log-sum-exp,
// over all or the last of the queries and over the query heads of the KV head.  The log-sum-exp is known from the attention itself, so nothing
// depends on another key: a workgroup owns 256 keys, which stay in registers, and the queries go by.
// A wave has 64 keys (twice 32, the right operand of v_mfma_f32_32x32x16_bf16), queries' heads are the left operand, so that a lane has 16 scores of
// one key and adds up their exponentials by itself.  Queries go from memory to LDS in tiles of 64 (query, head) rows, 16-byte chunks
// XORed with the row against bank conflicts, and serve the four waves.
// Sums go in order: 16 probabilities, those of a tile, of kSumTiles tiles, of a chunk of tiles, of the chunks; the results do not depend on timing.
// Bound by the vector units (an exponential, a product and a sum a score, 16 cycles for 64, and about 4 more) beside the matrix units (16
// cycles), at the clock that the power limit leaves: 33,625 tokens in three prompts, 32 heads on 8, 1.73 TFLOP of products, take 1.70 ms, 1.02
// PFLOP/s, where a library product of 16,384^3 reaches 1.39 (1.65 ms on another card).  The last 64 queries of 32,749 tokens take 27 us under the
// profiler, 25.5 a call one behind the other (their keys, 67 MB, alone 14).
#include "api_checks.h"
#include "kv_store.h"
#include <algorithm>
#include <type_traits>

namespace ihip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kKwThreads = 256, kKwWaves = kKwThreads / kWave;
template <int SETS> constexpr int kKwKeys = 32 * SETS * kKwWaves;         // of a workgroup
constexpr int kKwRows = 64;                          // rows of a tile
constexpr int kSumTiles = 16;

struct KeyWeightArgs {
    int B, Hq, Hkv, G, rows_q, rows_k, window;
    const int32_t *cu_q, *cu_k;
    const uint16_t *q, *k;
    int64_t q_sh, q_st, k_sh, k_st;
    const float *lse;                // [rows_q, Hq]
    float scale_log2e, decay;
    const float *before;             // [B, Hkv, weight_rows] or null
    float *weights;
    int weight_rows;
    int chunk_tiles, chunks;         // tiles of a chunk, from the sequence's end; chunks that a sequence can have
    float *part;                     // [chunk, Hkv, rows_k], or null: one chunk
    int window_rows, wg_keys, log2_G;        // rows in LDS, keys of a workgroup of the window's kernel; -1: G is not a power of two
    bool near;                       // G divides a tile's rows, whose queries are less than 2^31 bytes apart
};

// A log-sum-exp to base 2 with one rounding: that of log2 e would be a factor of all of a query's probabilities (1.4e-7 for one of 10)
__device__ inline float key_weight_r(float lse)
{
    constexpr float kLog2e = 1.44269504088896340736f, kRest = (float)(1.44269504088896340736 - (double)kLog2e);
    return fmaf(lse, kLog2e, lse * kRest);
}

// A sequence, and the tiles of its rows that count
struct KeyWeightSeq {
    int b, q_first, nq, k_first, nk, ahead, row0, rows;      // rows row0 .. rows - 1 count
    // The one that block `id` of `keys` keys belongs to (b: -1 if there is none).  Blocks are numbered so that sequence b's begin at first
    // key / keys + b, which leaves room for a part of a block in each
    __device__ KeyWeightSeq(const KeyWeightArgs &a, int keys, int id, int lane)
    {
        int q0 = 0, q1 = 0, k0 = 0, k1 = 0;          // of lane's sequence among the last 64 with one that begins at or before id
        b = -1;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            const int i = min(b0 + lane, a.B - 1);
            const int c0 = min(max(a.cu_k[i], 0), a.rows_k), c1 = a.cu_k[i + 1], d0 = a.cu_q[i], d1 = a.cu_q[i + 1];
            const int n = __popcll(__ballot(b0 + lane < a.B && c0 / keys + i <= id));
            if (n == 0) break;
            b = b0 + n - 1;
            k0 = c0; k1 = c1; q0 = d0; q1 = d1;
        }
        b = __builtin_amdgcn_readfirstlane(b);
        const int at = b & 63;
        q_first = min(max(__builtin_amdgcn_readlane(q0, at), 0), a.rows_q);
        nq = min(max(__builtin_amdgcn_readlane(q1, at), q_first), a.rows_q) - q_first;
        k_first = __builtin_amdgcn_readlane(k0, at);
        nk = min(max(__builtin_amdgcn_readlane(k1, at), k_first), a.rows_k) - k_first;
        ahead = nk - nq;                             // query i sees keys 0 .. i + ahead
        row0 = max(0, nq - a.window) * a.G;
        rows = nq * a.G;
    }
    __device__ int tiles() const { return (rows - row0 + kKwRows - 1) / kKwRows; }
    // the first tile with a query that sees key k
    __device__ int first_tile(const KeyWeightArgs &a, int k) const { return (int)min(max((int64_t)0, ((int64_t)k - ahead) * a.G - row0) / kKwRows, (int64_t)tiles()); }
};

// A wave's SETS times 32 keys and what has been added up for them.  Rows come half a tile at a time: the products of 32 rows with the keys, and between
// them, two scores after each, the exponentials of the half before.  Score i is that of row 8 (i / 4) + 4 half + i % 4.
struct KeyWeightTile { const uint16_t *q; const float *r; const int *last; };        // 64 rows in LDS: chunks XORed with the row; r; the last key
template <int SETS>
struct KeyWeightWave {
    static constexpr int kOps = 3;                   // operands that are read ahead of their use
    int n, half, kw;                                 // lane's key and half, first key
    float scale_log2e;
    bf16x8 kb[SETS][8];                              // (behind the last key: that one again)
    f32x16 c[2][SETS];                               // of the present and the previous half
    float part_sum[SETS], near_sum[SETS];
    bf16x8 x[kOps + 1];
    float4 r4[2];

    __device__ KeyWeightWave(int lane, float scale) : n(lane & 31), half(lane >> 5), scale_log2e(scale) {}
    __device__ void load_keys(const KeyWeightArgs &a, const KeyWeightSeq &seq, int g, int first, bf16x8 (&to)[SETS][8]) const
    {
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            const uint16_t *kp = a.k + (int64_t)(seq.k_first + min(first + 32 * s + n, seq.nk - 1)) * a.k_st + g * a.k_sh + half * 8;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) to[s][ks] = *reinterpret_cast<const bf16x8 *>(kp + ks * 16);
        }
    }
    __device__ void begin(int first)
    {
        kw = first;
#pragma unroll
        for (int s = 0; s < SETS; ++s) near_sum[s] = 0.f;
    }
    // The keys are waited for here: in the loop the compiler, which does not know what has been waited for in assembly, would wait for all loads at
    // their use
    __device__ void keys_are_there()
    {
#pragma unroll
        for (int s = 0; s < SETS; ++s)
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(kb[s][ks]));
    }
    __device__ bf16x8 operand(const KeyWeightTile &t, int h, int ks) const { return *reinterpret_cast<const bf16x8 *>(t.q + (32 * h + n) * kD + (((ks * 2 + half) ^ (n & 15)) << 3)); }
    __device__ float4 rows_r(const KeyWeightTile &t, int h, int i4) const { return *reinterpret_cast<const float4 *>(t.r + 32 * h + 8 * i4 + 4 * half); }
    static __device__ float element(const float4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    // score i of set s; r: that of its row
    template <bool MASKED>
    __device__ void exponential(const KeyWeightTile &t, int h, int i, int s, float r)
    {
        float w = __builtin_amdgcn_exp2f(fmaf(c[h][s][i], scale_log2e, -r));
        if constexpr (MASKED) w = kw + 32 * s + n <= t.last[32 * h + 8 * (i / 4) + 4 * half + i % 4] ? w : 0.f;
        part_sum[s] = i == 0 ? w : part_sum[s] + w;
        if (i == 15) near_sum[s] += part_sum[s];
    }
    // Of half h, and of the r of the half before, if there is one
    template <bool BEFORE>
    __device__ void first_operands(const KeyWeightTile &t, int h, const KeyWeightTile &before)
    {
#pragma unroll
        for (int ks = 0; ks < kOps; ++ks) x[ks] = operand(t, h, ks);
        if constexpr (BEFORE) r4[0] = rows_r(before, 1 - h, 0);
    }
    // products of half h, whose first operands have been asked for; exponentials of the half before, MASKED if not all of its rows see all keys
    template <bool MASKED, bool BEFORE>
    __device__ void half_tile(const KeyWeightTile &t, int h, const KeyWeightTile &before)
    {
#pragma unroll
        for (int i = 0; i < 8 * SETS; ++i) {
            const int ks = i / SETS, s = i % SETS, score = 2 * i / SETS;
            if (s == 0 && ks + kOps < 8) x[(ks + kOps) % (kOps + 1)] = operand(t, h, ks + kOps);
            if (BEFORE && score % 4 == 0 && score < 12) r4[(score / 4 + 1) % 2] = rows_r(before, 1 - h, score / 4 + 1);
            c[h][s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[ks % (kOps + 1)], kb[s][ks], ks == 0 ? f32x16{} : c[h][s], 0, 0, 0);
            if constexpr (BEFORE) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int e = (2 * i + u) / SETS;
                    exponential<MASKED>(before, 1 - h, e, (2 * i + u) % SETS, element(r4[(e / 4) % 2], e % 4));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __device__ void half_tile(const KeyWeightTile &t, int h, const KeyWeightTile &before, bool masked)
    {
        if (masked) half_tile<true, true>(t, h, before);
        else half_tile<false, true>(t, h, before);
    }
    template <bool MASKED>
    __device__ void last_half(const KeyWeightTile &t)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float4 r = rows_r(t, 1, i / 4);
#pragma unroll
            for (int s = 0; s < SETS; ++s) exponential<MASKED>(t, 1, i, s, element(r, i % 4));
        }
    }
    __device__ void last_half(const KeyWeightTile &t, bool masked)
    {
        if (masked) last_half<true>(t);
        else last_half<false>(t);
    }
    // f(key, sum), a lane a key
    template <class F>
    __device__ void for_keys(const float (&sum)[SETS], F f) const
    {
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            const float w = sum[s] + __shfl_xor(sum[s], 32, 64);
            if (half == s % 2) f(kw + 32 * s + n, w);
        }
    }
};
__device__ inline void store_key_weight(const KeyWeightArgs &a, int b, int g, int key, float w)
{
    if (key >= a.weight_rows) return;
    const int64_t at = ((int64_t)b * a.Hkv + g) * a.weight_rows + key;
    a.weights[at] = a.before ? fmaf(a.decay, a.before[at], w) : w;
}

// SETS of 32 keys a wave
template <int SETS>
__global__ __launch_bounds__(kKwThreads, SETS == 2 ? 2 : 3) void prompt_key_weights_kernel(const KeyWeightArgs a)
{
    __shared__ __attribute__((aligned(16))) uint16_t sh_q[2][kKwRows * kD];
    __shared__ __attribute__((aligned(16))) float sh_r[3][kKwRows];          // of a tile's rows: r, and the last key
    __shared__ __attribute__((aligned(16))) int sh_last[3][kKwRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x % a.Hkv, id = blockIdx.x / a.Hkv;
    constexpr int kKeys = kKwKeys<SETS>;
    const KeyWeightSeq seq(a, kKeys, id, lane);
    const int b = seq.b;
    if (b < 0) return;
    const int block = id - (seq.k_first / kKeys + b), k0 = block * kKeys;
    if (block < 0 || k0 >= seq.nk) return;
    const int tiles = seq.tiles(), begin = seq.first_tile(a, k0);
    const int end = tiles - (int)min((int64_t)blockIdx.y * a.chunk_tiles, (int64_t)tiles), t0 = max(begin, end - a.chunk_tiles);
    if (blockIdx.y > 0 && t0 >= end) return;
    KeyWeightWave<SETS> keys(lane, a.scale_log2e);
    keys.begin(k0 + wave * 32 * SETS);
    keys.load_keys(a, seq, g, keys.kw, keys.kb);

    // A thread's rows of a tile, of which it brings 16-byte pieces, and another one, whose r it brings.  The next tile's are 64 rows less: addresses go on
    // by differences (multiplications take four times as long as additions)
    constexpr int kPieces = kKwRows / (4 * kKwWaves);
    const int per_tile = kKwRows / a.G, heads_left = kKwRows % a.G, last_row = seq.row0 + (end - 1) * kKwRows;       // of the first tile, its first
    const int64_t q_step = per_tile * a.q_st + heads_left * a.q_sh, q_wrap = a.G * a.q_sh - a.q_st;
    const int r_step = per_tile * a.Hq + heads_left, r_wrap = a.G - a.Hq;
    const uint16_t *const qb = a.q + (int64_t)seq.q_first * a.q_st + (int64_t)g * a.G * a.q_sh;
    const float *const lse = a.lse + (int64_t)seq.q_first * a.Hq + g * a.G;
    auto in_tile = [&](int i) { return 4 * (wave + i * kKwWaves) + (lane >> 4); };
    auto q_of = [&](int query, int head, int i) { return qb + query * a.q_st + head * a.q_sh + (((lane & 15) ^ (in_tile(i) & 15)) << 3); };
    const uint16_t *q_at[kPieces];
    int q_head[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int row = last_row + in_tile(i), query = row / a.G;
        q_head[i] = row - query * a.G;
        q_at[i] = q_of(query, q_head[i], i);
    }
    int r_query = (last_row + (tid & (kKwRows - 1))) / a.G, r_head = last_row + (tid & (kKwRows - 1)) - r_query * a.G;
    const float *r_at = lse + (int64_t)r_query * a.Hq + r_head;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)&sh_q[0][0] + wave * 4 * kD * 2;
    auto stage_of = [&](int st, int i) { return lds0 + (st * kKwRows + i * 4 * kKwWaves) * kD * 2; };
    auto send = [&](int st, int i, const uint16_t *from) { global_to_lds(stage_of(st, i), from); };
    // where the heads of a query share tiles alike and are not far apart, addresses are a scalar and a lane's offset that stays
    const uint16_t *q_base = qb + (int64_t)(last_row / a.G) * a.q_st;
    uint32_t q_off[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) q_off[i] = (uint32_t)((const uint8_t *)q_at[i] - (const uint8_t *)q_base);
    auto request = [&](int st) {                     // the next tile
        if (a.near) {
            q_base -= q_step;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) global_to_lds(stage_of(st, i), q_base, q_off[i]);
            return;
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            q_at[i] -= q_step;
            q_head[i] -= heads_left;
            if (q_head[i] < 0) { q_head[i] += a.G; q_at[i] += q_wrap; }
            send(st, i, q_at[i]);
        }
    };
    auto row_info = [&](float &r, int &last) {
        r_at -= r_step;
        r_query -= per_tile;
        r_head -= heads_left;
        if (r_head < 0) { r_head += a.G; --r_query; r_at += r_wrap; }
        r = *r_at;
        last = r_query + seq.ahead;
    };

    float sum[SETS] = {};
    if (t0 < end) {                                  // the first tile: rows behind the last one stand for that one
#pragma unroll
        for (int i = 0; i < kPieces; ++i) send(0, i, last_row + in_tile(i) < seq.rows ? q_at[i] : q_of(seq.nq - 1, a.G - 1, i));
        if (tid < kKwRows) {
            const bool there = last_row + tid < seq.rows;
            sh_r[0][tid] = key_weight_r(there ? *r_at : lse[(int64_t)(seq.nq - 1) * a.Hq + a.G - 1]);
            sh_last[0][tid] = there ? r_query + seq.ahead : -1;
        }
    }
    keys.keys_are_there();

    int first_query = (seq.row0 + (end - 1) * kKwRows) / a.G;        // that of a tile's first row
    int first_head = seq.row0 + (end - 1) * kKwRows - first_query * a.G;
    bool masked_before = false;
    int st3 = 0;                                     // stage of r
    KeyWeightTile before{};
    for (int t = end - 1, st = 0; t >= t0; --t, st ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const KeyWeightTile tile{sh_q[st], sh_r[st3], sh_last[st3]};
        if (t == end - 1) keys.template first_operands<false>(tile, 0, before);
        else keys.template first_operands<true>(tile, 0, before);
        float r_next;
        int last_next;
        if (t > t0) {
            request(st ^ 1);
            if (tid < kKwRows) row_info(r_next, last_next);
        }
        // not all rows see all of the wave's keys, or the last tile's last rows are not there
        const bool masked = first_query + seq.ahead < keys.kw + 32 * SETS - 1 || seq.row0 + (t + 1) * kKwRows > seq.rows;
        if (t == end - 1) keys.template half_tile<true, false>(tile, 0, before);
        else keys.half_tile(tile, 0, before, masked_before);
        if ((end - t) % kSumTiles == 0) {
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                sum[s] += keys.near_sum[s];
                keys.near_sum[s] = 0.f;
            }
        }
        keys.template first_operands<true>(tile, 1, tile);
        keys.half_tile(tile, 1, tile, masked);
        masked_before = masked;
        before = tile;
        st3 = st3 == 2 ? 0 : st3 + 1;
        first_query -= per_tile;
        first_head -= heads_left;
        if (first_head < 0) { first_head += a.G; --first_query; }
        if (t > t0 && tid < kKwRows) {
            sh_r[st3][tid] = key_weight_r(r_next);      // (not before: the load would be waited for there)
            sh_last[st3][tid] = last_next;
        }
    }
    if (t0 < end) keys.last_half(before, masked_before);
#pragma unroll
    for (int s = 0; s < SETS; ++s) sum[s] += keys.near_sum[s];
    keys.for_keys(sum, [&](int key, float w) {
        if (key >= seq.nk) return;
        if (a.part) a.part[((int64_t)blockIdx.y * a.Hkv + g) * a.rows_k + seq.k_first + key] = w;
        else store_key_weight(a, b, g, key, w);
    });
}

// Few rows, as of a window: they stay in LDS, and each wave goes through keys by itself, the next 32 on their way under the products of the present ones
// (so many that a compute unit has room for two workgroups: 512 rows, one of them, 49 us where the other kernel takes 47)
constexpr int kWindowRows = 256;
__global__ __launch_bounds__(kKwThreads, 2) void prompt_key_weights_window_kernel(const KeyWeightArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x % a.Hkv, id = blockIdx.x / a.Hkv;
    const KeyWeightSeq seq(a, a.wg_keys, id, lane);
    const int b = seq.b;
    if (b < 0) return;
    const int block = id - (seq.k_first / a.wg_keys + b), k0 = block * a.wg_keys, k1 = min(k0 + a.wg_keys, seq.nk);
    if (block < 0 || k0 >= k1) return;
    constexpr int kStep = 32 * kKwWaves;
    KeyWeightWave<1> keys(lane, a.scale_log2e);
    int first = k0 + wave * 32;
    keys.load_keys(a, seq, g, first, keys.kb);
    // (of more rows than there is room for, which is what max_q says, the last)
    const int row0 = max(seq.row0, seq.rows - a.window_rows), rows = seq.rows - row0, tiles = (rows + kKwRows - 1) / kKwRows;
    float *const sh_r = reinterpret_cast<float *>(smem + a.window_rows * kD);
    int *const sh_last = reinterpret_cast<int *>(sh_r + a.window_rows);
    auto query_of = [&](int row) { return a.log2_G >= 0 ? row >> a.log2_G : row / a.G; };
    const uint16_t *const qb = a.q + (int64_t)seq.q_first * a.q_st + (int64_t)g * a.G * a.q_sh;
    const float *const lse = a.lse + (int64_t)seq.q_first * a.Hq + g * a.G;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
    for (int i = wave; i < tiles * (kKwRows / 4); i += kKwWaves) {         // four rows; those behind the last one stand for that one
        const int in_tile = 4 * i + (lane >> 4), row = row0 + min(in_tile, rows - 1), query = query_of(row);
        global_to_lds(lds0 + i * 4 * kD * 2, qb + query * a.q_st + (row - query * a.G) * a.q_sh + (((lane & 15) ^ (in_tile & 15)) << 3));
    }
    for (int i = tid; i < tiles * kKwRows; i += kKwThreads) {
        const int row = row0 + min(i, rows - 1), query = query_of(row);
        sh_r[i] = key_weight_r(lse[(int64_t)query * a.Hq + row - query * a.G]);
        sh_last[i] = i < rows ? query + seq.ahead : -1;
    }
    keys.keys_are_there();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    auto tile_of = [&](int t) { return KeyWeightTile{smem + t * kKwRows * kD, sh_r + t * kKwRows, sh_last + t * kKwRows}; };
    for (; first < k1; first += kStep) {
        keys.begin(first);
        bf16x8 next[1][8];
        keys.load_keys(a, seq, g, first + kStep, next);      // (behind the last key: that one again)
        bool masked_before = false;
        const int t0 = min((int)(max((int64_t)0, ((int64_t)first - seq.ahead) * a.G - row0) / kKwRows), tiles);
        for (int t = t0; t < tiles; ++t) {
            const KeyWeightTile tile = tile_of(t), before = tile_of(max(t - 1, 0));
            const bool masked = __builtin_amdgcn_readfirstlane(tile.last[0]) < first + 31 || (t + 1) * kKwRows > rows;
            if (t == t0) {
                keys.first_operands<false>(tile, 0, before);
                keys.half_tile<true, false>(tile, 0, before);
            } else {
                keys.first_operands<true>(tile, 0, before);
                keys.half_tile(tile, 0, before, masked_before);
            }
            keys.first_operands<true>(tile, 1, tile);
            keys.half_tile(tile, 1, tile, masked);
            masked_before = masked;
        }
        if (t0 < tiles) keys.last_half(tile_of(tiles - 1), masked_before);
        const float sum[1] = {keys.near_sum[0]};
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) keys.kb[0][ks] = next[0][ks];
        keys.keys_are_there();                       // (in front of the store, which would be waited for as well)
        keys.for_keys(sum, [&](int key, float w) {
            if (key < k1) store_key_weight(a, b, g, key, w);
        });
    }
}

// The chunks of a block of keys added up, a key a thread
template <int SETS>
__global__ __launch_bounds__(kKwKeys<SETS>) void prompt_key_weights_sum_kernel(const KeyWeightArgs a)
{
    const int g = blockIdx.x % a.Hkv, id = blockIdx.x / a.Hkv;
    const KeyWeightSeq seq(a, kKwKeys<SETS>, id, threadIdx.x & 63);
    const int b = seq.b;
    if (b < 0) return;
    const int k0 = (id - (seq.k_first / kKwKeys<SETS> + b)) * kKwKeys<SETS>, key = k0 + threadIdx.x;
    if (k0 < 0 || key >= seq.nk || key >= a.weight_rows) return;
    const int chunks = min(a.chunks, max(1, (seq.tiles() - seq.first_tile(a, k0) + a.chunk_tiles - 1) / a.chunk_tiles));
    float w = 0.f;
    for (int c = 0; c < chunks; ++c) w += a.part[((int64_t)c * a.Hkv + g) * a.rows_k + seq.k_first + key];
    store_key_weight(a, b, g, key, w);
}

// Wide blocks of keys, which read the queries half as often, where there is work for many rounds of workgroups, narrow ones otherwise; queries in
// chunks of about the tiles that give each compute unit 8 of them (48 where blocks are wide: the blocks of a long prompt differ).  us, wide / narrow:
// 33,625 tokens in three prompts 1,634 / 1,792, 7,401 in four 98 to 105 / 89, 1,024 27 / 16.  Rows that fit LDS: the window's kernel (the last 16,
// 32 and 64 queries of 32,749, 32 heads on 8, 15.3, 19.2 and 25.7 where narrow blocks take 18.4, 22.3 and 30.3), with two workgroups a compute unit.
struct KeyWeightPlan { int sets; int64_t blocks; int chunk_tiles, chunks; size_t bytes; int window_rows, wg_keys; };       // window_rows: 0, or the window's kernel
static KeyWeightPlan key_weight_plan(const ihip_packed &p, int rows_k, int window)
{
    constexpr int kLeast = 4;                        // tiles of a chunk
    const int64_t G = p.Hq / p.Hkv, most = std::max<int64_t>(1, ((int64_t)std::min({p.max_q, window, p.rows}) * G + kKwRows - 1) / kKwRows);
    KeyWeightPlan r{};
    if (most * kKwRows <= kWindowRows) {
        r.window_rows = (int)most * kKwRows;
        const int64_t each = 32 * kKwWaves, all = (rows_k / each + p.B) * p.Hkv;
        r.wg_keys = (int)(each * std::min<int64_t>(std::max<int64_t>(all / (2 * (int64_t)compute_units()), 1), 64));
        r.blocks = rows_k / r.wg_keys + p.B;
        r.chunks = 1;
        return r;
    }
    auto tiles = [&](int64_t keys) { return (r.blocks = rows_k / keys + p.B) * p.Hkv * most; };
    r.sets = tiles(kKwKeys<2>) >= 512 * (int64_t)compute_units() ? 2 : 1;
    const int64_t all = tiles(r.sets == 1 ? kKwKeys<1> : kKwKeys<2>), want = std::max<int64_t>(kLeast, all / ((r.sets == 1 ? 8 : 48) * (int64_t)compute_units()));
    r.chunks = (int)std::max<int64_t>(1, (most + want / 2) / want);
    r.chunk_tiles = (int)((most - 1) / r.chunks + 1);
    r.bytes = r.chunks > 1 ? (size_t)r.chunks * p.Hkv * rows_k * sizeof(float) : 0;
    return r;
}

}  // namespace ihip

using namespace ihip;

extern "C" size_t ihip_prompt_key_weights_workspace_bytes(const ihip_packed *packed, int32_t rows_k, int32_t window)
{
    const char *who = "ihip_prompt_key_weights_workspace_bytes";
    if (check_packed(who, packed) != IHIP_OK) return 0;
    if (rows_k < 0 || window < 1) {
        fail(IHIP_ERR_INVALID_ARG, "%s: rows_k = %d, window = %d", who, rows_k, window);
        return 0;
    }
    return std::max<size_t>(key_weight_plan(*packed, rows_k, window).bytes, 256);
}

extern "C" int32_t ihip_prompt_key_weights(const ihip_packed *packed, ihip_tensor q, ihip_tensor k, const int32_t *cu_k, int32_t rows_k,
                                           float sm_scale, const float *lse, int32_t window, const float *before, float decay,
                                           const ihip_kv_track *track, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ihip_prompt_key_weights";
    int32_t rc;
    if ((rc = check_packed(who, packed)) != IHIP_OK) return rc;
    if (rows_k < 0 || (!cu_k && rows_k != packed->rows))
        return fail(IHIP_ERR_INVALID_ARG, "%s: rows_k = %d (without cu_k: the %d rows of q)", who, rows_k, packed->rows);
    if (window < 1) return fail(IHIP_ERR_INVALID_ARG, "%s: window = %d", who, window);
    if (packed->B == 0 || rows_k == 0) return IHIP_OK;
    KeyWeightArgs a{};
    if ((rc = check_tensor(k, who, "k")) != IHIP_OK) return rc;
    if (packed->rows > 0 && (rc = check_tensor(q, who, "q")) != IHIP_OK) return rc;
    if (packed->rows > 0 && !lse) return fail(IHIP_ERR_INVALID_ARG, "%s: lse is NULL", who);
    if ((rc = check_track(who, track, 0, false)) != IHIP_OK) return rc;
    if ((rc = check_before(who, before, decay, track, (int64_t)packed->B * packed->Hkv)) != IHIP_OK) return rc;
    if ((rc = check_sm_scale(who, sm_scale, &a.scale_log2e)) != IHIP_OK) return rc;
    a.B = packed->B; a.Hq = packed->Hq; a.Hkv = packed->Hkv; a.G = packed->Hq / packed->Hkv;
    a.rows_q = packed->rows; a.rows_k = rows_k; a.window = window;
    a.cu_q = packed->cu_q; a.cu_k = cu_k ? cu_k : packed->cu_q;
    a.q = (const uint16_t *)q.ptr; a.q_sh = q.stride_h; a.q_st = q.stride_t;
    a.k = (const uint16_t *)k.ptr; a.k_sh = k.stride_h; a.k_st = k.stride_t;
    a.lse = lse;
    a.decay = decay;
    a.before = before; a.weights = track->weights; a.weight_rows = track->rows;
    if ((int64_t)a.rows_q * a.G > INT32_MAX - kKwRows)
        return fail(IHIP_ERR_UNSUPPORTED, "%s: %d rows of %d heads (%d KV heads) are too many", who, a.rows_q, a.Hq, a.Hkv);
    const KeyWeightPlan plan = key_weight_plan(*packed, rows_k, window);
    if (plan.blocks * a.Hkv > UINT32_MAX / kKwThreads || plan.chunks > 65535) return fail(IHIP_ERR_UNSUPPORTED, "%s: %lld workgroups are too many", who, (long long)plan.blocks * a.Hkv);
    const bool parts = plan.chunks > 1 && ws && !((uintptr_t)ws & 15) && ws_bytes >= plan.bytes;
    a.chunk_tiles = parts ? plan.chunk_tiles : INT32_MAX;
    a.near = kKwRows % a.G == 0 && a.q_st >= 0 && a.q_sh >= 0 && a.q_st < (1 << 22) && (int64_t)(a.G - 1) * a.q_sh < (1 << 28);
    a.chunks = parts ? plan.chunks : 1;
    a.part = parts ? (float *)ws : nullptr;
    const dim3 grid((uint32_t)(plan.blocks * a.Hkv), parts ? plan.chunks : 1);
    a.window_rows = plan.window_rows;
    a.wg_keys = plan.wg_keys;
    a.log2_G = pow2(a.G) ? __builtin_ctz(a.G) : -1;
    const hipStream_t st = (hipStream_t)stream;
    if (plan.window_rows > 0) {
        const int lds = plan.window_rows * (kD * (int)sizeof(uint16_t) + 8);
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(&prompt_key_weights_window_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        KernelTimer timer("prompt_key_weights_window", st);
        hipLaunchKernelGGL(prompt_key_weights_window_kernel, grid, dim3(kKwThreads), lds, st, a);
        return check_launch(who);
    }
    {
        KernelTimer timer("prompt_key_weights", st);
        if (plan.sets == 1) hipLaunchKernelGGL(prompt_key_weights_kernel<1>, grid, dim3(kKwThreads), 0, st, a);
        else hipLaunchKernelGGL(prompt_key_weights_kernel<2>, grid, dim3(kKwThreads), 0, st, a);
    }
    if ((rc = check_launch(who)) != IHIP_OK || !parts) return rc;
    KernelTimer timer("prompt_key_weights_sum", st);
    if (plan.sets == 1) hipLaunchKernelGGL(prompt_key_weights_sum_kernel<1>, dim3(grid.x), dim3(kKwKeys<1>), 0, st, a);
    else hipLaunchKernelGGL(prompt_key_weights_sum_kernel<2>, dim3(grid.x), dim3(kKwKeys<2>), 0, st, a);
    return check_launch(who);
}

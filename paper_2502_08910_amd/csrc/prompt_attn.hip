// Dense causal attention of packed prompts on v_mfma_f32_32x32x16_bf16.
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i k_j - r_i),   j <= i + (keys - queries),   c = sm_scale log2 e
// in one pass over the keys, for a reference r_i that is the row's maximum over its first tile (below).  A wave holds its rows (queries' heads; the right
// operand of the first product, K the left one), so that a lane has 16 of the 32 scores of one row, its exponentials are already
// the right operand of the second product with V^T (whose rows it takes in the order of the scores), and nothing of P goes through LDS.
// P is rounded to bf16 for it (2^-8 of each probability at most): what the rounding drops, as second operands, would be half as many matrix
// instructions again.  The sum that divides takes the probabilities as they were.
// K and V go from memory to LDS by themselves (global_load_lds), 16-byte chunks XORed with the row, so that both the rows of K and the
// transposed reads of V (ds_read_b64_tr_b16) are without conflicts.
// Bound by the matrix units (32 cycles an instruction) and the vector units (four instructions a product, 28 cycles, 16 of them for the
// exponential) of a SIMD's two waves, at the clock that the power limit leaves: one prompt of 32,749 with 32 heads, 8.79 TFLOP, takes
// 7.1 ms, 1.23 PFLOP/s, on a card where a library product of 16,384^3 reaches 1.37 and one of 8,192^3 1.39 (7.8 ms on another).
#include "api_checks.h"
#include "kv_store.h"
#include <algorithm>
#include <cmath>
#include <type_traits>

namespace ihip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPromptWaves = 4;

// A wave has one or two sets of 32 rows.  With one, two workgroups share a compute unit, each under the beginnings, ends and waits of the
// other; tiles have 64 keys, whose two halves take the place of two sets.  With two, a workgroup has a compute unit to itself (512 registers a
// lane), what is read from LDS serves two matrix instructions, and the keys are read half as often; tiles have 32 keys.
template <int SETS>
struct PromptShape {
    static constexpr int kSetRows = 32 * SETS, kRows = kSetRows * kPromptWaves;          // rows of a wave and of a workgroup
    static constexpr int kKeys = 64 / SETS, kEl = kKeys * kD;                            // of a tile
    static constexpr int kPerCu = 3 - SETS;                                              // workgroups of a compute unit
    static constexpr int kStages = SETS == 2 ? 4 : 2;                                    // tiles of K, and of V, in LDS
    static constexpr int kLds = (kStages * 2 * kEl + (SETS == 2 ? kRows * kD : 0)) * 2;  // bytes; behind the tiles, or in their place: the results
    // shares, in tiles: a block's beginning and end, the smallest part of one, the smallest share
    static constexpr int kBlockCost = 4, kMinPart = 4, kMinShare = 12;
};
constexpr int kOrderedSeqs = 64;                     // up to so many sequences, one a lane, blocks go in the order of their keys
constexpr float kPromptLowest = -3.4028234e38f;      // stand-in for -inf in maxima: no score is below it
// A block is done again where a sum of exponentials is outside 1/kPromptMaxSum .. kPromptMaxSum or a reference beyond +-kPromptMaxRef (whose
// rounding the exponentials would show), then with exponentials times 2^-kPromptShift: sums of up to a million of the largest values are finite
constexpr float kPromptMaxSum = 0x1p64f, kPromptMaxRef = 0x1p22f, kPromptShift = 20.f;

int32_t check_packed(const char *who, const ihip_packed *p);

struct PromptArgs {
    int B, Hq, Hkv, G, rows_q, rows_k;
    const int32_t *cu_q, *cu_k;
    const uint16_t *q, *k, *v;
    int64_t q_sh, q_st, k_sh, k_st, v_sh, v_st;
    int log2_G;                      // -1: G is not a power of two
    float scale_log2e;
    bool ordered;                    // blocks by themselves: in the order of their keys; otherwise
    int places;                      // of every sequence in the list of blocks, 0: as its rows are
    uint16_t *out;                   // [rows_q, Hq, d]
    float *lse;                      // [rows_q, Hq] or null
    // launches whose work is dealt out in equal shares: partial results of parts of blocks, two a workgroup
    float4 *part_o;                  // [part][wave][accumulators of a lane, four at a time: 16 a set][lane]
    float2 *part_ml;                 // [part][wave][set][32 rows]: reference of the exponentials (log2 units), sum
};

// ---- shares ------------------------------------------------------------------
// Where there are too few blocks x heads to keep the compute units busy to the end, the tiles of all blocks are dealt out in equal
// shares, one to each workgroup that the chip holds at a time, which begin and end inside blocks; a second kernel merges the
// parts of a block.  The list goes KV head by KV head, sequence by sequence, block by block; a block weighs its tiles and kBlockCost for
// its beginning and end.

// A sequence and its blocks of rows.  The G query heads of a KV head go together: row query * G + head.  Fewer keys that only some rows of a
// block see, fuller last blocks, and keys are read once for all of them.
template <int SETS>
struct PromptSeq {
    typedef PromptShape<SETS> Shape;
    int q_first, nq, k_first, nk, G, log2_G;
    int ahead, rows, blocks;
    __device__ PromptSeq() {}
    __device__ PromptSeq(const PromptArgs &a, int b)
    {
        q_first = min(max(a.cu_q[b], 0), a.rows_q);
        nq = min(max(a.cu_q[b + 1], q_first), a.rows_q) - q_first;
        k_first = min(max(a.cu_k[b], 0), a.rows_k);
        nk = min(max(a.cu_k[b + 1], k_first), a.rows_k) - k_first;
        G = a.G;
        log2_G = a.log2_G;
        derive();
    }
    __device__ void derive()
    {
        ahead = nk - nq;                             // query i sees keys 0 .. i + ahead
        rows = nq * G;
        blocks = (rows + Shape::kRows - 1) / Shape::kRows;
    }
    __device__ PromptSeq of_lane(int l) const        // that of lane l, in all lanes
    {
        PromptSeq r;
        r.q_first = __builtin_amdgcn_readlane(q_first, l);
        r.nq = __builtin_amdgcn_readlane(nq, l);
        r.k_first = __builtin_amdgcn_readlane(k_first, l);
        r.nk = __builtin_amdgcn_readlane(nk, l);
        r.G = G;
        r.log2_G = log2_G;
        r.derive();
        return r;
    }
    __device__ int query(int row) const { return log2_G >= 0 ? row >> log2_G : row / G; }
    __device__ int tiles(int m) const                // up to the last key that the block's last query sees
    {
        return (max(0, query(min((m + 1) * Shape::kRows, rows) - 1) + 1 + ahead) + Shape::kKeys - 1) / Shape::kKeys;
    }
    // Weight of blocks 0 .. m - 1, m <= blocks: the sum of (ahead + kKeys + kRows (j + 1) / G) / kKeys, which is no less than tiles(j), where
    // that is positive, rounded down, and kBlockCost for each: with that a block weighs no less than its tiles and kBlockCost
    __device__ int64_t weight_before(int m) const
    {
        const int64_t first = ahead + Shape::kKeys, none = first >= 0 ? 0 : min((int64_t)m, -first * G / Shape::kRows);
        const int64_t sum = 2 * G * first * (m - none) + Shape::kRows * (m * (m + 1ll) - none * (none + 1));
        constexpr int log2 = SETS == 2 ? 6 : 7;      // of 2 kKeys
        return (log2_G >= 0 ? sum >> (log2 + log2_G) : sum / ((int64_t)G << log2)) + (int64_t)Shape::kBlockCost * m;
    }
    __device__ int64_t weight() const { return weight_before(blocks); }
    // A part begins at a multiple of a tile, kMinPart or more from both ends of the block and not behind the tile that its first
    // query sees the end of (so that every query has a key in a part's first tile); w: weight from the block's beginning.
    // The block's number of tiles stands for its end.
    __device__ int part_begin(int m, int64_t w) const
    {
        const int t = tiles(m), c = (int)min<int64_t>(max<int64_t>(w - Shape::kBlockCost, 0), t);
        if (c < Shape::kMinPart) return 0;
        if (c > t - Shape::kMinPart) return t;
        const int last = min((query(m * Shape::kRows) + ahead) / Shape::kKeys, t - Shape::kMinPart);
        return c <= last ? c : last < Shape::kMinPart ? t : last;
    }
};
__device__ inline int64_t wave_sum_i64(int64_t v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ inline int64_t head_weight(const PromptArgs &a, int lane)
{
    int64_t w = 0;
    for (int b = lane; b < a.B; b += 64) w += PromptSeq<2>(a, b).weight();
    return wave_sum_i64(w);
}
struct PromptPlace { int head, b, m, tile; int64_t begin; };        // head in list order; begin: weight in front of the block
__device__ inline PromptPlace prompt_place(const PromptArgs &a, int64_t x, int64_t per_head, int lane)
{
    PromptPlace r{(int)(x / per_head), 0, 0, 0, 0};
    int64_t y = x % per_head;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int64_t w = b0 + lane < a.B ? PromptSeq<2>(a, b0 + lane).weight() : 0;
        int64_t incl = w;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t o = __shfl_up(incl, d, 64);
            if (lane >= d) incl += o;
        }
        const unsigned long long past = __ballot(incl > y);
        if (past != 0) {
            const int at = __builtin_ctzll(past);
            r.b = __builtin_amdgcn_readfirstlane(b0 + at);
            y -= __shfl(incl - w, at, 64);
            break;
        }
        y -= __shfl(incl, 63, 64);
    }
    const PromptSeq<2> q(a, r.b);
    int lo = 0, hi = q.blocks - 1;                   // the last block that begins at or before y
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (q.weight_before(mid) <= y) lo = mid;
        else hi = mid - 1;
    }
    r.m = __builtin_amdgcn_readfirstlane(lo);
    r.head = __builtin_amdgcn_readfirstlane(r.head);
    r.tile = __builtin_amdgcn_readfirstlane(q.part_begin(r.m, y - q.weight_before(r.m)));
    r.begin = x - (y - q.weight_before(r.m));
    return r;
}
// Shares that the whole weight is cut into, at most n
__device__ inline int prompt_shares(int64_t whole, int n) { return __builtin_amdgcn_readfirstlane((int)min<int64_t>(n, max<int64_t>(1, whole / PromptShape<2>::kMinShare))); }

// 16 bytes a lane from a scalar base and the lane's byte offset to the LDS byte address dst + 16 l (counts on vmcnt).  M0 is left as it is:
// nothing else in this kernel reads it, and it is not the compiler's to keep values in.
__device__ inline void prompt_to_lds(uint32_t dst, const uint16_t *base, uint32_t byte_off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(dst), "v"(byte_off), "s"(base) : "memory");
}

// A value and that of the lane 32 further, combined (commutatively: both lanes get the same)
template <class Op>
__device__ inline float half_swap(float x, Op op)
{
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Two sets: shares, as above; one: a workgroup a block and KV head, the heads of a block next to each other, those with most keys first.
template <int SETS>
__global__ __launch_bounds__(64 * kPromptWaves, PromptShape<SETS>::kPerCu) void prompt_attn_kernel(const PromptArgs a)
{
    typedef PromptShape<SETS> Shape;
    typedef PromptSeq<SETS> Seq;
    constexpr bool SHARES = SETS == 2;
    extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
    constexpr int kRows = Shape::kRows, kTileKeys = Shape::kKeys, kStages = Shape::kStages, kEl = Shape::kEl;
    constexpr int kLoads = kTileKeys / (4 * kPromptWaves);         // of a wave for K (and for V) of a tile
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    uint16_t *const rows = smem + (SETS == 2 ? kStages * 2 * kEl : 0) + wave * Shape::kSetRows * kD;       // this wave's results on their way out

    // which KV head, which sequence, which of its blocks, which tiles of the block
    int head, b = -1, m = 0, tile0 = 0, tile1 = 0, share = 0;
    PromptPlace end{};
    Seq seq;
    if constexpr (SHARES) {
        const int64_t per_head = head_weight(a, lane), whole = per_head * a.Hkv;
        const int shares = prompt_shares(whole, gridDim.x);
        // workgroups are dealt to the eight XCDs in turn: each gets shares that follow each other, of one KV head if there are eight
        share = shares % 8 == 0 && (int)gridDim.x == shares ? (blockIdx.x & 7) * (shares / 8) + (blockIdx.x >> 3) : blockIdx.x;
        if (share >= shares || __builtin_amdgcn_readfirstlane((int)(whole == 0)) != 0) return;
        const PromptPlace p = prompt_place(a, share * whole / shares, per_head, lane);
        head = p.head; b = p.b; m = p.m; tile0 = p.tile;
        if (share + 1 < shares) end = prompt_place(a, (share + 1) * whole / shares, per_head, lane);
        else end.head = a.Hkv;
        end.head = __builtin_amdgcn_readfirstlane(end.head);
        end.b = __builtin_amdgcn_readfirstlane(end.b);
        end.m = __builtin_amdgcn_readfirstlane(end.m);
        end.tile = __builtin_amdgcn_readfirstlane(end.tile);
    } else {
        head = blockIdx.x % a.Hkv;                   // neighbours read different KV heads, on the XCD of their own if there are eight
        int ti = blockIdx.x / a.Hkv;
        if (a.ordered) {
            // blocks in the order of their keys, a block's worth of them at a time: key class c of a sequence's block m is base + m
            const Seq q(a, min(lane, a.B - 1));
            const int blocks = lane < a.B ? q.blocks : 0, base = (int)min((int64_t)max(0, q.ahead) * a.G / kRows, (int64_t)1 << 30);
            auto at_least = [&](int c) { return (int)wave_sum_u32((uint32_t)min(max(base + blocks - c, 0), blocks)); };
            if (ti >= at_least(0)) return;
            int lo = 0, hi = (int)wave_reduce_bits((uint32_t)(base + blocks), [](uint32_t x, uint32_t y) { return max(x, y); });
            while (hi - lo > 1) {                    // at_least(lo) > ti >= at_least(hi)
                const int mid = lo + (hi - lo) / 2;
                if (at_least(mid) > ti) lo = mid;
                else hi = mid;
            }
            ti -= at_least(hi);
            const unsigned long long those = __ballot(base <= lo && lo < base + blocks);
            const int rank = __popcll(those & ((1ull << lane) - 1));
            b = __builtin_ctzll(__ballot(((those >> lane) & 1) && rank == ti));
            m = lo - __builtin_amdgcn_readlane(base, b);
            seq = q.of_lane(b);
        } else {
            // a sequence's longest blocks come first, of as many places as the longest sequence needs ...
            int at = ti % max(a.places, 1);
            if (a.places > 0) {
                b = ti / a.places;
                seq = Seq(a, b).of_lane(0);
            } else {
                // ... or from first row / kRows + b on, where there are at least as many as it has blocks
                b = 0;
                for (int range = a.B, step = 2; step > 1;) {         // the last one whose places begin at or before ti, of b .. b + range - 1
                    step = (range + 63) / 64;
                    const int i = lane * step;
                    const Seq q(a, min(b + i, a.B - 1));
                    const int c = __popcll(__ballot(lane == 0 || (i < range && q.q_first * a.G / kRows + b + i <= ti))) - 1;
                    b += c * step;
                    range = min(step, range - c * step);
                    seq = q.of_lane(c);
                }
                at = ti - seq.q_first * a.G / kRows - b;
            }
            m = __builtin_amdgcn_readfirstlane(seq.blocks - 1 - at);
            if (m < 0 || m >= seq.blocks) return;
        }
    }
    for (;;) {                                       // SHARES: blocks and parts of blocks; otherwise once
        // (the same in all lanes, which the compiler cannot see everywhere)
        head = __builtin_amdgcn_readfirstlane(head);
        b = __builtin_amdgcn_readfirstlane(b);
        m = __builtin_amdgcn_readfirstlane(m);
        tile0 = __builtin_amdgcn_readfirstlane(tile0);
        if (SHARES) seq = Seq(a, b).of_lane(0);
        const int nk = seq.nk, ahead = seq.ahead, n_rows = seq.rows;
        // the query of row i of the block, and its head among the KV head's
        const int query0 = seq.query(m * kRows), over0 = m * kRows - query0 * a.G, head0 = head * a.G;
        auto query_of = [&](int i, int &of) {
            const int q = seq.query(i + over0);
            of = i + over0 - q * a.G;
            return query0 + q;
        };
        const int all_tiles = __builtin_amdgcn_readfirstlane(seq.tiles(m));
        const bool is_end = SHARES && __builtin_amdgcn_readfirstlane((int)(head == end.head && b == end.b && m == end.m)) != 0;
        tile1 = __builtin_amdgcn_readfirstlane(is_end ? end.tile : all_tiles);
        if (all_tiles == 0 && !is_end) {                 // queries without keys
            for (int i = tid; i < min(kRows, n_rows - m * kRows) * kRowLanes; i += 64 * kPromptWaves) {
                int of;
                const int q = query_of(i / kRowLanes, of);
                const int64_t at = (int64_t)(seq.q_first + q) * a.Hq + head0 + of;
                reinterpret_cast<uint4 *>(a.out + at * kD)[i % kRowLanes] = make_uint4(0, 0, 0, 0);
                if (a.lse != nullptr && i % kRowLanes == 0) a.lse[at] = -INFINITY;
            }
        } else if (tile0 < tile1) {
            const int g = head;
            const int row0 = m * kRows + wave * Shape::kSetRows;           // this wave's first row
            const int n_tiles = tile1 - tile0;               // of this part, numbered from its first
            // Work goes in two turns s, for the two sets of queries or the two halves of a tile: their queries and first key
            auto qs = [](int s) { return SETS == 2 ? s : 0; };
            auto key0 = [](int s) { return SETS == 2 ? 0 : 32 * s; };

            bf16x8 qb[SETS][8];
            int last_key[SETS], first_last[SETS];            // the last key of a lane's query, and of a set's first
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                int of;
                last_key[s] = query_of(min(wave * Shape::kSetRows + s * 32 + n, n_rows - 1 - m * kRows), of) + ahead - tile0 * kTileKeys;
                first_last[s] = seq.query(row0 + s * 32) + ahead - tile0 * kTileKeys;
            }
            auto load_queries = [&] {
                int l = lane;                                // (not known to be it: what follows from it is computed here, not kept in registers all along)
                asm volatile("" : "+v"(l));
                const int n = l & 31, half = l >> 5;
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
                    int of;
                    const int q = query_of(min(wave * Shape::kSetRows + s * 32 + n, n_rows - 1 - m * kRows), of);
                    const uint16_t *qp = a.q + (int64_t)(seq.q_first + q) * a.q_st + (head0 + of) * a.q_sh + half * 8;
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) qb[s][ks] = *reinterpret_cast<const bf16x8 *>(qp + ks * 16);
                }
            };
            const int keys_here = nk - tile0 * kTileKeys;
            const uint16_t *kb = a.k + ((int64_t)seq.k_first + (int64_t)tile0 * kTileKeys) * a.k_st + g * a.k_sh;
            const uint16_t *vb = a.v + ((int64_t)seq.k_first + (int64_t)tile0 * kTileKeys) * a.v_st + g * a.v_sh;

            // Loads of a tile: four-row instructions for K and V, dealt to the waves.  Lane l brings 16 bytes of row
            // 4 j + l / 16 to base + 16 l.  The base of a tile is scalar; a lane's offset from it changes in a tile that reaches behind the last key
            // only, whose rows stand for the missing ones.  What would come after the last tile is the last one again, so that every period has
            // as many loads on their way as any other.
            auto offset = [&](int i, int rows, int64_t st, bool is_v) {
                const int key = 4 * (wave + i * kPromptWaves) + (lane >> 4), at = min(key, rows - 1), slot = lane & 15;
                return (uint32_t)(at * (int)st + ((slot ^ (is_v ? (key & 3) << 2 : key & 15)) << 3)) * 2u;
            };
            uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                k_off[i] = offset(i, kTileKeys, a.k_st, false);
                v_off[i] = offset(i, kTileKeys, a.v_st, true);
            }
            const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem + wave * 4 * kD * 2;
            const bool cut = n_tiles * kTileKeys > keys_here;       // the last tile reaches behind the last key
            const uint16_t *k_next = kb, *v_next = vb;       // of the tiles to be requested next
            int k_tile = 0, v_tile = 0;
            auto request = [&](bool is_v, int st) {
                int &tile = is_v ? v_tile : k_tile;
                const uint16_t *&next = is_v ? v_next : k_next;
                const int64_t stride = is_v ? a.v_st : a.k_st;
                uint32_t off[kLoads];
#pragma unroll
                for (int i = 0; i < kLoads; ++i) off[i] = is_v ? v_off[i] : k_off[i];
                if (cut && tile == n_tiles - 1) {
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) off[i] = offset(i, keys_here - tile * kTileKeys, stride, is_v);
                }
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    prompt_to_lds(lds0 + ((is_v ? kStages : 0) + st) * kEl * 2 + i * 4 * kPromptWaves * kD * 2, next, off[i]);
                const bool more = tile < n_tiles - 1;
                next += more ? kTileKeys * stride : 0;
                tile += more;
            };
            auto request_k = [&](int st) { request(false, st); };
            auto request_v = [&](int st) { request(true, st); };
            const uint16_t *k_at[8], *v_at[4];               // this lane's addresses in stage 0
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) k_at[ks] = smem + n * kD + ((ks * 2 + half) ^ (n & 15)) * 8;
            {
                const int i = lane & 15, key = 4 * half + (i >> 2);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const int chunk = dt * 4 + ((n >> 4) << 1) + ((i & 3) >> 1);
                    v_at[dt] = smem + kStages * kEl + key * kD + ((chunk ^ ((key & 3) << 2)) << 3) + ((i & 1) << 2);
                }
            }
            // operands of a stage for turn s; i: 4 kk + dt
            auto k_operand = [&](int st, int s, int ks) { return *reinterpret_cast<const bf16x8 *>(k_at[ks] + st * kEl + key0(s) * kD); };
            auto v_operand = [&](int st, int s, int i) {
                const uint16_t *at = v_at[i & 3] + st * kEl + (key0(s) + 16 * (i >> 2)) * kD;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 8 * kD));
                return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            };
            f32x16 o[SETS][4], sc[2];
            auto scores = [&](int st, int s) {
                sc[s] = f32x16{};
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(st, s, ks), qb[qs(s)][ks], sc[s], 0, 0, 0);
            };
            // Keys of a turn that a lane's query must not see, as bits: score r is that of key 8 (r / 4) + 4 half + r % 4
            auto hidden_keys = [&](int tile, int s) { return ~0u << min(max(last_key[qs(s)] - 4 * half - tile * kTileKeys - key0(s) + 1, 0), 31); };
            auto hide = [&](uint32_t bits, int r, float x) {         // v_bfe_i32, v_bfi_b32
                const int hidden = (int)(bits << (31 - (8 * (r >> 2) + (r & 3)))) >> 31;
                return __int_as_float((hidden & __float_as_int(-INFINITY)) | (~hidden & __float_as_int(x)));
            };
            auto mask = [&](int tile, int s) {
                if (tile * kTileKeys + key0(s) + 31 <= first_last[qs(s)]) return;
                const uint32_t bits = hidden_keys(tile, s);
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[s][r] = hide(bits, r, sc[s][r]);
            };
            auto row_max = [&](const f32x16 &s) {            // of both halves of the wave
                float mx = s[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
                return half_swap(mx, [](float x, float y) { return fmaxf(x, y); });
            };

            uint32_t pw[2][8];                               // the probabilities of a turn, in pairs of keys
            float m_ref[SETS], l_run[SETS], l_turn;          // (16 probabilities are added up before they go to a sum that may be long)
#pragma unroll
            for (int s = 0; s < SETS; ++s) m_ref[s] = kPromptLowest;
            // two scores -> two probabilities (exp2(-inf) = 0).  The empty assembly keeps them where they are called: left to themselves all
            // exponentials of a turn would be computed in front of the other's matrix instructions instead of under them.
            auto exponentials = [&](int s, int i, bool masked, uint32_t bits) {
                float x = fmaf(sc[s][2 * i], a.scale_log2e, -m_ref[qs(s)]), y = fmaf(sc[s][2 * i + 1], a.scale_log2e, -m_ref[qs(s)]);
                if (masked) {
                    x = hide(bits, 2 * i, x);
                    y = hide(bits, 2 * i + 1, y);
                }
                asm volatile("" : "+v"(x), "+v"(y));
                x = __builtin_amdgcn_exp2f(x);
                y = __builtin_amdgcn_exp2f(y);
                l_turn = i == 0 ? x + y : l_turn + x + y;
                pw[s][i] = pack_bf16x2(x, y);
                asm volatile("" : "+v"(pw[s][i]), "+v"(l_turn));
                if (i == 7) {
                    l_run[qs(s)] += l_turn;
                    asm volatile("" : "+v"(l_run[qs(s)]));
                }
            };
            auto probabilities = [&](int s, int kk) {
                return __builtin_bit_cast(bf16x8, make_uint4(pw[s][4 * kk], pw[s][4 * kk + 1], pw[s][4 * kk + 2], pw[s][4 * kk + 3]));
            };
            // Matrix instructions of the loop are written as assembly, so that each stays where it is, with its share of the vector
            // instructions under it, and that the accumulators of two sets are kept in the upper half of the 512 registers ("a") and everything else
            // in the lower one.  The compiler does not know the instructions' latency: a turn's scores are read by vector instructions eight
            // matrix instructions after their last one.
            auto score_step = [&](int s, int ks, const bf16x8 &x) {
                if (ks == 0) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=v"(sc[s]) : "v"(x), "v"(qb[qs(s)][0]));
                else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(sc[s]) : "v"(x), "v"(qb[qs(s)][ks]));
            };
            auto value_step = [&](int s, int i, const bf16x8 &x) {
                if constexpr (SETS == 2) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o[qs(s)][i & 3]) : "v"(x), "v"(probabilities(s, i >> 2)));
                else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(o[0][i & 3]) : "v"(x), "v"(probabilities(s, i >> 2)));
            };
            // Period t, in two turns: first product of tile t + 1 and second product of tile t, and under them the exponentials of the other
            // turn, 16 matrix instructions and 16 scores a lane at a time.
            // Two sets: K of tile t + 4 and V of tile t + 3 are requested into the stages that period t - 1 has read, and have landed when period
            // t + 1 ends; operands serve both turns, and the first ones of period t + 1 are read from LDS as this one ends.
            bf16x8 ka[8], va[8];
            auto first_operands = [&](int st, int st1) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    ka[i] = k_operand(st1, 0, i);
                    va[i] = v_operand(st, 0, i);
                }
            };
            auto period_of_sets = [&](int st, int st1, int st2, int st3, int t, bool masked) {     // stages of tiles t, t + 1, t + 2, t + 3
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint32_t bits = masked ? hidden_keys(t + s, 1 - s) : 0u;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if (s == 0 && r < 6) ka[r + 2] = k_operand(st1, 0, r + 2);
                        if (s == 0 && r >= 6 && r < 12) va[r - 4] = v_operand(st, 0, r - 4);
                        if (s == 1 && r == 10) first_operands(st1, st2);
                        if (r < 8) score_step(s, r, ka[r]);
                        else value_step(s, r & 7, va[r & 7]);
                        if (r % 2 == 0) exponentials(1 - s, r / 2, masked, bits);
                        if (s == 0 && r == 3) request_k(st);
                        if (s == 0 && r == 9) request_v(st3);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
                __syncthreads();
            };
            // One set: K of tile t + 2 and V of tile t + 1 are requested into the stages that period t - 1 has read, and have landed when this one
            // ends; operands are read from LDS four matrix instructions ahead.  What that and the barrier leave idle is the other workgroup's.
            auto period_of_halves = [&](int st, int t, bool masked) {                              // st: t % 2
                constexpr int kAhead = 4;
                auto operand = [&](int c) { return (c & 8) == 0 ? k_operand(st ^ 1, c >> 4, c & 7) : v_operand(st, c >> 4, c & 7); };
                bf16x8 x[kAhead];
#pragma unroll
                for (int c = 0; c < kAhead; ++c) x[c] = operand(c);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint32_t bits = masked ? hidden_keys(t + s, 1 - s) : 0u;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int c = 16 * s + r;
                        if (r < 8) score_step(s, r, x[c % kAhead]);
                        else value_step(s, r & 7, x[c % kAhead]);
                        if (c + kAhead < 32) x[c % kAhead] = operand(c + kAhead);
                        if (r % 2 == 0) exponentials(1 - s, r / 2, masked, bits);
                        if (s == 0 && r == 1) request_k(st);
                        if (s == 0 && r == 3) request_v(st ^ 1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
            };
            // One product step outside of the loop, whose operands vector instructions have just written
            auto product = [&](int s, int i, const bf16x8 &x, const bf16x8 &y) {
                if constexpr (SETS == 2) asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o[qs(s)][i & 3]) : "v"(x), "v"(y));
                else asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(o[0][i & 3]) : "v"(x), "v"(y));
            };
            // (the compiler does not know that there are matrix instructions in the assembly, whose results take up to 19 wait states)
            auto settle = [&] {
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
                    if constexpr (SETS == 2) asm volatile("s_nop 15\n\ts_nop 7" : "+a"(o[s][0]), "+a"(o[s][1]), "+a"(o[s][2]), "+a"(o[s][3]));
                    else asm volatile("s_nop 15\n\ts_nop 7" : "+v"(o[s][0]), "+v"(o[s][1]), "+v"(o[s][2]), "+v"(o[s][3]));
                }
            };
            auto clear = [&] {
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
                    l_run[s] = 0.f;
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt) o[s][dt] = f32x16{};
                }
                if constexpr (SETS == 2) {
#pragma unroll
                    for (int s = 0; s < SETS; ++s) asm volatile("" : "+a"(o[s][0]), "+a"(o[s][1]), "+a"(o[s][2]), "+a"(o[s][3]));
                }
            };
            // tiles that all queries of the block see whole; behind them scores are masked, under the matrix instructions as well
            const int seen = min(n_tiles, (query0 + ahead + 1) / kTileKeys - tile0);

            // Exponentials are taken against the row's maximum over the first tile (which holds a key of every query that has any), not
            // against a running one: bf16 and fp32 have exponents to spare, nothing is lost while the scores stay within 2^64 of it.
#pragma unroll
            for (int st = 0; st < kStages; ++st) request_k(st);
#pragma unroll
            for (int st = 0; st < kStages - 1; ++st) request_v(st);
            load_queries();
            clear();                                         // (while the loads are on their way)
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                scores(0, s);
                mask(0, s);
                m_ref[qs(s)] = fmaxf(m_ref[qs(s)], row_max(sc[s]) * a.scale_log2e);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) exponentials(0, i, false, 0);
            __syncthreads();                                 // K(0) has been read
            // This wave's last tile with a key that one of its queries sees.  Behind it, it only keeps the others company: the matrix units are
            // the other workgroup's meanwhile
            const int last_seen = seq.query(min(row0 + Shape::kSetRows, n_rows) - 1) + ahead - tile0 * kTileKeys;
            const int mine = row0 >= n_rows ? 1 : min(max(last_seen, 0) / kTileKeys + 1, n_tiles), unmasked = min(seen, mine);
            int t = 0;
            if constexpr (SETS == 2) {
                first_operands(0, 1);
                for (; t + 4 < unmasked; t += 4) {
                    period_of_sets(0, 1, 2, 3, t, false);
                    period_of_sets(1, 2, 3, 0, t + 1, false);
                    period_of_sets(2, 3, 0, 1, t + 2, false);
                    period_of_sets(3, 0, 1, 2, t + 3, false);
                }
                for (; t + 1 < mine; ++t) period_of_sets(t & 3, (t + 1) & 3, (t + 2) & 3, (t + 3) & 3, t, true);
            } else {
                for (; t + 2 < unmasked; t += 2) {
                    period_of_halves(0, t, false);
                    period_of_halves(1, t + 1, false);
                }
                for (; t + 1 < mine; ++t) period_of_halves(t & 1, t, true);
            }
            // its last tile, whose first products are done
            const uint32_t bits = hidden_keys(t, 1);
            // two sets: both products of an operand; one: one half after the other
            auto turn_of = [](int c) { return SETS == 2 ? c & 1 : c >> 3; };
            auto step_of = [](int c) { return SETS == 2 ? c >> 1 : c & 7; };
            bf16x8 x[16 / SETS];
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = v_operand(t & (kStages - 1), turn_of(c * SETS), step_of(c * SETS));
#pragma unroll
            for (int i = 0; i < 8; ++i) exponentials(1, i, true, bits);
#pragma unroll
            for (int c = 4; c < 16 / SETS; ++c) x[c] = v_operand(t & (kStages - 1), turn_of(c * SETS), step_of(c * SETS));
#pragma unroll
            for (int c = 0; c < 16; ++c) product(turn_of(c), step_of(c), x[c / SETS], probabilities(turn_of(c), step_of(c) >> 2));
            for (; t + 1 < n_tiles; ++t) {
                request_k(t & (kStages - 1));
                request_v((t + kStages - 1) & (kStages - 1));
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(SETS == 2 ? 2 * kLoads : 0) : "memory");
                __syncthreads();
            }
            settle();
            // Where a row's sum says that its scores left that range, or a result is not finite, the block is done again, a tile at a time and
            // against the maxima over all tiles.  What is not finite in V is for all queries that see it, however small its probability has
            // become in fp32, and for no others, for whom a probability of 0 times it would be NaN.  So the products take 0 in its place, and
            // infinity or NaN is added at the end for the queries that see some; which those are, and of what, say the products of "sees it" and a
            // code for "is +infinity", "-infinity" or "NaN".  (A sum that is NaN, from a query or a key that is, says all that there is to know of its row.)
            bool fine = true;
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                l_run[s] = half_swap(l_run[s], [](float x, float y) { return x + y; });
                float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < 16; ++r)
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt) zero[dt] = fmaf(o[s][dt][r], 0.f, zero[dt]);
                const bool in_range = last_key[s] < 0 || (l_run[s] >= 1 / kPromptMaxSum && l_run[s] <= kPromptMaxSum && fabsf(m_ref[s]) <= kPromptMaxRef);
                fine = fine && (l_run[s] != l_run[s] || (in_range && zero[0] + zero[1] + zero[2] + zero[3] == 0.f));
            }
            if (__syncthreads_or(!fine) != 0) {              // (all waves have read the stages)
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // (what was requested beyond the last tile)
                auto tile_here = [&] {
                    request_k(0);
                    request_v(0);
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __syncthreads();
                };
                // bf16 pairs: 1, 2^8 and 2^16 for +infinity, -infinity and NaN, 0 elsewhere (sums over a tile are exact); the values with 0 in their place
                auto code = [](uint32_t w) {
                    const uint32_t x = w & 0x7fffu, y = w >> 16 & 0x7fffu;
                    return (x < 0x7f80u ? 0u : x > 0x7f80u ? 0x4780u : (w & 0x8000u) != 0 ? 0x4380u : 0x3f80u) |
                           (y < 0x7f80u ? 0u : y > 0x7f80u ? 0x4780u : w >> 31 != 0 ? 0x4380u : 0x3f80u) << 16;
                };
                auto finite = [](uint32_t w) {
                    return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
                };
                auto of_words = [](const bf16x8 &x, auto f) {
                    const uint4 w = __builtin_bit_cast(uint4, x);
                    return __builtin_bit_cast(bf16x8, make_uint4(f(w.x), f(w.y), f(w.z), f(w.w)));
                };
                bool some = false;                           // values that are not finite
                uint32_t up[SETS][2], down[SETS][2];         // of the lane's 64 results: which get +infinity, -infinity (both: NaN)
#pragma unroll
                for (int s = 0; s < SETS; ++s) up[s][0] = up[s][1] = down[s][0] = down[s][1] = 0;
#pragma unroll
                for (int s = 0; s < SETS; ++s) m_ref[s] = kPromptLowest;
                k_next = kb; v_next = vb;
                k_tile = v_tile = 0;
                for (t = 0; t < n_tiles; ++t) {
                    tile_here();
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        scores(0, s);
                        mask(t, s);
                        m_ref[qs(s)] = fmaxf(m_ref[qs(s)], row_max(sc[s]));
                    }
                    bool found = false;                      // by any of the 256 threads in its share of the tile
#pragma unroll
                    for (int i = 0; i < kEl / (8 * 64 * kPromptWaves); ++i) {
                        const uint4 w = reinterpret_cast<const uint4 *>(smem + kStages * kEl)[i * 64 * kPromptWaves + tid];
                        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int c = 0; c < 4; ++c) found |= (x[c] & 0x7f80u) == 0x7f80u || (x[c] & 0x7f800000u) == 0x7f800000u;
                    }
                    if (__syncthreads_or(found) != 0) {
                        some = true;
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const uint32_t bits = hidden_keys(t, s);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                pw[s][i] = 0;
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int r = 2 * i + e;
                                    pw[s][i] |= (bits >> (8 * (r >> 2) + (r & 3)) & 1) != 0 ? 0u : 0x3f80u << (16 * e);
                                }
                            }
                        }
                        clear();
#pragma unroll
                        for (int s = 0; s < 2; ++s)
#pragma unroll
                            for (int i = 0; i < 8; ++i) product(s, i, of_words(v_operand(0, s, i), code), probabilities(s, i >> 2));
                        settle();
#pragma unroll
                        for (int s = 0; s < SETS; ++s)
#pragma unroll
                            for (int r = 0; r < 64; ++r) {
                                const uint32_t sum = (uint32_t)o[s][r / 16][r % 16];
                                up[s][r / 32] |= ((sum & 0xffu) != 0 || sum > 0xffffu ? 1u : 0u) << (r % 32);
                                down[s][r / 32] |= (sum > 0xffu ? 1u : 0u) << (r % 32);
                            }
                    }
                    __syncthreads();
                }
                clear();
                k_next = kb; v_next = vb;
                k_tile = v_tile = 0;
                for (t = 0; t < n_tiles; ++t) {
                    tile_here();
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        scores(0, s);
                        mask(t, s);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {        // against the maximum as it came from the products: scaled, it would be rounded
                            const float x = __builtin_amdgcn_exp2f(fmaf(sc[s][2 * i] - m_ref[qs(s)], a.scale_log2e, -kPromptShift));
                            const float y = __builtin_amdgcn_exp2f(fmaf(sc[s][2 * i + 1] - m_ref[qs(s)], a.scale_log2e, -kPromptShift));
                            l_turn = i == 0 ? x + y : l_turn + x + y;
                            pw[s][i] = pack_bf16x2(x, y);
                        }
                        l_run[qs(s)] += l_turn;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            bf16x8 x = v_operand(0, s, i);
                            if (some) x = of_words(x, finite);
                            product(s, i, x, probabilities(s, i >> 2));
                        }
                    }
                    __syncthreads();
                }
                settle();
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
                    m_ref[s] = fmaf(m_ref[s], a.scale_log2e, kPromptShift);
                    l_run[s] = half_swap(l_run[s], [](float x, float y) { return x + y; });
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            if ((up[s][dt / 2] >> (16 * (dt & 1) + r) & 1) != 0) o[s][dt][r] += INFINITY;
                            if ((down[s][dt / 2] >> (16 * (dt & 1) + r) & 1) != 0) o[s][dt][r] -= INFINITY;
                        }
                }
            }
            if (SHARES && n_tiles < all_tiles) {             // a part: its share's first (which does not begin the block) or last one
                const int64_t unit = (int64_t)(2 * share + (tile0 == 0)) * kPromptWaves + wave;
                float4 *to = a.part_o + unit * SETS * 16 * 64 + lane;
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                        for (int r4 = 0; r4 < 4; ++r4)
                            to[(s * 16 + dt * 4 + r4) * 64] = make_float4(o[s][dt][r4 * 4], o[s][dt][r4 * 4 + 1], o[s][dt][r4 * 4 + 2], o[s][dt][r4 * 4 + 3]);
                    if (half == 0) a.part_ml[(unit * SETS + s) * 32 + n] = make_float2(m_ref[s], l_run[s]);
                }
            } else {
                // The results go out through LDS, so that whole rows are written: 16-byte chunk c of row r at slot c ^ r % 16.  256 queries of 32 heads on 256
                // keys each 17.4 -> 15.9 us
                int l = lane;                                    // (as above)
                asm volatile("" : "+v"(l));
                const int n = l & 31, half = l >> 5;
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
                    const float inv = l_run[s] == 0.f ? 0.f : 1.0f / l_run[s];             // (a query without keys: 0)
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                        for (int r4 = 0; r4 < 4; ++r4)
                            *reinterpret_cast<uint2 *>(rows + (s * 32 + n) * kD + (((dt * 4 + r4) ^ (n & 15)) << 3) + half * 4) =
                                make_uint2(pack_bf16x2(o[s][dt][r4 * 4] * inv, o[s][dt][r4 * 4 + 1] * inv), pack_bf16x2(o[s][dt][r4 * 4 + 2] * inv, o[s][dt][r4 * 4 + 3] * inv));
                    int of;
                    const int q = query_of(wave * Shape::kSetRows + s * 32 + n, of);
                    if (a.lse != nullptr && half == 0 && row0 + s * 32 + n < n_rows)
                        a.lse[(int64_t)(seq.q_first + q) * a.Hq + head0 + of] = l_run[s] == 0.f ? -INFINITY : (m_ref[s] + log2f(l_run[s])) * 0.69314718055994530942f;
                }
                asm volatile("" ::: "memory");                   // lanes read what other lanes of the wave wrote (LDS keeps the order)
                // four rows at a time: 4 / G queries and 4 % G heads further, or a query more and G heads less
                const int row = l >> 4, slot = l & 15;
                int of;
                const int q = query_of(wave * Shape::kSetRows + row, of);
                uint16_t *out = a.out + ((int64_t)(seq.q_first + query0) * a.Hq + head0) * kD;
                int at = ((q - query0) * a.Hq + of) * kD + slot * 8;
                const int heads = 4 % a.G, step = (4 / a.G * a.Hq + heads) * kD, wrap = (a.Hq - a.G) * kD;
                auto row_piece = [&](int i) { return *reinterpret_cast<const uint4 *>(rows + (4 * i + row) * kD + ((slot ^ (4 * (i & 3) + row)) << 3)); };
                uint4 piece[Shape::kSetRows / 4];
#pragma unroll
                for (int i = 0; i < Shape::kSetRows / 4; ++i) piece[i] = row_piece(i);
#pragma unroll
                for (int i = 0; i < Shape::kSetRows / 4; ++i) {
                    if (row0 + 4 * i + row < n_rows) *reinterpret_cast<uint4 *>(out + at) = piece[i];
                    of += heads;
                    at += step + (of >= a.G ? wrap : 0);
                    of -= of >= a.G ? a.G : 0;
                }
            }
        }
        if (!SHARES || is_end) break;
        tile0 = 0;
        if (++m >= seq.blocks) {                         // on to the next block of the list
            m = 0;
            do {
                if (++b == a.B) { b = 0; ++head; }
            } while (head < a.Hkv && Seq(a, b).blocks == 0);
        }
        if (head >= a.Hkv) break;
        __syncthreads();                                 // the last tile's values have been read
    }
}

// The parts of the block that boundary `blockIdx.x` + 1 of the shares is the first to cut; the queries of one of its waves a workgroup, a
// quarter of each lane's accumulators a wave.
__global__ __launch_bounds__(256) void prompt_merge_kernel(const PromptArgs a, int workgroups)
{
    constexpr int kPieces = 8;                       // 16-byte pieces of a lane's accumulators, of which each of the four waves takes a quarter
    const int lane = threadIdx.x & 63, quarter = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = blockIdx.y;
    const int64_t per_head = head_weight(a, lane), whole = per_head * a.Hkv;
    const int shares = prompt_shares(whole, workgroups), j = blockIdx.x + 1;
    if (whole == 0 || j >= shares) return;
    const PromptPlace p = prompt_place(a, j * whole / shares, per_head, lane);
    const PromptSeq<2> seq(a, p.b);
    const int tiles = seq.tiles(p.m);
    if (p.tile == 0 || p.tile == tiles) return;      // cuts nothing
    auto tile_of = [&](int k) {                      // where share k begins in this block, its end if behind it
        const int64_t w = k * whole / shares - p.begin;
        return k >= shares || w >= (int64_t)tiles + PromptShape<2>::kBlockCost ? tiles : seq.part_begin(p.m, w);
    };
    if ((j - 1) * whole / shares >= p.begin) {
        const int before = tile_of(j - 1);
        if (before > 0) return;                      // not the first
    }
    const int n = lane & 31, half = lane >> 5, s = quarter * kPieces / 16;
    float M = kPromptLowest, L = 0.f;
    float4 acc[kPieces];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    };
    // share k's part of the block is [tile_of(k), tile_of(k + 1)), the first one's from 0; a lane finds that of one share.  f takes the parts
    // that a wave has found: the lanes that have one, and a lane's
    auto for_parts = [&](auto f) {
        int begun = 0;
        for (int k0 = j - 1; begun < tiles; k0 += 64) {
            const int end = tile_of(k0 + lane + 1);
            int begin = __shfl_up(end, 1, 64);
            if (lane == 0) begin = begun;
            begun = __builtin_amdgcn_readlane(end, 63);
            f(__ballot(begin < end), 2 * (k0 + lane) + (begin == 0));
        }
    };
    auto unit_of = [&](unsigned long long left, int part) { return (int64_t)__builtin_amdgcn_readlane(part, __builtin_ctzll(left)) * kPromptWaves + wave; };
    auto sums_of = [&](int64_t unit) { return a.part_ml[(unit * 2 + s) * 32 + n]; };
    auto results_of = [&](int64_t unit) { return a.part_o + (unit * 32 + quarter * kPieces) * 64 + lane; };
    // Up to four parts are read at a time: 64 queries on 60,064 keys, which are cut into 64 parts, 117 -> 107 us
    clear();
    for_parts([&](unsigned long long left, int part) {
        auto take = [&](auto count) {
            constexpr int N = decltype(count)::value;
            float2 ml[N];
            float4 x[N][kPieces];
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const int64_t unit = unit_of(left, part);
                left &= left - 1;
                ml[c] = sums_of(unit);
                const float4 *from = results_of(unit);
#pragma unroll
                for (int i = 0; i < kPieces; ++i) x[c][i] = from[i * 64];
            }
            float top = M;
#pragma unroll
            for (int c = 0; c < N; ++c) top = fmaxf(top, ml[c].x);
            const float old = __builtin_amdgcn_exp2f(M - top);
            M = top;
            L *= old;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) acc[i] = make_float4(acc[i].x * old, acc[i].y * old, acc[i].z * old, acc[i].w * old);
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float w = __builtin_amdgcn_exp2f(ml[c].x - top - kPromptShift);      // (for sums over the parts that are finite)
                L += ml[c].y * w;
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
                    acc[i] = make_float4(acc[i].x + x[c][i].x * w, acc[i].y + x[c][i].y * w, acc[i].z + x[c][i].z * w, acc[i].w + x[c][i].w * w);
            }
        };
        while (__popcll(left) >= 4) take(std::integral_constant<int, 4>{});
        if (__popcll(left) >= 2) take(std::integral_constant<int, 2>{});
        if (left != 0) take(std::integral_constant<int, 1>{});
    });
    // What is infinite, from an infinite value, stays so with any weight, where infinity times 0 would be NaN
    float zero = 0.f;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) zero = fmaf(acc[i].x, 0.f, fmaf(acc[i].y, 0.f, fmaf(acc[i].z, 0.f, fmaf(acc[i].w, 0.f, zero))));
    if (__any(zero != 0.f)) {
        clear();
        for_parts([&](unsigned long long left, int part) {
            for (; left != 0; left &= left - 1) {
                const int64_t unit = unit_of(left, part);
                const float w = __builtin_amdgcn_exp2f(sums_of(unit).x - M - kPromptShift);
                const float4 *from = results_of(unit);
                auto weighted = [&](float x) { return __builtin_isinf(x) ? x : x * w; };
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const float4 x = from[i * 64];
                    acc[i] = make_float4(acc[i].x + weighted(x.x), acc[i].y + weighted(x.y), acc[i].z + weighted(x.z), acc[i].w + weighted(x.w));
                }
            }
        });
    }
    const int row = p.m * PromptShape<2>::kRows + wave * PromptShape<2>::kSetRows + s * 32 + n;
    if (row >= seq.rows) return;
    const float inv = 1.0f / L;
    const int query = seq.query(row);
    const int64_t at = (int64_t)(seq.q_first + query) * a.Hq + p.head * a.G + (row - query * a.G);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int piece = quarter * kPieces + i - 16 * s;
        *reinterpret_cast<uint2 *>(a.out + at * kD + piece * 8 + half * 4) =
            L == 0.f ? make_uint2(0, 0) : make_uint2(pack_bf16x2(acc[i].x * inv, acc[i].y * inv), pack_bf16x2(acc[i].z * inv, acc[i].w * inv));
    }
    if (a.lse != nullptr && half == 0 && quarter * kPieces == 16 * s) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L * 0x1p20f)) * 0.69314718055994530942f;
}

// Blocks x KV heads of a call, at most: a part of a block in every sequence beyond the whole ones, and no more than max_q gives each
static int64_t prompt_blocks(const ihip_packed &p, int rows)
{
    const int64_t G = p.Hq / p.Hkv, by_rows = p.rows * G / rows + p.B, by_len = p.B * ((p.max_q * G - 1) / rows + 1);
    return std::min(by_rows, by_len) * p.Hkv;
}
// Whether a call is dealt out in shares.  From what the host knows of it, total tokens, keys and sequences, in units of 32 keys for 256
// rows of one compute unit (0.7 us; a launch takes 14 us): blocks by themselves (of 128 rows, one set a wave) take as long as the
// longest, or as the rounds of them that the compute units do (blocks of the same length in whole rounds; a whole prompt's blocks, of all
// lengths up to the longest, fill the rounds), and each begins and ends.  Shares take the mean, and some time for beginnings, ends and the
// merge.  The longest of several sequences with keys ahead is not known; it is taken for twice the mean, since shares cost a
// little where all are alike and the others a lot where they are not.  max_q may be a loose bound: no sequence is taken to bring more than
// 16 times the mean.  Of 65 calls the estimate takes the faster way on 62, and what is
// 1, 13 and 14 % slower on three.
// us by themselves / in shares, 32 heads on 8: 1,024 queries 24 / 53, 8,192 469 / 578; 64 on 2,064 keys 36 / 47, 512 on 4,608 66 / 75; 200 on 8,200
// 109 / 79; 128, 256, 64 and 500 on 3,000 to 12,000 156 / 102; one each of 16 sequences on 8,000 161 / 127; 8 heads, 64 on 60,064 681 /
// 109; 16 heads on 8, 1,500 on 13,500 and 700 on 20,700 326 / 267, 1,000 on 101,000 1,514 / 707.
static bool prompt_in_shares(const ihip_packed &p, int64_t keys)
{
    if (p.max_q <= 0 || p.rows <= 0 || p.B <= 0) return false;
    const double cu = compute_units(), before = std::max<double>(0, (double)(keys - p.rows)) / p.B, mean = (double)p.rows / p.B;
    const double most = std::min<double>(p.max_q, std::min<double>(p.rows, 16 * mean));
    const double longest = ((p.B > 1 ? 2 : 1) * before + most) / 32, tiles = (before + mean / 2) / 32, alike = before / (before + mean / 2);
    auto rounds_of = [&](int rows) {
        return std::min((double)prompt_blocks(p, rows), (double)p.rows * p.Hq / rows + 0.5 * p.B * p.Hkv) / cu;
    };
    const double one = rounds_of(128);
    const double alone = std::max(0.5 * longest, (0.5 * tiles + 4) * (one + alike * (std::ceil(one) - one)) - 4);
    return (1.1 * tiles + 6) * rounds_of(256) + 40 < alone;
}
// Parts of all workgroups of a launch in shares
static size_t prompt_part_bytes() { return (size_t)2 * compute_units() * kPromptWaves * 64 * (32 * sizeof(float4) + sizeof(float2)); }

}  // namespace ihip

using namespace ihip;

extern "C" size_t ihip_prompt_attn_workspace_bytes(const ihip_packed *packed, int32_t rows_k)
{
    if (check_packed("ihip_prompt_attn_workspace_bytes", packed) != IHIP_OK) return 0;
    return prompt_in_shares(*packed, rows_k) ? prompt_part_bytes() : 256;
}

extern "C" int32_t ihip_prompt_attn(const ihip_packed *packed, ihip_tensor q, ihip_tensor k, ihip_tensor v, const int32_t *cu_k,
                                    int32_t rows_k, float sm_scale, void *out, float *out_lse, void *ws, size_t ws_bytes,
                                    void *stream)
{
    const char *who = "ihip_prompt_attn";
    int32_t rc;
    if ((rc = check_packed(who, packed)) != IHIP_OK) return rc;
    if (rows_k < 0 || (!cu_k && rows_k != packed->rows))
        return fail(IHIP_ERR_INVALID_ARG, "%s: rows_k = %d (without cu_k: the %d rows of q)", who, rows_k, packed->rows);
    if (packed->B == 0 || packed->rows == 0 || packed->max_q == 0) return IHIP_OK;
    if ((rc = check_tensor(q, who, "q")) != IHIP_OK) return rc;
    if (rows_k > 0 && ((rc = check_tensor(k, who, "k")) != IHIP_OK || (rc = check_tensor(v, who, "v")) != IHIP_OK)) return rc;
    if (!out || ((uintptr_t)out & 15)) return fail(IHIP_ERR_INVALID_ARG, "%s: out is NULL or not 16-byte aligned", who);
    PromptArgs a;
    a.B = packed->B; a.Hq = packed->Hq; a.Hkv = packed->Hkv; a.G = packed->Hq / packed->Hkv;
    a.rows_q = packed->rows; a.rows_k = rows_k;
    a.cu_q = packed->cu_q; a.cu_k = cu_k ? cu_k : packed->cu_q;
    a.q = (const uint16_t *)q.ptr; a.q_sh = q.stride_h; a.q_st = q.stride_t;
    a.k = (const uint16_t *)k.ptr; a.k_sh = k.stride_h; a.k_st = k.stride_t;
    a.v = (const uint16_t *)v.ptr; a.v_sh = v.stride_h; a.v_st = v.stride_t;
    // the rows of a tile, and of a wave's queries, are addressed by 32-bit byte offsets from the first
    if ((a.q_st | a.k_st | a.v_st) < 0 || a.q_st >= (1 << 24) || a.k_st >= (1 << 24) || a.v_st >= (1 << 24))
        return fail(IHIP_ERR_UNSUPPORTED, "%s: rows of q, k and v must be less than 2^24 elements apart", who);
    const int64_t groups = prompt_blocks(*packed, PromptShape<1>::kRows);
    if (groups > INT32_MAX) return fail(IHIP_ERR_UNSUPPORTED, "%s: %lld workgroups are too many", who, (long long)groups);
    // so are a KV head's rows counted, and the results of a block, which are the heads of up to kRows / G + 2 queries
    constexpr int most = PromptShape<2>::kRows;
    if ((int64_t)a.rows_q * a.G > INT32_MAX - most || ((most / a.G + 2) * (int64_t)a.Hq + a.G) * kD > INT32_MAX)
        return fail(IHIP_ERR_UNSUPPORTED, "%s: %d rows of %d heads (%d KV heads) are too many", who, a.rows_q, a.Hq, a.Hkv);
    if ((rc = check_sm_scale(who, sm_scale, &a.scale_log2e)) != IHIP_OK) return rc;
    a.log2_G = pow2(a.G) ? __builtin_ctz(a.G) : -1;
    a.out = (uint16_t *)out;
    a.lse = out_lse;
    const hipStream_t st = (hipStream_t)stream;
    if (ws && !((uintptr_t)ws & 15) && ws_bytes >= prompt_part_bytes() && prompt_in_shares(*packed, rows_k)) {
        constexpr int lds = PromptShape<2>::kLds;
        static bool attr_set = false;        // allow more than 64 KiB of dynamic LDS, once
        if (!attr_set) {
            (void)hipFuncSetAttribute(reinterpret_cast<const void *>(&prompt_attn_kernel<2>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            attr_set = true;
        }
        const int n = PromptShape<2>::kPerCu * compute_units();
        a.part_o = (float4 *)ws;
        a.part_ml = (float2 *)(a.part_o + (size_t)2 * n * kPromptWaves * 32 * 64);
        {
            KernelTimer timer("prompt_attn_shares", st);
            hipLaunchKernelGGL(prompt_attn_kernel<2>, dim3(n), dim3(64 * kPromptWaves), lds, st, a);
        }
        if ((rc = check_launch(who)) != IHIP_OK) return rc;
        KernelTimer timer("prompt_merge", st);
        hipLaunchKernelGGL(prompt_merge_kernel, dim3(n, kPromptWaves), dim3(256), 0, st, a, n);
        return check_launch(who);
    }
    typedef PromptShape<1> Shape;
    // The order of the blocks matters where some compute unit has two.  Finding them without it is shorter: 512 queries, 32 heads 18.5 -> 17.6 us
    a.ordered = packed->B <= kOrderedSeqs && groups > compute_units();
    const int64_t places = ((int64_t)packed->max_q * a.G - 1) / Shape::kRows + 1;
    a.places = groups == places * packed->B * packed->Hkv ? (int)places : 0;
    KernelTimer timer("prompt_attn", st);
    hipLaunchKernelGGL(prompt_attn_kernel<1>, dim3((uint32_t)groups), dim3(64 * kPromptWaves), Shape::kLds, st, a);
    return check_launch(who);
}

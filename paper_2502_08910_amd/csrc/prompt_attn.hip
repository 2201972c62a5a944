// Dense causal attention of packed prompts on v_mfma_f32_32x32x16_bf16.
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
constexpr int kPromptRows = 64 * kPromptWaves;       // queries of a workgroup (two sets of 32 a wave)
constexpr int kTileKeys = 32;
constexpr int kTileEl = kTileKeys * kD;              // bf16 elements of a K or V tile in LDS
constexpr int kPromptStages = 4;
constexpr float kNegBigPrompt = -1.0e30f;            // finite stand-in for -inf in maxima
constexpr float kPromptMaxSum = 18446744073709551616.0f;      // 2^64: sum of exponentials beyond which a block is done again

int32_t check_packed(const char *who, const ihip_packed *p);

struct PromptArgs {
    int B, Hq, Hkv, G, rows_q, rows_k;
    const int32_t *cu_q, *cu_k;
    const uint16_t *q, *k, *v;
    int64_t q_sh, q_st, k_sh, k_st, v_sh, v_st;
    float scale_log2e;
    uint16_t *out;                   // [rows_q, Hq, d]
    float *lse;                      // [rows_q, Hq] or null
    // launches whose work is dealt out in equal shares: partial results of parts of blocks, two a workgroup
    float4 *part_o;                  // [part][wave][accumulators of a lane, four at a time: 32][lane]
    float2 *part_ml;                 // [part][wave][64 queries]: reference of the exponentials (log2 units), sum
};

// ---- shares ------------------------------------------------------------------
// Where there are too few blocks of 256 queries x heads to keep the compute units busy to the end, the tiles of all blocks are dealt out
// to one workgroup a unit in equal shares, which begin and end inside blocks; a second kernel merges the parts of a block.  The
// list goes head by head (the query heads of a KV head next to each other), sequence by sequence, block by block; a block weighs its
// tiles and kBlockCost for its beginning and end.
constexpr int kBlockCost = 4, kMinPart = 4, kMinShare = 12;      // tiles

template <int ROWS>
struct PromptSeqOf {
    int q_first, nq, k_first, nk;
    int ahead, blocks, ahead_tiles;
    __device__ PromptSeqOf() {}
    __device__ PromptSeqOf(const PromptArgs &a, int b)
    {
        q_first = min(max(a.cu_q[b], 0), a.rows_q);
        nq = min(max(a.cu_q[b + 1], q_first), a.rows_q) - q_first;
        k_first = min(max(a.cu_k[b], 0), a.rows_k);
        nk = min(max(a.cu_k[b + 1], k_first), a.rows_k) - k_first;
        derive();
    }
    __device__ void derive()
    {
        ahead = nk - nq;                             // query i sees keys 0 .. i + ahead
        blocks = (nq + ROWS - 1) / ROWS;
        ahead_tiles = (ahead + kTileKeys - 1) >> 5;  // rounded up, also below 0
    }
    __device__ PromptSeqOf of_lane(int l) const      // that of lane l, in all lanes
    {
        PromptSeqOf r;
        r.q_first = __builtin_amdgcn_readlane(q_first, l);
        r.nq = __builtin_amdgcn_readlane(nq, l);
        r.k_first = __builtin_amdgcn_readlane(k_first, l);
        r.nk = __builtin_amdgcn_readlane(nk, l);
        r.derive();
        return r;
    }
    __device__ int tiles(int m) const
    {
        return m + 1 < blocks ? max(0, ROWS / kTileKeys * (m + 1) + ahead_tiles) : (nk + kTileKeys - 1) / kTileKeys;
    }
    __device__ int64_t weight_before(int m) const    // of blocks 0 .. m - 1, m < blocks
    {
        constexpr int per = ROWS / kTileKeys;
        const int none = min(m, ahead_tiles < 0 ? -ahead_tiles / per : 0);        // blocks whose queries see nothing
        auto sum = [&](int64_t c) { return per / 2 * c * (c + 1) + ahead_tiles * c; };
        return sum(m) - sum(none) + (int64_t)kBlockCost * m;
    }
    __device__ int64_t weight() const { return blocks == 0 ? 0 : weight_before(blocks - 1) + tiles(blocks - 1) + kBlockCost; }
    // A part begins at a multiple of a tile, kMinPart or more from both ends of the block and not behind the tile that its first
    // query sees the end of (so that every query has a key in a part's first tile); w: weight from the block's beginning.
    // The block's number of tiles stands for its end.
    __device__ int part_begin(int m, int64_t w) const
    {
        const int t = tiles(m), c = (int)min<int64_t>(max<int64_t>(w - kBlockCost, 0), t);
        if (c < kMinPart) return 0;
        if (c > t - kMinPart) return t;
        const int last = min((m * ROWS + ahead) / kTileKeys, t - kMinPart);
        return c <= last ? c : last < kMinPart ? t : last;
    }
};
typedef PromptSeqOf<kPromptRows> PromptSeq;
__device__ inline int64_t wave_sum_i64(int64_t v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ inline int64_t head_weight(const PromptArgs &a, int lane)
{
    int64_t w = 0;
    for (int b = lane; b < a.B; b += 64) w += PromptSeq(a, b).weight();
    return wave_sum_i64(w);
}
struct PromptPlace { int head, b, m, tile; int64_t begin; };        // head in list order; begin: weight in front of the block
__device__ inline PromptPlace prompt_place(const PromptArgs &a, int64_t x, int64_t per_head, int lane)
{
    PromptPlace r{(int)(x / per_head), 0, 0, 0, 0};
    int64_t y = x % per_head;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int64_t w = b0 + lane < a.B ? PromptSeq(a, b0 + lane).weight() : 0;
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
    const PromptSeq q(a, r.b);
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
__device__ inline int prompt_shares(int64_t whole, int n) { return __builtin_amdgcn_readfirstlane((int)min<int64_t>(n, max<int64_t>(1, whole / kMinShare))); }

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

// SHARES: as above; otherwise a workgroup a block and head, the heads of a block next to each other, those with most keys first.
// SETS: sets of 32 queries of a wave, 2, or 1 where there are too few blocks otherwise.  With one, the two tiles of a group take the place of the
// two sets everywhere below: they are worked on in turn, and both go to the same queries.
template <int SETS, bool SHARES>
__global__ __launch_bounds__(64 * kPromptWaves, 1) void prompt_attn_kernel(const PromptArgs a)
{
    static_assert(SETS == 2 || (SETS == 1 && !SHARES), "shares are made of blocks of two sets a wave");
    constexpr int kSetRows = 32 * SETS, kRows = kSetRows * kPromptWaves;       // queries of a wave and of the workgroup
    constexpr int kGroup = 3 - SETS, kGroupKeys = kGroup * kTileKeys, kGroupEl = kGroup * kTileEl;
    constexpr int kLoads = kGroupKeys / (4 * kPromptWaves);                    // of a wave for K (and for V) of a group
    typedef PromptSeqOf<kRows> Seq;
    extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    // this wave's results on their way out: behind the stages, or, where those take all of LDS, in their place
    uint16_t *const rows = smem + (SETS == 2 ? kPromptStages * 2 * kGroupEl : 0) + wave * kSetRows * kD;

    // which head, which sequence, which of its blocks, which tiles of the block
    int head, b = -1, m = 0, tile0 = 0, tile1 = 0, share = 0;
    PromptPlace end{};
    Seq seq;
    if constexpr (SHARES) {
        const int64_t per_head = head_weight(a, lane), whole = per_head * a.Hq;
        const int shares = prompt_shares(whole, gridDim.x);
        // workgroups are dealt to the eight XCDs in turn: each gets shares that follow each other, of one KV head if there are eight
        share = shares % 8 == 0 && (int)gridDim.x == shares ? (blockIdx.x & 7) * (shares / 8) + (blockIdx.x >> 3) : blockIdx.x;
        if (share >= shares || __builtin_amdgcn_readfirstlane((int)(whole == 0)) != 0) return;
        const PromptPlace p = prompt_place(a, share * whole / shares, per_head, lane);
        head = p.head; b = p.b; m = p.m; tile0 = p.tile;
        if (share + 1 < shares) end = prompt_place(a, (share + 1) * whole / shares, per_head, lane);
        else end.head = a.Hq;
    } else {
        head = blockIdx.x % a.Hq;
        head = head % a.Hkv * a.G + head / a.Hkv;    // neighbours read different KV heads, on the XCD of their own if there are eight
        int ti = blockIdx.x / a.Hq;
        if (a.B <= 64) {
            // blocks in the order of their keys, a block's worth of them at a time: key class c of a sequence's block m is base + m
            const Seq q(a, min(lane, a.B - 1));
            const int blocks = lane < a.B ? q.blocks : 0, base = max(0, q.ahead) / kRows;
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
            for (int b0 = 0; b0 < a.B; b0 += 64) {
                const int blocks = b0 + lane < a.B ? Seq(a, b0 + lane).blocks : 0;
                const int incl = (int)wave_scan_u32((uint32_t)blocks, lane);
                const unsigned long long past = __ballot(incl > ti);
                if (past != 0) {
                    const int at = __builtin_ctzll(past);
                    b = b0 + at;
                    m = __builtin_amdgcn_readlane(incl, at) - 1 - ti;          // the longest blocks of a sequence come first
                    break;
                }
                ti -= __builtin_amdgcn_readlane(incl, 63);
            }
            if (b < 0) return;
            seq = Seq(a, b);
        }
    }
    for (;;) {                                       // SHARES: blocks and parts of blocks; otherwise once
    // (the same in all lanes, which the compiler cannot see everywhere)
    head = __builtin_amdgcn_readfirstlane(head);
    b = __builtin_amdgcn_readfirstlane(b);
    m = __builtin_amdgcn_readfirstlane(m);
    tile0 = __builtin_amdgcn_readfirstlane(tile0);
    if (SHARES) seq = Seq(a, b);
    const int nq = seq.nq, nk = seq.nk, ahead = seq.ahead;
    const int all_tiles = __builtin_amdgcn_readfirstlane(seq.tiles(m));
    const bool is_end = SHARES && __builtin_amdgcn_readfirstlane((int)(head == end.head && b == end.b && m == end.m)) != 0;
    tile1 = __builtin_amdgcn_readfirstlane(is_end ? end.tile : all_tiles);
    if (all_tiles == 0 && !is_end) {                 // queries without keys
        for (int i = tid; i < min(kRows, nq - m * kRows) * kRowLanes; i += 64 * kPromptWaves) {
            const int64_t at = (int64_t)(seq.q_first + m * kRows + i / kRowLanes) * a.Hq + head;
            reinterpret_cast<uint4 *>(a.out + at * kD)[i % kRowLanes] = make_uint4(0, 0, 0, 0);
            if (a.lse != nullptr && i % kRowLanes == 0) a.lse[at] = -INFINITY;
        }
    } else if (tile0 < tile1) {
    const int h = head, g = h / a.G;
    const int row0 = m * kRows + wave * kSetRows;    // this wave's first query
    const int n_groups = (tile1 - tile0 + kGroup - 1) / kGroup;      // of tiles of this part, numbered from its first
    auto qs = [](int s) { return SETS == 2 ? s : 0; };               // the queries of set s, and its tile in group t
    auto tile_of = [](int t, int s) { return SETS == 2 ? t : 2 * t + s; };

    bf16x8 qb[SETS][8];
    int last_key[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) last_key[s] = min(row0 + s * 32 + n, nq - 1) + ahead - tile0 * kTileKeys;
    auto load_queries = [&] {
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            const uint16_t *qp = a.q + (int64_t)(seq.q_first + min(row0 + s * 32 + n, nq - 1)) * a.q_st + h * a.q_sh + half * 8;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) qb[s][ks] = *reinterpret_cast<const bf16x8 *>(qp + ks * 16);
        }
    };
    const int first_last = row0 + ahead - tile0 * kTileKeys;       // the last key of the wave's first query
    const int keys_here = nk - tile0 * kTileKeys;
    const uint16_t *kb = a.k + ((int64_t)seq.k_first + (int64_t)tile0 * kTileKeys) * a.k_st + g * a.k_sh;
    const uint16_t *vb = a.v + ((int64_t)seq.k_first + (int64_t)tile0 * kTileKeys) * a.v_st + g * a.v_sh;

    // Loads of a group of tiles (32 keys with two sets, 64 with one): four-row instructions, dealt to the waves.  Lane l brings 16 bytes of row
    // 4 j + l / 16 to base + 16 l.  The base of a group is scalar; a lane's offset from it changes in a group that reaches behind the last key
    // only, whose rows stand for the missing ones.  What would come after the last group is the last one again, so that every period
    // has as many loads on their way as any other.
    auto offset = [&](int i, int rows, int64_t st, bool is_v) {
        const int key = 4 * (wave + i * kPromptWaves) + (lane >> 4), at = min(key, rows - 1), slot = lane & 15;
        return (uint32_t)(at * (int)st + ((slot ^ (is_v ? (key & 3) << 2 : key & 15)) << 3)) * 2u;
    };
    uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        k_off[i] = offset(i, kGroupKeys, a.k_st, false);
        v_off[i] = offset(i, kGroupKeys, a.v_st, true);
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem + wave * 4 * kD * 2;
    const bool cut = n_groups * kGroupKeys > keys_here;     // the last group reaches behind the last key
    const uint16_t *k_next = kb, *v_next = vb;       // of the groups to be requested next
    int k_group = 0, v_group = 0;
    auto request = [&](bool is_v, int st) {
        int &group = is_v ? v_group : k_group;
        const uint16_t *&next = is_v ? v_next : k_next;
        const int64_t stride = is_v ? a.v_st : a.k_st;
        uint32_t off[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) off[i] = is_v ? v_off[i] : k_off[i];
        if (cut && group == n_groups - 1) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) off[i] = offset(i, keys_here - group * kGroupKeys, stride, is_v);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            prompt_to_lds(lds0 + ((is_v ? kPromptStages : 0) + st) * kGroupEl * 2 + i * 4 * kPromptWaves * kD * 2, next, off[i]);
        const bool more = group < n_groups - 1;
        next += more ? kGroupKeys * stride : 0;
        group += more;
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
            v_at[dt] = smem + kPromptStages * kGroupEl + key * kD + ((chunk ^ ((key & 3) << 2)) << 3) + ((i & 1) << 2);
        }
    }
    // operand of a stage for set s (with two sets the same tile for both); i: 4 kk + dt
    auto k_operand = [&](int st, int s, int ks) { return *reinterpret_cast<const bf16x8 *>(k_at[ks] + st * kGroupEl + (SETS == 1 ? s * kTileEl : 0)); };
    auto v_operand = [&](int st, int s, int i) {
        const uint16_t *at = v_at[i & 3] + st * kGroupEl + (SETS == 1 ? s * kTileEl : 0) + 16 * (i >> 2) * kD;
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
    // Keys of a tile that a lane's query must not see, as bits: score r is that of key 8 (r / 4) + 4 half + r % 4
    auto hidden_keys = [&](int tile, int s) { return ~0u << min(max(last_key[qs(s)] - 4 * half - tile * kTileKeys + 1, 0), 31); };
    auto hide = [&](uint32_t bits, int r, float x) {         // v_bfe_i32, v_bfi_b32
        const int hidden = (int)(bits << (31 - (8 * (r >> 2) + (r & 3)))) >> 31;
        return __int_as_float((hidden & __float_as_int(-INFINITY)) | (~hidden & __float_as_int(x)));
    };
    auto mask = [&](int tile, int s) {
        if (tile * kTileKeys + kTileKeys - 1 <= first_last + qs(s) * 32) return;
        const uint32_t bits = hidden_keys(tile, s);
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[s][r] = hide(bits, r, sc[s][r]);
    };
    auto row_max = [&](const f32x16 &s) {            // scaled; of both halves
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        return half_swap(mx, [](float x, float y) { return fmaxf(x, y); }) * a.scale_log2e;
    };

    uint32_t pw[2][8];                               // the probabilities of a set, in pairs of keys
    float m_ref[SETS], l_run[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        m_ref[s] = kNegBigPrompt;
        l_run[s] = 0.f;
    }
    // two scores -> two probabilities (exp2(-inf) = 0).  The empty assembly keeps them where they are called: left to themselves all
    // exponentials of a phase would be computed in front of its matrix instructions instead of under them.
    auto exponentials = [&](int s, int i, bool masked, uint32_t bits) {
        float x = fmaf(sc[s][2 * i], a.scale_log2e, -m_ref[qs(s)]), y = fmaf(sc[s][2 * i + 1], a.scale_log2e, -m_ref[qs(s)]);
        if (masked) {
            x = hide(bits, 2 * i, x);
            y = hide(bits, 2 * i + 1, y);
        }
        asm volatile("" : "+v"(x), "+v"(y));
        x = __builtin_amdgcn_exp2f(x);
        y = __builtin_amdgcn_exp2f(y);
        l_run[qs(s)] += x;
        l_run[qs(s)] += y;
        pw[s][i] = pack_bf16x2(x, y);
        asm volatile("" : "+v"(pw[s][i]), "+v"(l_run[qs(s)]));
    };
    auto probabilities = [&](int s, int kk) {
        return __builtin_bit_cast(bf16x8, make_uint4(pw[s][4 * kk], pw[s][4 * kk + 1], pw[s][4 * kk + 2], pw[s][4 * kk + 3]));
    };
    // Period t, for the two sets of 32 queries in turn: first product of tile t + 1 and second product of tile t, and under them the
    // exponentials of the other set, 16 matrix instructions and 16 scores a lane at a time.  K of tile t + 4 and V of tile t + 3 are
    // requested into the stages that period t - 1 has read, and have landed when period t + 1 ends; the first operands of period
    // t + 1 are read from LDS as this one ends.  Matrix instructions are written as assembly: of the 512 registers that the one wave of
    // a SIMD has, they can keep the accumulators in the upper half ("a") and everything else in the lower one, and they stay where
    // they are, each with its share of the vector instructions under it.  The compiler does not know the instructions' latency: a set's
    // scores are read by vector instructions eight matrix instructions after their last one.
    bf16x8 ka[8], va[8];
    auto first_operands = [&](int st, int st1, int s) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            ka[i] = k_operand(st1, s, i);
            va[i] = v_operand(st, s, i);
        }
    };
    auto period = [&](int st, int st1, int st2, int st3, int t, bool masked) {      // stages of groups t, t + 1, t + 2, t + 3
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t bits = masked ? hidden_keys(tile_of(t + s, 1 - s), 1 - s) : 0u;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = r & 7;
                if ((s == 0 || SETS == 1) && r < 6) ka[r + 2] = k_operand(st1, s, r + 2);
                if ((s == 0 || SETS == 1) && r >= 6 && r < 12) va[r - 4] = v_operand(st, s, r - 4);
                if (s == 0 && SETS == 1 && r == 10) first_operands(st, st1, 1);
                if (s == 1 && r == 10) first_operands(st1, st2, 0);
                if (r == 0) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=v"(sc[s]) : "v"(ka[0]), "v"(qb[qs(s)][0]));
                else if (r < 8) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(sc[s]) : "v"(ka[r]), "v"(qb[qs(s)][r]));
                else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o[qs(s)][i & 3]) : "v"(va[i]), "v"(probabilities(s, i >> 2)));
                if (r % 2 == 0) exponentials(1 - s, r / 2, masked, bits);
                if (s == 0 && r == 3) request_k(st);
                if (s == 0 && r == 9) request_v(st3);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
        __syncthreads();
    };
    // Exponentials are taken against the row's maximum over the first tile (which holds a key of every query that has any), not
    // against a running one: bf16 and fp32 have exponents to spare, nothing is lost while the scores stay within 2^64 of it.  Where a
    // row's sum says that they did not, the block is done again against the maxima over all tiles.
    for (int again = 0; again < 2; ++again) {
        if (again) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // (what was requested beyond the last group)
            k_next = kb;
            k_group = 0;
#pragma unroll
            for (int s = 0; s < SETS; ++s) m_ref[s] = kNegBigPrompt;
            for (int t = 0; t < n_groups; ++t) {
                request_k(0);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    scores(0, s);
                    mask(tile_of(t, s), s);
                    m_ref[qs(s)] = fmaxf(m_ref[qs(s)], row_max(sc[s]));
                }
                __syncthreads();
            }
        }
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            l_run[s] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[s][dt] = f32x16{};
        }
        k_next = kb; v_next = vb;
        k_group = v_group = 0;
#pragma unroll
        for (int st = 0; st < 4; ++st) request_k(st);
#pragma unroll
        for (int st = 0; st < 3; ++st) request_v(st);
        if (!again) load_queries();
        // (the accumulators are cleared while the loads are on their way)
#pragma unroll
        for (int s = 0; s < SETS; ++s) asm volatile("" : "+a"(o[s][0]), "+a"(o[s][1]), "+a"(o[s][2]), "+a"(o[s][3]));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            scores(0, s);
            mask(tile_of(0, s), s);
            if (!again) m_ref[qs(s)] = fmaxf(SETS == 2 ? kNegBigPrompt : m_ref[0], row_max(sc[s]));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) exponentials(0, i, false, 0);
        __syncthreads();                             // K(0) has been read
        first_operands(0, 1, 0);
        int t = 0;
        // groups of whole tiles that all queries of the block see; behind them scores are masked, under the matrix instructions as well
        const int seen = min(n_groups, ((m * kRows + ahead + 1) / kTileKeys - tile0) / kGroup);
        for (; t + 4 < seen; t += 4) {
            period(0, 1, 2, 3, t, false);
            period(1, 2, 3, 0, t + 1, false);
            period(2, 3, 0, 1, t + 2, false);
            period(3, 0, 1, 2, t + 3, false);
        }
        for (; t + 1 < n_groups; ++t) period(t & 3, (t + 1) & 3, (t + 2) & 3, (t + 3) & 3, t, true);
        // the last group, whose first products are done
        const uint32_t bits = hidden_keys(tile_of(t, 1), 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) exponentials(1, i, true, bits);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            bf16x8 vt = v_operand(t & 3, 0, i);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (SETS == 1 && s == 1) vt = v_operand(t & 3, 1, i);
                asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o[qs(s)][i & 3]) : "v"(vt), "v"(probabilities(s, i >> 2)));
            }
        }
        // (the compiler does not know that there are matrix instructions in the assembly, whose results take up to 19 wait states)
#pragma unroll
        for (int s = 0; s < SETS; ++s) asm volatile("s_nop 15\n\ts_nop 7" : "+a"(o[s][0]), "+a"(o[s][1]), "+a"(o[s][2]), "+a"(o[s][3]));
        bool in_range = true;
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            l_run[s] = half_swap(l_run[s], [](float x, float y) { return x + y; });
            in_range = in_range && l_run[s] <= kPromptMaxSum;
        }
        if (again || __syncthreads_or(!in_range) == 0) break;
    }
    if (SHARES && n_groups < all_tiles) {             // a part: its share's first (which does not begin the block) or last one
        const int64_t unit = (int64_t)(2 * share + (tile0 == 0)) * kPromptWaves + wave;
        float4 *to = a.part_o + unit * 32 * 64 + lane;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4)
                    to[(s * 16 + dt * 4 + r4) * 64] = make_float4(o[s][dt][r4 * 4], o[s][dt][r4 * 4 + 1], o[s][dt][r4 * 4 + 2], o[s][dt][r4 * 4 + 3]);
            if (half == 0) a.part_ml[unit * 64 + s * 32 + n] = make_float2(m_ref[s], l_run[s]);
        }
    } else {
    // The results go out through LDS, so that whole rows are written: 16-byte chunk c of row r at slot c ^ r % 16.  256 queries of 32 heads on 256
    // keys each 17.4 -> 14.4 us
    if (SETS == 1) {                                 // in place of the stages, once they have been read and the last requests have come
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const float l = l_run[s];
        const int row = row0 + s * 32 + n;
        const float inv = l == 0.f ? 0.f : 1.0f / l;           // (a query without keys: 0)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<uint2 *>(rows + (s * 32 + n) * kD + (((dt * 4 + r4) ^ (n & 15)) << 3) + half * 4) =
                    make_uint2(pack_bf16x2(o[s][dt][r4 * 4] * inv, o[s][dt][r4 * 4 + 1] * inv), pack_bf16x2(o[s][dt][r4 * 4 + 2] * inv, o[s][dt][r4 * 4 + 3] * inv));
        if (a.lse != nullptr && half == 0 && row < nq)
            a.lse[(int64_t)(seq.q_first + row) * a.Hq + h] = l == 0.f ? -INFINITY : (m_ref[s] + log2f(l)) * 0.69314718055994530942f;
    }
    asm volatile("" ::: "memory");                   // lanes read what other lanes of the wave wrote (LDS keeps the order)
    uint16_t *out = a.out + ((int64_t)(seq.q_first + row0) * a.Hq + h) * kD;
    const int64_t step = (int64_t)4 * a.Hq * kD;     // four rows
    const int64_t mine = (int64_t)(lane >> 4) * a.Hq * kD + (lane & 15) * 8;
    auto row_piece = [&](int i) { return *reinterpret_cast<const uint4 *>(rows + (4 * i + (lane >> 4)) * kD + (((lane & 15) ^ (4 * (i & 3) + (lane >> 4))) << 3)); };
    if (row0 + kSetRows <= nq) {
#pragma unroll
        for (int i = 0; i < kSetRows / 4; ++i) *reinterpret_cast<uint4 *>(out + i * step + mine) = row_piece(i);
    } else {
        for (int i = 0; i < kSetRows / 4; ++i)
            if (row0 + 4 * i + (lane >> 4) < nq) *reinterpret_cast<uint4 *>(out + i * step + mine) = row_piece(i);
    }
    }
    }
    if (!SHARES || is_end) break;
    tile0 = 0;
    if (++m >= seq.blocks) {                         // on to the next block of the list
        m = 0;
        do {
            if (++b == a.B) { b = 0; ++head; }
        } while (head < a.Hq && Seq(a, b).blocks == 0);
    }
    if (head >= a.Hq) break;
    __syncthreads();                                 // the last tile's values have been read
    }
}

// The parts of the block that boundary `blockIdx.x` + 1 of the shares is the first to cut; a wave's 64 queries a workgroup.
// Wave w of it takes accumulators 8 w .. 8 w + 7 of each lane.
__global__ __launch_bounds__(256) void prompt_merge_kernel(const PromptArgs a, int workgroups)
{
    const int lane = threadIdx.x & 63, quarter = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = blockIdx.y;
    const int64_t per_head = head_weight(a, lane), whole = per_head * a.Hq;
    const int shares = prompt_shares(whole, workgroups), j = blockIdx.x + 1;
    if (whole == 0 || j >= shares) return;
    const PromptPlace p = prompt_place(a, j * whole / shares, per_head, lane);
    const PromptSeq seq(a, p.b);
    const int tiles = seq.tiles(p.m);
    if (p.tile == 0 || p.tile == tiles) return;      // cuts nothing
    auto tile_of = [&](int k) {                      // where share k begins in this block, its end if behind it
        const int64_t w = k * whole / shares - p.begin;
        return k >= shares || w >= (int64_t)tiles + kBlockCost ? tiles : seq.part_begin(p.m, w);
    };
    if ((j - 1) * whole / shares >= p.begin) {
        const int before = tile_of(j - 1);
        if (before > 0) return;                      // not the first
    }
    const int n = lane & 31, half = lane >> 5, s = quarter >> 1;
    float M = kNegBigPrompt, L = 0.f;
    float4 acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    int begin = 0;
    for (int k = j - 1; begin < tiles; ++k) {
        const int end = tile_of(k + 1);
        if (begin < end) {
            const int64_t unit = (int64_t)(2 * k + (begin == 0)) * kPromptWaves + wave;
            const float2 ml = a.part_ml[unit * 64 + s * 32 + n];
            const float4 *from = a.part_o + (unit * 32 + quarter * 8) * 64 + lane;
            const float top = fmaxf(M, ml.x), old = __builtin_amdgcn_exp2f(M - top), w = __builtin_amdgcn_exp2f(ml.x - top);
            M = top;
            L = L * old + ml.y * w;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 x = from[i * 64];
                acc[i] = make_float4(acc[i].x * old + x.x * w, acc[i].y * old + x.y * w, acc[i].z * old + x.z * w, acc[i].w * old + x.w * w);
            }
        }
        begin = end;
    }
    const int row = p.m * kPromptRows + wave * 64 + s * 32 + n;
    if (row >= seq.nq) return;
    const float inv = 1.0f / L;
    const int64_t at = (int64_t)(seq.q_first + row) * a.Hq + p.head;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int dt = (quarter & 1) * 2 + i / 4, r4 = i & 3;
        *reinterpret_cast<uint2 *>(a.out + at * kD + dt * 32 + r4 * 8 + half * 4) =
            L == 0.f ? make_uint2(0, 0) : make_uint2(pack_bf16x2(acc[i].x * inv, acc[i].y * inv), pack_bf16x2(acc[i].z * inv, acc[i].w * inv));
    }
    if (a.lse != nullptr && half == 0 && (quarter & 1) == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994530942f;
}

// Blocks x heads of a call, at most: a part of a block in every sequence beyond the whole ones, and no more than max_q gives each
static int64_t prompt_blocks(const ihip_packed &p, int block = kPromptRows)
{
    const int64_t by_rows = (int64_t)p.rows / block + p.B, by_len = (int64_t)p.B * ((p.max_q - 1) / block + 1);
    return (by_rows < by_len ? by_rows : by_len) * p.Hq;
}
// How a call is done, from what the host knows of it: total tokens, keys and sequences.  The estimates are in tiles of 32 keys for a block of 256
// queries (0.7 us, and 14 us for a launch): a launch takes as long as its longest block, or as the rounds of blocks that the compute units do
// (blocks of the same length in whole rounds; a whole prompt's blocks, of all lengths up to the longest, fill the rounds), where a full chip
// runs slower than a few blocks and each block begins and ends.  A block of 128 queries takes 0.6 of the time for the same keys: it
// wins while there are too few blocks of 256.  Equal shares take the mean, and 50 tiles for beginnings, ends and the merge.
// us with two sets / one / shares, 32 heads: 256 queries 18 / 16 / 40, 512 26 / 19 / 52, 1,024 37 / 26 / 52, 2,048 60 / 51 / 79, 3,000
// 87 / 99 / 117, 8,192 476 / 545 / 537; 8 heads, 4,096 99 / 64 / 72; 512 on 4,608 keys 109 / 69 / 73; 200 on 8,200 180 / 114 / 81;
// 16 heads, 1,500 on 13,500 and 700 on 20,700 438 / 353 / 269; 8 heads, 64 on 60,064 1,216 / 734 / 118.
enum class PromptWay { kTwoSets, kOneSet, kShares };
static PromptWay prompt_way(const ihip_packed &p, int64_t keys, bool scratch = true)
{
    if (p.max_q <= 0 || p.rows <= 0 || p.B <= 0) return PromptWay::kTwoSets;
    const double cu = compute_units(), before = std::max<double>(0, (double)(keys - p.rows)) / p.B, mean = (double)p.rows / p.B;
    const double longest = (before + p.max_q) / kTileKeys, tiles = (before + mean / 2) / kTileKeys, alike = before / (before + mean / 2);
    auto rounds_of = [&](int block) { return std::min<double>((double)prompt_blocks(p, block), ((double)p.rows / block + 0.5 * p.B) * p.Hq) / cu; };
    auto whole = [&](int block, double per_tile, double busy) {
        constexpr double fixed = 8;                  // tiles that a block's beginning and end take
        const double rounds = rounds_of(block), filled = rounds + alike * (std::ceil(rounds) - rounds);
        return std::max(per_tile * longest, busy * (per_tile * tiles + fixed) * filled - fixed);
    };
    const double two = whole(kPromptRows, 1, 1.3), one = whole(kPromptRows / 2, 0.6, 1.1), shares = 1.4 * tiles * rounds_of(kPromptRows) + 50;
    if (scratch && shares < two && shares < one) return PromptWay::kShares;
    return one < two ? PromptWay::kOneSet : PromptWay::kTwoSets;
}
static size_t prompt_part_bytes() { return (size_t)2 * compute_units() * kPromptWaves * 64 * (32 * sizeof(float4) + sizeof(float2)); }

}  // namespace ihip

using namespace ihip;

extern "C" size_t ihip_prompt_attn_workspace_bytes(const ihip_packed *packed, int32_t rows_k)
{
    if (check_packed("ihip_prompt_attn_workspace_bytes", packed) != IHIP_OK) return 0;
    return prompt_way(*packed, rows_k) == PromptWay::kShares ? prompt_part_bytes() : 256;
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
    a.scale_log2e = sm_scale * 1.44269504088896340736f;
    a.out = (uint16_t *)out;
    a.lse = out_lse;
    const PromptWay way = prompt_way(*packed, rows_k, ws && !((uintptr_t)ws & 15) && ws_bytes >= prompt_part_bytes());
    const bool one_set = way == PromptWay::kOneSet;
    const int64_t groups = prompt_blocks(*packed, one_set ? kPromptRows / 2 : kPromptRows);
    if (groups > INT32_MAX) return fail(IHIP_ERR_UNSUPPORTED, "%s: %lld workgroups are too many", who, (long long)groups);
    const hipStream_t st = (hipStream_t)stream;
    const dim3 threads(64 * kPromptWaves);
    constexpr int lds = kPromptStages * 4 * kTileEl * 2;       // with two sets half of it is the results'
    static_assert(kPromptStages * 2 * kTileEl >= kPromptRows * kD, "the results of a block fit behind the stages");
    static bool attr_set = false;        // allow more than 64 KiB of dynamic LDS, once
    if (!attr_set) {
        for (auto kernel : {&prompt_attn_kernel<2, false>, &prompt_attn_kernel<1, false>, &prompt_attn_kernel<2, true>})
            (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        attr_set = true;
    }
    if (way == PromptWay::kShares) {
        const int n = compute_units();
        a.part_o = (float4 *)ws;
        a.part_ml = (float2 *)(a.part_o + (size_t)2 * n * kPromptWaves * 32 * 64);
        {
            KernelTimer timer("prompt_attn_shares", st);
            hipLaunchKernelGGL((prompt_attn_kernel<2, true>), dim3(n), threads, lds, st, a);
        }
        if ((rc = check_launch(who)) != IHIP_OK) return rc;
        KernelTimer timer("prompt_merge", st);
        hipLaunchKernelGGL(prompt_merge_kernel, dim3(n, kPromptWaves), dim3(256), 0, st, a, n);
        return check_launch(who);
    }
    KernelTimer timer("prompt_attn", st);
    if (one_set) hipLaunchKernelGGL((prompt_attn_kernel<1, false>), dim3((uint32_t)groups), threads, lds, st, a);
    else hipLaunchKernelGGL((prompt_attn_kernel<2, false>), dim3((uint32_t)groups), threads, lds, st, a);
    return check_launch(who);
}

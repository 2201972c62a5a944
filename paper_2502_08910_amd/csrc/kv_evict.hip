// A cache cut down to the rows that are worth most: the first tokens, the last ones, and of the others those with most attention weight.
//
// Kept rows stay where they are if that is below `keep`; the i-th evicted row below `keep` is filled with the i-th kept row from behind it.
// No row is both read and written, so all moves go at once and in any order, and a cache that drops 64 of 1,088 rows moves 64 of them.
//
// The threshold is found by its digits, most significant first, in a histogram of all rows and then among the rows of one bin; a row's key is
// its weight in an order-preserving map over its number from the end, so that no two are the same and ties go to the lower row.  What is
// kept goes down as one bit a row, and the holes below `keep` are matched to the kept rows above it by their ranks.
//   up to kHeld rows    kv_evict_select_kernel, a workgroup a (sequence, KV head), keys in LDS.  Few rows move within it.
//   more                in chunks, one workgroup each: digits, candidates, ranks (a launch each: what all chunks have found is read by the next);
//                       of very many rows two digits.  Only where more than kEvictList rows have them does each workgroup look at all rows for the rest.
//   many moves          kv_evict_move_kernel, 16 lanes a row, four rows of each on their way.
// 1,088 rows to 1,024, 32 sequences of 8 KV heads, take 9 us, phases between barriers; 32,749 to 4,096 bf16 rows 27, four launches of 5 to 8;
// 77,777 to 131,072 E4M3 rows of four sequences to 16,384 each 100, of which 63 move 450,000 rows of K and of V (4.0 TB/s) and 38 are three passes
// over 28 MB of weights and positions.  That is where weights spread over octaves.  A first digit is an eighth of an octave: of the sums that 64 queries of
// random vectors leave, 11,500 of 32,749 rows have the threshold's, 45,400 of 131,072, and the two calls take 61 and 224.
#include "api_checks.h"
#include "kv_store.h"
#include <algorithm>
#include <cstdlib>
#include <type_traits>

namespace ihip {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;
constexpr int kEvictBins = 4096, kEvictList = 4096;  // of the first digit; rows of one bin that are looked at on their own
constexpr int kAhead = 8;                            // rows of a thread that are on their way together
constexpr int kHeld = 2 * kAhead * kEvictThreads;    // rows whose keys stay in LDS
constexpr int kEvictWords = 2048;                    // words of bits in LDS, those of 131,072 rows
constexpr int kFewMoves = 512;                       // of a (sequence, KV head): within the first kernel
constexpr int kMoveThreads = 256, kMoveAhead = 4, kMoveRows = kMoveThreads / kRowLanes * kMoveAhead;     // places of a workgroup
constexpr int kEvictLeast = 4096;                    // rows of a chunk
constexpr int64_t kEvictOneDigit = 131072;           // rows up to which one digit leaves no more than kEvictList of them if weights spread over octaves
constexpr int kEvictMostChunks = 16;                // (all of them look at the histograms of all)
static_assert(kMoveRows == 64, "a workgroup moves into the rows of one word");

// What is known of a (sequence, KV head) between launches
struct EvictState {
    int32_t n;                       // rows
    uint32_t bin, need, count;       // the threshold's first digits, how many rows are kept of those that have them, how many have them
};
struct EvictArgs {
    int B, Hkv, max_len, keep, n_sink, n_recent;
    const int32_t *lens, *seen;
    const float *weights;
    const int32_t *positions;
    int rows;                        // of a head in weights and positions
    float *to_weights;
    int32_t *to_positions;
    int to_rows;
    int32_t *kept;                   // [P, keep]
    int32_t *new_lens;
    EvictState *state;               // [P]
    uint64_t *bits;                  // [P, words]
    uint2 *before;                   // [P, words]: holes and movers in front of a word
    int32_t *movers;                 // [P, most]
    int words, most;
    int chunks;
    uint2 *listed;                   // [P, kEvictList]: key and row of the rows with the first digit
    uint32_t *hist;                  // [digits, P, chunks, kEvictBins]
    int digits;                      // of 12 bits each that histograms of all rows find: 1 or 2
    uint2 *sure;                     // [P, chunks]: rows above the first digit, below `keep` and from there on
    bool set_lens;                   // the select kernel writes new_lens
    StoreView store;
};

// Larger is kept: protected rows before all weights, NaN behind them; -0 as +0
__device__ inline uint32_t evict_key(float w, int pos, int n_sink, int recent_from)
{
    if (pos < n_sink || pos >= recent_from) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct EvictDigits {
    uint32_t hist[kEvictBins];
    uint32_t wave_tot[2][kEvictWaves];
    uint32_t digit, left, count, listed;
    uint32_t sum[2];
};
struct EvictShared : EvictDigits {
    union {
        struct { uint32_t key[kEvictList]; int32_t row[kEvictList]; } list;      // while the threshold is looked for
        struct { int32_t movers[kFewMoves], holes[kFewMoves]; } moves;           // behind that
    };
    uint64_t bits[kEvictWords];
};
struct EvictHeldShared : EvictShared {
    uint2 before[kHeld / 64];
    uint32_t held[kHeld];
};

// Sum of what the waves before this one have left
__device__ inline uint32_t evict_waves_before(const uint32_t (&tot)[kEvictWaves], int lane, int wv)
{
    static_assert(kEvictWaves == 16, "a row of 16 lanes");
    uint32_t v = (lane & 15) < wv ? tot[lane & 15] : 0u;
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true);       // quad_perm [1,0,3,2]
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true);       // quad_perm [2,3,0,1]
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true);      // row_half_mirror
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true);        // row_mirror
}
// Of `bins` bins, the one from which the `need`-th largest comes: its number, what of `need` is left in it, and its rows
__device__ inline void evict_find_bin(EvictDigits &sh, int bins, uint32_t need)
{
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, per = max(1, bins / kEvictThreads);
    uint32_t h[4] = {0, 0, 0, 0}, mine = 0;          // bins in descending order: thread t has bins - 1 - per t and on
    if (per * tid < bins)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < per) mine += h[i] = sh.hist[bins - 1 - per * tid - i];
    uint32_t incl = wave_scan_u32(mine, lane);
    if (lane == 63) sh.wave_tot[0][wv] = incl;
    __syncthreads();
    incl += evict_waves_before(sh.wave_tot[0], lane, wv);
    uint32_t above = incl - mine;
    if (above < need && incl >= need) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < per && above < need && above + h[i] >= need) {
                sh.digit = bins - 1 - per * tid - i;
                sh.left = need - above;
                sh.count = h[i];
            }
            above += h[i];
        }
    }
    __syncthreads();
}
__device__ inline void evict_clear(EvictDigits &sh, int bins)
{
    for (int i = threadIdx.x; i < bins; i += kEvictThreads) sh.hist[i] = 0;
    __syncthreads();
}
// adds a wave's digits; the first one's like at once (rows of weight 0 are often many)
__device__ inline void evict_count(EvictDigits &sh, uint32_t digit, bool on)
{
    const unsigned long long there = __ballot(on);
    if (there == 0) return;
    const uint32_t first = __builtin_amdgcn_readlane(digit, __builtin_ctzll(there));
    const unsigned long long same = __ballot(on && digit == first);
    if (on && digit != first) atomicAdd(&sh.hist[digit], 1u);
    if ((threadIdx.x & 63) == __builtin_ctzll(there)) atomicAdd(&sh.hist[first], (uint32_t)__popcll(same));
}
// A row's key over its number from the end: 63 bits, the first digit the upper 12
__device__ inline uint64_t evict_composite(uint32_t key, int row) { return (uint64_t)key << 31 | (uint32_t)(0x7fffffff - row); }
constexpr int kEvictShift = 63 - 12;

// The threshold: rows whose composite is at least that are kept, `need` of the `count` rows that have the digits in `from` down to bit `shift`.
// in_list: they are all listed; otherwise for_rows(f) goes over all rows with f(key, row, there)
template <class ForRows>
__device__ inline uint64_t evict_threshold(EvictShared &sh, uint64_t from, int shift, uint32_t need, uint32_t count, int in_list, ForRows for_rows)
{
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    while (need < count && shift > 0) {              // (all of a bin: the threshold is the bin's lowest)
        const int width = min(shift, 10), low = shift - width;
        evict_clear(sh, 1 << width);                 // (with a barrier, behind which the list is there as well)
        auto look = [&](uint64_t c, bool on) { evict_count(sh, (uint32_t)(c >> low) & ((1u << width) - 1), on && c >> shift == from >> shift); };
        if (in_list != 0) {
            for (int i0 = wv * 64; i0 < in_list; i0 += kEvictThreads) {
                const int i = min(i0 + lane, in_list - 1);
                look(evict_composite(sh.list.key[i], sh.list.row[i]), i0 + lane < in_list);
            }
        } else {
            for_rows([&](uint32_t key, int row, bool there) { look(evict_composite(key, row), there); });
        }
        __syncthreads();
        evict_find_bin(sh, 1 << width, need);
        from |= (uint64_t)sh.digit << low;
        need = sh.left;
        count = sh.count;
        shift = low;
        __syncthreads();
    }
    return from;
}

// Of word w of the bits: which rows are below `keep`
__device__ inline uint64_t evict_below(int keep, int w) { return keep - 64 * w >= 64 ? ~0ull : keep <= 64 * w ? 0ull : (1ull << (keep - 64 * w)) - 1; }
// Ranks of words [w0, w1), bits[w - w0], of holes and movers that follow hole_at and mover_at
__device__ inline void evict_ranks(EvictDigits &sh, const uint64_t *bits, uint2 *before, int w0, int w1, int keep, uint32_t hole_at, uint32_t mover_at)
{
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, per = (w1 - w0 + kEvictThreads - 1) / kEvictThreads;
    const int first = min(w0 + tid * per, w1), end = min(first + per, w1);
    uint32_t holes = 0, movers = 0;
    for (int w = first; w < end; ++w) {
        const uint64_t x = bits[w - w0], mask = evict_below(keep, w);
        holes += __popcll(~x & mask);
        movers += __popcll(x & ~mask);
    }
    const uint32_t holes_incl = wave_scan_u32(holes, lane), movers_incl = wave_scan_u32(movers, lane);
    if (lane == 63) { sh.wave_tot[0][wv] = holes_incl; sh.wave_tot[1][wv] = movers_incl; }
    __syncthreads();
    hole_at += holes_incl - holes;
    mover_at += movers_incl - movers;
    hole_at += evict_waves_before(sh.wave_tot[0], lane, wv);
    mover_at += evict_waves_before(sh.wave_tot[1], lane, wv);
    for (int w = first; w < end; ++w) {
        const uint64_t x = bits[w - w0], mask = evict_below(keep, w);
        before[w - w0] = make_uint2(hole_at, mover_at);
        hole_at += __popcll(~x & mask);
        mover_at += __popcll(x & ~mask);
    }
    __syncthreads();
}
// The movers of words [w0, w1) in their places of the list
__device__ inline void evict_movers(const uint64_t *bits, const uint2 *before, int w0, int w1, int keep, int32_t *movers, int most)
{
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (int w = max(w0, keep / 64) + wv; w < w1; w += kEvictWaves) {
        const uint64_t x = bits[w - w0] & ~evict_below(keep, w);
        const uint32_t at = before[w - w0].y + __popcll(x & ((1ull << lane) - 1));
        if (((x >> lane) & 1) && at < (uint32_t)most) movers[at] = 64 * w + lane;
    }
}

// Keys of a (sequence, KV head)
struct EvictKeys {
    const float *weights;
    const int32_t *positions;
    int n_sink, recent_from;
    __device__ EvictKeys(const EvictArgs &a, int p)
        : weights(a.weights + (int64_t)p * a.rows), positions(a.positions + (int64_t)p * a.rows), n_sink(a.n_sink), recent_from(a.seen[p / a.Hkv] - a.n_recent) {}
    // f(key, row, there) for rows [r0, r1): a thread has every 1024th, a wave 64 neighbours, kAhead of a thread are on their way together
    template <class F>
    __device__ void for_rows(int r0, int r1, F f) const
    {
        for (int at = r0; at < r1; at += kAhead * kEvictThreads) {
            float w[kAhead];
            int pos[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int row = min(at + i * kEvictThreads + (int)threadIdx.x, r1 - 1);
                w[i] = weights[row];
                pos[i] = positions[row];
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int row = at + i * kEvictThreads + (int)threadIdx.x;
                if (at + i * kEvictThreads >= r1) break;
                f(evict_key(w[i], pos[i], n_sink, recent_from), row, row < r1);
            }
        }
    }
};

// Rows of a store that are copied
template <int FORMAT>
struct EvictRow {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef typename std::conditional<FORMAT == IHIP_KV_BF16, u32x4, typename std::conditional<FORMAT == IHIP_KV_E4M3, u32x2, uint32_t>::type>::type word;
    int64_t k_to, v_to;
    word k, v;
    uint32_t scales;
    bool on;
    // one of 16 lanes of row src on its way to row dst
    __device__ void load(const EvictArgs &a, int b, int g, int src, int dst, int l16)
    {
        const StoreView &s = a.store;
        int64_t from = b, to = b, from_in = src, to_in = dst;
        if (s.paged.block_table) {
            const int32_t *table = s.paged.block_table + (int64_t)b * s.paged.table_stride;
            const int in_page = (1 << s.paged.page_log2) - 1;
            from = table[src >> s.paged.page_log2];
            to = table[dst >> s.paged.page_log2];
            from_in = src & in_page;
            to_in = dst & in_page;
        }
        on = from >= 0 && to >= 0;
        if (!on) return;
        const int64_t k_from = from * s.k_sb + g * s.k_sh + from_in * s.k_st, v_from = from * s.v_sb + g * s.v_sh + from_in * s.v_st;
        k_to = to * s.k_sb + g * s.k_sh + to_in * s.k_st;
        v_to = to * s.v_sb + g * s.v_sh + to_in * s.v_st;
        k = reinterpret_cast<const word *>(s.k + k_from)[l16];
        v = reinterpret_cast<const word *>(s.v + v_from)[l16];
        if (FORMAT == IHIP_KV_MX4 && l16 < 2) scales = *reinterpret_cast<const uint32_t *>(l16 == 0 ? s.ks + k_from / 16 : s.vs + v_from / 16);
    }
    __device__ void store(const EvictArgs &a, int l16) const
    {
        if (!on) return;
        reinterpret_cast<word *>(a.store.k + k_to)[l16] = k;
        reinterpret_cast<word *>(a.store.v + v_to)[l16] = v;
        if (FORMAT == IHIP_KV_MX4 && l16 < 2) *reinterpret_cast<uint32_t *>(l16 == 0 ? a.store.ks + k_to / 16 : a.store.vs + v_to / 16) = scales;
    }
};
__device__ inline void evict_beside(const EvictArgs &a, int p, int source, int at)       // weight and position of a place
{
    const int64_t from = (int64_t)p * a.rows + source, to = (int64_t)p * a.to_rows + at;
    if (source != at || a.to_weights != a.weights) a.to_weights[to] = a.weights[from];
    if (source != at || a.to_positions != a.positions) a.to_positions[to] = a.positions[from];
}
__device__ inline int evict_len(const EvictArgs &a, int b) { return min(max(a.lens[b], 0), a.max_len); }

// FORMAT: that of the rows that are moved here, -1: none are
template <int FORMAT>
__global__ __launch_bounds__(kEvictThreads) void kv_evict_select_kernel(const EvictArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    EvictHeldShared &sh = *reinterpret_cast<EvictHeldShared *>(smem);
    const int p = blockIdx.x, b = p / a.Hkv, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int n = evict_len(a, b), keep = a.keep;
    if (a.set_lens && p % a.Hkv == 0 && tid == 0) a.new_lens[b] = min(n, keep);
    if (FORMAT < 0 && tid == 0) a.state[p].n = n;
    int32_t *kept = a.kept + (int64_t)p * keep;
    if (n <= keep) {
        if (FORMAT >= 0)
            for (int i = tid; i < keep; i += kEvictThreads) {
                kept[i] = i < n ? i : -1;
                if (i < n) evict_beside(a, p, i, i);
            }
        return;
    }
    if (tid == 0) sh.listed = 0;
    evict_clear(sh, kEvictBins);
    EvictKeys(a, p).for_rows(0, n, [&](uint32_t key, int row, bool there) {
        evict_count(sh, key >> 20, there);
        sh.held[row] = key;
    });
    __syncthreads();
    evict_find_bin(sh, kEvictBins, keep);
    const uint32_t bin = sh.digit, need = sh.left, count = sh.count;
    auto for_rows = [&](auto f) {
        for (int row0 = wv * 64; row0 < n; row0 += kEvictThreads) f(sh.held[row0 + lane], row0 + lane, row0 + lane < n);
    };
    const int words = (n + 63) / 64, in_list = need < count && count <= kEvictList ? count : 0;
    for_rows([&](uint32_t key, int row, bool there) {        // those above the bin are kept, the bin's listed
        const uint64_t word = __ballot(there && key >> 20 > bin);
        if (lane == 0) sh.bits[row >> 6] = word;
        if (in_list != 0 && there && key >> 20 == bin) {
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            sh.list.key[at] = key;
            sh.list.row[at] = row;
        }
    });
    const uint64_t from = evict_threshold(sh, (uint64_t)bin << kEvictShift, kEvictShift, need, count, in_list, for_rows);
    __syncthreads();
    if (in_list != 0) {
        for (int i = tid; i < in_list; i += kEvictThreads) {
            const int row = sh.list.row[i];
            if (evict_composite(sh.list.key[i], row) >= from) atomicOr(reinterpret_cast<uint32_t *>(sh.bits) + (row >> 5), 1u << (row & 31));
        }
    } else {
        for_rows([&](uint32_t key, int row, bool there) {
            const uint64_t word = __ballot(there && evict_composite(key, row) >= from);
            if (lane == 0) sh.bits[row >> 6] = word;
        });
    }
    __syncthreads();
    evict_ranks(sh, sh.bits, sh.before, 0, words, keep, 0, 0);
    if constexpr (FORMAT < 0) {
        for (int w = tid; w < words; w += kEvictThreads) {
            a.bits[(int64_t)p * a.words + w] = sh.bits[w];
            a.before[(int64_t)p * a.words + w] = sh.before[w];
        }
        evict_movers(sh.bits, sh.before, 0, words, keep, a.movers + (int64_t)p * a.most, a.most);
    } else {
        evict_movers(sh.bits, sh.before, 0, words, keep, sh.moves.movers, kFewMoves);
        __syncthreads();
        for (int w = wv; 64 * w < keep; w += kEvictWaves) {
            const uint64_t x = ~sh.bits[w];
            const int row = 64 * w + lane;
            if (row >= keep) continue;
            const uint32_t at = sh.before[w].x + __popcll(x & ((1ull << lane) - 1));
            const bool hole = ((x >> lane) & 1) && at < (uint32_t)kFewMoves;
            const int source = hole ? sh.moves.movers[at] : row;
            kept[row] = source;
            evict_beside(a, p, source, row);
            if (hole) sh.moves.holes[at] = row;
        }
        __syncthreads();
        const int last = (keep - 1) / 64, l16 = tid & 15, grp = tid >> 4;
        const int moves = min((int)(sh.before[last].x + __popcll(~sh.bits[last] & evict_below(keep, last))), kFewMoves);
        for (int i0 = grp; i0 < moves; i0 += kEvictThreads / kRowLanes * kMoveAhead) {
            EvictRow<FORMAT> row[kMoveAhead];
#pragma unroll
            for (int i = 0; i < kMoveAhead; ++i) {
                const int at = i0 + i * (kEvictThreads / kRowLanes);
                row[i].on = false;
                if (at < moves) row[i].load(a, b, p % a.Hkv, sh.moves.movers[at], sh.moves.holes[at], l16);
            }
#pragma unroll
            for (int i = 0; i < kMoveAhead; ++i) row[i].store(a, l16);
        }
    }
}

// ---- in chunks -----------------------------------------------------------------
// Rows of chunk c of n rows: whole words
__device__ inline int evict_chunk(const EvictArgs &a, int n, int c)
{
    const int64_t size = (((int64_t)n + a.chunks - 1) / a.chunks + 63) & ~63ll;
    return (int)min(c * size, (int64_t)n);
}

// The histograms of all chunks added up, and the bin in which the `need`-th largest is
__device__ inline void evict_find_in_chunks(EvictDigits &sh, const EvictArgs &a, int p, int digit, uint32_t need)
{
    const int tid = threadIdx.x;
    const uint4 *hist = reinterpret_cast<const uint4 *>(a.hist + ((int64_t)digit * gridDim.x + p) * a.chunks * kEvictBins) + tid;
    uint4 all = make_uint4(0, 0, 0, 0);
    for (int i0 = 0; i0 < a.chunks; i0 += kAhead) {
        uint4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = hist[(int64_t)min(i0 + i, a.chunks - 1) * (kEvictBins / 4)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (i0 + i < a.chunks) all = make_uint4(all.x + x[i].x, all.y + x[i].y, all.z + x[i].z, all.w + x[i].w);
    }
    __syncthreads();
    reinterpret_cast<uint4 *>(sh.hist)[tid] = all;
    __syncthreads();
    evict_find_bin(sh, kEvictBins, need);
}
static_assert(kEvictBins == 4 * kEvictThreads, "");

// How many of a chunk's rows have which first digit, or which second one of those that have the threshold's first
template <int DIGIT>
__global__ __launch_bounds__(kEvictThreads) void kv_evict_digits_kernel(const EvictArgs a)
{
    __shared__ __attribute__((aligned(16))) EvictDigits sh;
    const int p = blockIdx.x, c = blockIdx.y, tid = threadIdx.x, n = DIGIT == 0 ? evict_len(a, p / a.Hkv) : a.state[p].n;
    if (DIGIT == 0 && c == 0 && tid == 0) a.state[p].n = n;
    if (n <= a.keep) return;
    uint32_t bin = 0;
    if (DIGIT == 1) {
        evict_find_in_chunks(sh, a, p, 0, a.keep);
        bin = sh.digit;
    }
    evict_clear(sh, kEvictBins);
    EvictKeys(a, p).for_rows(evict_chunk(a, n, c), evict_chunk(a, n, c + 1), [&](uint32_t key, int, bool there) {
        if constexpr (DIGIT == 0) evict_count(sh, key >> 20, there);
        else evict_count(sh, key >> 8 & (kEvictBins - 1), there && key >> 20 == bin);
    });
    __syncthreads();
    reinterpret_cast<uint4 *>(a.hist + (((int64_t)DIGIT * gridDim.x + p) * a.chunks + c) * kEvictBins)[tid] = reinterpret_cast<const uint4 *>(sh.hist)[tid];
}

// The threshold's first digits; rows above them are kept, those that have them are listed, each chunk's in its place
__global__ __launch_bounds__(kEvictThreads) void kv_evict_candidates_kernel(const EvictArgs a)
{
    __shared__ __attribute__((aligned(16))) EvictDigits sh;
    const int p = blockIdx.x, c = blockIdx.y, tid = threadIdx.x, lane = tid & 63, n = a.state[p].n, keep = a.keep;
    if (n <= keep) return;
    if (tid == 0) sh.listed = sh.sum[0] = sh.sum[1] = 0;
    evict_find_in_chunks(sh, a, p, 0, keep);
    uint32_t bin = sh.digit, need = sh.left, count = sh.count;
    if (a.digits == 2) {
        evict_find_in_chunks(sh, a, p, 1, need);
        bin = bin << 12 | sh.digit;
        need = sh.left;
        count = sh.count;
    }
    const int shift = 32 - 12 * a.digits;
    if (c == 0 && tid == 0) {
        a.state[p].bin = bin;
        a.state[p].need = need;
        a.state[p].count = count;
    }
    const bool list = need < count && count <= kEvictList;
    uint32_t at0 = 0;
    if (list) {
        const uint32_t *hist = a.hist + ((int64_t)(a.digits - 1) * gridDim.x + p) * a.chunks * kEvictBins + (bin & (kEvictBins - 1));
        for (int i = lane; i < c; i += 64) at0 += hist[(int64_t)i * kEvictBins];
    }
    at0 = wave_sum_u32(at0);
    uint64_t *bits = a.bits + (int64_t)p * a.words;
    uint2 *listed = a.listed + (int64_t)p * kEvictList;
    uint32_t below = 0, beyond = 0;                  // of this wave
    EvictKeys(a, p).for_rows(evict_chunk(a, n, c), evict_chunk(a, n, c + 1), [&](uint32_t key, int row, bool there) {
        // (a bin that is kept whole goes with those above it)
        const bool has = key >> shift == bin;
        const uint64_t word = __ballot(there && (key >> shift > bin || (need == count && has)));
        if (lane == 0 && there) {
            bits[row >> 6] = word;
            const uint64_t mask = evict_below(keep, row >> 6);
            below += __popcll(word & mask);
            beyond += __popcll(word & ~mask);
        }
        if (list && there && has) {
            const uint32_t at = at0 + atomicAdd(&sh.listed, 1u);
            if (at < kEvictList) listed[at] = make_uint2(key, row);
        }
    });
    if (lane == 0) {
        atomicAdd(&sh.sum[0], below);
        atomicAdd(&sh.sum[1], beyond);
    }
    __syncthreads();
    if (tid == 0) a.sure[(int64_t)p * a.chunks + c] = make_uint2(sh.sum[0], sh.sum[1]);
}

// The whole threshold; a chunk's bits, the ranks of its holes and movers, and its movers in their places
__global__ __launch_bounds__(kEvictThreads) void kv_evict_ranks_kernel(const EvictArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    EvictShared &sh = *reinterpret_cast<EvictShared *>(smem);
    const int p = blockIdx.x, c = blockIdx.y, tid = threadIdx.x, lane = tid & 63, keep = a.keep;
    const EvictState state = a.state[p];
    const int n = state.n;
    if (n <= keep) return;
    const int r0 = evict_chunk(a, n, c), r1 = evict_chunk(a, n, c + 1), w0 = r0 / 64, w1 = (r1 + 63) / 64;
    if (r0 >= r1) return;
    const int in_list = state.need < state.count && state.count <= kEvictList ? state.count : 0;
    const uint2 *listed = a.listed + (int64_t)p * kEvictList;
    for (int i = tid; i < in_list; i += kEvictThreads) {
        const uint2 x = listed[i];
        sh.list.key[i] = x.x;
        sh.list.row[i] = x.y;
    }
    uint64_t *bits = a.bits + (int64_t)p * a.words;
    for (int w = w0 + tid; w < w1; w += kEvictThreads) sh.bits[w - w0] = bits[w];
    // kept rows in front of the chunk, below `keep` and from there on
    uint32_t below = 0, beyond = 0;
    for (int i = tid; i < c; i += kEvictThreads) {
        const uint2 x = a.sure[(int64_t)p * a.chunks + i];
        below += x.x;
        beyond += x.y;
    }
    if (tid == 0) sh.sum[0] = sh.sum[1] = 0;
    const EvictKeys keys(a, p);
    const int shift = 63 - 12 * a.digits;
    const uint64_t from = evict_threshold(sh, (uint64_t)state.bin << shift, shift, state.need, state.count, in_list, [&](auto f) { keys.for_rows(0, n, f); });
    __syncthreads();
    if (in_list != 0) {
        for (int i = tid; i < in_list; i += kEvictThreads) {
            const int row = sh.list.row[i];
            if (evict_composite(sh.list.key[i], row) < from) continue;
            if (row < r0) (row < keep ? below : beyond) += 1;
            else if (row < r1) atomicOr(reinterpret_cast<uint32_t *>(sh.bits) + ((row - r0) >> 5), 1u << (row & 31));
        }
    } else if (state.need < state.count) {           // more rows than are listed: all are looked at again
        below = beyond = 0;
        keys.for_rows(0, r1, [&](uint32_t key, int row, bool there) {
            const bool on = there && evict_composite(key, row) >= from;
            if (on && row < r0) (row < keep ? below : beyond) += 1;
            const uint64_t word = __ballot(on);
            if (lane == 0 && row >= r0 && row < r1) sh.bits[(row - r0) >> 6] = word;
        });
    }
    below = wave_sum_u32(below);
    beyond = wave_sum_u32(beyond);
    if (lane == 0) {
        atomicAdd(&sh.sum[0], below);
        atomicAdd(&sh.sum[1], beyond);
    }
    __syncthreads();
    for (int w = w0 + tid; w < w1; w += kEvictThreads) bits[w] = sh.bits[w - w0];
    uint2 *before = a.before + (int64_t)p * a.words + w0;
    evict_ranks(sh, sh.bits, before, w0, w1, keep, min(r0, keep) - sh.sum[0], sh.sum[1]);
    evict_movers(sh.bits, before, w0, w1, keep, a.movers + (int64_t)p * a.most, a.most);
}

// The 64 rows of a word of bits
template <int FORMAT>
__global__ __launch_bounds__(kMoveThreads) void kv_evict_move_kernel(const EvictArgs a)
{
    __shared__ int sh_source[kMoveRows];
    const int p = blockIdx.x, b = p / a.Hkv, g = p % a.Hkv, w = blockIdx.y, tid = threadIdx.x, l16 = tid & 15, grp = tid >> 4;
    if (g == 0 && w == 0 && tid == 0) a.new_lens[b] = min(evict_len(a, b), a.keep);
    const int n = a.state[p].n;                      // (the lengths are not looked at: they may be written above)
    if (tid < kMoveRows) {
        const int at = w * kMoveRows + tid;
        int source = at < n && at < a.keep ? at : -1;
        if (n > a.keep && source >= 0) {
            const uint64_t x = ~a.bits[(int64_t)p * a.words + w];
            const uint32_t rank = a.before[(int64_t)p * a.words + w].x + __popcll(x & ((1ull << tid) - 1));
            if (((x >> tid) & 1) && rank < (uint32_t)a.most) source = a.movers[(int64_t)p * a.most + rank];
        }
        sh_source[tid] = source;
        if (at < a.keep) a.kept[(int64_t)p * a.keep + at] = source;
        if (source >= 0) evict_beside(a, p, source, at);
    }
    __syncthreads();
    EvictRow<FORMAT> row[kMoveAhead];
#pragma unroll
    for (int i = 0; i < kMoveAhead; ++i) {
        const int in_word = grp * kMoveAhead + i, at = w * kMoveRows + in_word, source = sh_source[in_word];
        row[i].on = false;
        if (source >= 0 && source != at) row[i].load(a, b, g, source, at, l16);
    }
#pragma unroll
    for (int i = 0; i < kMoveAhead; ++i) row[i].store(a, l16);
}

__global__ __launch_bounds__(kMoveThreads) void kv_evict_lens_kernel(const EvictArgs a)
{
    const int b = blockIdx.x * kMoveThreads + threadIdx.x;
    if (b < a.B) a.new_lens[b] = min(evict_len(a, b), a.keep);
}

struct EvictPlan {
    bool few, chunked;
    int64_t words, most, chunks;
    int digits;
    size_t bytes, listed, hist, sure, state, bits, before, movers;   // all of scratch, and where in it
};
static EvictPlan evict_plan(int64_t B, int64_t Hkv, int64_t max_len, int64_t keep)
{
    const int64_t P = B * Hkv;
    EvictPlan r{};
    r.words = (max_len + 63) / 64;
    r.most = std::max<int64_t>(0, std::min(keep, max_len - keep));
    r.chunked = r.most > 0 && max_len > kHeld;
    r.few = !r.chunked && r.most <= kFewMoves;
    // as many workgroups as there are compute units, of kEvictLeast rows or more; a chunk's bits are in LDS
    r.chunks = std::max<int64_t>({std::min<int64_t>({kEvictMostChunks, max_len / kEvictLeast, compute_units() / std::max<int64_t>(P, 1)}), r.words / (kEvictWords - 1) + 1, 2});
    auto take = [&](size_t bytes) {
        const size_t at = r.bytes;
        r.bytes += (bytes + 15) / 16 * 16;
        return at;
    };
    if (r.few) return r;
    r.state = take(P * sizeof(EvictState));
    r.bits = take(P * r.words * sizeof(uint64_t));
    r.before = take(P * r.words * sizeof(uint2));
    r.movers = take(P * r.most * sizeof(int32_t));
    if (!r.chunked) return r;
    r.listed = take(P * kEvictList * sizeof(uint2));
    r.sure = take(P * r.chunks * sizeof(uint2));
    r.digits = max_len > kEvictOneDigit ? 2 : 1;
    r.hist = take(r.digits * P * r.chunks * kEvictBins * sizeof(uint32_t));
    return r;
}
// (dynamic LDS beyond the 64 KiB that need no leave)
template <class Kernel>
static void launch_evict(Kernel *kernel, dim3 grid, size_t lds, hipStream_t st, const EvictArgs &a)
{
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    hipLaunchKernelGGL(kernel, grid, dim3(kEvictThreads), lds, st, a);
}
static int32_t check_evict(const char *who, int32_t B, int32_t Hkv, int32_t d, int32_t max_seq_len, int32_t keep)
{
    if (B < 0 || Hkv <= 0) return fail(IHIP_ERR_INVALID_ARG, "%s: bad B/Hkv = %d/%d", who, B, Hkv);
    if (d != kD) return fail(IHIP_ERR_UNSUPPORTED, "%s: d = %d, only 128 is built", who, d);
    if (max_seq_len < 0 || keep < 1) return fail(IHIP_ERR_INVALID_ARG, "%s: max_seq_len = %d, keep = %d", who, max_seq_len, keep);
    return IHIP_OK;
}

}  // namespace ihip

using namespace ihip;

extern "C" size_t ihip_kv_evict_workspace_bytes(int32_t B, int32_t Hkv, int32_t max_seq_len, int32_t keep)
{
    if (check_evict("ihip_kv_evict_workspace_bytes", B, Hkv, kD, max_seq_len, keep) != IHIP_OK) return 0;
    return std::max<size_t>(evict_plan(B, Hkv, max_seq_len, keep).bytes, 256);
}

extern "C" int32_t ihip_kv_evict(const ihip_kv_store *store, const ihip_kv_track *track, int32_t B, int32_t Hkv, int32_t d,
                                 const int32_t *seq_lens, int32_t max_seq_len, int32_t keep, int32_t n_sink, int32_t n_recent,
                                 const ihip_kv_track *to, int32_t *new_lens, int32_t *kept, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ihip_kv_evict";
    int32_t rc;
    if ((rc = check_evict(who, B, Hkv, d, max_seq_len, keep)) != IHIP_OK) return rc;
    if (n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > keep)
        return fail(IHIP_ERR_INVALID_ARG, "%s: n_sink = %d and n_recent = %d of keep = %d rows", who, n_sink, n_recent, keep);
    if (B == 0) return IHIP_OK;
    if (!seq_lens || !new_lens || !kept) return fail(IHIP_ERR_INVALID_ARG, "%s: seq_lens, new_lens or kept is NULL", who);
    EvictArgs a{};
    ihip_shape lengths{};
    lengths.max_seq_len = max_seq_len;
    if ((rc = check_store(who, store, lengths, &a.store)) != IHIP_OK) return rc;
    if ((rc = check_track(who, track, max_seq_len, true)) != IHIP_OK) return rc;
    if (!to) to = track;
    if ((rc = check_track(who, to, std::min(keep, max_seq_len), false)) != IHIP_OK) return rc;
    if (!to->positions) return fail(IHIP_ERR_INVALID_ARG, "%s: an array of to is NULL", who);
    if ((to->weights == track->weights || to->positions == track->positions) && to->rows != track->rows)
        return fail(IHIP_ERR_INVALID_ARG, "%s: to and track share arrays of %d and %d rows", who, to->rows, track->rows);
    const int64_t here = (int64_t)B * Hkv * track->rows * 4, there = (int64_t)B * Hkv * to->rows * 4;
    if (overlap_in_part(to->weights, there, track->weights, here) || overlap_in_part(to->positions, there, track->positions, here))
        return fail(IHIP_ERR_INVALID_ARG, "%s: to and track overlap in part", who);
    const int64_t row = store->format == IHIP_KV_BF16 ? 2 * kD : store->format == IHIP_KV_E4M3 ? kD : kD / 2;
    if (Hkv > 1 && (std::abs(a.store.k_sh) < row || std::abs(a.store.v_sh) < row))
        return fail(IHIP_ERR_INVALID_ARG, "%s: the heads of the store overlap", who);
    const int64_t lens_bytes = B * (int64_t)sizeof(int32_t);
    const bool apart = new_lens != seq_lens;
    if (overlap_in_part(new_lens, lens_bytes, seq_lens, lens_bytes)) return fail(IHIP_ERR_INVALID_ARG, "%s: new_lens overlaps seq_lens in part", who);
    const EvictPlan plan = evict_plan(B, Hkv, max_seq_len, keep);
    if (plan.bytes > 0 && (!ws || ((uintptr_t)ws & 15) || ws_bytes < plan.bytes))
        return fail(IHIP_ERR_WORKSPACE, "%s: workspace of %zu bytes, 16-byte aligned, needed, %zu given", who, plan.bytes, ws_bytes);
    const int64_t P = (int64_t)B * Hkv, moves = ((int64_t)keep - 1) / kMoveRows + 1;
    if (P > INT32_MAX / kEvictThreads || moves > 65535) return fail(IHIP_ERR_UNSUPPORTED, "%s: B * Hkv = %lld, keep = %d are too large", who, (long long)P, keep);
    // (the tokens seen are read while lengths are written, and would be the cut ones afterwards)
    if (new_lens == track->seen || overlap_in_part(new_lens, lens_bytes, track->seen, lens_bytes))
        return fail(IHIP_ERR_INVALID_ARG, "%s: new_lens overlaps the tokens seen", who);
    a.B = B; a.Hkv = Hkv; a.max_len = max_seq_len; a.keep = keep; a.n_sink = n_sink; a.n_recent = n_recent;
    a.lens = seq_lens; a.seen = track->seen;
    a.weights = track->weights; a.positions = track->positions; a.rows = track->rows;
    a.to_weights = to->weights; a.to_positions = to->positions; a.to_rows = to->rows;
    a.kept = kept; a.new_lens = new_lens;
    uint8_t *const scratch = (uint8_t *)ws;
    a.words = (int)plan.words; a.most = (int)plan.most; a.chunks = (int)plan.chunks; a.digits = plan.digits;
    a.state = (EvictState *)(scratch + plan.state);
    a.bits = (uint64_t *)(scratch + plan.bits);
    a.before = (uint2 *)(scratch + plan.before);
    a.movers = (int32_t *)(scratch + plan.movers);
    a.listed = (uint2 *)(scratch + plan.listed);
    a.sure = (uint2 *)(scratch + plan.sure);
    a.hist = (uint32_t *)(scratch + plan.hist);
    const hipStream_t st = (hipStream_t)stream;
    // lengths that are read by one workgroup are not written by another of the same launch
    a.set_lens = plan.few && apart;
    if (!plan.chunked) {
        KernelTimer timer("kv_evict_select", st);
        const dim3 grid((uint32_t)P);
        if (!plan.few) launch_evict(kv_evict_select_kernel<-1>, grid, sizeof(EvictHeldShared), st, a);
        else if (store->format == IHIP_KV_BF16) launch_evict(kv_evict_select_kernel<IHIP_KV_BF16>, grid, sizeof(EvictHeldShared), st, a);
        else if (store->format == IHIP_KV_E4M3) launch_evict(kv_evict_select_kernel<IHIP_KV_E4M3>, grid, sizeof(EvictHeldShared), st, a);
        else launch_evict(kv_evict_select_kernel<IHIP_KV_MX4>, grid, sizeof(EvictHeldShared), st, a);
    } else {
        const dim3 grid((uint32_t)P, (uint32_t)plan.chunks);
        {
            KernelTimer timer("kv_evict_digits", st);
            hipLaunchKernelGGL(kv_evict_digits_kernel<0>, grid, dim3(kEvictThreads), 0, st, a);
            if (a.digits == 2) hipLaunchKernelGGL(kv_evict_digits_kernel<1>, grid, dim3(kEvictThreads), 0, st, a);
        }
        if ((rc = check_launch(who)) != IHIP_OK) return rc;
        {
            KernelTimer timer("kv_evict_candidates", st);
            hipLaunchKernelGGL(kv_evict_candidates_kernel, grid, dim3(kEvictThreads), 0, st, a);
        }
        if ((rc = check_launch(who)) != IHIP_OK) return rc;
        KernelTimer timer("kv_evict_ranks", st);
        launch_evict(kv_evict_ranks_kernel, grid, sizeof(EvictShared), st, a);
    }
    if ((rc = check_launch(who)) != IHIP_OK || a.set_lens) return rc;
    if (plan.few) {
        KernelTimer timer("kv_evict_lens", st);
        hipLaunchKernelGGL(kv_evict_lens_kernel, dim3((B - 1) / kMoveThreads + 1), dim3(kMoveThreads), 0, st, a);
        return check_launch(who);
    }
    KernelTimer timer("kv_evict_move", st);
    const dim3 grid((uint32_t)P, (uint32_t)moves);
    if (store->format == IHIP_KV_BF16) hipLaunchKernelGGL(kv_evict_move_kernel<IHIP_KV_BF16>, grid, dim3(kMoveThreads), 0, st, a);
    else if (store->format == IHIP_KV_E4M3) hipLaunchKernelGGL(kv_evict_move_kernel<IHIP_KV_E4M3>, grid, dim3(kMoveThreads), 0, st, a);
    else hipLaunchKernelGGL(kv_evict_move_kernel<IHIP_KV_MX4>, grid, dim3(kMoveThreads), 0, st, a);
    return check_launch(who);
}

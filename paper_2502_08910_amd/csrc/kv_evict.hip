// A cache cut down to the rows that are worth most: the first tokens, the last ones, and of the others those with most attention weight.
//
// Kept rows stay where they are if that is below `keep`; the i-th evicted row below `keep` is filled with the i-th kept row from behind it.
// No row is both read and written, so all moves go at once and in any order, and a cache that drops 64 of 1,088 rows moves 64 of them.
//
// Two launches.  kv_evict_select_kernel, a workgroup a (sequence, KV head): the threshold is found by its digits, most significant first, in a
// histogram of all rows and then among the rows of one bin; a row's key is its weight in an order-preserving map over its number from
// the end, so that no two are the same and ties go to the lower row.  What is kept goes down as one bit a row, and the holes below
// `keep` are matched to the kept rows above it by their ranks.  kv_evict_move_kernel: 64 places a wave, 16 lanes a row that moves.
#include "api_checks.h"
#include "kv_store.h"
#include <algorithm>
#include <cstdlib>
#include <type_traits>

namespace ihip {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;
constexpr int kEvictBins = 4096, kEvictList = 4096;  // of the first digit; rows of one bin that are looked at on their own
constexpr int kMoveThreads = 256, kMoveRows = 256;   // places of a workgroup

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
    uint64_t *bits;                  // [P, words]
    int32_t *movers;                 // [P, most]
    int words, most;
    StoreView store;
    int row_bytes;                   // 4-bit rows: and 4 of scales
};

// Larger is kept: protected rows before all weights, NaN behind them; -0 as +0
__device__ inline uint32_t evict_key(float w, int pos, int n_sink, int recent_from)
{
    if (pos < n_sink || pos >= recent_from) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct EvictShared {
    uint32_t hist[kEvictBins];
    uint32_t list_key[kEvictList];
    int32_t list_row[kEvictList];
    uint32_t wave_tot[2][kEvictWaves];
    uint32_t digit, left, count, listed;
};

// Of `bins` bins, the one from which the `need`-th largest comes: its number, what of `need` is left in it, and its rows
__device__ inline void evict_find_bin(EvictShared &sh, int bins, uint32_t need, int tid)
{
    const int lane = tid & 63, wv = tid >> 6, per = max(1, bins / kEvictThreads);
    uint32_t h[4] = {0, 0, 0, 0}, mine = 0;          // bins in descending order: thread t has bins - 1 - per t and on
    if (per * tid < bins)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < per) mine += h[i] = sh.hist[bins - 1 - per * tid - i];
    uint32_t incl = wave_scan_u32(mine, lane);
    if (lane == 63) sh.wave_tot[0][wv] = incl;
    __syncthreads();
    for (int w = 0; w < wv; ++w) incl += sh.wave_tot[0][w];
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

__global__ __launch_bounds__(kEvictThreads) void kv_evict_select_kernel(const EvictArgs a)
{
    __shared__ EvictShared sh;
    const int p = blockIdx.x, b = p / a.Hkv, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int n = min(max(a.lens[b], 0), a.max_len), keep = a.keep;
    int32_t *kept = a.kept + (int64_t)p * keep;
    const int stays = min(n, keep);
    for (int i = tid; i < keep; i += kEvictThreads) kept[i] = i < stays ? i : -1;
    if (n <= keep) return;
    const float *weights = a.weights + (int64_t)p * a.rows;
    const int32_t *positions = a.positions + (int64_t)p * a.rows;
    const int recent_from = a.seen[b] - a.n_recent;
    auto key_at = [&](int i) { return evict_key(weights[i], positions[i], a.n_sink, recent_from); };

    // The threshold as a (key, complement of the row) pair: rows at or above it are kept.  `from` is its digits so far
    uint32_t need = keep;
    auto clear = [&](int bins) {
        for (int i = tid; i < bins; i += kEvictThreads) sh.hist[i] = 0;
        __syncthreads();
    };
    auto composite = [&](uint32_t key, int row) { return (uint64_t)key << 31 | (uint32_t)(0x7fffffff - row); };
    // adds a wave's digits; the first one's like at once (rows of weight 0 are often many)
    auto add = [&](uint32_t digit, bool on) {
        const unsigned long long there = __ballot(on);
        if (there == 0) return;
        const uint32_t first = __builtin_amdgcn_readlane(digit, __builtin_ctzll(there));
        const unsigned long long same = __ballot(on && digit == first);
        if (on && digit != first) atomicAdd(&sh.hist[digit], 1u);
        if (lane == __builtin_ctzll(there)) atomicAdd(&sh.hist[first], (uint32_t)__popcll(same));
    };
    uint64_t from = 0;
    int shift = 63 - 12;
    if (tid == 0) sh.listed = 0;
    clear(kEvictBins);
    for (int i0 = wv * 64; i0 < n; i0 += kEvictThreads) {
        const int i = i0 + lane;
        add(i < n ? key_at(i) >> 20 : 0, i < n);
    }
    __syncthreads();
    evict_find_bin(sh, kEvictBins, need, tid);
    from = (uint64_t)sh.digit << shift;
    need = sh.left;
    uint32_t count = sh.count;
    uint32_t in_list = 0;
    while (need < count && shift > 0) {              // (all of a bin: the threshold is the bin's lowest)
        if (in_list == 0 && count <= kEvictList) {
            in_list = count;
            for (int i = tid; i < n; i += kEvictThreads) {
                const uint32_t key = key_at(i);
                if (composite(key, i) >> shift != from >> shift) continue;
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                if (at < kEvictList) { sh.list_key[at] = key; sh.list_row[at] = i; }
            }
        }
        const int width = min(shift, 10), low = shift - width, m = in_list != 0 ? in_list : n;
        clear(1 << width);                           // (with a barrier, behind which the list is there as well)
        for (int i0 = wv * 64; i0 < m; i0 += kEvictThreads) {
            const int i = i0 + lane;
            uint64_t c = 0;
            if (i < m) c = in_list != 0 ? composite(sh.list_key[i], sh.list_row[i]) : composite(key_at(i), i);
            add((uint32_t)(c >> low) & ((1u << width) - 1), i < m && c >> shift == from >> shift);
        }
        __syncthreads();
        evict_find_bin(sh, 1 << width, need, tid);
        from |= (uint64_t)sh.digit << low;
        need = sh.left;
        count = sh.count;
        shift = low;
        __syncthreads();
    }

    // one bit a row
    uint64_t *bits = a.bits + (int64_t)p * a.words;
    for (int i0 = wv * 64; i0 < n; i0 += kEvictThreads) {
        const int i = i0 + lane;
        const uint64_t word = __ballot(i < n && composite(key_at(i), i) >= from);
        if (lane == 0) bits[i0 >> 6] = word;
    }
    __syncthreads();
    // holes below `keep`, kept rows from there on, counted by their words in order
    const int words = (n + 63) / 64, per = (words + kEvictThreads - 1) / kEvictThreads, w0 = min(tid * per, words), w1 = min(w0 + per, words);
    auto below = [&](int w) { return keep >= 64 * w + 64 ? ~0ull : keep <= 64 * w ? 0ull : (1ull << (keep - 64 * w)) - 1; };
    uint32_t holes = 0, movers = 0;
    for (int w = w0; w < w1; ++w) {
        const uint64_t x = bits[w], mask = below(w);
        holes += __popcll(~x & mask);
        movers += __popcll(x & ~mask);
    }
    const uint32_t holes_incl = wave_scan_u32(holes, lane), movers_incl = wave_scan_u32(movers, lane);
    if (lane == 63) { sh.wave_tot[0][wv] = holes_incl; sh.wave_tot[1][wv] = movers_incl; }
    __syncthreads();
    uint32_t hole_at = holes_incl - holes, mover_at = movers_incl - movers;
    for (int w = 0; w < wv; ++w) { hole_at += sh.wave_tot[0][w]; mover_at += sh.wave_tot[1][w]; }
    int32_t *list = a.movers + (int64_t)p * a.most;
    for (int w = w0; w < w1; ++w)
        for (uint64_t x = bits[w] & ~below(w); x != 0; x &= x - 1, ++mover_at)
            if (mover_at < (uint32_t)a.most) list[mover_at] = 64 * w + __builtin_ctzll(x);
    __syncthreads();
    for (int w = w0; w < w1; ++w)
        for (uint64_t x = ~bits[w] & below(w); x != 0; x &= x - 1, ++hole_at)
            if (hole_at < (uint32_t)a.most) kept[64 * w + __builtin_ctzll(x)] = list[hole_at];
}

template <int FORMAT>
__global__ __launch_bounds__(kMoveThreads) void kv_evict_move_kernel(const EvictArgs a)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef typename std::conditional<FORMAT == IHIP_KV_BF16, u32x4, typename std::conditional<FORMAT == IHIP_KV_E4M3, u32x2, uint32_t>::type>::type word;
    const int p = blockIdx.x, b = p / a.Hkv, g = p % a.Hkv, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    if (g == 0 && blockIdx.y == 0 && tid == 0) a.new_lens[b] = min(min(max(a.lens[b], 0), a.max_len), a.keep);
    const int at = blockIdx.y * kMoveRows + wv * 64 + lane;          // (the lengths are not looked at: they may be written above)
    const int source = at < a.keep ? a.kept[(int64_t)p * a.keep + at] : -1;
    if (source >= 0) {
        const int64_t from = (int64_t)p * a.rows + source, to = (int64_t)p * a.to_rows + at;
        const float w = a.weights[from];
        const int32_t pos = a.positions[from];
        if (source != at || a.to_weights != a.weights) a.to_weights[to] = w;
        if (source != at || a.to_positions != a.positions) a.to_positions[to] = pos;
    }
    // rows, four at a time
    const int32_t *table = a.store.paged.block_table ? a.store.paged.block_table + (int64_t)b * a.store.paged.table_stride : nullptr;
    auto row_of = [&](int row, int64_t sb, int64_t sh, int64_t st) {
        int64_t first = b, in_page = row;
        if (table) {
            first = table[row >> a.store.paged.page_log2];
            in_page = row & ((1 << a.store.paged.page_log2) - 1);
        }
        return first < 0 ? (int64_t)-1 : first * sb + g * sh + in_page * st;
    };
    const int l16 = lane & 15, quarter = lane >> 4;
    for (unsigned long long left = __ballot(source >= 0 && source != at); left != 0;) {
        unsigned long long mine = left;
        for (int i = 0; i < quarter; ++i) mine &= mine - 1;
        const bool on = mine != 0;
        const int which = on ? __builtin_ctzll(mine) : 0;
        const int src = __shfl(source, which, 64), dst = __shfl(at, which, 64);
        if (on) {
            const int64_t ks = row_of(src, a.store.k_sb, a.store.k_sh, a.store.k_st), kd = row_of(dst, a.store.k_sb, a.store.k_sh, a.store.k_st);
            const int64_t vs = row_of(src, a.store.v_sb, a.store.v_sh, a.store.v_st), vd = row_of(dst, a.store.v_sb, a.store.v_sh, a.store.v_st);
            if (ks != -1 && kd != -1) {
                const word x = reinterpret_cast<const word *>(a.store.k + ks)[l16], y = reinterpret_cast<const word *>(a.store.v + vs)[l16];
                reinterpret_cast<word *>(a.store.k + kd)[l16] = x;
                reinterpret_cast<word *>(a.store.v + vd)[l16] = y;
                if (FORMAT == IHIP_KV_MX4 && l16 < 2) {
                    if (l16 == 0) *reinterpret_cast<uint32_t *>(a.store.ks + kd / 16) = *reinterpret_cast<const uint32_t *>(a.store.ks + ks / 16);
                    else *reinterpret_cast<uint32_t *>(a.store.vs + vd / 16) = *reinterpret_cast<const uint32_t *>(a.store.vs + vs / 16);
                }
            }
        }
        for (int i = 0; i < 4; ++i) left &= left - 1;
    }
}

struct EvictPlan { int64_t words, most; size_t bytes; };
static EvictPlan evict_plan(int64_t B, int64_t Hkv, int64_t max_len, int64_t keep)
{
    EvictPlan r;
    r.words = (max_len + 63) / 64;
    r.most = std::max<int64_t>(0, std::min(keep, max_len - keep));
    r.bytes = (size_t)(B * Hkv) * (r.words * sizeof(uint64_t) + r.most * sizeof(int32_t));
    return r;
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
    const int64_t row = store->format == IHIP_KV_BF16 ? 2 * kD : store->format == IHIP_KV_E4M3 ? kD : kD / 2;
    if (Hkv > 1 && (std::abs(a.store.k_sh) < row || std::abs(a.store.v_sh) < row))
        return fail(IHIP_ERR_INVALID_ARG, "%s: the heads of the store overlap", who);
    const EvictPlan plan = evict_plan(B, Hkv, max_seq_len, keep);
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < plan.bytes)
        return fail(IHIP_ERR_WORKSPACE, "%s: workspace of %zu bytes, 16-byte aligned, needed, %zu given", who, plan.bytes, ws_bytes);
    const int64_t P = (int64_t)B * Hkv, moves = ((int64_t)keep - 1) / kMoveRows + 1;
    if (P > INT32_MAX / kEvictThreads || moves > 65535) return fail(IHIP_ERR_UNSUPPORTED, "%s: B * Hkv = %lld, keep = %d are too large", who, (long long)P, keep);
    a.B = B; a.Hkv = Hkv; a.max_len = max_seq_len; a.keep = keep; a.n_sink = n_sink; a.n_recent = n_recent;
    a.lens = seq_lens; a.seen = track->seen;
    a.weights = track->weights; a.positions = track->positions; a.rows = track->rows;
    a.to_weights = to->weights; a.to_positions = to->positions; a.to_rows = to->rows;
    a.kept = kept; a.new_lens = new_lens;
    a.bits = (uint64_t *)ws; a.words = (int)plan.words; a.most = (int)plan.most;
    a.movers = (int32_t *)(a.bits + P * plan.words);
    const hipStream_t st = (hipStream_t)stream;
    {
        KernelTimer timer("kv_evict_select", st);
        hipLaunchKernelGGL(kv_evict_select_kernel, dim3((uint32_t)P), dim3(kEvictThreads), 0, st, a);
    }
    if ((rc = check_launch(who)) != IHIP_OK) return rc;
    KernelTimer timer("kv_evict_move", st);
    const dim3 grid((uint32_t)P, (uint32_t)moves);
    if (store->format == IHIP_KV_BF16) hipLaunchKernelGGL(kv_evict_move_kernel<IHIP_KV_BF16>, grid, dim3(kMoveThreads), 0, st, a);
    else if (store->format == IHIP_KV_E4M3) hipLaunchKernelGGL(kv_evict_move_kernel<IHIP_KV_E4M3>, grid, dim3(kMoveThreads), 0, st, a);
    else hipLaunchKernelGGL(kv_evict_move_kernel<IHIP_KV_MX4>, grid, dim3(kMoveThreads), 0, st, a);
    return check_launch(who);
}

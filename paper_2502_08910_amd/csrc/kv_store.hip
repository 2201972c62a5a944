// Filling a KV cache with new tokens (rotated and quantised on the way) and reading it back as bf16.
//
// Both are one pass over memory: 16 lanes share a row of 128 elements, eight elements a lane, so that a row is read and written in whole
// lines and a scale's 32 elements are four neighbouring lanes.  Bound by memory: 7,937 tokens with 32 query and 8 KV heads into
// bf16 pages, 172 MB, take 35 us (4.9 TB/s; a copy of 4 GB moves 4.8), 128K tokens of 8 heads out of 4 bits, 679 MB, 135 us
// (5.0).  One token of each of 32 sequences takes 5.4 us, a chain of latencies: offsets, lengths, page, rows (5.9 with the tokens seen, weights
// and positions beside them).
#include "api_checks.h"
#include "kv_store.h"
#include <algorithm>
#include <cstdlib>
#include <type_traits>

namespace ihip {

constexpr int kStoreThreads = 256;
constexpr int kStoreGroups = kStoreThreads / kRowLanes;      // rows that a workgroup has in hand at a time

// bf16 rows that are more than the L2 caches keep go past them (non-temporal stores): 128K tokens of 8 heads widened from 4 bits 139 -> 135 us
// (5.0 TB/s; 142 -> 102 us where the rows are in the memory-side cache), 32K tokens of 32/8 heads appended to 4 bits and read back
// 197 -> 186 us, 7,937 tokens into bf16 pages 39.2 -> 37.1 us.  The narrow rows of the caches go through them
// (so do smaller results, which are read next).
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ inline void store_row16(void *row, int l16, const uint4 &w, bool past)
{
    const u32x4_t x = {w.x, w.y, w.z, w.w};
    if (past) __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t *>(row) + l16);
    else reinterpret_cast<u32x4_t *>(row)[l16] = x;
}
constexpr int64_t kPastBytes = 16 << 20;             // half of the eight L2 caches

struct AppendArgs {
    int B, Hq, Hkv, rows, max_len;
    const int32_t *cu, *lens;
    const uint16_t *q, *k, *v;
    int64_t q_sh, q_st, k_sh, k_st, v_sh, v_st;
    const float *cos, *sin;
    StoreView to;
    uint16_t *qo, *ko;               // may be null
    int64_t qo_sh, qo_st, ko_sh, ko_st;
    int first, per_wg;               // first head slot (Hq without queries) and head slots of a workgroup
    bool past;
    // tracked: what stands beside the rows
    const int32_t *seen;
    float *weights;
    int32_t *positions;
    int track_rows, n_pos;           // rows of a head; positions that can be rotated to
};

__device__ inline void append_row(uint8_t *row, uint8_t *scales, const uint4 &raw, const float (&f)[8], bool turned, int l16, int format, float scale, bool past)
{
    if (format == IHIP_KV_BF16) {
        uint4 w = raw;
        if (turned) w = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        store_row16(row, l16, w, past);
    } else if (format == IHIP_KV_E4M3) {
        reinterpret_cast<uint2 *>(row)[l16] = e4m3_quantise(f, scale);
    } else {
        uint32_t s;
        reinterpret_cast<uint32_t *>(row)[l16] = mx4_quantise(f, s);
        if ((l16 & 3) == 0) scales[l16 >> 2] = (uint8_t)s;
    }
}

// A workgroup takes 16 tokens, 16 lanes each, and a.per_wg of the Hq + 2 Hkv rows that each of them has: its queries, keys, values.
// TRACKED: a token's position is not its row, and both are written down.
template <int FORMAT, bool ROPE, bool TRACKED>
__global__ __launch_bounds__(kStoreThreads) void kv_append_kernel(const AppendArgs a)
{
    constexpr int kBatch = 4;        // rows that a lane asks for at once
    const int tid = threadIdx.x, l16 = tid & 15, grp = tid >> 4;
    const int t0 = blockIdx.x * kStoreGroups, tok = t0 + grp;
    const int s0 = a.first + blockIdx.y * a.per_wg, s1 = min(s0 + a.per_wg, a.Hq + 2 * a.Hkv);
    __shared__ int sh_b[kStoreGroups], sh_pos[kStoreGroups], sh_at[TRACKED ? kStoreGroups : 1];

    uint4 raw[kBatch];
    auto load = [&](int s) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            raw[u] = make_uint4(0, 0, 0, 0);
            const int slot = s + u;
            if (slot >= s1 || tok >= a.rows) continue;
            const uint16_t *src = slot < a.Hq ? a.q + slot * a.q_sh + tok * a.q_st
                                  : slot < a.Hq + a.Hkv ? a.k + (slot - a.Hq) * a.k_sh + tok * a.k_st
                                                        : a.v + (slot - a.Hq - a.Hkv) * a.v_sh + tok * a.v_st;
            raw[u] = reinterpret_cast<const uint4 *>(src)[l16];
        }
    };
    load(s0);                        // on their way while the tokens' places are looked up

    if (tid < kStoreGroups) sh_b[tid] = -1;
    __syncthreads();
    for (int b = tid; b < a.B; b += kStoreThreads) {
        const int c0 = min(max(a.cu[b], 0), a.rows), c1 = min(max(a.cu[b + 1], c0), a.rows), len = a.lens[b];
        for (int t = max(c0, t0); t < min(c1, t0 + kStoreGroups); ++t) {
            sh_b[t - t0] = b;
            sh_pos[t - t0] = len - (c1 - t);
            if constexpr (TRACKED) sh_at[t - t0] = a.seen[b] - (c1 - t);
        }
    }
    __syncthreads();
    const int b = sh_b[grp], pos = sh_pos[grp];
    int at = pos;                    // position in the sequence (pos: row)
    if constexpr (TRACKED) at = sh_at[grp];
    const bool there = b >= 0 && pos >= 0 && pos < a.max_len && (!TRACKED || (at >= 0 && at < a.n_pos));
    if (!there) return;              // (no barrier below)
    float4 c, n;
    if constexpr (ROPE) {
        c = reinterpret_cast<const float4 *>(a.cos + (int64_t)at * (kD / 2))[l16];
        n = reinterpret_cast<const float4 *>(a.sin + (int64_t)at * (kD / 2))[l16];
    }
    int64_t first = b, in_page = pos;
    if (a.to.paged.block_table) {
        first = a.to.paged.block_table[(int64_t)b * a.to.paged.table_stride + (pos >> a.to.paged.page_log2)];
        in_page = pos & ((1 << a.to.paged.page_log2) - 1);
    }
    const bool kept = first >= 0;    // else no page
    const int64_t k_row = first * a.to.k_sb + in_page * a.to.k_st, v_row = first * a.to.v_sb + in_page * a.to.v_st;

    for (int s = s0; s < s1; s += kBatch) {
        if (s > s0) load(s);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int slot = s + u;
            if (slot >= s1) break;
            float f[8];
            unpack_bf16x8(raw[u], f);
            if (slot < a.Hq + a.Hkv) {
                if constexpr (ROPE) turn_f32x8(f, c, n);
                const bool is_q = slot < a.Hq;
                uint16_t *out = is_q ? a.qo : a.ko;
                if (out) {
                    out += is_q ? slot * a.qo_sh + tok * a.qo_st : (slot - a.Hq) * a.ko_sh + tok * a.ko_st;
                    uint4 w = raw[u];
                    if constexpr (ROPE) w = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
                    store_row16(out, l16, w, a.past);
                }
                if (!is_q && kept) {
                    const int64_t o = k_row + (slot - a.Hq) * a.to.k_sh;
                    append_row(a.to.k + o, a.to.ks + o / 16, raw[u], f, ROPE, l16, FORMAT, a.to.k_scale, a.past);
                    if constexpr (TRACKED) {
                        const int64_t r = ((int64_t)b * a.Hkv + slot - a.Hq) * a.track_rows + pos;
                        if (l16 == 0) a.weights[r] = 0.f;
                        if (l16 == 1) a.positions[r] = at;
                    }
                }
            } else if (kept) {
                const int64_t o = v_row + (slot - a.Hq - a.Hkv) * a.to.v_sh;
                append_row(a.to.v + o, a.to.vs + o / 16, raw[u], f, false, l16, FORMAT, a.to.v_scale, a.past);
            }
        }
    }
}

struct GatherArgs {
    int BH, Hkv, max_len, groups;
    bool past;
    const int32_t *lens;
    StoreView from;
    uint16_t *k, *v;                 // may be null
    int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;
};

constexpr int kGatherRows = 2;       // rows of K, and as many of V, that a lane asks for at once (4-bit rows: 2 97 us, 4 103, 8 103)
template <int FORMAT>
__global__ __launch_bounds__(kStoreThreads) void kv_gather_kernel(const GatherArgs a)
{
    constexpr int kRows = kGatherRows;
    using word = typename std::conditional<FORMAT == IHIP_KV_BF16, uint4, typename std::conditional<FORMAT == IHIP_KV_E4M3, uint2, uint32_t>::type>::type;
    const int l16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const uint32_t group = blockIdx.y * gridDim.x + blockIdx.x;
    if (group >= (uint32_t)a.groups) return;
    const int bh = group % a.BH, b = bh / a.Hkv, g = bh % a.Hkv;
    const int t0 = group / a.BH * (kRows * kStoreGroups);
    const int len = min(a.lens[b], a.max_len);
    word x[2][kRows];
    uint32_t s[2][kRows];
    bool there[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int t = t0 + u * kStoreGroups + grp;
        there[u] = t < len;
        if (!there[u]) continue;
        int64_t first = b, in_page = t;
        if (a.from.paged.block_table) {
            first = a.from.paged.block_table[(int64_t)b * a.from.paged.table_stride + (t >> a.from.paged.page_log2)];
            in_page = t & ((1 << a.from.paged.page_log2) - 1);
            there[u] = first >= 0;
            if (!there[u]) continue;
        }
        const int64_t ko = first * a.from.k_sb + g * a.from.k_sh + in_page * a.from.k_st;
        const int64_t vo = first * a.from.v_sb + g * a.from.v_sh + in_page * a.from.v_st;
        if (a.k) {
            x[0][u] = reinterpret_cast<const word *>(a.from.k + ko)[l16];
            if constexpr (FORMAT == IHIP_KV_MX4) s[0][u] = a.from.ks[ko / 16 + (l16 >> 2)];
        }
        if (a.v) {
            x[1][u] = reinterpret_cast<const word *>(a.from.v + vo)[l16];
            if constexpr (FORMAT == IHIP_KV_MX4) s[1][u] = a.from.vs[vo / 16 + (l16 >> 2)];
        }
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        uint16_t *to = kv == 0 ? a.k : a.v;
        if (!to) continue;
        to += kv == 0 ? b * a.k_sb + g * a.k_sh : b * a.v_sb + g * a.v_sh;
        const int64_t st = kv == 0 ? a.k_st : a.v_st;
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (!there[u]) continue;
            uint4 w;
            if constexpr (FORMAT == IHIP_KV_BF16) {
                w = x[kv][u];
            } else if constexpr (FORMAT == IHIP_KV_E4M3) {
                const float scale = kv == 0 ? a.from.k_scale : a.from.v_scale;
                float f[8];
                unpack8_fp8(x[kv][u], f);
                w = make_uint4(pack_bf16x2(f[0] * scale, f[1] * scale), pack_bf16x2(f[2] * scale, f[3] * scale),
                               pack_bf16x2(f[4] * scale, f[5] * scale), pack_bf16x2(f[6] * scale, f[7] * scale));
            } else {
                w = mx4_to_bf16x8(x[kv][u], mx4_scale(s[kv][u]));
                if (s[kv][u] == 255u) w = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
            }
            store_row16(to + (int64_t)(t0 + u * kStoreGroups + grp) * st, l16, w, a.past);
        }
    }
}

// ---- argument checks ------------------------------------------------------------
int32_t check_packed(const char *who, const ihip_packed *p)
{
    if (!p) return fail(IHIP_ERR_INVALID_ARG, "%s: packed is NULL", who);
    if (p->B < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->Hq % p->Hkv != 0)
        return fail(IHIP_ERR_INVALID_ARG, "%s: bad B/Hq/Hkv = %d/%d/%d", who, p->B, p->Hq, p->Hkv);
    if (p->d != kD) return fail(IHIP_ERR_UNSUPPORTED, "%s: d = %d, only 128 is built", who, p->d);
    if (p->rows < 0 || p->max_q < 0) return fail(IHIP_ERR_INVALID_ARG, "%s: rows = %d, max_q = %d", who, p->rows, p->max_q);
    if (p->B > 0 && !p->cu_q) return fail(IHIP_ERR_INVALID_ARG, "%s: cu_q is NULL", who);
    return IHIP_OK;
}

// a bf16 tensor that is written: rows of their own
int32_t check_output(const ihip_tensor &t, const char *who, const char *name, int heads)
{
    const int32_t rc = check_tensor(t, who, name);
    if (rc != IHIP_OK) return rc;
    if (t.stride_t < kD) return fail(IHIP_ERR_INVALID_ARG, "%s: %s.stride_t = %lld < d", who, name, (long long)t.stride_t);
    if (heads > 1 && t.stride_h < kD && t.stride_h > -kD)
        return fail(IHIP_ERR_INVALID_ARG, "%s: the heads of %s overlap (stride_h = %lld)", who, name, (long long)t.stride_h);
    return IHIP_OK;
}

int32_t check_track(const char *who, const ihip_kv_track *track, int64_t rows, bool whole)
{
    if (!track) return fail(IHIP_ERR_INVALID_ARG, "%s: track is NULL", who);
    if (!track->weights || (whole && (!track->positions || !track->seen)))
        return fail(IHIP_ERR_INVALID_ARG, "%s: an array of track is NULL", who);
    if (track->rows < 0 || track->rows < rows) return fail(IHIP_ERR_INVALID_ARG, "%s: track has %d rows, %lld are needed", who, track->rows, (long long)rows);
    return IHIP_OK;
}

int32_t check_before(const char *who, const float *before, float decay, const ihip_kv_track *track, int64_t heads)
{
    if (!(decay >= 0.f) || decay > 3.4028234e38f) return fail(IHIP_ERR_INVALID_ARG, "%s: decay = %g", who, decay);
    const int64_t bytes = heads * track->rows * (int64_t)sizeof(float);
    if (before && overlap_in_part(before, bytes, track->weights, bytes)) return fail(IHIP_ERR_INVALID_ARG, "%s: before overlaps the weights in part", who);
    return IHIP_OK;
}

int32_t check_store(const char *who, const ihip_kv_store *store, const ihip_shape &for_lengths, StoreView *view)
{
    int32_t rc;
    if (!store) return fail(IHIP_ERR_INVALID_ARG, "%s: store is NULL", who);
    StoreView w{};
    w.k_scale = w.v_scale = 1.0f;
    int unit = 1;
    if (store->format == IHIP_KV_BF16) {
        if ((rc = check_output(store->k, who, "k", 1)) != IHIP_OK || (rc = check_output(store->v, who, "v", 1)) != IHIP_OK) return rc;
        unit = 2;
    } else if (store->format == IHIP_KV_E4M3) {
        if ((rc = check_tensor8(store->k, who, "k")) != IHIP_OK || (rc = check_tensor8(store->v, who, "v")) != IHIP_OK) return rc;
        if ((rc = check_scales(who, store->k_scale, store->v_scale)) != IHIP_OK) return rc;
        w.k_scale = store->k_scale;
        w.v_scale = store->v_scale;
    } else if (store->format == IHIP_KV_MX4) {
        for (const ihip_tensor *t : {&store->k, &store->v}) {
            const char *name = t == &store->k ? "k" : "v";
            if (!t->ptr) return fail(IHIP_ERR_INVALID_ARG, "%s: %s.ptr is NULL", who, name);
            if (((uintptr_t)t->ptr & 15) || ((t->stride_b | t->stride_h | t->stride_t) & 63) || t->stride_t < kD / 2)
                return fail(IHIP_ERR_INVALID_ARG, "%s: %s: 4-bit rows are 16-byte aligned and their strides multiples of 64 bytes", who, name);
        }
        if (store->k.stride_b != store->v.stride_b || store->k.stride_h != store->v.stride_h || store->k.stride_t != store->v.stride_t)
            return fail(IHIP_ERR_INVALID_ARG, "%s: the strides of 4-bit k and v differ", who);
        if (!store->k_scales || !store->v_scales || (((uintptr_t)store->k_scales | (uintptr_t)store->v_scales) & 3))
            return fail(IHIP_ERR_INVALID_ARG, "%s: k_scales and v_scales must be 4-byte aligned arrays", who);
        w.ks = (uint8_t *)store->k_scales;
        w.vs = (uint8_t *)store->v_scales;
    } else {
        return fail(IHIP_ERR_INVALID_ARG, "%s: format = %d", who, store->format);
    }
    w.k = (uint8_t *)const_cast<void *>(store->k.ptr);
    w.v = (uint8_t *)const_cast<void *>(store->v.ptr);
    w.k_sb = store->k.stride_b * unit; w.k_sh = store->k.stride_h * unit; w.k_st = store->k.stride_t * unit;
    w.v_sb = store->v.stride_b * unit; w.v_sh = store->v.stride_h * unit; w.v_st = store->v.stride_t * unit;
    if (store->paged) {
        KvFormat fmt;
        if ((rc = check_paged(who, &for_lengths, store->paged, &fmt)) != IHIP_OK) return rc;
        w.paged = fmt.paged;
    }
    *view = w;
    return IHIP_OK;
}

}  // namespace ihip

using namespace ihip;

// track: NULL, or what ihip_kv_append_tracked was given
static int32_t append_entry(const char *who, const ihip_packed *packed, ihip_tensor q, ihip_tensor k, ihip_tensor v, const int32_t *seq_lens,
                            int32_t max_seq_len, const ihip_rope *rope, const ihip_kv_store *store, const ihip_kv_track *track,
                            ihip_tensor q_out, ihip_tensor k_out, void *stream)
{
    int32_t rc;
    if ((rc = check_packed(who, packed)) != IHIP_OK) return rc;
    if (packed->B == 0 || packed->rows == 0) return IHIP_OK;
    if ((rc = check_tensor(k, who, "k")) != IHIP_OK || (rc = check_tensor(v, who, "v")) != IHIP_OK) return rc;
    const bool with_q = q_out.ptr != nullptr;
    if (with_q && ((rc = check_tensor(q, who, "q")) != IHIP_OK || (rc = check_output(q_out, who, "q_out", packed->Hq)) != IHIP_OK)) return rc;
    if (k_out.ptr && (rc = check_output(k_out, who, "k_out", packed->Hkv)) != IHIP_OK) return rc;
    if (!seq_lens) return fail(IHIP_ERR_INVALID_ARG, "%s: seq_lens is NULL", who);
    if (max_seq_len <= 0) return fail(IHIP_ERR_INVALID_ARG, "%s: max_seq_len = %d", who, max_seq_len);
    if (rope && (!rope->cos || !rope->sin || (((uintptr_t)rope->cos | (uintptr_t)rope->sin) & 15)))
        return fail(IHIP_ERR_INVALID_ARG, "%s: rope tables are NULL or not 16-byte aligned", who);
    if (rope && !track && rope->n_pos < max_seq_len)
        return fail(IHIP_ERR_INVALID_ARG, "%s: rope table has %d positions, max_seq_len is %d", who, rope->n_pos, max_seq_len);
    AppendArgs a{};
    ihip_shape lengths{};
    lengths.max_seq_len = max_seq_len;
    if ((rc = check_store(who, store, lengths, &a.to)) != IHIP_OK) return rc;
    const int64_t row = store->format == IHIP_KV_BF16 ? 2 * kD : store->format == IHIP_KV_E4M3 ? kD : kD / 2;
    if (packed->Hkv > 1 && (std::abs(a.to.k_sh) < row || std::abs(a.to.v_sh) < row))
        return fail(IHIP_ERR_INVALID_ARG, "%s: the heads of the store overlap", who);
    if (track) {
        a.seen = track->seen; a.weights = track->weights; a.positions = track->positions; a.track_rows = track->rows;
        a.n_pos = rope ? rope->n_pos : INT32_MAX;
    }
    a.B = packed->B; a.Hq = packed->Hq; a.Hkv = packed->Hkv; a.rows = packed->rows; a.max_len = max_seq_len;
    a.cu = packed->cu_q; a.lens = seq_lens;
    a.q = (const uint16_t *)q.ptr; a.q_sh = q.stride_h; a.q_st = q.stride_t;
    a.k = (const uint16_t *)k.ptr; a.k_sh = k.stride_h; a.k_st = k.stride_t;
    a.v = (const uint16_t *)v.ptr; a.v_sh = v.stride_h; a.v_st = v.stride_t;
    a.qo = (uint16_t *)const_cast<void *>(q_out.ptr); a.qo_sh = q_out.stride_h; a.qo_st = q_out.stride_t;
    a.ko = (uint16_t *)const_cast<void *>(k_out.ptr); a.ko_sh = k_out.stride_h; a.ko_st = k_out.stride_t;
    a.cos = rope ? rope->cos : nullptr;
    a.sin = rope ? rope->sin : nullptr;
    a.first = with_q ? 0 : a.Hq;
    const int slots = a.Hq + 2 * a.Hkv - a.first, groups = (a.rows - 1) / kStoreGroups + 1;
    // Longer runs of heads use a token's place and angles longer, as long as there are workgroups enough (32K tokens, 48 heads, 4 to a
    // workgroup / 16: 186 / 169 us; a decode step is slower with 16)
    a.per_wg = 4;
    while (a.per_wg < 16 && (int64_t)groups * slots / (2 * a.per_wg) >= 8 * (int64_t)compute_units()) a.per_wg *= 2;
    a.past = (int64_t)a.rows * (slots - 2 * a.Hkv + (k_out.ptr ? a.Hkv : 0) + (store->format == IHIP_KV_BF16 ? 2 * a.Hkv : 0)) * kD * 2 > kPastBytes;
    const dim3 grid(groups, (slots + a.per_wg - 1) / a.per_wg);
    if (grid.y > 65535) return fail(IHIP_ERR_UNSUPPORTED, "%s: %d heads are too many", who, slots);
    KernelTimer timer("kv_append", (hipStream_t)stream);
#define IHIP_KA(FMT)                                                                                                                   \
    if (rope && track) hipLaunchKernelGGL((kv_append_kernel<FMT, true, true>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a);  \
    else if (rope) hipLaunchKernelGGL((kv_append_kernel<FMT, true, false>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a);     \
    else if (track) hipLaunchKernelGGL((kv_append_kernel<FMT, false, true>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a);    \
    else hipLaunchKernelGGL((kv_append_kernel<FMT, false, false>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a)
    if (store->format == IHIP_KV_BF16) { IHIP_KA(IHIP_KV_BF16); }
    else if (store->format == IHIP_KV_E4M3) { IHIP_KA(IHIP_KV_E4M3); }
    else { IHIP_KA(IHIP_KV_MX4); }
#undef IHIP_KA
    return check_launch(who);
}

extern "C" {

int32_t ihip_kv_append(const ihip_packed *packed, ihip_tensor q, ihip_tensor k, ihip_tensor v, const int32_t *seq_lens,
                       int32_t max_seq_len, const ihip_rope *rope, const ihip_kv_store *store, ihip_tensor q_out,
                       ihip_tensor k_out, void *stream)
{
    return append_entry("ihip_kv_append", packed, q, k, v, seq_lens, max_seq_len, rope, store, nullptr, q_out, k_out, stream);
}

int32_t ihip_kv_append_tracked(const ihip_packed *packed, ihip_tensor q, ihip_tensor k, ihip_tensor v, const int32_t *seq_lens,
                               int32_t max_seq_len, const ihip_rope *rope, const ihip_kv_store *store,
                               const ihip_kv_track *track, ihip_tensor q_out, ihip_tensor k_out, void *stream)
{
    const char *who = "ihip_kv_append_tracked";
    int32_t rc;
    if ((rc = check_packed(who, packed)) != IHIP_OK) return rc;
    if (packed->B == 0 || packed->rows == 0) return IHIP_OK;
    if ((rc = check_track(who, track, max_seq_len, true)) != IHIP_OK) return rc;
    return append_entry(who, packed, q, k, v, seq_lens, max_seq_len, rope, store, track, q_out, k_out, stream);
}

int32_t ihip_kv_gather(const ihip_kv_store *store, int32_t B, int32_t Hkv, int32_t d, const int32_t *seq_lens,
                       int32_t max_seq_len, ihip_tensor k_out, ihip_tensor v_out, void *stream)
{
    const char *who = "ihip_kv_gather";
    int32_t rc;
    if (B < 0 || Hkv <= 0) return fail(IHIP_ERR_INVALID_ARG, "%s: bad B/Hkv = %d/%d", who, B, Hkv);
    if (d != kD) return fail(IHIP_ERR_UNSUPPORTED, "%s: d = %d, only 128 is built", who, d);
    if (max_seq_len < 0) return fail(IHIP_ERR_INVALID_ARG, "%s: max_seq_len = %d", who, max_seq_len);
    if (B == 0 || max_seq_len == 0) return IHIP_OK;
    if (!seq_lens) return fail(IHIP_ERR_INVALID_ARG, "%s: seq_lens is NULL", who);
    if (k_out.ptr && (rc = check_output(k_out, who, "k_out", Hkv)) != IHIP_OK) return rc;
    if (v_out.ptr && (rc = check_output(v_out, who, "v_out", Hkv)) != IHIP_OK) return rc;
    GatherArgs a{};
    ihip_shape lengths{};
    lengths.max_seq_len = max_seq_len;
    if ((rc = check_store(who, store, lengths, &a.from)) != IHIP_OK) return rc;
    if (!k_out.ptr && !v_out.ptr) return IHIP_OK;
    const int64_t groups = (int64_t)B * Hkv * ((max_seq_len - 1) / (kGatherRows * kStoreGroups) + 1);
    if ((int64_t)B * Hkv > INT32_MAX || groups > INT32_MAX) return fail(IHIP_ERR_UNSUPPORTED, "%s: B * Hkv * max_seq_len is too large", who);
    a.past = (int64_t)B * Hkv * max_seq_len * kD * 2 * ((k_out.ptr != nullptr) + (v_out.ptr != nullptr)) > kPastBytes;
    a.groups = (int)groups; a.BH = B * Hkv; a.Hkv = Hkv; a.max_len = max_seq_len; a.lens = seq_lens;
    a.k = (uint16_t *)const_cast<void *>(k_out.ptr); a.k_sb = k_out.stride_b; a.k_sh = k_out.stride_h; a.k_st = k_out.stride_t;
    a.v = (uint16_t *)const_cast<void *>(v_out.ptr); a.v_sb = v_out.stride_b; a.v_sh = v_out.stride_h; a.v_st = v_out.stride_t;
    constexpr uint32_t row = 1u << 23;                       // (a dimension has fewer than 2^32 threads)
    const dim3 grid(std::min((uint32_t)groups, row), (uint32_t)(groups - 1) / row + 1);
    KernelTimer timer("kv_gather", (hipStream_t)stream);
    if (store->format == IHIP_KV_BF16) hipLaunchKernelGGL((kv_gather_kernel<IHIP_KV_BF16>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a);
    else if (store->format == IHIP_KV_E4M3) hipLaunchKernelGGL((kv_gather_kernel<IHIP_KV_E4M3>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((kv_gather_kernel<IHIP_KV_MX4>), grid, dim3(kStoreThreads), 0, (hipStream_t)stream, a);
    return check_launch(who);
}

}  // extern "C"

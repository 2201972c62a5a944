// Block-sparse decode attention over 4-bit (MX FP4) K and V rows: sink + kept blocks + window, or all keys.
//
// As in the decode attention over bf16 and E4M3 rows, the attended tokens of a problem (sequence, KV head) form a virtual slot list
// [sink | kept blocks | window], cut into splits, one workgroup each, whose partial results a second kernel merges.  A wave takes 32 slots
// at a time; no value crosses lanes between the loads, the products and the softmax:
//   scores   v_mfma_f32_16x16x32_bf16, 16 K rows x twice 8 heads (fewer repeat the last).  Lane (n, g) = (l % 16, l / 16) brings the 16
//            bytes of row n that are one scale's 32 elements, and widens them to bf16 with that scale (exact).  The contraction takes
//            the dims in the order 32 g + 8 j + i for step j, the same for the queries.  Column n, rows 4 g + r: lane (n, g)
//            gets head n % 8's scores of keys 4 g + r and 16 + 4 g + r.
//   output   v_mfma_f32_16x16x32_bf16 again, 16 rows x 32 keys x 16 dims, eight times: a lane's eight probabilities are its part of
//            the left operand as they are (rounded to bf16 in rows 0 .. 7, what that dropped in rows 8 .. 15; the two are added in
//            LDS), key 16 (i / 4) + 4 g + i % 4 for element i; for the right one it brings the
//            four bytes of dims 8 n .. 8 n + 7 of the same keys, and column n of product j is dim 8 n + j.
// So a probability is off by at most 2^-16 of it, and a result as good as its last rounding (0.0017, root mean square and relative; 0.0022 with
// probabilities of one part).  The sum that divides takes the probabilities as they were.
// Bound by memory: 68 bytes a row.  32 sequences of 7,383 to 16,384 tokens, 8 KV heads, 416 MB, take 92 us (4.5 TB/s; a copy of 4 GB
// moves 4.8; also 92 with probabilities of one part) and 5 for the merge; one of 4,099 takes 6.3 (5.8) and 5.1, chains of latencies.
#include "api_checks.h"
#include "decode_softmax.h"
#include "kv_store.h"
#include <algorithm>

namespace ihip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMxThreads = 256, kMxWaves = kMxThreads / kWave;
constexpr int kMxStep = 32;                          // slots of a wave at a time
constexpr int kMxMaxSplit = 4096, kMxMinSplit = 128; // slots of a split (multiples of 128: a step of every wave)
constexpr int kMxPerCu = 3;                          // workgroups that a compute unit holds

struct AttnMx4Args {
    Geometry ge;
    const uint16_t *q; int64_t q_sb, q_sh;
    const uint8_t *k, *v, *ks, *vs;
    uint32_t sb, st;                 // rows (64 bytes) between sequences or pages, and between tokens
    int64_t sh;                      // ... between KV heads
    const int32_t *block_starts;
    int n_blocks, block, block_log2;
    float scale_log2e;
    int n_splits;
    DecodeGrid grid;
    PagedView paged;
    float *part_ml, *part_acc;       // [P, n_splits, G, 2] (reference, unscaled, and sum), [P, n_splits, G, 128]
    uint16_t *out;
    float *out_lse;
};

// One wave's operands of 32 slots on their way
struct MxRows {
    uint4 k[2];                      // rows n and 16 + n, this lane's 32 elements
    uint32_t k_scale[2];
    uint32_t v[8], v_scale[8];       // dims 8 n .. of keys 4 g + r and 16 + 4 g + r
};

template <int HEADS>
__global__ __launch_bounds__(kMxThreads, kMxPerCu) void attn_decode_mx4_kernel(const AttnMx4Args a)
{
    const int p = a.grid.problem(), split = a.grid.part();
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const Problem pr = problem_of(a.ge, p);
    const int G = a.ge.G;
    const int n_sink_eff = min(a.ge.n_sink, pr.E), w0 = max(pr.hi, a.ge.n_sink);
    const int block_slots = a.n_blocks << a.block_log2;
    const int total = n_sink_eff + block_slots + max(0, pr.E - w0);
    // every problem's own slots in equal parts (the host's bound makes none longer than kMxMaxSplit)
    const int per = min(kMxMaxSplit, max(kMxMinSplit, ((total + a.n_splits - 1) / a.n_splits + kMxMinSplit - 1) / kMxMinSplit * kMxMinSplit));
    const int s0 = split * per;
    const int slots = min(per, total - s0), steps = (slots + kMxStep - 1) / kMxStep;
    const int64_t pbase = ((int64_t)p * a.n_splits + split) * G;

    __shared__ __attribute__((aligned(16))) uint32_t sh_row[kMxMaxSplit];     // row of every slot
    __shared__ uint32_t sh_there[kMxMaxSplit / 32];                           // which slots of a step hold a key
    __shared__ float sh_m[kMxWaves][HEADS], sh_l[kMxWaves][HEADS];
    __shared__ __attribute__((aligned(16))) float sh_acc[kMxWaves][2][HEADS][kD];      // of the two parts

    bf16x8 qb[4];
    {
        const uint16_t *qp = a.q + pr.b * a.q_sb + (int64_t)(pr.g * G + min(n & 7, G - 1)) * a.q_sh + 32 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) qb[j] = *reinterpret_cast<const bf16x8 *>(qp + 8 * j);
    }
    const int32_t *table = a.paged.block_table ? a.paged.block_table + (int64_t)pr.b * a.paged.table_stride : nullptr;
    const int32_t *starts = a.block_starts + (int64_t)p * a.n_blocks;
    for (int i = tid; i < steps * kMxStep; i += kMxThreads) {
        int slot = s0 + i, pos;
        if (slot < n_sink_eff) pos = slot;
        else if (slot < n_sink_eff + block_slots) {
            slot -= n_sink_eff;
            const int start = starts[slot >> a.block_log2];
            pos = start + (slot & (a.block - 1));
            pos = start >= 0 && pos < pr.hi ? pos : -1;
        } else {
            pos = w0 + (slot - n_sink_eff - block_slots);
            pos = pos < pr.E ? pos : -1;
        }
        uint32_t row = 0;                            // (without a key: some row that can be read)
        if (pos >= 0) {
            int first = pr.b, in_page = pos;
            if (table) {
                first = table[pos >> a.paged.page_log2];
                in_page = pos & ((1 << a.paged.page_log2) - 1);
            }
            if (first >= 0) row = (uint32_t)first * a.sb + (uint32_t)in_page * a.st;
            else pos = -1;                           // no page
        }
        sh_row[i] = row;
        const unsigned long long there = __ballot(pos >= 0);
        if ((lane & 31) == 0) sh_there[i >> 5] = (uint32_t)(there >> (lane & 32));
    }
    const uint8_t *kb = a.k + pr.g * a.sh * 64 + g * 16, *vb = a.v + pr.g * a.sh * 64 + n * 4;
    const uint8_t *ksb = a.ks + pr.g * a.sh * 4 + g, *vsb = a.vs + pr.g * a.sh * 4 + (n >> 2);
    __syncthreads();

    auto load = [&](int step, MxRows &r) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint64_t row = sh_row[step * kMxStep + 16 * t + n];
            r.k[t] = *reinterpret_cast<const uint4 *>(kb + row * 64);
            r.k_scale[t] = ksb[row * 4];
            const uint4 rows = *reinterpret_cast<const uint4 *>(&sh_row[step * kMxStep + 16 * t + 4 * g]);
            const uint32_t of[4] = {rows.x, rows.y, rows.z, rows.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r.v[4 * t + i] = *reinterpret_cast<const uint32_t *>(vb + (uint64_t)of[i] * 64);
                r.v_scale[4 * t + i] = vsb[(uint64_t)of[i] * 4];
            }
        }
    };

    const uint32_t second = n < 8 ? 0u : ~0u;        // lanes that bring the second parts of the probabilities
    f32x4 acc[8];                                    // rows 4 g + r, dim 8 n + j
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kSoftmaxLowest, l = 0.f;                    // of head n (m: the same in the four lanes of a head; l: of this lane's keys)
    MxRows r, nx;
    if (wv < steps) load(wv, r);
    for (int step = wv; step < steps; step += kMxWaves) {
        if (step + kMxWaves < steps) load(step + kMxWaves, nx);
        f32x4 c[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            const uint32_t w[4] = {r.k[t].x, r.k[t].y, r.k[t].z, r.k[t].w};
            const float s = mx4_scale(r.k_scale[t]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, mx4_to_bf16x8(w[j], s)), qb[j], c[t], 0, 0, 0);
        }
        const uint32_t there = __builtin_amdgcn_readfirstlane(sh_there[step]);
        if (there != ~0u) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!((there >> (16 * (i >> 2) + 4 * g + (i & 3))) & 1)) {
                    c[i >> 2][i & 3] = -INFINITY;
                    r.v_scale[i] = 127;              // what stands in the row is not used, but has to be finite
                }
        }
        float w[8], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = softmax_exp(c[i >> 2][i & 3], m, a.scale_log2e);        // of -inf: 0
            sum += w[i];
        }
        if (__any(!(sum <= kSoftmaxMaxSum))) {            // the reference follows where the scores outgrew it
            float top = c[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, c[i >> 2][i & 3]);
            const float mn = fmaxf(m, max_over_rows(top));
            const float corr = softmax_weight(m, mn, a.scale_log2e);
            m = mn;
            l *= corr;
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = softmax_exp(c[i >> 2][i & 3], m, a.scale_log2e);
                sum += w[i];
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const float x = __shfl(corr, 4 * g + h, 64);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j][h] *= x;
            }
        }
        l += sum;
        uint32_t part[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t first = pack_bf16x2(w[2 * i], w[2 * i + 1]) & second;
            part[i] = pack_bf16x2(w[2 * i] - __uint_as_float(first << 16), w[2 * i + 1] - __uint_as_float(first & 0xffff0000u));
        }
        const bf16x8 pw = __builtin_bit_cast(bf16x8, make_uint4(part[0], part[1], part[2], part[3]));
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = mx4_scale(r.v_scale[i]);
#define IHIP_MX_DIMS(B)                                                                                                                     \
        {                                                                                                                                   \
            uint32_t x[8], lo[4], hi[4];                                                                                                    \
            _Pragma("unroll") for (int i = 0; i < 8; ++i) x[i] = mx4_pair<B>(r.v[i], s[i]);                                                 \
            _Pragma("unroll") for (int i = 0; i < 4; ++i) {                                                                                 \
                lo[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);                                                         \
                hi[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);                                                         \
            }                                                                                                                               \
            acc[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pw, __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), acc[2 * B], 0, 0, 0);             \
            acc[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pw, __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), acc[2 * B + 1], 0, 0, 0); \
        }
        IHIP_MX_DIMS(0)
        IHIP_MX_DIMS(1)
        IHIP_MX_DIMS(2)
        IHIP_MX_DIMS(3)
#undef IHIP_MX_DIMS
        r = nx;
    }

    // the waves and both parts are merged through LDS
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (lane < HEADS) { sh_m[wv][lane] = m; sh_l[wv][lane] = l; }
    if (4 * (g & 1) < HEADS) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float *to = &sh_acc[wv][g >> 1][4 * (g & 1) + h][8 * n];
            *reinterpret_cast<float4 *>(to) = make_float4(acc[0][h], acc[1][h], acc[2][h], acc[3][h]);
            *reinterpret_cast<float4 *>(to + 4) = make_float4(acc[4][h], acc[5][h], acc[6][h], acc[7][h]);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < G * kD; idx += kMxThreads) {
        const int h = idx / kD, c = idx % kD;
        float M = kSoftmaxLowest;
#pragma unroll
        for (int w = 0; w < kMxWaves; ++w) M = fmaxf(M, sh_m[w][h]);
        float L = 0.f, A = 0.f;
#pragma unroll
        for (int w = 0; w < kMxWaves; ++w) {
            const float x = softmax_weight(sh_m[w][h], M, a.scale_log2e);
            L = fmaf(x, sh_l[w][h], L);
            A = fmaf(x, sh_acc[w][0][h][c] + sh_acc[w][1][h][c], A);
        }
        if (a.n_splits == 1) {                       // nothing to merge
            const int64_t hq = (int64_t)pr.b * a.ge.Hq + pr.g * G + h;
            a.out[hq * kD + c] = (uint16_t)f32_to_bf16_bits(L == 0.f ? 0.f : A / L);
            if (a.out_lse != nullptr && c == 0) a.out_lse[hq] = softmax_lse(M, L, a.scale_log2e);
            continue;
        }
        a.part_acc[(pbase + h) * kD + c] = A;
        if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + (pbase + h) * 2) = make_float2(M, L);
    }
}

// Merge of the splits: one workgroup per (problem, head), a thread a dim; groups of 128 threads share the splits
constexpr int kMxMergeGroups = 4, kMxMergeAhead = 8;
__global__ __launch_bounds__(kD * kMxMergeGroups) void attn_decode_mx4_merge_kernel(const AttnMx4Args a)
{
    const int G = a.ge.G, p = blockIdx.x / G, h = blockIdx.x % G, c = threadIdx.x % kD, grp = threadIdx.x / kD;
    const int64_t pbase = (int64_t)p * a.n_splits * G;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
    float M = kSoftmaxLowest, L = 0.f, A = 0.f;
    for (int s0 = grp; s0 < a.n_splits; s0 += kMxMergeGroups * kMxMergeAhead) {
        float2 x[kMxMergeAhead];
        float v[kMxMergeAhead], top = M;
#pragma unroll
        for (int i = 0; i < kMxMergeAhead; ++i) {
            const int64_t at = pbase + (int64_t)min(s0 + i * kMxMergeGroups, a.n_splits - 1) * G + h;
            x[i] = ml[at];
            v[i] = a.part_acc[at * kD + c];
        }
#pragma unroll
        for (int i = 0; i < kMxMergeAhead; ++i)
            if (s0 + i * kMxMergeGroups < a.n_splits) top = fmaxf(top, x[i].x);
        const float corr = softmax_weight(M, top, a.scale_log2e);
        L *= corr;
        A *= corr;
        M = top;
#pragma unroll
        for (int i = 0; i < kMxMergeAhead; ++i) {
            if (s0 + i * kMxMergeGroups >= a.n_splits) break;
            const float w = softmax_weight(x[i].x, M, a.scale_log2e);
            L = fmaf(w, x[i].y, L);
            A = fmaf(w, v[i], A);
        }
    }
    __shared__ float sh_m[kMxMergeGroups], sh_l[kMxMergeGroups], sh_a[kMxMergeGroups][kD];
    sh_a[grp][c] = A;
    if (c == 0) { sh_m[grp] = M; sh_l[grp] = L; }
    __syncthreads();
    if (grp != 0) return;
    M = kSoftmaxLowest;
#pragma unroll
    for (int i = 0; i < kMxMergeGroups; ++i) M = fmaxf(M, sh_m[i]);
    L = A = 0.f;
#pragma unroll
    for (int i = 0; i < kMxMergeGroups; ++i) {
        const float w = softmax_weight(sh_m[i], M, a.scale_log2e);
        L = fmaf(w, sh_l[i], L);
        A = fmaf(w, sh_a[i][c], A);
    }
    const int64_t hq = (int64_t)(p / a.ge.Hkv) * a.ge.Hq + (p % a.ge.Hkv) * G + h;
    a.out[hq * kD + c] = (uint16_t)f32_to_bf16_bits(L == 0.f ? 0.f : A / L);       // an idle place: 0
    if (a.out_lse != nullptr && c == 0) a.out_lse[hq] = softmax_lse(M, L, a.scale_log2e);
}

// Most slots that a problem has: sink and window are not longer than the sequence, whatever they are given as
static int64_t mx4_slots(const ihip_shape &s, int n_blocks, int block)
{
    return std::min<int64_t>((int64_t)s.n_sink + s.n_stream, s.max_seq_len) + (int64_t)n_blocks * block;
}
// Splits of a problem, which the kernel makes equally long.  A workgroup that has a compute unit to itself takes 10.7 ns a slot (it waits
// for its loads), three that share one 21 ns (they wait for the memory); a round of workgroups 2 us more than its slots, the launch 3, and the
// merge with its launch 10.  The least of that over one split (no merge), the splits that give every compute unit one, two or three
// workgroups, and those that fill two and more rounds.  One split / 768 workgroups or more (us), 8 problems a sequence: 8 sequences of 1,000
// keys 14.7 / 21.2, 16 of 2,000 25.5 / 20.9, 32 of 1,000 16.9 / 20.2, 32 of 4,000 44.6 / 37.9, 96 of 4,000 88 / 99; 32 of 7,383 to 16,384 in 4, 6
// (two rounds), 9, 12, 15 and 18 splits 120, 101, 103, 105, 109 and 112.
struct MxSplits { int best, most; };                 // most: no less than the best of any shorter list, for the scratch
static MxSplits mx4_splits(const ihip_shape &s, int n_blocks, int block)
{
    const int64_t total = mx4_slots(s, n_blocks, block), P = std::max(1, s.B * s.Hkv);
    const int64_t cu = compute_units(), places = cu * kMxPerCu;
    const int64_t fewest = (total + kMxMaxSplit - 1) / kMxMaxSplit, finest = (total + kMxMinSplit - 1) / kMxMinSplit;
    const int64_t rounds = (P * fewest + places - 1) / places;
    int64_t best = fewest;
    double least = 1e300;
    auto consider = [&](int64_t n) {
        n = std::min(std::max(n, fewest), finest);
        const int64_t size = ((total + n - 1) / n + kMxMinSplit - 1) / kMxMinSplit * kMxMinSplit;
        const double share = (double)std::min(P * n, places) / cu, slot = 0.0107 + 0.00515 * std::max(0.0, share - 1);
        const double time = (double)((P * n + places - 1) / places) * ((double)size * slot + 2) + 3 + (n > 1 ? 10 : 0);
        if (time < least) {
            least = time;
            best = n;
        }
    };
    consider(1);
    for (int k = 1; k <= kMxPerCu; ++k) consider(k * cu / P);
    for (int64_t r = std::max<int64_t>(rounds, 2); r < rounds + 4; ++r) consider(r * places / P);
    return {(int)best, (int)std::min(std::max((rounds + 3) * places / P, fewest), finest)};
}

size_t attn_decode_mx4_workspace(const ihip_shape &s, int n_blocks, int block)
{
    return (size_t)s.B * s.Hq * mx4_splits(s, n_blocks, block).most * (2 + kD) * sizeof(float);
}

}  // namespace ihip

using namespace ihip;

extern "C" int32_t ihip_sparse_attn_decode_mx4kv(const ihip_shape *shape, ihip_tensor q, const ihip_kv_store *store,
                                                 const int32_t *block_starts, int32_t n_blocks, int32_t block, float sm_scale,
                                                 void *out, float *out_lse, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ihip_sparse_attn_decode_mx4kv";
    int32_t rc;
    if ((rc = check_shape(shape, who)) != IHIP_OK) return rc;
    if (shape->B == 0) return IHIP_OK;
    if (shape->Tq != 1 || shape->b_q != 1) return fail(IHIP_ERR_INVALID_ARG, "%s: needs Tq == b_q == 1", who);
    if ((rc = check_tensor(q, who, "q")) != IHIP_OK) return rc;
    StoreView w;
    if ((rc = check_store(who, store, *shape, &w)) != IHIP_OK) return rc;
    if (store->format != IHIP_KV_MX4) return fail(IHIP_ERR_INVALID_ARG, "%s: the store holds no 4-bit rows (format %d)", who, store->format);
    if ((w.k_sb | w.k_st | w.k_sh) < 0 || w.k_sb / 64 > UINT32_MAX || w.k_st / 64 > UINT32_MAX)
        return fail(IHIP_ERR_UNSUPPORTED, "%s: strides must be from 0 to 2^32 rows of 64 bytes", who);
    if (n_blocks < 0 || !pow2(block)) return fail(IHIP_ERR_INVALID_ARG, "%s: n_blocks = %d, block = %d", who, n_blocks, block);
    if (n_blocks > 0 && !block_starts) return fail(IHIP_ERR_INVALID_ARG, "%s: block_starts is NULL", who);
    if (mx4_slots(*shape, n_blocks, block) > INT32_MAX - kMxMaxSplit)
        return fail(IHIP_ERR_UNSUPPORTED, "%s: more than 2^31 slots", who);
    if (!out) return fail(IHIP_ERR_INVALID_ARG, "%s: out is NULL", who);
    const size_t need = attn_decode_mx4_workspace(*shape, n_blocks, block);
    if (!ws || ((uintptr_t)ws & 7) || ws_bytes < need)
        return fail(IHIP_ERR_WORKSPACE, "%s: workspace of %zu bytes, 8-byte aligned, needed, %zu given", who, need, ws_bytes);
    AttnMx4Args a{};
    a.ge = make_geometry(*shape);
    a.q = (const uint16_t *)q.ptr; a.q_sb = q.stride_b; a.q_sh = q.stride_h;
    a.k = w.k; a.v = w.v; a.ks = w.ks; a.vs = w.vs;
    a.sb = (uint32_t)(w.k_sb / 64); a.sh = w.k_sh / 64; a.st = (uint32_t)(w.k_st / 64);
    a.block_starts = block_starts;
    a.n_blocks = n_blocks; a.block = block; a.block_log2 = __builtin_ctz(block);
    if ((rc = check_sm_scale(who, sm_scale, &a.scale_log2e)) != IHIP_OK) return rc;
    a.n_splits = mx4_splits(*shape, n_blocks, block).best;
    a.grid = decode_grid(a.ge, a.n_splits, false);
    a.paged = w.paged;
    const int P = shape->B * shape->Hkv;
    a.part_ml = (float *)ws;
    a.part_acc = a.part_ml + (size_t)P * a.n_splits * a.ge.G * 2;
    a.out = (uint16_t *)out;
    a.out_lse = out_lse;
    const dim3 grid = a.grid.dims(P, a.n_splits);
    if (grid.y > 65535) return fail(IHIP_ERR_UNSUPPORTED, "%s: %d sequences x KV heads are too many", who, P);
    const hipStream_t st = (hipStream_t)stream;
    {
        KernelTimer timer("attn_decode_mx4", st);
        if (a.ge.G <= 4) hipLaunchKernelGGL(attn_decode_mx4_kernel<4>, grid, dim3(kMxThreads), 0, st, a);
        else hipLaunchKernelGGL(attn_decode_mx4_kernel<8>, grid, dim3(kMxThreads), 0, st, a);
    }
    if ((rc = check_launch(who)) != IHIP_OK || a.n_splits == 1) return rc;
    KernelTimer timer("attn_decode_mx4_merge", st);
    hipLaunchKernelGGL(attn_decode_mx4_merge_kernel, dim3(P * a.ge.G), dim3(kD * kMxMergeGroups), 0, st, a);
    return check_launch(who);
}

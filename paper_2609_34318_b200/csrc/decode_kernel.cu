// Attention of one new token per sequence over a paged key / value cache.
//
//   s_j = scale <q_a, k_j>,  LSE = ln sum_j exp(s_j),  O = sum_j exp(s_j - LSE) v_j
//
// over the cached positions j of the sequence, for every query head a; the g query heads that share a K / V head read its
// rows together. Every K / V row is needed once, 2 (d_qk + d_v) bytes for 2 g (d_qk + d_v) FLOP: memory bounds it for every
// grouping, and what counts is that all SMs load all the time, whatever the lengths are.
//
// Work. The keys of a (sequence, K / V head) pair are cut into tiles of 64; all tiles of a call, one pair after the other,
// are dealt out to the thread blocks (one per SM) in equal runs. A run covers the end of one pair, some whole pairs and the
// beginning of another. Whole pairs are written straight to out / lse; the two cut ones leave (O, LSE) in fp32 in the
// workspace, and hydra_decode_join_kernel joins what belongs together, in the order of the keys: results do not depend on
// timing. The lengths are read on the device, so a captured call follows them.
//
// A thread block: one warp reads the page table and loads K, V (boxes of 16 or 8 rows, 128-byte swizzle) and, with the first
// tile of a pair, its q rows into a ring of stages; four warps take 16 keys of every tile each, with a running maximum, sum
// and accumulator of their own, joined once per pair. Products on mma.sync: 16 query rows (the group, padded) against 16
// keys are far below what a tcgen05 product computes at once, and the tensor cores idle either way (1 to 16 FLOP per byte).
#include <cuda_bf16.h>

#include <algorithm>

#include "hydra_internal.h"
#include "sm100_ptx.cuh"

namespace hydra {
namespace {

constexpr int kSmemOfSm = 228 * 1024;        // of which the system takes 1 KB per thread block
constexpr float kRaise = 8.f;               // the running maximum is raised when it grew by more than 2^8

enum : int32_t { FLAG_FIRST = 1, FLAG_LAST = 2, FLAG_END = 4, FLAG_PARTIAL = 8, FLAG_SECOND_SLOT = 16 };
struct __align__(16) StageDesc {
    uint64_t seen;                          // keys of the tile that count
    int32_t item;                           // (sequence * kv_heads + kv head) * chunks + chunk
    int32_t flags;
};

// Thread blocks of one kind. kNTiles: tiles of eight query heads per warp; kHeadWarps: warps that share a key's query heads;
// kKeyWarps: warps that share a tile's keys, 16 each; kPerSm: thread blocks per SM.
template <int kDqk_, int kNTiles_, int kHeadWarps_, int kKeyWarps_, int kPerSm_>
struct Shape {
    static constexpr int kDqk = kDqk_, kNTiles = kNTiles_, kHeadWarps = kHeadWarps_, kKeyWarps = kKeyWarps_, kPerSm = kPerSm_;
    static constexpr int kKeys = 16 * kKeyWarps;                        // of a tile
    static constexpr int kRows = 8 * kNTiles * kHeadWarps;              // query heads of a block
    static constexpr int kConsumers = kKeyWarps * kHeadWarps;           // warps
    static constexpr int kThreads = 32 * (kConsumers + 1);
    static constexpr int kKBytes = kKeys * kDqk * 2, kVBytes = kKeys * D_V * 2, kQBytes = kRows * kDqk * 2;
    static constexpr int kStage = kKBytes + kVBytes + kQBytes;
    // floats between rows of the join buffer: 2 * 132 = 8 (mod 32), the eight values and four heads of a warp's store meet 32 banks
    static constexpr int kJoinStride = D_V + 4;
    static constexpr int kJoin = kKeyWarps * kRows * kJoinStride * 4;
    static constexpr int kFixed = 1024 + 512 + 16 * kKeyWarps * kRows;      // alignment of the ring; barriers and descriptors; (m, l)
    static constexpr int kFit = (kSmemOfSm / kPerSm - 1024 - kJoin - kFixed) / kStage;
    static constexpr int kStages = kFit < 8 ? kFit : 8;
    static constexpr int kSmem = kStages * kStage + kJoin + 1024;
    static_assert(kStage % 1024 == 0 && kStages >= 2, "ring");
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// an 8 x 8 matrix of 16-bit values, a thread's two of row lane / 4, becomes its transpose
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// c[16 x 8] += a[16 x 16] b[16 x 8]
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }

// Tiles of a sequence. Lengths outside the table's reach count as its ends.
__device__ __forceinline__ int32_t seq_len_of(const DecodeParams& p, int32_t b)
{
    return min(max(__ldcg(p.seq_lens + b), 0), p.max_len);
}
__device__ __forceinline__ int32_t tiles_of(const DecodeParams& p, int32_t len) { return (len + p.tile_keys - 1) / p.tile_keys; }

// The run of thread block c of n: tiles [total c / n, total (c + 1) / n); the block that has tile t.
__device__ __forceinline__ int64_t run_start(int64_t total, int64_t c, int64_t n) { return total * c / n; }
__device__ __forceinline__ int64_t block_of(int64_t total, int64_t t, int64_t n) { return ((t + 1) * n - 1) / total; }

struct Start { int32_t seq; int32_t pad; int64_t before; int64_t total; };

template <class S>
__global__ void __launch_bounds__(S::kThreads, S::kPerSm)
hydra_decode_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const DecodeParams p,
                    const uint64_t call_tag)
{
    constexpr int kDqk = S::kDqk, kKeys = S::kKeys, kKeyWarps = S::kKeyWarps, kNT = S::kNTiles;
    constexpr int kBoxesK = kDqk / 64, kBoxesV = D_V / 64, kBox = kKeys * 128;      // 64 columns of a tile
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 2];
    __shared__ StageDesc s_desc[S::kStages];
    __shared__ float2 s_ml[2][kKeyWarps][S::kRows];      // of two pairs in turn: the slowest warp may still read the last one's
    __shared__ int64_t s_scan[S::kThreads / 32];
    __shared__ Start s_start;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    float* const join = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)) + S::kStages * S::kStage);
    auto full = [&](int s) { return smem_u32(&bars[s]); };
    auto empty = [&](int s) { return smem_u32(&bars[S::kStages + s]); };
    const uint32_t join_bar[2] = {smem_u32(&bars[2 * S::kStages]), smem_u32(&bars[2 * S::kStages + 1])};
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), S::kConsumers); }
        mbar_init(join_bar[0], S::kConsumers);
        mbar_init(join_bar[1], S::kConsumers);
        fence_mbar_init();
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
        abort_flag = 0;
        s_start.total = 0;
    }
    wait_for_previous_launch();
    overlap_next_launch();                              // (the join's blocks wait for this grid's end)
    if (call_tag && blockIdx.x == 0 && tid == 0) {      // nothing has cleared the status block
        p.status->call_tag = call_tag;
        for (int i = 0; i < 4; ++i) p.status->probe_cycles[i] = p.status->probe_ns[i] = 0;
    }

    // ------------------------------------------------------------------ this block's run of tiles
    const int32_t per_seq = p.kv_heads * p.chunks;      // pairs of a sequence
    int64_t n_blocks;
    {
        const int per = (p.n_seqs + S::kThreads - 1) / S::kThreads;
        const int b0 = min(tid * per, p.n_seqs), b1 = min(b0 + per, p.n_seqs);
        int64_t mine = 0;
        for (int b = b0; b < b1; ++b) mine += tiles_of(p, seq_len_of(p, b));
        int64_t sum = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t up = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += up;
        }
        if (lane == 31) s_scan[warp] = sum;
        __syncthreads();
        int64_t before = sum - mine, all = 0;
        for (int w = 0; w < S::kThreads / 32; ++w) {
            if (w < warp) before += s_scan[w];
            all += s_scan[w];
        }
        const int64_t total = all * per_seq;
        n_blocks = min(static_cast<int64_t>(gridDim.x), total);
        if (blockIdx.x >= n_blocks) return;
        const int64_t first = run_start(total, blockIdx.x, n_blocks) / per_seq;     // in tiles of a head
        if (first >= before && first < before + mine) {
            int64_t at = before;
            int b = b0;
            for (;; ++b) {
                const int n = tiles_of(p, seq_len_of(p, b));
                if (first < at + n) break;
                at += n;
            }
            s_start.seq = b;
            s_start.before = at;
            s_start.total = total;
        }
        __syncthreads();
    }
    const int64_t total = s_start.total;
    const int64_t lo = run_start(total, blockIdx.x, n_blocks), hi = run_start(total, blockIdx.x + 1, n_blocks);
    const uint64_t limit = p.wait_limit_ns;
    volatile int* abort_p = &abort_flag;

    if (warp == S::kConsumers) {
        // ------------------------------------------------------------------ page table and loads
        if (p.debug_stall_ns) {
            debug_stall(p.debug_stall_ns);              // test hook: load nothing; the other warps' waits run out
        } else {
            const int32_t boxes = kKeys / p.box_rows;   // of a tile; lane j asks for box j's page
            const int32_t key_in_tile = lane * p.box_rows;
            int32_t b = s_start.seq, len = seq_len_of(p, b), n_tiles = tiles_of(p, len);
            int64_t base = s_start.before * per_seq;    // first tile of sequence b
            int32_t in_seq = static_cast<int32_t>((lo - base) / n_tiles);           // pair of the sequence, and tile of the pair
            int32_t tile = static_cast<int32_t>((lo - base) - static_cast<int64_t>(in_seq) * n_tiles);
            auto page_at = [&](int32_t seq, int32_t key, int32_t seq_len) -> int32_t {
                return lane < boxes && key < seq_len ? __ldcg(p.page_table + static_cast<int64_t>(seq) * p.max_pages + key / p.page_size) : -1;
            };
            int32_t page = page_at(b, tile * kKeys + key_in_tile, len);
            bool ok = true;
            for (int64_t t = lo; t <= hi; ++t) {
                const int st = static_cast<int>((t - lo) % S::kStages);
                const uint32_t turn = static_cast<uint32_t>((t - lo) / S::kStages);
                if (lane == 0) ok = mbar_wait(empty(st), (turn & 1u) ^ 1u, abort_p, limit);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                if (t == hi) {
                    if (lane == 0) { s_desc[st].flags = FLAG_END; mbar_arrive(full(st)); }
                    break;
                }
                const int32_t key = tile * kKeys + key_in_tile;
                const bool there = lane < boxes && key < len && page >= 0 && page < p.n_pages;
                const uint64_t mask = there ? (~0ull >> (64 - min(p.box_rows, len - key))) << key_in_tile : 0ull;
                const uint32_t seen_lo = __reduce_or_sync(0xffffffffu, static_cast<uint32_t>(mask));
                const uint32_t seen_hi = __reduce_or_sync(0xffffffffu, static_cast<uint32_t>(mask >> 32));
                const int n_boxes = __popc(__ballot_sync(0xffffffffu, there));
                const bool first = tile == 0 || t == lo, last = tile == n_tiles - 1 || t == hi - 1;
                const int32_t kvh = in_seq / p.chunks, chunk = in_seq - kvh * p.chunks;
                const int32_t q_rows = min(S::kRows, p.group - chunk * S::kRows);
                const uint32_t stage = ring + static_cast<uint32_t>(st) * S::kStage;
                if (lane == 0) {
                    // does another block have tiles of this pair?
                    const int64_t pair0 = t - tile;
                    const bool cut = pair0 < lo || pair0 + n_tiles > hi;
                    s_desc[st].seen = static_cast<uint64_t>(seen_hi) << 32 | seen_lo;
                    s_desc[st].item = b * per_seq + in_seq;
                    s_desc[st].flags = (first ? FLAG_FIRST : 0) | (last ? FLAG_LAST : 0) | (cut ? FLAG_PARTIAL : 0) |
                                       (pair0 >= lo ? FLAG_SECOND_SLOT : 0);
                    const uint32_t q_bytes = first ? static_cast<uint32_t>(q_rows) * kDqk * 2 : 0u;
                    mbar_arrive_expect_tx(full(st), static_cast<uint32_t>(n_boxes * p.box_rows) * (kDqk + D_V) * 2 + q_bytes);
                    if (first)
                        bulk_load(stage + S::kKBytes + S::kVBytes,
                                  p.q + b * p.q_stride + static_cast<int64_t>(kvh * p.group + chunk * S::kRows) * kDqk, q_bytes, full(st));
                }
                __syncwarp();
                if (there) {
                    const int32_t row = static_cast<int32_t>((static_cast<int64_t>(page) * p.kv_heads + kvh) * p.page_size + key % p.page_size);
                    const uint32_t dst = stage + static_cast<uint32_t>(key_in_tile) * 128;
#pragma unroll
                    for (int c = 0; c < kBoxesK; ++c) tma_load_2d(dst + c * kBox, &map_k, full(st), c * 64, row);
#pragma unroll
                    for (int c = 0; c < kBoxesV; ++c) tma_load_2d(dst + S::kKBytes + c * kBox, &map_v, full(st), c * 64, row);
                }
                // the next tile, and its pages while the ring is waited for
                if (++tile == n_tiles) {
                    tile = 0;
                    if (++in_seq == per_seq) {
                        in_seq = 0;
                        if (t + 1 < hi) {
                            do { len = seq_len_of(p, ++b); } while (len == 0);
                            n_tiles = tiles_of(p, len);
                        }
                    }
                }
                if (t + 1 < hi) page = page_at(b, tile * kKeys + key_in_tile, len);
            }
        }
    } else {
        // ------------------------------------------------------------------ scores, softmax, O
        // Keys stand on the 16 rows of a product and query heads on its 8 columns: S^T = K Q^T, O^T = V^T P^T. A thread has the
        // heads 2 (lane mod 4) and the one after it, of every tile of eight, and of a product the rows lane / 4 and 8 more.
        const int kw = warp % kKeyWarps, head_of_warp = warp / kKeyWarps * 8 * kNT, key_of_lane = lane >> 2;
        uint32_t q[kDqk / 16][kNT][2];
        float o[D_V / 16][kNT][4];
        float m[kNT][2], l[kNT][2];
        const uint32_t k_row = static_cast<uint32_t>(kw * 16 + (lane & 15)), k_unit = (lane >> 4) & 1;
        const uint32_t v_row = static_cast<uint32_t>(kw * 16 + (lane & 7) + ((lane >> 4) & 1) * 8), v_unit = (lane >> 3) & 1;
        uint32_t joins = 0;
        for (uint32_t n = 0;; ++n) {
            const int st = static_cast<int>(n % S::kStages);
            if (!mbar_wait(full(st), (n / S::kStages) & 1u, abort_p, limit)) break;
            const StageDesc d = s_desc[st];
            if (d.flags & FLAG_END) break;
            const uint32_t stage = ring + static_cast<uint32_t>(st) * S::kStage;
            if (d.flags & FLAG_FIRST) {
#pragma unroll
                for (int t = 0; t < kNT; ++t) {
                    const uint32_t q_at = stage + S::kKBytes + S::kVBytes + static_cast<uint32_t>(head_of_warp + t * 8 + (lane & 7)) * (kDqk * 2) + (lane >> 3) * 16;
#pragma unroll
                    for (int ks = 0; ks < kDqk / 16; ks += 2) {
                        uint32_t f[4];
                        ldmatrix_x4(q_at + ks * 32, f);
                        q[ks][t][0] = f[0]; q[ks][t][1] = f[1]; q[ks + 1][t][0] = f[2]; q[ks + 1][t][1] = f[3];
                    }
                }
#pragma unroll
                for (int i = 0; i < D_V / 16 * kNT * 4; ++i) o[i / (4 * kNT)][i / 4 % kNT][i % 4] = 0.f;
#pragma unroll
                for (int t = 0; t < kNT; ++t) {
                    m[t][0] = m[t][1] = neg_inf();
                    l[t][0] = l[t][1] = 0.f;
                }
            }
            const uint32_t seen = static_cast<uint32_t>(d.seen >> (kw * 16)) & 0xffffu;
            if (seen) {
                float s[2][kNT][4];                     // even and odd steps: two chains of products per tile of heads
#pragma unroll
                for (int i = 0; i < 8 * kNT; ++i) s[i / (4 * kNT)][i / 4 % kNT][i % 4] = 0.f;
#pragma unroll
                for (int ks = 0; ks < kDqk / 16; ++ks) {
                    uint32_t kf[4];
                    ldmatrix_x4(stage + (ks / 4) * kBox + k_row * 128 + ((((ks % 4) * 2 + k_unit) ^ (k_row & 7)) << 4), kf);
#pragma unroll
                    for (int t = 0; t < kNT; ++t) mma_bf16(s[ks & 1][t], kf, q[ks][t][0], q[ks][t][1]);
                }
                const uint32_t bits = seen >> key_of_lane;      // bit 0: this thread's first key, bit 8: its second
                uint32_t ph[kNT][2], pl[kNT][2];
#pragma unroll
                for (int t = 0; t < kNT; ++t) {
                    float x[4];                         // [key][head]
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = (s[0][t][e] + s[1][t][e]) * p.scale_log2;
                        if (!(bits >> (8 * (e >> 1)) & 1u)) x[e] = neg_inf();
                    }
                    // The reference of the exponentials is raised when a score is more than 2^8 above it: until then, no warp-wide
                    // maximum is needed, one vote says so.
                    const float top0 = fmaxf(x[0], x[2]), top1 = fmaxf(x[1], x[3]);
                    if (__any_sync(0xffffffffu, top0 > m[t][0] + kRaise || top1 > m[t][1] + kRaise)) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float top = c ? top1 : top0;
#pragma unroll
                            for (int g = 4; g < 32; g *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, g));
                            if (top > m[t][c] + kRaise) {
                                const float f = ex2_approx(m[t][c] - top);
                                m[t][c] = top;
                                l[t][c] *= f;
#pragma unroll
                                for (int j = 0; j < D_V / 16; ++j) { o[j][t][c] *= f; o[j][t][c + 2] *= f; }
                            }
                        }
                    }
                    const float ref0 = m[t][0] == neg_inf() ? 0.f : m[t][0], ref1 = m[t][1] == neg_inf() ? 0.f : m[t][1];
                    float pr[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) pr[e] = ex2_approx(x[e] - (e & 1 ? ref1 : ref0));
                    l[t][0] += pr[0] + pr[2];
                    l[t][1] += pr[1] + pr[3];
                    // P as the sum of two bf16 (2^-17 of it is lost): the tensor cores have time for a second product, and with
                    // one the rounding of P alone is as large as that of the bf16 result
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t h = pack_bf16x2(pr[2 * e], pr[2 * e + 1]);
                        ph[t][e] = transpose_8x8(h);
                        pl[t][e] = transpose_8x8(pack_bf16x2(pr[2 * e] - __uint_as_float(h << 16), pr[2 * e + 1] - __uint_as_float(h & 0xffff0000u)));
                    }
                }
                // rows behind the end hold anything: 0 * NaN must not reach the sums
                const uint32_t v_bits = seen >> (2 * (lane & 3));
                const uint32_t keep0 = (v_bits & 1u ? 0xffffu : 0u) | (v_bits & 2u ? 0xffff0000u : 0u);
                const uint32_t keep1 = (v_bits & 0x100u ? 0xffffu : 0u) | (v_bits & 0x200u ? 0xffff0000u : 0u);
#pragma unroll
                for (int j = 0; j < D_V / 16; ++j) {
                    uint32_t vf[4];
                    ldmatrix_x4_trans(stage + S::kKBytes + (j / 4) * kBox + v_row * 128 + ((((j % 4) * 2 + v_unit) ^ (v_row & 7)) << 4), vf);
                    if (seen != 0xffffu) { vf[0] &= keep0; vf[1] &= keep0; vf[2] &= keep1; vf[3] &= keep1; }
#pragma unroll
                    for (int t = 0; t < kNT; ++t) {
                        mma_bf16(o[j][t], vf, ph[t][0], ph[t][1]);
                        mma_bf16(o[j][t], vf, pl[t][0], pl[t][1]);
                    }
                }
            }
            mbar_arrive_warp(empty(st));
            if (!(d.flags & FLAG_LAST)) continue;

            // ---------------------------------------------------------------- the warps' shares of the pair, joined
            const int32_t chunk = d.item % p.chunks, bh = d.item / p.chunks, b = bh / p.kv_heads, kvh = bh - b * p.kv_heads;
            const int32_t head0 = kvh * p.group + chunk * S::kRows, q_rows = min(S::kRows, p.group - chunk * S::kRows);
            auto& ml_of = s_ml[joins & 1u];
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int g = 4; g < 32; g *= 2) l[t][c] += __shfl_xor_sync(0xffffffffu, l[t][c], g);
                    if (lane < 4) ml_of[kw][head_of_warp + t * 8 + 2 * lane + c] = make_float2(m[t][c], l[t][c]);
                }
            mbar_arrive_warp(join_bar[0]);
            if (!mbar_wait(join_bar[0], joins & 1u, abort_p, limit)) break;
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int row = head_of_warp + t * 8 + 2 * (lane & 3) + c;
                    if (row >= q_rows) continue;
                    float top = neg_inf();
#pragma unroll
                    for (int w = 0; w < kKeyWarps; ++w) top = fmaxf(top, ml_of[w][row].x);
                    const float f = m[t][c] == neg_inf() ? 0.f : ex2_approx(m[t][c] - top);
                    float* dst = join + (kw * S::kRows + row) * S::kJoinStride + key_of_lane;
#pragma unroll
                    for (int j = 0; j < D_V / 16; ++j) {
                        dst[16 * j] = o[j][t][c] * f;
                        dst[16 * j + 8] = o[j][t][c + 2] * f;
                    }
                }
            mbar_arrive_warp(join_bar[1]);
            if (!mbar_wait(join_bar[1], joins & 1u, abort_p, limit)) break;
            ++joins;
            const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (d.flags & FLAG_SECOND_SLOT ? 1 : 0);
            for (int e = warp; e < q_rows; e += S::kConsumers) {
                float top = neg_inf(), sum = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kKeyWarps; ++w) top = fmaxf(top, ml_of[w][e].x);
#pragma unroll
                for (int w = 0; w < kKeyWarps; ++w) {
                    const float2 ml = ml_of[w][e];
                    if (ml.x != neg_inf()) sum += ml.y * ex2_approx(ml.x - top);
                    const float4 x = *reinterpret_cast<const float4*>(join + (w * S::kRows + e) * S::kJoinStride + 4 * lane);
                    acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
                }
                const float inv = top == neg_inf() ? 0.f : 1.f / sum, lse2 = top == neg_inf() ? top : top + log2f(sum);
                acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
                if (d.flags & FLAG_PARTIAL) {
                    reinterpret_cast<float4*>(p.part_o + (slot * S::kRows + e) * D_V)[lane] = acc;
                    if (lane == 0) p.part_lse2[slot * S::kRows + e] = lse2;
                } else {
                    reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(b) * p.h + head0 + e) * D_V)[lane] =
                        make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
                    if (lane == 0) p.lse[static_cast<int64_t>(head0 + e) * p.n_seqs + b] = lse2 * 0.6931471805599453f;
                }
            }
        }
    }
    __syncthreads();
    if (abort_flag) {
        // A wait ran out. Give copies still in flight time to land, then report and leave.
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 50000ull) { }
        if (tid == 0) {
            p.status->detail = blockIdx.x;
            p.status->error_tag = call_tag;
            p.status->status = HYDRA_ERR_DEVICE_TIMEOUT;
        }
        __syncthreads();
    }
}

// Rows (sequence, query head) whose keys several thread blocks had: (O, LSE) of the parts joined in the order of the keys.
// Rows without a key: O = 0, LSE = -inf. The others have been written. kWarps per row.
constexpr int kJoinThreads = 256;
template <int kWarps>
__global__ void __launch_bounds__(kJoinThreads)
hydra_decode_join_kernel(const DecodeParams p, int32_t n_blocks_max)
{
    constexpr int kRowsPerBlock = kJoinThreads / 32 / kWarps;
    __shared__ float4 s_acc[kWarps > 1 ? kWarps : 1][32];
    __shared__ float s_sum[kWarps > 1 ? kWarps : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp % kWarps;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRowsPerBlock + warp / kWarps;
    const bool valid = row < static_cast<int64_t>(p.n_seqs) * p.h;
    const int32_t b = valid ? static_cast<int32_t>(row / p.h) : 0, a = valid ? static_cast<int32_t>(row - static_cast<int64_t>(b) * p.h) : 0;
    const int32_t per_seq = p.kv_heads * p.chunks;
    int64_t before = 0, all = 0;
    for (int32_t i = lane; i < p.n_seqs; i += 32) {
        const int32_t n = tiles_of(p, seq_len_of(p, i));
        all += n;
        if (i < b) before += n;
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        all += __shfl_xor_sync(0xffffffffu, all, d);
        before += __shfl_xor_sync(0xffffffffu, before, d);
    }
    const int32_t n_tiles = tiles_of(p, seq_len_of(p, b));
    const int32_t kvh = a / p.group, in_group = a - kvh * p.group, chunk = in_group / p.chunk_rows, r = in_group - chunk * p.chunk_rows;
    const int64_t total = all * per_seq, n_blocks = min(static_cast<int64_t>(n_blocks_max), total);
    const int64_t t0 = before * per_seq + static_cast<int64_t>(kvh * p.chunks + chunk) * n_tiles;
    const int64_t c0 = n_tiles ? block_of(total, t0, n_blocks) : 0, c1 = n_tiles ? block_of(total, t0 + n_tiles - 1, n_blocks) : 0;
    uint2* const out = reinterpret_cast<uint2*>(p.out + row * D_V) + lane;
    float* const lse = p.lse + static_cast<int64_t>(a) * p.n_seqs + b;
    wait_for_previous_launch();
    if (!valid || (n_tiles > 0 && c0 == c1)) return;    // (all warps of a row leave together)
    if (n_tiles == 0) {
        if (w == 0) {
            *out = make_uint2(0u, 0u);
            if (lane == 0) *lse = neg_inf();
        }
        return;
    }
    const int32_t parts = static_cast<int32_t>(c1 - c0) + 1;
    // part i is the beginning of block c0 + i's run, but the first is the end of its block's
    auto at = [&](int32_t i) { return (2 * (c0 + i) + (i == 0 ? 1 : 0)) * p.chunk_rows + r; };
    float top = neg_inf();
    for (int32_t i = lane; i < parts; i += 32) top = fmaxf(top, __ldcg(p.part_lse2 + at(i)));
#pragma unroll
    for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float ref = top == neg_inf() ? 0.f : top;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int32_t i = w; i < parts; i += kWarps) {
        const float f = ex2_approx(__ldcg(p.part_lse2 + at(i)) - ref);
        const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part_o + at(i) * D_V) + lane);
        sum += f;
        acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
    }
    if (kWarps > 1) {
        s_acc[w][lane] = acc;
        if (lane == 0) s_sum[w] = sum;
        __syncthreads();
        if (w) return;
        for (int i = 1; i < kWarps; ++i) {
            const float4 x = s_acc[i][lane];
            acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
            sum += s_sum[i];
        }
    }
    const float inv = top == neg_inf() ? 0.f : 1.f / sum;
    *out = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (lane == 0) *lse = top == neg_inf() ? top : (top + log2f(sum)) * 0.6931471805599453f;
}

struct Form {
    int32_t rows, tile_keys, per_sm;
    cudaError_t (*launch)(const CUtensorMap&, const CUtensorMap&, const DecodeParams&, uint64_t, int, cudaStream_t);
};
template <class S>
cudaError_t launch_one(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& p, uint64_t call_tag, int grid,
                       cudaStream_t stream)
{
    static OncePerDevice configured;
    const auto kernel = hydra_decode_kernel<S>;
    if (cudaError_t e = allow_dynamic_smem(kernel, S::kSmem, configured)) return e;
    return launch_overlapped(kernel, grid, S::kThreads, S::kSmem, stream, mk, mv, p, call_tag);
}
template <class S>
constexpr Form form_of() { return {S::kRows, S::kKeys, S::kPerSm, launch_one<S>}; }

// by query heads per K / V head
template <int kDqk>
const Form& form_for(int32_t group)
{
    static constexpr Form one = form_of<Shape<kDqk, 1, 1, 4, 2>>(), two = form_of<Shape<kDqk, 2, 1, 2, 3>>(),
                          four = form_of<Shape<kDqk, 2, 2, 4, 1>>();
    return group <= 8 ? one : group <= 16 ? two : four;
}
const Form& form_for(int32_t d_qk, int32_t group) { return d_qk == 192 ? form_for<192>(group) : form_for<128>(group); }

}  // namespace

DecodeForm decode_form(int32_t d_qk, int32_t group)
{
    const Form& f = form_for(d_qk, group);
    return {f.rows, f.tile_keys, f.per_sm};
}

cudaError_t launch_decode(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& p, int32_t d_qk, uint64_t call_tag,
                          int grid, cudaStream_t stream)
{
    return form_for(d_qk, p.group).launch(mk, mv, p, call_tag, grid, stream);
}

cudaError_t launch_decode_join(const DecodeParams& p, int grid_of_parts, cudaStream_t stream)
{
    const int64_t rows = static_cast<int64_t>(p.n_seqs) * p.h;
    // few pairs have many parts each: eight warps share a row
    if (static_cast<int64_t>(p.n_seqs) * p.kv_heads * p.chunks < grid_of_parts / 4)
        return launch_overlapped(hydra_decode_join_kernel<8>, static_cast<int>(rows), kJoinThreads, 0, stream, p, grid_of_parts);
    return launch_overlapped(hydra_decode_join_kernel<1>, static_cast<int>((rows + 7) / 8), kJoinThreads, 0, stream, p, grid_of_parts);
}

}  // namespace hydra

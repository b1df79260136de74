// Attention of one new token per sequence over a paged key / value cache.
//
//   s_j = scale <q_a, k_j>,  LSE = ln sum_j exp(s_j),  O = sum_j exp(s_j - LSE) v_j
//
// over the cached positions j of the sequence, for every query head a; the g query heads that share a K / V head read its
// rows together. Every K / V row is needed once, 2 (d_qk + d_v) bytes for 2 g (d_qk + d_v) FLOP: memory bounds it for every
// grouping, and what counts is that all SMs load all the time, whatever the lengths are.
//
// Work. A unit is a sequence and up to four neighbouring K / V heads (their rows of a page lie side by side: a unit's loads are four
// times as long, and its pages are looked up and translated once for all of them). Its keys are cut into tiles of 64 rows (keys
// times heads); all tiles of a call, one unit after the other, are cut into pieces (struct Pieces): every thread block, one per
// SM, has one of seven eighths of its share, and the rest is popped from a counter in ever smaller pieces, because SMs do not
// read equally fast (equal shares of 256K tokens ended between 342 and 381 us). A piece covers the end of one unit, some whole units and the
// beginning of another. Whole units are written straight to out / lse; cut ones leave (O, LSE) in fp32 in the workspace, and
// hydra_decode_join_kernel joins what belongs together, in the order of the keys: who ran a piece changes nothing. The lengths are
// read on the device, so a captured call follows them.
//
// A thread block. One warp plans ahead: lengths, page table, the q rows of every unit. One loads the tiles into a ring. Eight
// warps, two sets of four, take 16 rows of a tile each, one head's, with a running maximum, sum and O of their own (the sets take
// tiles in turn, or, with more than eight query heads per K / V head, each half of the query heads). When a unit is through they
// leave them in shared memory and each joins some of the query heads, while the ring goes on being filled.
// Products on mma.sync: up to eight query heads per K / V head the loads bound the kernel (the tensor pipe is active for 8 % of the
// time with eight) and the accumulators stay in the registers that rescale them. From 16 on the products bound it; 128 keys against
// 8 to 64 query heads would be a shape for tcgen05, which this kernel does not have.
//
// Measured (16 heads of 192 / 128, on two GPUs): 256K tokens 377 to 385 us, 7.0 to 7.1 TB/s read; 230 sequences of 64 to 512 tokens
// 207 to 213 us, 6.3 to 6.5 TB/s; 19 sequences of a 32K batch 63 us for 345 MB, of which 5 pass before the first tile (lengths, page,
// load) and 4 for the join; one sequence of 1000 tokens 10.9 us, nearly all of it that chain. On K / V heads of 128 with 1, 8, 16, 17,
// 32, 64 query heads each, 524288 tokens take 329, 331, 382, 494, 503, 968 us (the copy rate gives 327): more than 32 are read once
// per 32.
#include <cuda_bf16.h>

#include <algorithm>

#include "hydra_internal.h"
#include "sm100_ptx.cuh"

namespace hydra {
namespace {

constexpr int kSlices = 4, kSlice = 16;     // a tile: four slices of 16 rows, each 16 keys of one K / V head
constexpr int kTileRows = kSlices * kSlice;
constexpr int kSmemLimit = 227 * 1024;
constexpr float kRaise = 8.f;               // the running maximum is raised when it grew by more than 2^8

constexpr int kJoinWarps = 4, kJoinParts = 8;      // of hydra_decode_join_kernel: warps of a block, parts that a warp asks for at once
constexpr int kJoinChunk = kJoinWarps * kJoinParts;     // parts that a block joins of a row

struct __align__(16) TileDesc {
    uint64_t seen;                          // keys of the tile that count
    uint32_t unit;                          // number of its unit, counted over the block's pieces; or kEnd
    uint32_t set;                           // of the warps that take it in turn
};
constexpr uint32_t kLastOfUnit = 1u << 31;  // added to the unit: the last of its tiles in this piece
constexpr uint32_t kEnd = 0x7fffffffu;      // no tile is left
struct __align__(16) UnitDesc {
    int32_t seq, unit;                      // unit of the sequence
    int32_t slot;                           // of a partial result; negative: the whole unit is here
};
// What the planning warp hands to the loading warp at a time: up to eight tiles of one unit. (No more of them: the pieces that a
// block pops are to depend on how far it is.)
constexpr int kBatches = 2, kBatchTiles = 8;
struct __align__(16) BatchDesc {
    int32_t tiles;                          // of the batch; negative: no tile is left
    uint32_t unit;
    int32_t left;                           // tiles of the unit in this piece, those of the batch and behind it
    int32_t head;                           // its first K / V head
    uint32_t set;                           // of the warps that take the first tile (by its number in the piece: which warp takes a
};                                          // tile, and with it the order of the sums, does not depend on what the block ran before)
struct __align__(16) BoxDesc {
    int32_t page, row;                      // page < 0: nothing to load
    int32_t rows;                           // that count; fewer than a box's at the end of a sequence
    uint32_t loaded;                        // rows per head that are loaded of the box's tile
};

// kNTiles: tiles of eight query heads per warp; kHeadSets: sets of warps that share a tile, each with query heads of its own (one:
// the two sets take tiles in turn)
template <int kDqk_, int kNTiles_, int kHeadSets_>
struct Shape {
    static constexpr int kDqk = kDqk_, kNTiles = kNTiles_, kHeadSets = kHeadSets_, kTurns = 2 / kHeadSets;
    static constexpr int kWarpRows = 8 * kNTiles;                       // query heads of a warp
    static constexpr int kRows = kNTiles * kHeadSets == 4 ? 32 : 16;    // most query heads of a unit (decode_unit_kv_heads)
    static constexpr int kConsumers = 2 * kSlices;                      // warps
    static constexpr int kThreads = 32 * (kConsumers + 2);
    static constexpr int kKBytes = kTileRows * kDqk * 2, kVBytes = kTileRows * D_V * 2, kStage = kKBytes + kVBytes;
    // Bytes between rows of q: eight rows meet all banks. (Without the 16 they met the same four: eight warps' matrix loads took some
    // 1000 cycles per unit. One sequence of 1000 tokens 12.3 -> 10.9 us, 19 of a 32K batch 65.9 -> 63.5, 230 of 64 to 512 tokens 211 -> 208.)
    static constexpr int kQRow = kDqk * 2 + 16;
    static constexpr int kQBytes = (kRows == 32 ? kRows : kRows + kWarpRows) * kQRow;  // (the last rows that a product takes may be padding)
    // floats between rows of the join buffer: 2 * 132 = 8 (mod 32), the eight values and four heads of a warp's store meet 32 banks
    static constexpr int kJoinStride = D_V + 4;
    static constexpr int kJoinBytes = kConsumers * kWarpRows * kJoinStride * 4;
    static constexpr int kQSlots = kRows == 16 ? 3 : 2;                 // units that are loaded or being computed
    static constexpr int kFixed = 1024 + 2304 + 8 * kConsumers * kWarpRows;    // alignment of the ring; barriers, descriptors; (m, l)
    static constexpr int kStages = (kSmemLimit - kFixed - kQSlots * kQBytes - kJoinBytes) / kStage;
    static constexpr int kSmem = kStages * kStage + kQSlots * kQBytes + kJoinBytes + 1024;
    static_assert(kStages >= 3 && kStage % 1024 == 0 && kQBytes % 16 == 0, "ring");
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
// 16 bytes of a 128-byte unit of a tile, where the 128-byte swizzle puts them (base: a multiple of 1024)
__device__ __forceinline__ uint32_t swizzled(uint32_t base, uint32_t unit, uint32_t part)
{
    return base + unit * 128 + ((part ^ (unit & 7)) << 4);
}
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// Lengths outside the table's reach count as its ends.
__device__ __forceinline__ int32_t seq_len_of(const DecodeParams& p, int32_t b)
{
    return min(max(__ldcg(p.seq_lens + b), 0), p.max_len);
}
__device__ __forceinline__ int32_t tiles_of(const DecodeParams& p, int32_t len) { return (len + p.tile_keys - 1) >> p.tile_shift; }

// The lengths of all sequences, as a warp has read them: a lane has the sum of its share of the sequences, and the sum up to there,
// in tiles of one unit.
struct Lengths {
    int32_t share, my_len, mine, sum, total;
    static __device__ __forceinline__ int32_t scan(int32_t x, int lane)
    {
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int32_t up = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += up;
        }
        return x;
    }
    __device__ __forceinline__ Lengths(const DecodeParams& p, int lane) : share((p.n_seqs + 31) / 32), my_len(0), mine(0)
    {
#pragma unroll 4
        for (int i = 0; i < share; ++i)
            if (lane * share + i < p.n_seqs) mine += tiles_of(p, my_len = seq_len_of(p, lane * share + i));
        sum = scan(mine, lane);
        total = __shfl_sync(0xffffffffu, sum, 31);
    }
    // the sequence that has tile `at` (of one unit each), its length, and the tiles before it
    __device__ __forceinline__ void find(const DecodeParams& p, int lane, int32_t at, int32_t& b, int32_t& len, int32_t& before) const
    {
        const int owner = __ffs(__ballot_sync(0xffffffffu, sum > at)) - 1;
        before = __shfl_sync(0xffffffffu, sum - mine, owner);
        if (share == 1) {
            b = owner;
            len = __shfl_sync(0xffffffffu, my_len, owner);
            return;
        }
        for (b = owner * share;; b += 32) {
            const int32_t its = b + lane < p.n_seqs ? seq_len_of(p, b + lane) : 0, n = tiles_of(p, its), s = scan(n, lane);
            const uint32_t past = __ballot_sync(0xffffffffu, before + s > at);
            if (past) {
                const int first = __ffs(past) - 1;
                b += first;
                len = __shfl_sync(0xffffffffu, its, first);
                before += __shfl_sync(0xffffffffu, s - n, first);
                return;
            }
            before += __shfl_sync(0xffffffffu, s, 31);
        }
    }
};

// How the tiles of a call are cut: into equal shares, one per thread block, and a share of 64 tiles or more into pieces of 7/8,
// 1/16, 1/32, 1/64 and 1/64 of it (of 32 or more, of 7/8, 1/16, 1/32 and 1/32), which are run in that order: the first pieces of all
// shares, then the second ones, ... Pieces are numbered in the order of their tiles; none in front of the last tile is empty, for
// a unit's parts are counted by them.
struct Pieces {
    int32_t total, blocks, share, levels, start[DECODE_LEVELS + 1];
    __device__ __forceinline__ Pieces(const DecodeParams& p, int32_t tiles_of_a_unit)
        : total(tiles_of_a_unit * p.units), blocks(p.blocks), share(p.by_blocks(total + p.blocks - 1))
    {
        levels = share < 32 ? 1 : share < 64 ? DECODE_LEVELS - 1 : DECODE_LEVELS;
        start[0] = 0;
#pragma unroll
        for (int l = 1; l <= DECODE_LEVELS; ++l) start[l] = share - (l < levels ? share >> (l + 2) : 0);
    }
    __device__ __forceinline__ int32_t count() const { return total ? (total + share - 1) / share * levels : 0; }
    // the i-th piece to be run: its number and tiles (none: it lies behind the end)
    __device__ __forceinline__ int32_t in_order(int32_t i, int32_t& lo, int32_t& hi) const
    {
        int32_t level = 0, of = i;
        for (; of >= blocks; of -= blocks) ++level;
        range(of, level, lo, hi);
        return of * levels + level;
    }
    __device__ __forceinline__ void range(int32_t piece, int32_t& lo, int32_t& hi) const
    {
        const int32_t of = piece / levels;
        range(of, piece - of * levels, lo, hi);
    }
    __device__ __forceinline__ void range(int32_t of, int32_t level, int32_t& lo, int32_t& hi) const
    {
        lo = hi = 0;
#pragma unroll
        for (int l = 0; l < DECODE_LEVELS; ++l)
            if (l == level) { lo = start[l]; hi = start[l + 1]; }
        lo = min(of * share + lo, total);
        hi = min(of * share + hi, total);
    }
    __device__ __forceinline__ int32_t piece_of(int32_t tile) const
    {
        const int32_t of = tile / share, at = tile - of * share;
        int32_t level = 0;
#pragma unroll
        for (int l = 1; l < DECODE_LEVELS; ++l) level += l < levels && at >= start[l] ? 1 : 0;
        return of * levels + level;
    }
};

// The counter of popped pieces: the call's number above kCountBits, the count below. Whatever a workspace held before counts as
// zero; where the launches are recorded the number is zero and a launch of their own clears it. `old` is what atomicAdd(word, 1)
// has returned; the result is the count before it.
constexpr int kCountBits = 20;
__device__ __forceinline__ int32_t popped(unsigned long long* word, unsigned long long old, uint64_t call_tag)
{
    const unsigned long long tag = call_tag >> kCountBits;
    while (old >> kCountBits != tag) {
        const unsigned long long seen = atomicCAS(word, old + 1, (tag << kCountBits) + 1);
        if (seen == old + 1) return 0;
        old = seen >> kCountBits == tag ? atomicAdd(word, 1ull) : seen - 1;
    }
    return static_cast<int32_t>(old & ((1u << kCountBits) - 1));
}

// What (O, log2 of the sum) of several parts is together; 0 and -inf of none
struct Joined { float4 o; float lse2; };
template <int kN>
__device__ __forceinline__ Joined join_of(const float (&part)[kN], const float4 (&x)[kN])
{
    float top = part[0];
#pragma unroll
    for (int j = 1; j < kN; ++j) top = fmaxf(top, part[j]);
    const float ref = top == neg_inf() ? 0.f : top;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
        const float f = ex2_approx(part[j] - ref);
        sum += f;
        o.x += f * x[j].x; o.y += f * x[j].y; o.z += f * x[j].z; o.w += f * x[j].w;
    }
    const float inv = top == neg_inf() ? 0.f : 1.f / sum;
    return {make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv), top == neg_inf() ? top : top + log2f(sum)};
}

template <class S>
__global__ void __launch_bounds__(S::kThreads, 1)
hydra_decode_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_k8, const __grid_constant__ CUtensorMap map_v8, const DecodeParams p,
                    const uint64_t call_tag)
{
    constexpr int kDqk = S::kDqk, kNT = S::kNTiles;
    constexpr uint32_t kUnitsK = kDqk / 64, kUnitsV = D_V / 64;      // 128-byte units of a row
    extern __shared__ uint8_t smem_raw[];
    enum { B_FULL = 0, B_EMPTY = S::kStages, B_QFULL = 2 * S::kStages, B_QEMPTY = B_QFULL + S::kQSlots, B_JFULL = B_QEMPTY + S::kQSlots,
           B_JEMPTY, B_BFULL, B_BEMPTY = B_BFULL + kBatches,
           B_COUNT = B_BEMPTY + kBatches };
    __shared__ __align__(8) uint64_t bars[B_COUNT];
    __shared__ TileDesc s_tile[S::kStages];
    __shared__ UnitDesc s_unit[S::kQSlots];
    __shared__ BatchDesc s_batch[kBatches];
    __shared__ BoxDesc s_box[kBatches][32];
    __shared__ float2 s_ml[S::kConsumers][S::kWarpRows];
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, q_ring = ring + S::kStages * S::kStage;
    float* const join = reinterpret_cast<float*>(smem_raw + (q_ring - smem_u32(smem_raw)) + S::kQSlots * S::kQBytes);
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    if (tid == 0) {
        for (int i = 0; i < S::kStages; ++i) { mbar_init(bar(B_FULL + i), 1); mbar_init(bar(B_EMPTY + i), S::kConsumers); }
        for (int i = 0; i < S::kQSlots; ++i) { mbar_init(bar(B_QFULL + i), 1); mbar_init(bar(B_QEMPTY + i), S::kConsumers); }
        mbar_init(bar(B_JFULL), S::kConsumers);
        mbar_init(bar(B_JEMPTY), S::kConsumers);
        for (int i = 0; i < kBatches; ++i) { mbar_init(bar(B_BFULL + i), 1); mbar_init(bar(B_BEMPTY + i), 1); }
        fence_mbar_init();
        tma_prefetch_desc(&map_k); tma_prefetch_desc(&map_v); tma_prefetch_desc(&map_k8); tma_prefetch_desc(&map_v8);
        abort_flag = 0;
    }
    __syncthreads();
    wait_for_previous_launch();
    overlap_next_launch();                              // (the join's blocks wait for this grid's end)
    if (call_tag && blockIdx.x == 0 && tid == 0) {      // nothing has cleared the status block
        p.status->call_tag = call_tag;
        for (int i = 0; i < 4; ++i) p.status->probe_cycles[i] = p.status->probe_ns[i] = 0;
    }
    // The page table into L2 while the lengths are on their way (a line per thread, more is left to the lookups).
    if (const int64_t at = (static_cast<int64_t>(tid) * gridDim.x + blockIdx.x) * 32; at < static_cast<int64_t>(p.n_seqs) * p.max_pages)
        prefetch_l2(p.page_table + at);
    const uint64_t limit = p.wait_limit_ns;
    volatile int* abort_p = &abort_flag;
    auto wait = [&](int i, uint32_t parity) { return mbar_wait(bar(i), parity & 1u, abort_p, limit); };
    // Lanes that have seen a phase end at different polls have to come together again: the next matrix load or product wants the
    // whole warp.
    auto wait_together = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, wait(i, parity)) != 0; };

    if (warp == S::kConsumers) {
        // ------------------------------------------------------------------ pieces, page table, q
        // Runs ahead of the loading warp, which must not wait for anything but places in the ring: what it does not issue for a
        // moment, the memory does not catch up on.
        if (p.debug_stall_ns) {
            debug_stall(p.debug_stall_ns);              // test hook: plan nothing; the other warps' waits run out
        } else {
            const Lengths lengths(p, lane);
            const Pieces pieces(p, lengths.total);
            const int32_t box_rows = p.box_rows, boxes = p.boxes, most = min(kBatchTiles, 32 / boxes);
            unsigned long long* const counter = reinterpret_cast<unsigned long long*>(&p.status->pieces);
            uint32_t n_unit = 0, n_batch = 0;           // of this block so far
            bool ok = true;
            auto hand_over = [&](const BatchDesc& d, const BoxDesc& box) {
                const uint32_t at = n_batch % kBatches;
                if (lane == 0) ok = wait(B_BEMPTY + at, (n_batch / kBatches) ^ 1u);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) return;
                s_box[at][lane] = box;
                if (lane == 0) s_batch[at] = d;
                mbar_arrive_warp(bar(B_BFULL + at));
                ++n_batch;
            };
            auto plan = [&](int32_t piece, int32_t lo, int32_t hi) {
                int32_t b = 0, len = 0, n_tiles = 0, unit = 0, tile = 0;                // unit of the sequence, tile of the unit
                if (lane == 0) p.arrived[piece] = 0;    // (for the join, which counts with it)
                for (int32_t t = lo; t < hi && ok;) {
                    // The sequence is looked up at the piece's beginning and behind a row without a key. Of those there may be any number:
                    // one after the other, each would be a load that the next one waits for (262144 of them: the call took 42.7 ms, 2.6 so).
                    if (n_tiles == 0) {
                        int32_t before;
                        lengths.find(p, lane, p.by_units(t), b, len, before);
                        n_tiles = tiles_of(p, len);
                        const int32_t in_seq = t - before * p.units;
                        unit = in_seq / n_tiles;
                        tile = in_seq - unit * n_tiles;
                    }
                    // ------------------------------------------------ a unit's tiles in this piece: q rows, what the joining warp needs
                    int32_t left = min(n_tiles - tile, hi - t);
                    const int32_t end = t += left;
                    const int32_t q_slot = n_unit % S::kQSlots, rows = p.rows_of(unit);
                    if (lane == 0) {
                        ok = wait(B_QEMPTY + q_slot, (n_unit / S::kQSlots) ^ 1u);
                        if (ok) {
                            s_unit[q_slot] = {b, unit, left < n_tiles ? 2 * piece + (tile == 0 ? 1 : 0) : -1};
                            mbar_arrive_expect_tx(bar(B_QFULL + q_slot), static_cast<uint32_t>(rows) * kDqk * 2);
                        }
                    }
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (ok && lane < rows)
                        bulk_load(q_ring + static_cast<uint32_t>(q_slot) * S::kQBytes + lane * S::kQRow,
                                  p.q + b * p.q_stride + static_cast<int64_t>(p.first_head(unit) + lane) * kDqk, kDqk * 2, bar(B_QFULL + q_slot));
                    while (left > 0 && ok) {
                        const int32_t n = min(left, most), key = (tile << p.tile_shift) + lane * box_rows;
                        const int32_t rows = lane < n * boxes ? min(box_rows, len - key) : 0;
                        BoxDesc box{-1, 0, rows, 0u};
                        if (rows > 0) {
                            const int32_t col = p.by_page(key);
                            const int32_t page = __ldcg(p.page_table + static_cast<int64_t>(b) * p.max_pages + col);
                            if (page >= 0 && page < p.n_pages) {
                                box.page = page;
                                box.row = key - col * p.page_size;
                                box.loaded = static_cast<uint32_t>((rows + 7) & ~7);
                            }
                        }
                        for (int d = 1; d < boxes; d *= 2) box.loaded += __shfl_xor_sync(0xffffffffu, box.loaded, d);
                        hand_over({n, n_unit, left, p.first_kv_head(unit), static_cast<uint32_t>(end - left - lo) % S::kTurns}, box);
                        tile += n;
                        left -= n;
                    }
                    ++n_unit;
                    if (tile == n_tiles) {
                        tile = 0;
                        if (++unit == p.units && t < hi) {
                            unit = 0;
                            len = seq_len_of(p, ++b);
                            n_tiles = tiles_of(p, len);
                        }
                    }
                }
            };
            for (int32_t i = blockIdx.x; ok && i < pieces.levels * pieces.blocks;) {
                unsigned long long pop = 0;
                const bool more = pieces.levels > 1;
                if (more && lane == 0) pop = atomicAdd(counter, 1ull);          // (looked at when this piece has been planned)
                int32_t lo, hi;
                const int32_t piece = pieces.in_order(i, lo, hi);
                i = more ? -1 : INT32_MAX;
                if (lo < hi) plan(piece, lo, hi);
                if (more) {
                    if (lane == 0) i = pieces.blocks + popped(counter, pop, call_tag);
                    i = __shfl_sync(0xffffffffu, i, 0);
                }
            }
            if (ok) hand_over({-1, 0u, 0, 0, 0u}, {});          // no tile is left
        }
    } else if (warp == S::kConsumers + 1) {
        // ------------------------------------------------------------------ loads
        // The lanes issue the copies of a tile's boxes side by side: 121 us for 300 sequences of 1500 tokens, two K / V heads of 128 with 16
        // query heads each, on pages of 8 tokens (eight boxes per tile), where pages of 16 or 64 take 115; one thread alone took 180 us.
        // With one or two boxes per tile either way takes the same.
        const int32_t box_rows = p.box_rows, boxes = p.boxes;
        const uint32_t row_bytes = static_cast<uint32_t>(p.unit_kv_heads) * (kDqk + D_V) * 2;      // of a key
        const uint32_t k_box = static_cast<uint32_t>(box_rows * p.unit_kv_heads) * kDqk * 2, v_box = static_cast<uint32_t>(box_rows * p.unit_kv_heads) * D_V * 2;
        const int32_t of_tile = lane / boxes, j = lane - of_tile * boxes;       // this lane's box: the tile of the batch, its number in the tile
        uint32_t st = 0, turn = 0;                  // place in the ring
        for (uint32_t n_batch = 0;; ++n_batch) {
            const uint32_t at = n_batch % kBatches;
            if (!wait_together(B_BFULL + at, n_batch / kBatches)) break;
            const BatchDesc batch = s_batch[at];
            const BoxDesc d = s_box[at][lane];
            if (batch.tiles < 0) {
                if (wait_together(B_EMPTY + st, turn ^ 1u) && lane == 0) {
                    s_tile[st].unit = kEnd;
                    mbar_arrive(bar(B_FULL + st));
                }
                break;
            }
            mbar_arrive_warp(bar(B_BEMPTY + at));
            const uint64_t seen = d.page < 0 ? 0ull : (~0ull >> (64 - d.rows)) << (j * box_rows);
            const int32_t pieces = d.page < 0 || d.rows > box_rows - 8 ? 0 : (d.rows + 7) / 8;     // of eight rows; 0: the whole box
            uint32_t lo = static_cast<uint32_t>(seen), hi = static_cast<uint32_t>(seen >> 32);
            for (int x = 1; x < boxes; x *= 2) {
                lo |= __shfl_xor_sync(0xffffffffu, lo, x);
                hi |= __shfl_xor_sync(0xffffffffu, hi, x);
            }
            bool ok = true;
            for (int32_t i = 0; i < batch.tiles; ++i) {
                ok = wait_together(B_EMPTY + st, turn ^ 1u);
                if (!ok) break;
                const uint32_t full = bar(B_FULL + st);
                if (of_tile == i && j == 0) {
                    mbar_expect_tx(full, d.loaded * row_bytes);
                    s_tile[st].seen = static_cast<uint64_t>(hi) << 32 | lo;
                    s_tile[st].unit = batch.unit | (batch.left - i == 1 ? kLastOfUnit : 0u);
                    s_tile[st].set = (batch.set + i) % S::kTurns;
                }
                __syncwarp();
                if (of_tile == i && d.page >= 0) {
                    const uint32_t k_dst = ring + st * S::kStage + j * k_box, v_dst = ring + st * S::kStage + S::kKBytes + j * v_box;
                    if (pieces == 0) {
                        tma_load_5d(k_dst, &map_k, full, 0, 0, d.row, batch.head, d.page);
                        tma_load_5d(v_dst, &map_v, full, 0, 0, d.row, batch.head, d.page);
                    }
                }
                // a sequence's last rows, where they need not a whole box: eight at a time, head by head
                if (const uint32_t cut = __ballot_sync(0xffffffffu, of_tile == i && pieces > 0)) {
                    const int32_t from = __ffs(cut) - 1, n = __shfl_sync(0xffffffffu, pieces, from), box = from - i * boxes;
                    const int32_t row = __shfl_sync(0xffffffffu, d.row, from), page = __shfl_sync(0xffffffffu, d.page, from);
                    const int32_t h = lane / n, r = (lane - h * n) * 8;
                    if (h < p.unit_kv_heads) {
                        const uint32_t to = static_cast<uint32_t>((box * p.unit_kv_heads + h) * box_rows + r);
                        tma_load_5d(ring + st * S::kStage + to * kDqk * 2, &map_k8, full, 0, 0, row + r, batch.head + h, page);
                        tma_load_5d(ring + st * S::kStage + S::kKBytes + to * D_V * 2, &map_v8, full, 0, 0, row + r, batch.head + h, page);
                    }
                }
                __syncwarp();
                if (of_tile == i && j == 0) mbar_arrive(full);
                if (++st == S::kStages) { st = 0; ++turn; }
            }
            if (!ok) break;
        }
    } else {
        // ------------------------------------------------------------------ scores, softmax, O
        // Keys stand on the 16 rows of a product and query heads on its 8 columns: S^T = K Q^T, O^T = V^T P^T. A thread has the
        // heads 2 (lane mod 4) and the one after it, of every tile of eight, and of a product the rows lane / 4 and 8 more.
        const int slice = warp % kSlices, key_of_lane = lane >> 2;
        const uint32_t set = warp / kSlices;
        const int first_row = S::kHeadSets == 1 ? 0 : set * S::kWarpRows;      // of its K / V head's query heads
        const int kv_head = slice >> p.key_slices_log2, key_slice = slice & ((1 << p.key_slices_log2) - 1);     // of the unit, of its head
        const int q_row = kv_head * p.group + first_row;
        // Rows of the tile: boxes one after the other, in a box head by head. Of the slice's 16 keys, this lane addresses key r.
        auto tile_row = [&](int r) {
            const int key = key_slice * kSlice + r, box = key / p.box_rows;
            return static_cast<uint32_t>((box * p.unit_kv_heads + kv_head) * p.box_rows + key - box * p.box_rows);
        };
        const uint32_t k_unit0 = tile_row(lane & 15) * kUnitsK, k_part = (lane >> 4) & 1;
        const uint32_t v_unit0 = tile_row((lane & 7) + ((lane >> 4) & 1) * 8) * kUnitsV, v_part = (lane >> 3) & 1;
        uint32_t q[kDqk / 16][kNT][2];
        float o[D_V / 16][kNT][4];
        float m[kNT][2], l[kNT][2];
        if (warp == 0)                                  // sequences without a key
            for (int32_t b0 = blockIdx.x; b0 < p.n_seqs; b0 += 32 * gridDim.x) {
                const int32_t mine = b0 + lane * gridDim.x;
                uint32_t none = __ballot_sync(0xffffffffu, mine < p.n_seqs && seq_len_of(p, mine) == 0);
                for (; none; none &= none - 1) {
                    const int32_t b = b0 + (__ffs(none) - 1) * gridDim.x;
                    for (int32_t a = 0; a < p.h; ++a) {
                        reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(b) * p.h + a) * D_V)[lane] = make_uint2(0u, 0u);
                        if (lane == 0) p.lse[static_cast<int64_t>(a) * p.n_seqs + b] = neg_inf();
                    }
                }
            }
        const int key_slices = 1 << p.key_slices_log2;
        UnitDesc of{};
        uint32_t unit = kEnd;
        for (uint32_t n = 0;; ++n) {
            const int st = static_cast<int>(n % S::kStages);
            if (!wait_together(B_FULL + st, n / S::kStages)) break;
            const TileDesc d = s_tile[st];
            if (d.unit == kEnd) break;
            if ((d.unit & ~kLastOfUnit) != unit) {
                unit = d.unit & ~kLastOfUnit;
                const int q_slot = static_cast<int>(unit % S::kQSlots);
                if (!wait_together(B_QFULL + q_slot, unit / S::kQSlots)) break;
                of = s_unit[q_slot];
#pragma unroll
                for (int t = 0; t < kNT; ++t) {
                    const uint32_t q_at = q_ring + static_cast<uint32_t>(q_slot) * S::kQBytes +
                                          static_cast<uint32_t>(q_row + t * 8 + (lane & 7)) * S::kQRow + (lane >> 3) * 16;
#pragma unroll
                    for (int ks = 0; ks < kDqk / 16; ks += 2) {
                        uint32_t f[4];
                        ldmatrix_x4(q_at + ks * 32, f);
                        q[ks][t][0] = f[0]; q[ks][t][1] = f[1]; q[ks + 1][t][0] = f[2]; q[ks + 1][t][1] = f[3];
                    }
                }
                // Nothing has waited for the loads of the rows yet. Without the fence they can still be on their way when an asynchronous
                // copy of a later unit's rows lands in the slot, as happened with short units in one of some ten calls.
                fence_proxy_async_smem();
                mbar_arrive_warp(bar(B_QEMPTY + q_slot));
#pragma unroll
                for (int i = 0; i < D_V / 16 * kNT * 4; ++i) o[i / (4 * kNT)][i / 4 % kNT][i % 4] = 0.f;
#pragma unroll
                for (int t = 0; t < kNT; ++t) {
                    m[t][0] = m[t][1] = neg_inf();
                    l[t][0] = l[t][1] = 0.f;
                }
            }
            const uint32_t seen = static_cast<uint32_t>(d.seen >> (key_slice * kSlice)) & 0xffffu;
            if (seen && (S::kTurns == 1 || d.set == set)) {
                const uint32_t stage = ring + static_cast<uint32_t>(st) * S::kStage;
                float s[2][kNT][4];                     // even and odd steps: two chains of products per tile of heads
#pragma unroll
                for (int i = 0; i < 8 * kNT; ++i) s[i / (4 * kNT)][i / 4 % kNT][i % 4] = 0.f;
#pragma unroll
                for (int ks = 0; ks < kDqk / 16; ++ks) {
                    uint32_t kf[4];
                    ldmatrix_x4(swizzled(stage, k_unit0 + ks / 4, ks % 4 * 2 + k_part), kf);
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
                    float top[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])};
                    if (__any_sync(0xffffffffu, top[0] > m[t][0] + kRaise || top[1] > m[t][1] + kRaise)) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
#pragma unroll
                            for (int g = 4; g < 32; g *= 2) top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], g));
                            if (top[c] > m[t][c] + kRaise) {
                                const float f = ex2_approx(m[t][c] - top[c]);
                                m[t][c] = top[c];
                                l[t][c] *= f;
#pragma unroll
                                for (int j = 0; j < D_V / 16; ++j) { o[j][t][c] *= f; o[j][t][c + 2] *= f; }
                            }
                        }
                    }
                    const float ref[2] = {m[t][0] == neg_inf() ? 0.f : m[t][0], m[t][1] == neg_inf() ? 0.f : m[t][1]};
                    float pr[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) pr[e] = ex2_approx(x[e] - ref[e & 1]);
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
                // rows that do not count hold anything: 0 * NaN must not reach the sums
                const uint32_t v_bits = seen >> (2 * (lane & 3));
                const uint32_t keep0 = (v_bits & 1u ? 0xffffu : 0u) | (v_bits & 2u ? 0xffff0000u : 0u);
                const uint32_t keep1 = (v_bits & 0x100u ? 0xffffu : 0u) | (v_bits & 0x200u ? 0xffff0000u : 0u);
#pragma unroll
                for (int j = 0; j < D_V / 16; ++j) {
                    uint32_t vf[4];
                    ldmatrix_x4_trans(swizzled(stage + S::kKBytes, v_unit0 + j / 4, j % 4 * 2 + v_part), vf);
                    if (seen != 0xffffu) { vf[0] &= keep0; vf[1] &= keep0; vf[2] &= keep1; vf[3] &= keep1; }
#pragma unroll
                    for (int t = 0; t < kNT; ++t) {
                        mma_bf16(o[j][t], vf, ph[t][0], ph[t][1]);
                        mma_bf16(o[j][t], vf, pl[t][0], pl[t][1]);
                    }
                }
            }
            mbar_arrive_warp(bar(B_EMPTY + st));
            if (!(d.unit & kLastOfUnit)) continue;
            // ---------------------------------------------------------------- what the warp has of its unit, into shared memory
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int g = 4; g < 32; g *= 2) l[t][c] += __shfl_xor_sync(0xffffffffu, l[t][c], g);
            if (!wait_together(B_JEMPTY, unit ^ 1u)) break;
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int row = t * 8 + 2 * (lane & 3) + c;
                    if (first_row + row >= p.group) continue;       // padding
                    if (lane < 4) s_ml[warp][row] = make_float2(m[t][c], l[t][c]);
                    float* dst = join + (warp * S::kWarpRows + row) * S::kJoinStride + key_of_lane;
#pragma unroll
                    for (int j = 0; j < D_V / 16; ++j) {
                        dst[16 * j] = o[j][t][c];
                        dst[16 * j + 8] = o[j][t][c + 2];
                    }
                }
            mbar_arrive_warp(bar(B_JFULL));
            if (!wait_together(B_JFULL, unit)) break;
            // ---------------------------------------------------------------- the warps that share a head, joined; a row per warp
            const int32_t head0 = p.first_head(of.unit), rows = p.rows_of(of.unit);
            for (int32_t e = warp; e < rows; e += S::kConsumers) {
                const int32_t head = e / p.group, in_group = e - head * p.group, r = in_group % S::kWarpRows;
                const int warp0 = (S::kHeadSets == 1 ? 0 : in_group / S::kWarpRows * kSlices) + (head << p.key_slices_log2);
                float2 ml[S::kTurns * kSlices];
                float top = neg_inf(), sum = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < S::kTurns * kSlices; ++w) {
                    ml[w] = w % kSlices < key_slices ? s_ml[warp0 + w][r] : make_float2(neg_inf(), 0.f);
                    top = fmaxf(top, ml[w].x);
                }
                const float ref = top == neg_inf() ? 0.f : top;
#pragma unroll
                for (int w = 0; w < S::kTurns * kSlices; ++w) {
                    if (w % kSlices >= key_slices) continue;
                    const float f = ex2_approx(ml[w].x - ref);
                    const float4 x = *reinterpret_cast<const float4*>(join + ((warp0 + w) * S::kWarpRows + r) * S::kJoinStride + 4 * lane);
                    sum += f * ml[w].y;
                    acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
                }
                const float inv = top == neg_inf() ? 0.f : 1.f / sum, lse2 = top == neg_inf() ? top : top + log2f(sum);
                acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
                if (of.slot >= 0) {
                    const int64_t row = static_cast<int64_t>(of.slot) * p.unit_rows + e;
                    reinterpret_cast<float4*>(p.part_o + row * D_V)[lane] = acc;
                    if (lane == 0) p.part_lse2[row] = lse2;
                } else {
                    reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(of.seq) * p.h + head0 + e) * D_V)[lane] =
                        make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
                    if (lane == 0) p.lse[static_cast<int64_t>(head0 + e) * p.n_seqs + of.seq] = lse2 * 0.6931471805599453f;
                }
            }
            mbar_arrive_warp(bar(B_JEMPTY));
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

struct DecodeJoin {
    int32_t item;                           // sequence * units of a sequence + unit of the sequence
    int32_t piece, parts;                   // the first piece with tiles of it, and how many there are (0: nothing to join)
};

// (O, LSE) of the parts of cut units, joined in the order of the keys. Part i of a unit is the beginning of piece c0 + i, but the
// first the end of its piece. A thread block per piece: those whose piece goes on with a unit share its rows. A row of up to
// eight parts has a warp, of up to 32 a block; of more, every 32 have a block that puts their join in the place of the first, and
// the block that comes last joins those. The blocks are small enough to stand beside those of the kernel before, and find out
// what they have to do while that one still runs.
__global__ void __launch_bounds__(32 * kJoinWarps, 9)
hydra_decode_join_kernel(const DecodeParams p)
{
    __shared__ float4 s_o[kJoinWarps][32];
    __shared__ float s_lse2[kJoinWarps];
    __shared__ int32_t s_last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ DecodeJoin s_join;
    if (warp == 0) {                                    // the unit that this block's piece went on with
        const Lengths lengths(p, lane);
        const Pieces pieces(p, lengths.total);
        DecodeJoin join{0, 0, 0};
        int32_t lo = 0, hi = 0;
        if (static_cast<int32_t>(blockIdx.x) < pieces.count()) pieces.range(blockIdx.x, lo, hi);
        if (lo < hi) {
            int32_t b, before, len;
            lengths.find(p, lane, p.by_units(lo), b, len, before);
            const int32_t n_tiles = tiles_of(p, len), in_seq = lo - before * p.units, unit = in_seq / n_tiles, tile = in_seq - unit * n_tiles;
            if (tile > 0) {
                join.item = b * p.units + unit;
                join.piece = pieces.piece_of(lo - tile);
                join.parts = pieces.piece_of(lo - tile + n_tiles - 1) - join.piece + 1;
            }
        }
        if (lane == 0) s_join = join;
    }
    __syncthreads();
    const DecodeJoin join = s_join;
    const int32_t b = join.item / p.units, unit = join.item - b * p.units;
    wait_for_previous_launch();
    if (join.parts == 0) return;
    const int32_t rows = p.rows_of(unit), parts = join.parts, chunks = (parts + kJoinChunk - 1) / kJoinChunk;
    const bool by_warp = parts <= kJoinParts;

    // the join of parts first, first + step, ... (count of them, at most kJoinParts)
    auto join_parts = [&](int32_t r, int32_t first, int32_t step, int32_t count) -> Joined {
        float part[kJoinParts];
        float4 x[kJoinParts];
#pragma unroll
        for (int j = 0; j < kJoinParts; ++j) {
            const int32_t i = first + j * step, at = (2 * (join.piece + i) + (i == 0 ? 1 : 0)) * p.unit_rows + r;
            part[j] = j < count ? __ldcg(p.part_lse2 + at) : neg_inf();
            x[j] = j < count ? __ldcg(reinterpret_cast<const float4*>(p.part_o + static_cast<int64_t>(at) * D_V) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return join_of(part, x);
    };
    auto write = [&](int32_t r, const Joined& v) {
        const int32_t a = p.first_head(unit) + r;
        reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(b) * p.h + a) * D_V)[lane] =
            make_uint2(pack_bf16x2(v.o.x, v.o.y), pack_bf16x2(v.o.z, v.o.w));
        if (lane == 0) p.lse[static_cast<int64_t>(a) * p.n_seqs + b] = v.lse2 * 0.6931471805599453f;
    };
    // warp w's share of a row's parts first + step * [0, count)
    auto join_block = [&](int32_t r, int32_t first, int32_t step, int32_t count) -> Joined {
        const int32_t mine = count > warp ? (count - warp + kJoinWarps - 1) / kJoinWarps : 0;
        __syncthreads();                                // (what the block joined before has been read)
        const Joined v = join_parts(r, first + warp * step, step * kJoinWarps, mine);
        s_o[warp][lane] = v.o;
        if (lane == 0) s_lse2[warp] = v.lse2;
        __syncthreads();
        float part[kJoinWarps];
        float4 x[kJoinWarps];
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) { part[w] = s_lse2[w]; x[w] = s_o[w][lane]; }
        return join_of(part, x);
    };

    const int32_t helpers = parts - 1, tasks = by_warp ? (rows + kJoinWarps - 1) / kJoinWarps : rows * chunks;
    for (int32_t task = static_cast<int32_t>(blockIdx.x) - join.piece - 1; task < tasks; task += helpers) {
        if (by_warp) {
            const int32_t r = task * kJoinWarps + warp;
            if (r < rows) write(r, join_parts(r, 0, 1, parts));
            continue;
        }
        const int32_t r = task / chunks, first = (task - r * chunks) * kJoinChunk;
        Joined v = join_block(r, first, 1, min(kJoinChunk, parts - first));
        if (chunks > 1) {
            if (warp == 0) {
                const int32_t at = (2 * (join.piece + first) + (first == 0 ? 1 : 0)) * p.unit_rows + r;
                reinterpret_cast<float4*>(p.part_o + static_cast<int64_t>(at) * D_V)[lane] = v.o;
                if (lane == 0) p.part_lse2[at] = v.lse2;
                __threadfence();
                __syncwarp();
                if (lane == 0) s_last = atomicAdd(p.arrived + join.piece + 1 + r, 1) == chunks - 1;
            }
            __syncthreads();
            if (!s_last) continue;
            __threadfence();
            v = join_block(r, 0, kJoinChunk, chunks);   // (at most 24 of them)
        }
        if (warp == 0) write(r, v);
    }
}

using LaunchFn = cudaError_t (*)(const CUtensorMap (&)[4], const DecodeParams&, uint64_t, cudaStream_t);
template <class S>
cudaError_t launch_one(const CUtensorMap (&maps)[4], const DecodeParams& p, uint64_t call_tag, cudaStream_t stream)
{
    static OncePerDevice configured;
    const auto kernel = hydra_decode_kernel<S>;
    if (cudaError_t e = allow_dynamic_smem(kernel, S::kSmem, configured)) return e;
    return launch_overlapped(kernel, p.blocks, S::kThreads, S::kSmem, stream, maps[0], maps[1], maps[2], maps[3], p, call_tag);
}
template <int kDqk>
LaunchFn form_for(int32_t group)
{
    return group <= 8 ? launch_one<Shape<kDqk, 1, 1>> : group <= 16 ? launch_one<Shape<kDqk, 1, 2>> : launch_one<Shape<kDqk, 2, 2>>;
}

}  // namespace

cudaError_t launch_decode(const CUtensorMap (&maps)[4], const DecodeParams& p, int32_t d_qk, uint64_t call_tag, cudaStream_t stream)
{
    return (d_qk == 192 ? form_for<192>(p.group) : form_for<128>(p.group))(maps, p, call_tag, stream);
}

cudaError_t launch_decode_join(const DecodeParams& p, cudaStream_t stream)
{
    return launch_overlapped(hydra_decode_join_kernel, DECODE_LEVELS * p.blocks, 32 * kJoinWarps, 0, stream, p);
}

}  // namespace hydra

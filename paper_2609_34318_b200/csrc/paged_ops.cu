// Rotary positions with several axes, and the way of new keys and values into a paged cache.
//
// All forms move rows of bf16 (one row per token and head) once, turning the rotary columns on the way; they are bound by
// memory, and with a few tokens (a step of generation) by the chain of loads in front of the first row. Pair i of the rotary
// columns belongs to one axis and turns by that axis's position times theta^(-2i / rope_dim); the angle is formed and reduced
// in double precision as in hydra_mla_rope, whose results those of one axis equal bit for bit. Where a token's rows go in the
// cache is found on the device (its sequence by a search of cu_new with the 32 lanes of a warp, its place from the sequence's
// length, its page from the page table), so that a captured call follows the lengths. Rows without a place are not written.
//
// Every warp works by itself on a few tokens (or some heads of one): it asks for its first rows, finds the tokens' places, puts
// cosines and sines of their angles into shared memory, and only then needs the rows. Blocks that did this together, with
// barriers between the steps, had two of them on an SM at a time and no more than 4 KB to move between two barriers.
#include <algorithm>
#include <cmath>

#include "elementwise.cuh"

namespace hydra {
namespace {

enum : int { PLACE_ROPE = 0, PLACE_ROPE_IN_PLACE, PLACE_KV, PLACE_MLA };
constexpr int kPlaceWarps = 8;              // of a block
constexpr int kMaxTokens = 16;              // that a warp takes at once
constexpr int kMaxAngles = 512;             // tokens times rotary pairs
constexpr int kMaxPairs = 128;
// Blocks per SM. 32K prompt tokens of 16 MLA heads take 112 us (5.4 TB/s), with five blocks (48 registers) 130, with six 137; a
// thread moves a vector at a time, more of them in flight gained nothing. A step of 230 tokens 4.8 us; 65536 patches of a video, two
// heads of 128, 35 us, of which 8 are their angles and the rotation's products; their 16 query heads rotated 90 to 93 us (5.8 to 6.0
// TB/s); as many tokens of text, whose angles all have to be formed, into two heads of 128, 43 us.
constexpr int kPlaceBlocks = 4;

// Strides, offsets and columns in vectors of 2 kWords elements.
struct PlaceParams {
    const uint16_t *k, *v, *pe;             // pe: the rotary key of PLACE_MLA (whose k has rows of position-free part and value)
    uint16_t *y, *y_v;                      // rows, or the pages of K and V
    int64_t k_stride, v_stride, pe_stride;  // between tokens (pe: in elements)
    int64_t y_stride;                       // PLACE_ROPE: between tokens
    int64_t y_head, y_v_head;               // between the heads of a token at its destination
    int32_t k_vecs, y_vecs, v_vecs;         // of a row of k, of y, of y_v
    int32_t rot0, rot_vecs;                 // rotary vectors [rot0, rot0 + rot_vecs) of a row of y
    const int32_t* positions;               // [axes, n_tokens], or null: the place in the sequence
    int64_t n_tokens;
    int32_t pairs, inverse, axes;
    int32_t axis_first[HYDRA_MAX_AXES];     // first pair of every axis (the number of pairs from the last axis on)
    double log_theta;
    // the cache
    const int32_t *page_table, *seq_lens, *cu_new;
    int32_t n_seqs, max_pages, page_size, n_pages, heads;
    // a warp's share: `tokens` tokens, or share_heads heads (the last of the splits: what is left) of one; vectors of a token's share in
    // k, in v, and its rotary ones
    int32_t tokens, splits, share_heads;
    Div by_k_token, by_k_row, by_v_token, by_v_row, by_rot_token, by_rot_row;
};

// The last sequence that begins at or before token t, by one warp: every round tries 32 places of what is left.
__device__ __forceinline__ int32_t sequence_of(const int32_t* cu, int32_t n_seqs, int64_t t, int lane)
{
    int32_t lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const int found = __popc(__ballot_sync(0xffffffffu, at < hi && cu[at] <= t));
        lo += max(found - 1, 0) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

template <int kWords, int kMode>
__global__ void __launch_bounds__(32 * kPlaceWarps, kPlaceBlocks)
hydra_place_rows_kernel(const PlaceParams p)
{
    constexpr bool kPaged = kMode == PLACE_KV || kMode == PLACE_MLA;
    __shared__ double s_freq[kMaxPairs];
    __shared__ __align__(32) float s_cos_of[kPlaceWarps][kMaxAngles], s_sin_of[kPlaceWarps][kMode == PLACE_MLA ? 1 : kMaxAngles];
    __shared__ int64_t s_k_to[kPlaceWarps][kMaxTokens], s_v_to[kPlaceWarps][kMaxTokens];   // a token's rows at its destination; -1: nowhere
    __shared__ int32_t s_position[kPlaceWarps][HYDRA_MAX_AXES * kMaxTokens];    // [axis][token]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* const s_cos = s_cos_of[warp];                // (PLACE_MLA: the turned key itself, a pair in each)
    float* const s_sin = s_sin_of[warp];
    if (static_cast<int>(threadIdx.x) < p.pairs) s_freq[threadIdx.x] = exp(-p.log_theta * static_cast<int>(threadIdx.x) / p.pairs);
    __syncthreads();
    wait_for_previous_launch();

    const int64_t n_shares = (p.n_tokens + p.tokens - 1) / p.tokens * p.splits, n_warps = static_cast<int64_t>(gridDim.x) * kPlaceWarps;
    for (int64_t share = static_cast<int64_t>(blockIdx.x) * kPlaceWarps + warp; share < n_shares; share += n_warps) {
        const int64_t t0 = share / p.splits * p.tokens;
        const int32_t head0 = static_cast<int32_t>(share % p.splits) * p.share_heads;
        const uint32_t n_tok = static_cast<uint32_t>(min(static_cast<int64_t>(p.tokens), p.n_tokens - t0));
        const uint32_t n_heads = static_cast<uint32_t>(min(p.share_heads, p.heads - head0)), n_k = n_tok * n_heads * p.k_vecs;
        const int64_t k_from = t0 * p.k_stride + static_cast<int64_t>(head0) * p.k_vecs;
        // rows of k, in the order in which they lie there
        auto load_k = [&](uint32_t e) {
            const uint32_t tok = p.by_k_token(e);
            const int64_t at = k_from + tok * p.k_stride + (e - tok * p.by_k_token.d);
            return kMode == PLACE_ROPE_IN_PLACE ? ld_words_coherent<kWords>(p.k, at) : ld_words<kWords>(p.k, at);
        };
        auto rotary = [&](uint32_t e) {                 // in place, only the rotary vectors move
            if (kMode != PLACE_ROPE_IN_PLACE) return true;
            const uint32_t c = e - p.by_k_row(e) * p.k_vecs;
            return c >= static_cast<uint32_t>(p.rot0) && c < static_cast<uint32_t>(p.rot0 + p.rot_vecs);
        };
        const bool has_first = static_cast<uint32_t>(lane) < n_k && rotary(lane);
        Words<kWords> first;
        if (has_first) first = load_k(lane);
        int32_t position[HYDRA_MAX_AXES * kMaxTokens / 32];
        const uint32_t n_positions = p.positions ? n_tok * p.axes : 0;
#pragma unroll
        for (int j = 0; j < HYDRA_MAX_AXES * kMaxTokens / 32; ++j)
            if (const uint32_t i = lane + 32 * j; i < n_positions) {
                const uint32_t axis = i / n_tok;
                position[j] = p.positions[axis * p.n_tokens + t0 + (i - axis * n_tok)];
            }
        __syncwarp();                                   // the tables of the tokens before are no longer read
#pragma unroll
        for (int j = 0; j < HYDRA_MAX_AXES * kMaxTokens / 32; ++j)
            if (const uint32_t i = lane + 32 * j; i < n_positions) s_position[warp][i] = position[j];
        if (kPaged) {
            int32_t b = 0;
            int64_t place = -1;
            const int64_t t = t0 + lane;
            if (p.cu_new) {
                b = sequence_of(p.cu_new, p.n_seqs, t0, lane);
                if (lane < static_cast<int>(n_tok)) {
                    // A lane's token is of the same sequence as the first or of one close behind, but for rows that append
                    // nothing: any number of those may lie between, and after a few steps the rest is searched by halves.
                    int32_t end = p.cu_new[b + 1];
                    for (int step = 0; t >= end && b + 1 < p.n_seqs; ++step) {
                        if (step == kMaxTokens) {
                            for (int32_t hi = p.n_seqs; hi - b > 1;) {
                                const int32_t mid = b + (hi - b) / 2;
                                (p.cu_new[mid] <= t ? b : hi) = mid;
                            }
                            end = p.cu_new[b + 1];
                            break;
                        }
                        end = p.cu_new[++b + 1];
                    }
                    if (t >= p.cu_new[b] && t < end) place = static_cast<int64_t>(p.seq_lens[b]) - (end - t);
                }
            } else if (lane < static_cast<int>(n_tok) && t < p.n_seqs) {
                b = static_cast<int32_t>(t);
                place = static_cast<int64_t>(p.seq_lens[b]) - 1;
            }
            if (lane < static_cast<int>(n_tok)) {
                int64_t to_k = -1, to_v = -1;
                if (place >= 0 && place < static_cast<int64_t>(p.max_pages) * p.page_size) {
                    const int32_t col = static_cast<int32_t>(place / p.page_size), row = static_cast<int32_t>(place % p.page_size);
                    const int32_t page = p.page_table[static_cast<int64_t>(b) * p.max_pages + col];
                    if (page >= 0 && page < p.n_pages) {
                        to_k = (static_cast<int64_t>(page) * p.heads + head0) * p.y_head + static_cast<int64_t>(row) * p.y_vecs;
                        to_v = (static_cast<int64_t>(page) * p.heads + head0) * p.y_v_head + static_cast<int64_t>(row) * p.v_vecs;
                    }
                }
                s_k_to[warp][lane] = to_k;
                s_v_to[warp][lane] = to_v;
                if (!p.positions) s_position[warp][lane] = static_cast<int32_t>(place);
            }
        }
        __syncwarp();
        // A lane takes a pair of every token (with fewer pairs than lanes, of every n-th); neighbouring patches of an image or a video
        // share most of their positions, and an angle that the token before had is not formed again.
        const uint32_t abreast = p.pairs >= 32 ? 1 : p.pairs ? 32 / p.pairs : 0;
        for (uint32_t pair = p.pairs >= 32 ? lane : p.pairs ? lane % p.pairs : 0; pair < static_cast<uint32_t>(p.pairs); pair += 32) {
            int axis = 0;
#pragma unroll
            for (int a = 1; a < HYDRA_MAX_AXES; ++a) axis += static_cast<int32_t>(pair) >= p.axis_first[a] ? 1 : 0;
            const double freq = s_freq[pair];
            const int32_t* const its = s_position[warp] + axis * n_tok;
            int32_t last = 0;
            float cs = 1.f, sn = 0.f;                   // of position 0
            uint32_t tok = p.pairs >= 32 ? 0 : lane / p.pairs;
            if (tok >= abreast) tok = n_tok;
            for (; tok < n_tok; tok += abreast) {
                const int32_t at = its[tok];
                if (at != last) rope_angle(last = at, freq, cs, sn);
                const uint32_t i = tok * p.pairs + pair;
                if (kMode == PLACE_MLA) {
                    const float2 w = bf2_to_f2(*reinterpret_cast<const uint32_t*>(p.pe + (t0 + tok) * p.pe_stride + 2 * pair));
                    s_cos[i] = __uint_as_float(f2_to_bf2(w.x * cs - w.y * sn, w.x * sn + w.y * cs));
                } else {
                    s_cos[i] = cs;
                    s_sin[i] = p.inverse ? -sn : sn;
                }
            }
        }
        __syncwarp();
        // where vector c of a head's row of y goes
        auto to = [&](uint32_t tok, uint32_t head, uint32_t c) -> int64_t {
            if (!kPaged) return (t0 + tok) * p.y_stride + static_cast<int64_t>(head0 + head) * p.y_head + c;
            const int64_t base = s_k_to[warp][tok];
            return base < 0 ? -1 : base + static_cast<int64_t>(head) * p.y_head + c;
        };
        auto to_v = [&](uint32_t tok, uint32_t head, uint32_t c) -> int64_t {
            const int64_t base = s_v_to[warp][tok];
            return base < 0 ? -1 : base + static_cast<int64_t>(head) * p.y_v_head + c;
        };
        auto store_k = [&](uint32_t e, const Words<kWords>& w) {
            const uint32_t tok = p.by_k_token(e), in = e - tok * p.by_k_token.d, head = p.by_k_row(in), c = in - head * p.k_vecs;
            if (kMode == PLACE_MLA && c >= static_cast<uint32_t>(p.rot0)) {     // the value's part of the row
                if (const int64_t at = to_v(tok, head, c - p.rot0); at >= 0) st_words<kWords>(p.y_v, at, w);
                return;
            }
            const int64_t at = to(tok, head, c);
            if (kPaged && at < 0) return;
            if (kMode != PLACE_MLA && c >= static_cast<uint32_t>(p.rot0) && c < static_cast<uint32_t>(p.rot0 + p.rot_vecs)) {
                const uint32_t i = tok * p.pairs + (c - p.rot0) * kWords;
                st_words<kWords>(p.y, at, rotate_vec<kWords>(w, s_cos + i, s_sin + i));
            } else if (kMode != PLACE_ROPE_IN_PLACE) {
                st_words<kWords>(p.y, at, w);
            }
        };
        if (has_first) store_k(lane, first);
        for (uint32_t e = lane + 32; e < n_k; e += 32)
            if (rotary(e)) store_k(e, load_k(e));
        if (kMode == PLACE_KV) {                        // rows of v
            const uint32_t n_v = n_tok * n_heads * p.v_vecs;
            for (uint32_t e = lane; e < n_v; e += 32) {
                const uint32_t tok = p.by_v_token(e), in = e - tok * p.by_v_token.d, head = p.by_v_row(in);
                const auto w = ld_words<kWords>(p.v, (t0 + tok) * p.v_stride + static_cast<int64_t>(head0) * p.v_vecs + in);
                if (const int64_t at = to_v(tok, head, in - head * p.v_vecs); at >= 0) st_words<kWords>(p.y_v, at, w);
            }
        }
        if (kMode == PLACE_MLA) {                       // the turned key, for every head
            const uint32_t n_rot = n_tok * n_heads * p.rot_vecs;
            for (uint32_t e = lane; e < n_rot; e += 32) {
                const uint32_t tok = p.by_rot_token(e), in = e - tok * p.by_rot_token.d, head = p.by_rot_row(in), c = in - head * p.rot_vecs;
                const float* src = s_cos + tok * p.pairs + c * kWords;
                Words<kWords> w;
#pragma unroll
                for (int j = 0; j < kWords; ++j) w.w[j] = __float_as_uint(src[j]);
                if (const int64_t at = to(tok, head, p.rot0 + c); at >= 0) st_words<kWords>(p.y, at, w);
            }
        }
    }
    overlap_next_launch();
}

// What all forms have in common. k_elems: of a row of k; row_elems: of a row of y.
PlaceParams place_params(int64_t n_tokens, int32_t n_heads, const hydra_rope_t* rope, const int32_t* positions, int words,
                         int32_t k_elems, int32_t row_elems, int32_t v_elems, int32_t rot0_elems)
{
    const int32_t elems = 2 * words, rot_elems = rope ? rope->dim : 0, pairs = rot_elems / 2;
    const int32_t per_head = (row_elems + v_elems) / elems;
    // Some eight vectors per thread of a warp: several tokens where they are short, part of the heads where they are long. But
    // with few tokens the work is spread over the warps of all SMs first, down to two vectors per thread. (Half as many: 115 us for
    // the prompts above and 92 for the video's queries; four times as many: 130 and 96.)
    constexpr int64_t kWarps = 148 * kPlaceWarps * 2, kVectors = 32 * 8;
    int64_t tokens = std::min<int64_t>({kVectors / (int64_t{n_heads} * per_head), n_tokens / kWarps, kMaxTokens});
    if (pairs) tokens = std::min<int64_t>(tokens, kMaxAngles / pairs);
    tokens = std::max<int64_t>(tokens, 1);
    const int64_t steps = (n_tokens + tokens - 1) / tokens;
    int32_t splits = 1;
    auto share_heads = [&] { return (n_heads + splits - 1) / splits; };
    auto vectors = [&] { return tokens * share_heads() * per_head; };
    while (tokens == 1 && 2 * splits <= n_heads && (vectors() > 2 * kVectors || (steps * splits < kWarps && vectors() > 64))) splits *= 2;
    const int32_t share = share_heads(), k = k_elems / elems, v = v_elems / elems, rot = rot_elems / elems;
    splits = (n_heads + share - 1) / share;
    PlaceParams p{nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, 0, 0, 0, 0, k, row_elems / elems, v, rot0_elems / elems, rot,
                  positions, n_tokens, pairs, 0, rope ? rope->n_axes : 0, {}, 0.0, nullptr, nullptr, nullptr, 0, 0, 1, 0, n_heads,
                  static_cast<int32_t>(tokens), splits, share, Div(share * k), Div(k), Div(share * v), Div(v), Div(share * rot), Div(rot)};
    if (rope) {
        p.log_theta = std::log(static_cast<double>(rope->theta));
        for (int a = 0, first = 0; a < HYDRA_MAX_AXES; ++a) {
            p.axis_first[a] = a < rope->n_axes ? first : INT32_MAX;
            if (a < rope->n_axes) first += rope->axis_pairs[a];
        }
    }
    return p;
}

template <int kMode>
cudaError_t launch_place(const PlaceParams& p, int words, cudaStream_t stream)
{
    const int64_t shares = (p.n_tokens + p.tokens - 1) / p.tokens * p.splits;
    const int grid = static_cast<int>(std::min<int64_t>((shares + kPlaceWarps - 1) / kPlaceWarps, 148 * kPlaceBlocks));
    return launch_overlapped(words == 8 ? hydra_place_rows_kernel<8, kMode> : hydra_place_rows_kernel<4, kMode>, grid, 32 * kPlaceWarps, 0,
                             stream, p);
}

// 8 where the strides too are multiples of 16 elements
int words_of(std::initializer_list<int32_t> dims, std::initializer_list<int64_t> strides, std::initializer_list<const void*> ptrs)
{
    int64_t bits = 0;
    for (int64_t s : strides) bits |= s;
    return bits % 16 == 0 && words_for(dims, ptrs) == 8 ? 8 : 4;
}

}  // namespace

cudaError_t launch_rope_axes(const void* x, int64_t x_stride, const int32_t* positions, int64_t n_tokens, int32_t n_heads,
                             int32_t head_dim, const hydra_rope_t& rope, int inverse, void* y, int64_t y_stride, cudaStream_t stream)
{
    if (n_tokens == 0) return cudaSuccess;
    const int words = words_of({head_dim, rope.offset, rope.dim}, {x_stride, y_stride}, {x, y}), elems = 2 * words;
    PlaceParams p = place_params(n_tokens, n_heads, &rope, positions, words, head_dim, head_dim, 0, rope.offset);
    p.k = static_cast<const uint16_t*>(x);
    p.y = static_cast<uint16_t*>(y);
    p.k_stride = x_stride / elems;
    p.y_stride = y_stride / elems;
    p.y_head = head_dim / elems;
    p.inverse = inverse;
    return x == y ? launch_place<PLACE_ROPE_IN_PLACE>(p, words, stream) : launch_place<PLACE_ROPE>(p, words, stream);
}

cudaError_t launch_kv_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* pe, int64_t pe_stride,
                             const int32_t* positions, const int32_t* cu_new, int64_t n_tokens, const hydra_rope_t* rope,
                             const hydra_paged_cache_t& c, cudaStream_t stream)
{
    if (n_tokens == 0 || c.n_seqs == 0) return cudaSuccess;
    const int32_t dim = rope ? rope->dim : 0, offset = rope ? rope->offset : c.d_qk;
    const int words = words_of({c.d_qk, c.d_v, offset, dim}, {k_stride, v_stride}, {k, v, c.k, c.v}), elems = 2 * words;
    PlaceParams p = place_params(n_tokens, c.n_kv_heads, rope, positions, words, pe ? offset + c.d_v : c.d_qk, c.d_qk, c.d_v, offset);
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    p.pe = static_cast<const uint16_t*>(pe);
    p.y = static_cast<uint16_t*>(c.k);
    p.y_v = static_cast<uint16_t*>(c.v);
    p.k_stride = k_stride / elems;
    p.v_stride = v_stride / elems;
    p.pe_stride = pe_stride;
    p.y_head = static_cast<int64_t>(c.page_size) * (c.d_qk / elems);
    p.y_v_head = static_cast<int64_t>(c.page_size) * (c.d_v / elems);
    p.page_table = c.page_table;
    p.seq_lens = c.seq_lens;
    p.cu_new = cu_new;
    p.n_seqs = c.n_seqs;
    p.max_pages = c.max_pages;
    p.page_size = c.page_size;
    p.n_pages = c.n_pages;
    return pe ? launch_place<PLACE_MLA>(p, words, stream) : launch_place<PLACE_KV>(p, words, stream);
}

}  // namespace hydra

// Rotary positions with several axes, and the way of new keys and values into a paged cache.
//
// All three forms move rows of bf16 (one row per token and head) once, turning the rotary columns on the way; they are bound by
// memory, and with a few tokens (a step of generation) by the chain of loads in front of the first row. Pair i of the rotary
// columns belongs to one axis and turns by that axis's position times theta^(-2i / rope_dim); the angle is formed and reduced
// in double precision as in hydra_mla_rope, whose results those of one axis equal bit for bit. Where a token's rows go in the
// cache is found on the device (its sequence by a search of cu_new with the 32 lanes of a warp, its place from the sequence's
// length, its page from the page table), so that a captured call follows the lengths. Rows without a place are not written.
#include <algorithm>
#include <cmath>

#include "elementwise.cuh"

namespace hydra {
namespace {

enum : int { PLACE_ROPE = 0, PLACE_ROPE_IN_PLACE, PLACE_KV, PLACE_MLA };
constexpr int kMaxItem = 64;                // tokens that a block takes at once

// Strides, offsets and columns in vectors of 2 kWords elements.
struct PlaceParams {
    const uint16_t *k, *v, *pe;             // pe: the rotary key of PLACE_MLA (the position-free part and v lie in k's rows)
    uint16_t *y, *y_v;                      // rows, or the pages of K and V
    int64_t k_stride, v_stride, pe_stride;  // between tokens (pe: in elements)
    int64_t y_stride;                       // PLACE_ROPE: between tokens
    int64_t y_head, y_v_head;               // between the heads of a token at its destination
    int32_t k_head;                         // between the heads of a token in k
    int32_t k_vecs, v_vecs, rot0, rot_vecs; // of a row of y, of y_v; rotary vectors [rot0, rot0 + rot_vecs) of a row of y
    const int32_t* positions;               // [axes, n_tokens], or null: the place in the sequence
    int64_t n_tokens;
    int32_t pairs, inverse;
    int32_t axis_first[HYDRA_MAX_AXES];     // first pair of every axis (the number of pairs from the last axis on)
    double log_theta;
    // the cache
    const int32_t *page_table, *seq_lens, *cu_new;
    int32_t n_seqs, max_pages, page_size, n_pages;
    // a block's share: per_item tokens, heads_per_item heads
    int32_t per_item, splits;
    Div by_heads, by_rot, by_copy, by_v;
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

// n vectors of a block: load(e, at) gives vector e and where it goes, store(e, at, v) puts it there. (Two in flight: what
// a thread has in registers is what the SM's other blocks lack.)
template <int kWords, class Load, class Store>
__device__ __forceinline__ void move_rows(uint32_t n, Load load, Store store)
{
    constexpr int kUnroll = 2;
    for (uint32_t e0 = threadIdx.x; e0 < n; e0 += kUnroll * kVecThreads) {
        Words<kWords> v[kUnroll];
        int64_t at[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (e0 + u * kVecThreads < n) v[u] = load(e0 + u * kVecThreads, at[u]);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (e0 + u * kVecThreads < n) store(e0 + u * kVecThreads, at[u], v[u]);
    }
}

template <int kWords, int kMode>
__global__ void __launch_bounds__(kVecThreads)
hydra_place_rows_kernel(const PlaceParams p)
{
    constexpr bool kPaged = kMode == PLACE_KV || kMode == PLACE_MLA;
    __shared__ __align__(32) float s_cos[kVecThreads], s_sin[kVecThreads];      // (PLACE_MLA: s_cos holds the turned key)
    __shared__ int64_t s_k[kMaxItem], s_v[kMaxItem];                            // where a token's rows go; -1: nowhere
    __shared__ int32_t s_pos[kMaxItem];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int my_tok = p.pairs ? threadIdx.x / p.pairs : kMaxItem, my_pair = threadIdx.x - my_tok * p.pairs;
    const double freq = p.pairs ? exp(-p.log_theta * my_pair / p.pairs) : 0.0;
    int axis = 0;
#pragma unroll
    for (int a = 1; a < HYDRA_MAX_AXES; ++a) axis += my_pair >= p.axis_first[a] ? 1 : 0;
    const int32_t heads = p.by_heads.d;                                         // of a block
    wait_for_previous_launch();

    const int64_t n_items = (p.n_tokens + p.per_item - 1) / p.per_item * p.splits;
    for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
        const int64_t t0 = item / p.splits * p.per_item;
        const int32_t head0 = static_cast<int32_t>(item % p.splits) * heads;
        const int n_tok = static_cast<int>(min(static_cast<int64_t>(p.per_item), p.n_tokens - t0));
        const uint32_t rows = static_cast<uint32_t>(n_tok) * heads;
        __syncthreads();                                // the tables of the tokens before are no longer read
        if (kPaged) {
            for (int i = warp; i < n_tok; i += kVecThreads / 32) {
                const int64_t t = t0 + i;
                int32_t b;
                int64_t place = -1;
                if (p.cu_new) {
                    b = sequence_of(p.cu_new, p.n_seqs, t, lane);
                    const int32_t end = p.cu_new[b + 1];
                    if (t >= p.cu_new[b] && t < end) place = static_cast<int64_t>(p.seq_lens[b]) - (end - t);
                } else {
                    b = static_cast<int32_t>(min(t, static_cast<int64_t>(p.n_seqs - 1)));
                    if (t < p.n_seqs) place = static_cast<int64_t>(p.seq_lens[b]) - 1;
                }
                if (lane == 0) {
                    int64_t to_k = -1, to_v = -1;
                    if (place >= 0 && place < static_cast<int64_t>(p.max_pages) * p.page_size) {
                        const int32_t col = static_cast<int32_t>(place / p.page_size), row = static_cast<int32_t>(place % p.page_size);
                        const int32_t page = p.page_table[static_cast<int64_t>(b) * p.max_pages + col];
                        if (page >= 0 && page < p.n_pages) {
                            to_k = static_cast<int64_t>(page) * p.y_head * (heads * p.splits) + static_cast<int64_t>(row) * p.k_vecs;
                            to_v = static_cast<int64_t>(page) * p.y_v_head * (heads * p.splits) + static_cast<int64_t>(row) * p.v_vecs;
                        }
                    }
                    s_k[i] = to_k;
                    s_v[i] = to_v;
                    s_pos[i] = static_cast<int32_t>(place);
                }
            }
            if (!p.positions) __syncthreads();
        }
        if (my_tok < n_tok) {
            float cs, sn;
            rope_angle(p.positions ? p.positions[axis * p.n_tokens + t0 + my_tok] : s_pos[my_tok], freq, cs, sn);
            if (kMode == PLACE_MLA) {
                const float2 w = bf2_to_f2(*reinterpret_cast<const uint32_t*>(p.pe + (t0 + my_tok) * p.pe_stride + 2 * my_pair));
                s_cos[threadIdx.x] = __uint_as_float(f2_to_bf2(w.x * cs - w.y * sn, w.x * sn + w.y * cs));
            } else {
                s_cos[threadIdx.x] = cs;
                s_sin[threadIdx.x] = p.inverse ? -sn : sn;
            }
        }
        __syncthreads();
        // rows of y: row r is token by_heads(r) of the item; to(r, c) is its vector c, or -1
        auto to = [&](uint32_t r, uint32_t c) -> int64_t {
            const uint32_t tok = p.by_heads(r), head = head0 + r - tok * heads;
            if (!kPaged) return (t0 + tok) * p.y_stride + static_cast<int64_t>(head) * p.y_head + c;
            const int64_t base = s_k[tok];
            return base < 0 ? -1 : base + static_cast<int64_t>(head) * p.y_head + c;
        };
        auto from = [&](uint32_t r, uint32_t c) -> int64_t {
            const uint32_t tok = p.by_heads(r), head = head0 + r - tok * heads;
            return (t0 + tok) * p.k_stride + static_cast<int64_t>(head) * p.k_head + c;
        };
        // the rotary columns
        if (kMode == PLACE_MLA) {
            for (uint32_t e = threadIdx.x; e < rows * p.by_rot.d; e += kVecThreads) {
                const uint32_t r = p.by_rot(e), i = e - r * p.by_rot.d;
                const float* src = s_cos + p.by_heads(r) * p.pairs + i * kWords;
                Words<kWords> w;
#pragma unroll
                for (int j = 0; j < kWords; ++j) w.w[j] = __float_as_uint(src[j]);
                const int64_t at = to(r, p.rot0 + i);
                if (at >= 0) st_words<kWords>(p.y, at, w);
            }
        } else {
            move_rows<kWords>(rows * p.by_rot.d, [&](uint32_t e, int64_t& at) {
                const uint32_t r = p.by_rot(e), c = p.rot0 + e - r * p.by_rot.d;
                at = to(r, c);
                return kMode == PLACE_ROPE_IN_PLACE ? ld_words_coherent<kWords>(p.k, from(r, c)) : ld_words<kWords>(p.k, from(r, c));
            }, [&](uint32_t e, int64_t at, const Words<kWords>& w) {
                const uint32_t r = p.by_rot(e), c = p.by_heads(r) * p.pairs + (e - r * p.by_rot.d) * kWords;
                if (at >= 0) st_words<kWords>(p.y, at, rotate_vec<kWords>(w, s_cos + c, s_sin + c));
            });
        }
        // the others
        if (kMode != PLACE_ROPE_IN_PLACE)
            move_rows<kWords>(rows * p.by_copy.d, [&](uint32_t e, int64_t& at) {
                const uint32_t r = p.by_copy(e), j = e - r * p.by_copy.d, c = j < static_cast<uint32_t>(p.rot0) ? j : j + p.rot_vecs;
                at = to(r, c);
                return ld_words<kWords>(p.k, from(r, c));
            }, [&](uint32_t, int64_t at, const Words<kWords>& w) { if (at >= 0) st_words<kWords>(p.y, at, w); });
        if (kPaged)
            move_rows<kWords>(rows * p.by_v.d, [&](uint32_t e, int64_t& at) {
                const uint32_t r = p.by_v(e), c = e - r * p.by_v.d, tok = p.by_heads(r), head = head0 + r - tok * heads;
                const int64_t base = s_v[tok];
                at = base < 0 ? -1 : base + static_cast<int64_t>(head) * p.y_v_head + c;
                return kMode == PLACE_MLA ? ld_words<kWords>(p.k, from(r, p.rot0 + c))
                                          : ld_words<kWords>(p.v, (t0 + tok) * p.v_stride + static_cast<int64_t>(head) * p.v_vecs + c);
            }, [&](uint32_t, int64_t at, const Words<kWords>& w) { if (at >= 0) st_words<kWords>(p.y_v, at, w); });
    }
    overlap_next_launch();
}

// What all forms have in common. `vecs` vectors of a token are moved.
PlaceParams place_params(int64_t n_tokens, int32_t n_heads, const hydra_rope_t* rope, const int32_t* positions, int words,
                         int32_t copy_elems, int32_t v_elems, int32_t rot0_elems, int32_t row_elems)
{
    const int32_t elems = 2 * words, rot_elems = rope ? rope->dim : 0;
    // eight vectors per thread where the tokens are short, but no fewer than two blocks per SM for that; a token of many
    // vectors is shared by blocks, no fewer than a vector per thread, where there are few
    const int64_t vecs = int64_t{n_heads} * ((copy_elems + rot_elems + v_elems) / elems);
    const int32_t pairs = rot_elems / 2;
    int64_t per_item = std::min<int64_t>({8 * kVecThreads / vecs, n_tokens / (148 * 2), kMaxItem});
    if (pairs) per_item = std::min<int64_t>(per_item, kVecThreads / pairs);
    per_item = std::max<int64_t>(per_item, 1);
    const int64_t items = (n_tokens + per_item - 1) / per_item;
    int32_t splits = 1;
    while (n_heads % (2 * splits) == 0 && items * splits < 148 * 2 && per_item * vecs / (2 * splits) >= kVecThreads) splits *= 2;
    PlaceParams p{nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, 0, 0, 0, 0, 0, row_elems / elems, v_elems / elems,
                  rot0_elems / elems, rot_elems / elems, positions, n_tokens, pairs, 0, {}, 0.0, nullptr, nullptr, nullptr, 0, 0, 1, 0,
                  static_cast<int32_t>(per_item), splits, Div(n_heads / splits), Div(rot_elems / elems), Div(copy_elems / elems),
                  Div(v_elems / elems)};
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
    const int64_t items = (p.n_tokens + p.per_item - 1) / p.per_item * p.splits;
    const int grid = static_cast<int>(std::min<int64_t>(items, 148 * 32));
    return launch_overlapped(words == 8 ? hydra_place_rows_kernel<8, kMode> : hydra_place_rows_kernel<4, kMode>, grid, kVecThreads, 0,
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
    PlaceParams p = place_params(n_tokens, n_heads, &rope, positions, words, head_dim - rope.dim, 0, rope.offset, head_dim);
    p.k = static_cast<const uint16_t*>(x);
    p.y = static_cast<uint16_t*>(y);
    p.k_stride = x_stride / elems;
    p.y_stride = y_stride / elems;
    p.k_head = head_dim / elems;
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
    PlaceParams p = place_params(n_tokens, c.n_kv_heads, rope, positions, words, c.d_qk - dim, c.d_v, offset, c.d_qk);
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    p.pe = static_cast<const uint16_t*>(pe);
    p.y = static_cast<uint16_t*>(c.k);
    p.y_v = static_cast<uint16_t*>(c.v);
    p.k_stride = k_stride / elems;
    p.v_stride = v_stride / elems;
    p.pe_stride = pe_stride;
    p.k_head = (pe ? c.d_qk - dim + c.d_v : c.d_qk) / elems;
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

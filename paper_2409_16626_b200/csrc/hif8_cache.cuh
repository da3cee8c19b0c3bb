// What the kernels of the key/value cache share: where a token of a sequence lies in the pages, and how a block finds the
// sequence that its share of a ragged batch belongs to.
//
// Everything that comes from device memory (lengths, starts, page numbers, exponents) is clamped to what the host was told, so
// that wrong contents give wrong results and never an access outside the caller's buffers.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "hif8.h"
#include "hif8_internal.cuh"

namespace hif8 {

struct CacheView {
    uint8_t* k;             // [pages, heads, page tokens, dim]
    uint8_t* v;
    int* k_exp;             // [pages, heads]
    int* v_exp;
    const int* table;       // [sequences, table_stride] page numbers
    long long table_stride;
    int pages, heads, shift, dim;  // shift: log2 of the tokens of a page

    __host__ __device__ long long page_bytes() const { return ((long long)heads * dim) << shift; }
    size_t pool_bytes() const { return (size_t)pages * (size_t)page_bytes(); }
    size_t exp_bytes() const { return (size_t)pages * (size_t)heads * sizeof(int); }
    size_t table_bytes(int seqs) const { return (size_t)seqs * (size_t)table_stride * sizeof(int); }
    // first byte of a block: one page's tokens of one head
    __device__ long long block_at(int page, int head) const { return ((long long)page * heads + head) * dim << shift; }
    // page of the tokens block << shift .. of a sequence; -1 where the table names none
    __device__ int page_of(int seq, int block) const
    {
        if ((unsigned)block >= (unsigned long long)table_stride) return -1;
        const int p = table[(long long)seq * table_stride + block];
        return (unsigned)p < (unsigned)pages ? p : -1;
    }
    // most tokens that a row of the table can name (up to 2^30), and a length within that
    __host__ __device__ int capacity() const { return table_stride >= (1 << 30) >> shift ? 1 << 30 : (int)table_stride << shift; }
    __device__ int length(int n) const { return max(0, min(n, capacity())); }
};

namespace {

__device__ __forceinline__ int clamp_cache_exp(int e) { return max(-HIF8_CACHE_EXP_MAX, min(HIF8_CACHE_EXP_MAX, e)); }

// A ragged batch of tokens, sequence s's being start[s] .. start[s + 1] - 1, cut into pieces that lie within one page each.  Sequence s gets
// the piece numbers from (start[s] >> shift) + 2 s on: with c tokens it touches at most (c >> shift) + 2 pages, so no two sequences
// share a number, a block needs no prefix sum over the batch, and few numbers are empty.
struct Piece {
    int seq, token, count, pos;  // tokens token .. + count of the batch, at position pos .. of the sequence; count 0: nothing
};
__host__ __device__ inline long long piece_numbers(int n_tokens, int n_seqs, int shift) { return (long long)(n_tokens >> shift) + 2ll * n_seqs; }

__device__ __forceinline__ int start_at(const int* start, int s, int n_tokens) { return max(0, min(start[s], n_tokens)); }

// All lanes of a warp together: one probe a lane and round, so a search over 1024 sequences waits for memory twice.
__device__ __forceinline__ Piece find_piece(long long number, const int* start, const int* first, int n_seqs, int n_tokens, int shift, int lane)
{
    int lo = 0, n = n_seqs;  // the sequence is among lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) >> 5, at = lo + lane * step;
        const bool below = lane * step < n && (lane == 0 || (long long)(start_at(start, at, n_tokens) >> shift) + 2ll * at <= number);
        const int last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, below));  // (with starts in order the lanes below form a prefix)
        lo += last * step;
        n = min(step, n - last * step);
    }
    Piece p;
    p.seq = lo;
    const int b = start_at(start, lo, n_tokens), e = start_at(start, lo + 1, n_tokens), pos0 = max(0, first[lo]);
    const long long i = number - ((b >> shift) + 2ll * lo), page0 = pos0 >> shift;  // the piece's number within the sequence
    const long long from = i <= 0 ? pos0 : (page0 + i) << shift, to = (page0 + i + 1) << shift, end = (long long)pos0 + max(0, e - b);
    const long long stop = to < end ? to : end;
    p.count = i < 0 || from >= stop ? 0 : (int)(stop - from);
    p.pos = (int)from;
    p.token = b + (int)(from - pos0);
    return p;
}

// The units (a piece's tokens of one head of K or V) of team `me` of `teams`: consecutive ones, so that a piece is looked for once and not for each of its units
// (27.7 K tokens of 8 heads of 128, appended and read back: 89 -> 81 us).
struct UnitWalk {
    long long number, left;  // the piece's number; units to come, this one included
    int part, parts;         // of the piece: head and K or V; parts of a piece
    bool fresh;              // the first unit of its piece here
    __device__ UnitWalk(long long units, int parts_, long long me, long long teams) : parts(parts_), fresh(true)
    {
        const long long each = units / teams, rest = units - each * teams, u = me * each + (me < rest ? me : rest);
        left = each + (me < rest ? 1 : 0);
        number = u / parts;
        part = (int)(u - number * parts);
    }
    __device__ void next()
    {
        left--;
        fresh = ++part == parts;
        if (fresh) { part = 0; number++; }
    }
};

}  // namespace

// Whether something that a call writes lies where it writes something else, or reads.
struct ByteRange { const void* at; size_t bytes; };
inline bool written_over(std::initializer_list<ByteRange> written, std::initializer_list<ByteRange> read)
{
    for (const ByteRange* w = written.begin(); w != written.end(); w++) {
        for (const ByteRange* o = w + 1; o != written.end(); o++)
            if (ranges_overlap(w->at, w->bytes, o->at, o->bytes)) return true;
        for (const ByteRange& r : read)
            if (ranges_overlap(w->at, w->bytes, r.at, r.bytes)) return true;
    }
    return false;
}

// Arguments that describe the cache, checked before anything is launched; fills in the view.
inline int check_cache(const void* k, const void* v, const void* k_exp, const void* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim, const void* table,
                       int64_t table_stride, CacheView* out)
{
    if (n_pages < 0 || kv_heads < 1 || kv_heads > HIF8_CACHE_MAX_HEADS || table_stride < 1) return HIF8_ERR_SHAPE;
    if (page_tokens != 16 && page_tokens != 32 && page_tokens != 64 && page_tokens != 128) return HIF8_ERR_SHAPE;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return HIF8_ERR_SHAPE;
    if (!k || !v || !k_exp || !v_exp || !table) return HIF8_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u) return HIF8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(k_exp) | reinterpret_cast<uintptr_t>(v_exp) | reinterpret_cast<uintptr_t>(table)) & 3u) return HIF8_ERR_ALIGN;
    out->k = (uint8_t*)k; out->v = (uint8_t*)v; out->k_exp = (int*)k_exp; out->v_exp = (int*)v_exp;
    out->table = (const int*)table; out->table_stride = table_stride;
    out->pages = n_pages; out->heads = kv_heads; out->dim = head_dim;
    out->shift = page_tokens == 16 ? 4 : page_tokens == 32 ? 5 : page_tokens == 64 ? 6 : 7;
    return HIF8_OK;
}

}  // namespace hif8

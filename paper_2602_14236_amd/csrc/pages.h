// Paged K/V cache of text tokens: what its host API and its kernel files share.  The layout of a block of 16 tokens stands in sali.h.
#pragma once

#include "sali_internal.h"

#include "pages_arith.h"

namespace sali {

// a layer's pages
struct PageGeom {
    char* pool;
    uint64_t page_bytes;
    uint32_t head_bytes;                    // of one head in a page
    int32_t n_pages, n_kv, blocks_log2;     // blocks of a page
};

// a batch of sequences, and where faults are noted
struct PageSeqs {
    const int32_t* start;
    const int32_t* length;
    const int32_t* table;
    uint32_t* status;
    int32_t n_seqs, width, n_tokens, max_q, max_kv;
};

struct RowsIn {
    const char* d;
    int64_t token_bytes, head_bytes;
};
struct RowsOut {
    char* d;
    int64_t token_bytes, head_bytes;
};

struct PagesAttend {
    PageGeom geom;
    PageSeqs seqs;
    RowsIn q;
    RowsOut out;
    float* lse;                             // or NULL
    const float* prior;                     // or NULL
    const float* prior_lse;
    float scale2;                           // |softmax_scale| * log2(e), 1 for a scale of zero
    uint32_t q_keep, q_flip;                // what is done to the queries' bits: a negative scale flips their signs, a scale of zero makes them zero
    int32_t window, sinks;                  // window 0: none
    int32_t heads, group;                   // query heads, and of one K/V head
    float* partial;
    int32_t* records;
    const uint64_t* seen;                   // of drafted tokens, a mask each
};

// rotary positions of queries and keys
struct Rotate {
    RowsIn q, k;
    RowsOut q_out, k_out;
    const double* frequency;
    const int32_t* position;
    int64_t axis_stride;
    int32_t q_heads, k_heads, dim, pairs, adjacent, inverse, n_tokens;
    int32_t until[3];                       // first pair of the second, third and fourth axis
};

// attention weights of keys, summed
struct PagesWeigh {
    PageGeom geom;
    PageSeqs seqs;
    RowsIn q;
    const float* lse;
    float* weights;                         // [page][K/V head][token]
    float scale2;                           // softmax_scale * log2(e)
    int32_t window, sinks, heads, group, add;
    float* partial;                         // room for sums of chunks of rows
    size_t partial_bytes;
};

struct PagesSelect {
    PageGeom geom;
    PageSeqs seqs;
    const float* weights;
    int32_t* keep;
    int32_t budget, sinks, recent;
};

struct PagesKeep {
    PageGeom geom;
    PageSeqs seqs;
    const int32_t* keep;
    const int32_t* to;                      // table of the places where rows go
    float* weights;                         // or NULL
    int32_t width, keep_heads, to_width, in_place;
};

// scratch of the pages object: the status word, a row of zeros, then the partial results of attention
constexpr size_t kPagesZeros = 256, kPagesStatusBytes = kPagesZeros + 256;
struct PagesScratch {
    size_t partial, records, bytes;         // where the two areas start
};
PagesScratch pages_scratch(int64_t n_pages, int page_tokens, int n_kv, int group, int dim);

hipError_t launch_pages_append(int dtype, int store, int dim, const PageGeom& g, const PageSeqs& seqs, const RowsIn& k, const RowsIn& v, hipStream_t s);
hipError_t launch_pages_read(int dtype, int store, int dim, const PageGeom& g, const PageSeqs& seqs, const RowsOut& k, const RowsOut& v, hipStream_t s);
hipError_t launch_pages_attend_fp16(int store, int dim, const PagesAttend& a, hipStream_t s);
hipError_t launch_pages_attend_bf16(int store, int dim, const PagesAttend& a, hipStream_t s);
hipError_t launch_pages_attend_tree_fp16(int store, int dim, const PagesAttend& a, hipStream_t s);
hipError_t launch_pages_attend_tree_bf16(int store, int dim, const PagesAttend& a, hipStream_t s);
constexpr int kWeighTokens = 128;           // keys of a thread block at the least
inline int64_t weigh_blocks(const PageSeqs& q) { return ((int64_t)q.max_kv + kWeighTokens - 1) / kWeighTokens; }
constexpr int kKeepTokens = 64;             // rows of a thread block, if they go to other pages
inline int64_t keep_chunks(const PageSeqs& q, int32_t width, bool in_place) {
    // (a sequence's first place may lie inside a block of 16)
    return in_place ? 1 : (least((int64_t)width, (int64_t)q.max_q) + kBlockTokens - 1 + kKeepTokens - 1) / kKeepTokens;
}
inline int keep_strips(int dim, bool weights) { return 2 * (dim / 32) + (weights ? 1 : 0); }
constexpr int64_t kMostBlocks = (1 << 24) - 1;      // thread blocks of 256 threads that a launch takes
hipError_t launch_rotate(int dtype, const Rotate& r, hipStream_t s);
hipError_t launch_pages_weigh(int dtype, int store, int dim, const PagesWeigh& a, hipStream_t s);
hipError_t launch_pages_select(const PagesSelect& a, hipStream_t s);
hipError_t launch_pages_keep(int store, int dim, const PagesKeep& a, hipStream_t s);

#ifdef __HIPCC__
// Does the start of one of the sequences i, i + step .. lie behind the next one's?  Nobody knows then whose rows are whose: the batch is left out whole.
// (The first of them is asked for when this is made; a sequence that is alone has it checked with its other numbers.)
struct StartFalls {
    const int32_t* start;
    int n_seqs, i, step, first, next;
    __device__ __forceinline__ StartFalls(const int32_t* start, int n_seqs, int i, int step) : start(start), n_seqs(n_seqs), i(i), step(step), first(0), next(0) {
        if (n_seqs > 1 && i < n_seqs) {
            first = start[i];
            next = start[i + 1];
        }
    }
    __device__ __forceinline__ bool some() const {
        bool falls = first > next;
        for (int k = i + step; k < n_seqs; k += step) falls |= start[k] > start[k + 1];
        return falls;
    }
};
__device__ __forceinline__ PageSeq read_seq(const PageSeqs& q, const PageGeom& g, int s, bool& fits) {
    const int64_t a = q.start[s], b = q.start[s + 1], len = q.length[s];
    const int64_t in_table = (int64_t)q.width * (kBlockTokens << g.blocks_log2), room = in_table < q.max_kv ? in_table : q.max_kv;
    fits = page_seq_holds(a, b, len, q.n_tokens, q.max_q, room);
    return {(int32_t)a, fits ? (int32_t)(b - a) : 0, (int32_t)len};
}
__device__ __forceinline__ PageSeq load_seq(const PageSeqs& q, const PageGeom& g, int s, bool note) {
    bool fits;
    const PageSeq r = read_seq(q, g, s, fits);
    if (note && !fits) atomicOr(q.status, SALI_FAULT_BATCH);
    return r;
}
#endif

}  // namespace sali

// Paged attention of half-precision tokens; the kernels stand in pages_stream.h and pages_tile.h.
#include "pages_attn_launch.h"

namespace sali {

hipError_t launch_pages_attend_fp16(int store, int dim, const PagesAttend& a, hipStream_t s) { return launch_pages_attend<false>(store, dim, a, s); }

PagesScratch pages_scratch(int64_t n_pages, int page_tokens, int n_kv, int group, int dim) {
    auto align = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t row = (size_t)(dim + 4) * sizeof(float);
    size_t parts = (size_t)2 * kStreamMostBlocks * 32, records = (size_t)kStreamMostBlocks * sizeof(StreamRecord);
    for (int waves : {4, 12}) {
        parts = max(parts, (size_t)tile_parts(n_kv, waves) * n_kv * tile_rows(waves));       // stretches have as many at the most
        records = max(records, tile_scratch_bytes(tile_slots(n_pages * page_tokens, group, n_pages, tile_rows(waves)), n_kv, waves));
    }
    PagesScratch p;
    p.partial = kPagesStatusBytes;
    p.records = align(p.partial + parts * row);
    p.bytes = align(p.records + records);
    return p;
}

}  // namespace sali

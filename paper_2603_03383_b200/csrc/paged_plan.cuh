// How a call of the paged attention divides its workspace: plain arithmetic, for the host, the kernels and a host compiler alone.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <cuda_runtime.h>

namespace mtv {

constexpr int TH_ROWS = 16;            // query rows of a thin item

struct PaPhase {
    int prefix_items, seq_items;       // items of the prefix, and of each sequence
    int prefix_per_head, seq_per_head;
    int prefix_tile0, seq_tile0;       // row tile of a head's first item (0 where an item is a pair)
    int rows;                          // of a slot
    int workers;                       // at most: their numbers are below this
    float *o;                          // [slots][D / 8][rows][8]
    float2 *ml;                        // [slots][rows]
    int2 *span;                        // [items]: first and last worker that has a piece of it
};

// The phases of a call and the layout of its workspace; returns the bytes.
static inline size_t pa_plan(PaPhase (&ph)[3], int sms, int T, int B, int G, int Hkv, int D, int shared, char *ws) {
    const int npc = 128 / G;
    // at most 16 rows: thin items (64 single tokens of 4 rows a KV head behind 8192 shared keys: the whole call 77 us, and 94 as row tiles)
    const bool thin_seq = T * G <= TH_ROWS, thin_prefix = shared && B * T * G <= TH_ROWS;
    const int prefix_tiles = shared && !thin_prefix ? (B * T + npc - 1) / npc : 0, seq_tiles = thin_seq ? 0 : (T + npc - 1) / npc;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = ws + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    for (int f = 0; f < 3; ++f) {
        PaPhase &x = ph[f];
        x.prefix_per_head = f == 2 ? thin_prefix : f ? prefix_tiles % 2 : prefix_tiles / 2;
        x.seq_per_head = f == 2 ? thin_seq : f ? seq_tiles % 2 : seq_tiles / 2;
        x.prefix_items = Hkv * x.prefix_per_head;
        x.seq_items = Hkv * x.seq_per_head;
        x.prefix_tile0 = f ? prefix_tiles - 1 : 0;
        x.seq_tile0 = f ? seq_tiles - 1 : 0;
        x.rows = f == 2 ? TH_ROWS : f ? 128 : 256;
        const size_t items = (size_t)x.prefix_items + (size_t)B * x.seq_items;
        x.workers = items ? (f ? 2 : 1) * sms : 0;
        const size_t slots = items + x.workers;      // a piece's slot: its item's number plus its worker's
        x.o = reinterpret_cast<float *>(take(slots * x.rows * D * sizeof(float)));
        x.ml = reinterpret_cast<float2 *>(take(slots * x.rows * sizeof(float2)));
        x.span = reinterpret_cast<int2 *>(take(items * sizeof(int2)));
    }
    return at;
}

// Whether an item's span can be followed.  Every item that is attended to has one, unless a wait of the kernel that makes the pieces ran out:
// then the workspace may hold anything there.  Slots up to the item's number plus span.y are inside the workspace if it can.
static __host__ __device__ inline bool pa_span_ok(const PaPhase &f, int2 span) { return 0 <= span.x && span.x <= span.y && span.y < f.workers; }

}  // namespace mtv

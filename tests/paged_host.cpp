// paged_host.cpp -- the paged attention's entry points with their launches replaced: the split
// that every workgroup of the launch for few rows would work out is worked out here, by the
// same code, from sequences in host memory.  Built and read by test_paged_split.py.
#include "wave.h"

#include "../paper_2605_09681_amd/csrc/fkv_paged_api.hip"

namespace {

struct Item {
    int32_t seq, start, n, len, first, y, rt, part, parts, slot, step, join;
};
struct Plan {
    int32_t rows, n_work, n_slots, n_joins, lo, hi, count, tiles;   // tiles: of the launch for many rows, 0: not launched
};
Plan plan_out;
std::vector<Item> items;

template <int ROWS>
void split_rows(const fkv::PagedArgs &a) {
    wave::run([&](int lane) {                // (a workgroup's wave each, in turn)
        const fkv::paged::Split<ROWS, 32> split(a);
        const int n = a.target > 0 ? split.cut_items(a) : 0;
        if (lane == 0) plan_out.count = n;
        for (int b = 0; b < a.n_work; ++b) {
            const fkv::paged::Work w = split.locate(a, b);
            if (lane == 0 && w.ok)
                items.push_back({w.i, w.s.start, w.s.n, w.s.len, w.s.first, w.y, w.rt, w.part, w.parts, w.slot, w.step, w.join});
        }
    });
}

hipError_t split(const fkv::PagedArgs &a, int rows) {
    plan_out = Plan{rows, a.n_work, a.n_slots, a.n_joins, a.lo, a.hi, 0, plan_out.tiles};
    if (rows == 16) split_rows<16>(a);
    else if (rows == 32) split_rows<32>(a);
    else if (rows == 48) split_rows<48>(a);
    else split_rows<64>(a);
    return hipSuccess;
}

std::vector<int32_t> owners, blocks;
int32_t block_tokens;
std::vector<int64_t> first_rows;

}  // namespace

extern "C" hipError_t hipGetLastError() { return hipSuccess; }
extern "C" const char *hipGetErrorString(hipError_t) { return ""; }

namespace fkv {

fkv_status api_error(fkv_status st, const char *message) {
    fprintf(stderr, "%s\n", message);
    return st;
}
fkv_status api_ok() { return FKV_OK; }
fkv_status api_compute_units(int *n) {
    *n = 256;
    return FKV_OK;
}
hipError_t launch_paged_attention(const PagedArgs &a, int, int rows, hipStream_t) { return split(a, rows); }
hipError_t launch_latent_rows(const PagedArgs &a, int, int rows, hipStream_t) { return split(a, rows); }
hipError_t launch_paged_tiles(const PagedArgs &, int, int rows, hipStream_t) {
    plan_out.tiles = rows;
    return hipSuccess;
}
hipError_t launch_expanded_tiles(const PagedArgs &a, int, hipStream_t) {
    plan_out.tiles = 256;
    for (int i = 0; i < a.n_seqs; ++i)
        wave::run([&](int lane) {
            const int64_t row = paged::first_row(a, i);
            if (lane == 0) first_rows.push_back(row);
        });
    for (int b = 0; b < a.head_rows / paged::kSeqRows; ++b)
        wave::run([&](int lane) {
            paged::Seq s;
            int i = -1;
            const int key = paged::locate_block(a, b, &s, &i);
            if (lane == 0) blocks.insert(blocks.end(), {key < 0 ? -1 : i, key});
        });
    return hipSuccess;
}
hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t) {
    block_tokens = a.block_tokens;
    if (owners.empty()) return hipSuccess;
    for (int t0 = 0; t0 < a.batch.n_tokens; t0 += wave::kLanes)
        wave::run([&](int lane) {
            paged::Seq s;
            const int n = std::min(wave::kLanes, a.batch.n_tokens - t0);
            const int i = paged::owner_of(a.batch, lane < n ? t0 + lane : -1, t0, t0 + n, &s);
            if (lane < n) owners[t0 + lane] = i;
        });
    return hipSuccess;
}
hipError_t launch_latent_absorb(const LatentArgs &, int, hipStream_t) { return hipSuccess; }
hipError_t launch_latent_unabsorb(const LatentArgs &, int, hipStream_t) { return hipSuccess; }
hipError_t launch_latent_expand(const LatentArgs &, int, hipStream_t) { return hipSuccess; }

}  // namespace fkv

extern "C" {

// The calls below take any pointer for what only the kernels would read.
static void *const kAny = (void *)0x1000;
static fkv_rows rows_of(int heads, int width) { return fkv_rows{kAny, width, (int64_t)heads * width}; }

int host_attend(const fkv_batch *b, int heads, int kv, int d, const fkv_span *spans, int split_keys) {
    items.clear();
    plan_out = Plan{};
    const fkv_rows r = rows_of(heads, d);
    return fkv_paged_attention(b, heads, kv, d, &r, kAny, kAny, 1, spans, 0.1f, &r, nullptr, split_keys ? kAny : nullptr,
                               (size_t)1 << 50, nullptr);
}
int host_latent(const fkv_batch *b, int heads, int d, int R, int form) {
    items.clear();
    first_rows.clear();
    blocks.clear();
    plan_out = Plan{};
    const fkv_rows q = rows_of(heads, d + FKV_LATENT_ROT), o = rows_of(heads, d);
    return fkv_latent_attention(b, heads, d, R, &q, kAny, kAny, kAny, 1, nullptr, 0.1f, &o, form, kAny, (size_t)1 << 50, nullptr);
}
int host_append(const fkv_batch *b, int heads, int d, int dtype, int owned) {
    owners.assign(owned ? b->n_tokens : 0, -2);
    const fkv_rows r = rows_of(heads, d);
    return fkv_append_paged(b, heads, d, dtype, &r, &r, kAny, kAny, nullptr);
}
int host_block_tokens() { return block_tokens; }
const Plan *host_plan() { return &plan_out; }
int host_items(const Item **p) {
    *p = items.data();
    return (int)items.size();
}
int host_owners(const int32_t **p) {
    *p = owners.data();
    return (int)owners.size();
}
int host_first_rows(const int64_t **p) {
    *p = first_rows.data();
    return (int)first_rows.size();
}
int host_blocks(const int32_t **p) {
    *p = blocks.data();
    return (int)blocks.size() / 2;
}

}  // extern "C"

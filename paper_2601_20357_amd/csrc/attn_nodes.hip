// Attention over trees: which variant, and how many ranges of keys.
#include "attn_nodes.h"

namespace tabed {

constexpr size_t kRangesBytes = 8192;                                    // of the rows of a call that is split
constexpr int kMaxSplitRows = kRangesBytes / 8;
constexpr int kMinRange = 512, kWholeRow = 1024, kLongRow = 8192;        // tokens

template <typename F>
static auto with_hd(int hd, F&& f) {
    switch (hd) {
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        case 96: return f(std::integral_constant<int, 96>{});
        case 128: return f(std::integral_constant<int, 128>{});
        default: return f(std::integral_constant<int, 256>{});
    }
}

struct NodesVariant {
    int queries, unit, tokens, room;                                     // of a workgroup, of a wave, of a tile; workgroups that run at a time
};
static NodesVariant variant_of(const tabed_cache_paged& c, int queries, bool few) {
    auto take = [](auto v) {
        using T = decltype(v);
        return NodesVariant{T::kQueries, T::kUnit, T::kTokens, 256 * std::max(1, std::min(163840 / (int)(T::kLds + sizeof(NodesShared)), 512 / T::kThreads))};
    };
    return with_hd(c.head_dim, [&](auto hd) {
        return c.type == 2 ? with_nodes_variant<decltype(hd)::value, true>(queries, few, take) : with_nodes_variant<decltype(hd)::value, false>(queries, few, take);
    });
}
// Tiles of the longest row there can be.
static int64_t most_tiles(const tabed_cache_paged& c, int tokens) { return ((int64_t)c.max_blocks * TABED_CACHE_BLOCK + tokens - 1) / tokens; }

struct NodesPlan {
    int tiles, per_tile, slots, split, fill, min_tiles, whole_tiles;
};
static NodesPlan plan_of(const tabed_cache_paged& c, int rows, int N, int q_heads) {
    const int queries = N * (q_heads / c.kv_heads);
    const NodesVariant v = variant_of(c, queries, few_units(rows, c.kv_heads));
    NodesPlan p{};
    p.per_tile = v.queries;
    p.tiles = (queries + p.per_tile - 1) / p.per_tile;
    if (p.tiles > 1) p.per_tile = ((queries + p.tiles - 1) / p.tiles + v.unit - 1) / v.unit * v.unit;      // (as even as whole units of a wave leave them)
    const int64_t units = (int64_t)c.kv_heads * p.tiles;                 // workgroups of a slot
    const int64_t most = most_tiles(c, v.tokens);
    p.min_tiles = std::max(1, kMinRange / v.tokens);
    p.whole_tiles = std::max(1, kWholeRow / v.tokens);
    p.slots = rows;
    p.fill = (int)std::max<int64_t>(v.room / units, 2 * rows);
    // Ranges of 512 tokens or more (4 rows of 4000 tokens, 16 nodes, 32 / 8 heads of 128: 34 us; of 1024 or more 44, of 256 or more 36), of rows of more than 1024 (one row
    // of 600, 6 nodes, 12 heads of 64, four waves: whole 7.6 us, in two 12).  Where rows alone fill the chip they are cut only if one can be so long that the others would
    // wait for it: of more than 8192 (64 rows of 2000, 12 nodes, 12 heads of 64: whole 72 us, cut 92).  How long a row can be goes by the table's width, since the lengths
    // are known on the GPU alone: under a table of more than 8192 tokens those 64 rows are cut (101 us), and short rows, which never are, pay for the second launch (64
    // rows of 256 to 768, 16 nodes 24 us, then 37).  No more ranges than run at a time, also where a row's last tile of queries has little to do: the others' workgroups
    // would wait for a second round (tiles of 96 and 36 queries, 16 rows of 300 to 5000: 93 us with as many as the queries would fill, 77 so).
    if (rows <= kMaxSplitRows && most > std::max(1, (v.room / units > rows ? kWholeRow : kLongRow) / v.tokens)) {
        p.split = 1;
        p.slots = (int)std::min<int64_t>(p.fill, rows * ((most + p.min_tiles - 1) / p.min_tiles));
    }
    return p;
}

NodesAttnLayout nodes_attn_layout(const tabed_cache_paged& c, int rows, int N, int q_heads) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const NodesPlan p = plan_of(c, rows, N, q_heads);
    NodesAttnLayout L{kRangesBytes, kRangesBytes};
    if (p.split) L.off_o = L.off_ml + up((size_t)p.slots * c.kv_heads * p.tiles * p.per_tile * 16);
    return L;
}
// Bytes that calls of up to so many rows and nodes need: the most that any variant of them has of places for ranges' results, not less for more of either.
size_t nodes_attn_bytes(const tabed_cache_paged& c, int rows, int N, int q_heads) {
    const int64_t queries = (int64_t)N * (q_heads / c.kv_heads), split_rows = std::min(rows, kMaxSplitRows);
    int64_t places = 0;
    for (int64_t some : {(int64_t)16, (int64_t)32, queries}) {
        some = std::min(some, queries);
        const NodesVariant v = variant_of(c, (int)some, false);          // (few units: no more places)
        const int64_t most = most_tiles(c, v.tokens), least = std::max(1, kMinRange / v.tokens);
        if (most <= std::max(1, kWholeRow / v.tokens)) continue;
        const int64_t room = (int64_t)v.room * v.queries, row = (some + v.queries - 1) / v.queries * v.queries * c.kv_heads;      // places of as many as run, of a range
        int64_t twice = 2 * split_rows * row;
        if (most <= std::max(1, kLongRow / v.tokens)) twice = std::min(twice, 2 * room);      // (more rows than that are not cut)
        places = std::max(places, std::min(std::max(room, twice), split_rows * ((most + least - 1) / least) * row));
    }
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    return kRangesBytes + up((size_t)places * 16) + up((size_t)places * c.head_dim * 4);
}
int64_t nodes_attn_workgroups(const tabed_cache_paged& c, int rows, int N, int q_heads) {
    const NodesPlan p = plan_of(c, rows, N, q_heads);
    return ((int64_t)p.slots * c.kv_heads + 7) / 8 * 8 * p.tiles;
}
hipError_t launch_nodes_attn_init(char*, hipStream_t) { return hipSuccess; }         // (nothing is expected in it)

hipError_t launch_attention_nodes(const tabed_cache_paged& c, int layer, char* ws, int rows, int N, int q_heads, const uint16_t* q, int64_t q_row,
                                  int64_t q_tok, const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float scale, uint16_t* out,
                                  int64_t out_row, int64_t out_tok, float* lse, hipStream_t s) {
    ProfScope prof(TABED_K_BODY, s);
    const NodesPlan p = plan_of(c, rows, N, q_heads);
    const NodesAttnLayout L = nodes_attn_layout(c, rows, N, q_heads);
    const NodesAttnArgs a{paged_view(c, layer), rows, N, q_heads, q_heads / c.kv_heads, p.tiles, p.per_tile, p.slots, p.split, p.fill, p.min_tiles, p.whole_tiles, q, out, lse,
                          q_row, q_tok, out_row, out_tok, ctx_len, parents, n_nodes, scale * 1.44269504088896340736f, reinterpret_cast<int2*>(ws),
                          reinterpret_cast<float4*>(ws + L.off_ml), reinterpret_cast<float*>(ws + L.off_o)};
    return with_hd(c.head_dim, [&](auto hd) { return launch_nodes_hd<decltype(hd)::value>(c.type == 2, &prof, a, s); });
}

}  // namespace tabed

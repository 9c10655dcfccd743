// sa_chunk_attention: checks, and the launches of the kernels in sa_chunk.cuh.
#include "sa_chunk.cuh"

namespace sa {

static size_t chunk_workspace(const Plan& p, int64_t rows_most, int blocks) {
    return kChunkCutBytes + 2 * (size_t)blocks * sizeof(float) * chunk_slot_floats(p.d, rows_most <= chunk_rows(true));
}
static int chunk_blocks_most() { return sm_count() < kChunkBlocksMost ? sm_count() : kChunkBlocksMost; }

static int chunk_format(const Plan& p) {
    if (p.fp16) return FMT_FP16;
    if (p.fp4) return FMT_FP4;
    if (p.int8) return FMT_INT8;
    if (p.nibble) return p.k == 0 ? FMT_NIBBLE : p.k == 1 ? FMT_PLANAR1 : FMT_PLANAR2;
    return FMT_BYTE;
}

// The sequences of one kind (SPLIT: of at most 128 rows; or the others), kChunkBatch a launch.
static bool launch_kind(const Plan& p, ChunkArgs& a, const int64_t* cu, bool split, bool lost, cudaStream_t s) {
    const int fmt = chunk_format(p);
    int64_t most = 0;
    for (int b = 0; b < a.c.batch; ++b) {
        const int64_t rows = (cu[b + 1] - cu[b]) * p.G;
        if ((rows <= chunk_rows(true)) == split && rows > most) most = rows;
    }
    if (most == 0) return true;
    a.copies = !split || most > 64 ? 1 : most > 32 ? 2 : 4;
    const int per_tile = chunk_rows(split) / a.copies;
    const int64_t tiles_most = ((int64_t)a.c.max_pages + 1) / 2, blocks_most = chunk_blocks_most();
    for (int b = 0; b < a.c.batch;) {
        a.s.n = 0;
        a.s.tiles[0] = 0;
        int64_t work = 0, longest = 0;                                          // key tiles, by what the cache has room for
        int64_t least = 0, reach = 0;                                           // ... where it holds the new tokens only; the most that a unit has beyond what its sequence then adds to a block's share
        for (; b < a.c.batch && a.s.n < kChunkBatch; ++b) {
            const int64_t n = cu[b + 1] - cu[b], rows = n * p.G;
            if (n == 0 || (rows <= chunk_rows(true)) != split) continue;
            const int i = a.s.n, tiles = (int)((rows + per_tile - 1) / per_tile);
            if (i && a.s.tiles[i] > 0x7ffffff0 - tiles) break;
            a.s.b[i] = b;
            a.s.tokens[i] = (int)n;
            a.s.row0[i] = cu[b];
            a.s.tiles[i + 1] = a.s.tiles[i] + tiles;
            a.s.n = i + 1;
            const int64_t window = a.window ? ((int64_t)a.window + per_tile / p.G + 1) / kChunkTile + 2 + ((int64_t)a.sinks + kChunkTile - 1) / kChunkTile : tiles_most;
            const int64_t keys = window < tiles_most ? window : tiles_most;
            work += (int64_t)tiles * (kChunkUnitCost + keys);
            longest = keys > longest ? keys : longest;
            const int64_t own = (n - 1) / kChunkTile + 1, last = own < keys ? own : keys, beyond = keys * blocks_most - tiles * (keys - last) * p.Hkv;
            least += tiles * kChunkUnitCost + tiles * (1 + last) / 2;           // (causal: from one tile to `last`)
            reach = beyond > reach ? beyond : reach;
        }
        if (a.s.n == 0) break;
        // A unit a block, none of them cut, where that is as good.  Only the device knows the lengths and can decide on that, for which it needs the second launch, that of the merge, which
        // costs 2.5 us even where nothing is cut.  So not where the longest unit cannot be much longer than an equal share whatever the lengths are (worst: one sequence fills
        // the cache, the others hold their new tokens only; 2.5 tiles more than what cutting costs: a prompt of 2048 tokens, 16 / 2 heads of 128, binary16, 44.3 us whole, 46.4 cut); nor for few rows where that holds for equal lengths and units are short, as windows make them: 32 single tokens with a
        // window of 4096 32.9 us, 35.4 with the second launch, for which one sequence at its window beside 36 of 300 tokens takes 32.2, which 22.1 would do.
        const int64_t units = (int64_t)a.s.tiles[a.s.n] * p.Hkv, bound = (2 * (chunk_cut_cost(p.d, split) - kChunkUnitCost) + 5) * blocks_most / 2;
        const bool worst = reach - least * p.Hkv <= bound, equal = longest * blocks_most - work * p.Hkv <= bound;
        a.whole = units <= blocks_most && (worst || (split && equal && longest <= (p.d == 64 ? 40 : 20)));
        const int blocks = (int)(a.whole ? units : work * p.Hkv < blocks_most ? work * p.Hkv : blocks_most);
        a.merged = !a.whole && blocks > 1;
        const bool pot = !p.fp16 && !p.fp4 && !p.int8;
        const int rows_most = (int)(most < per_tile ? most : per_tile);
        const cudaError_t e = lost ? launch_chunk_lost(split, a, blocks, rows_most, s)
                              : pot ? launch_chunk_pot(p.d, fmt, split, a, blocks, rows_most, s) : launch_chunk_plain(p.d, fmt, split, a, blocks, rows_most, s);
        if (e != cudaSuccess) return false;
    }
    return true;
}

// lost: null, or {b, kv_head, tile} of sa_debug_chunk_lost_copy.
static sa_status chunk_attention(const sa_config* cfg, const sa_cache* cache, const uint16_t* Q, const int64_t* cu_lens_host, int window, int sinks, void* O, int o_dtype, void* workspace,
                                 size_t workspace_bytes, const int* lost, sa_stream stream) {
    Plan p;
    sa_status st = make_plan(cfg, &p);
    if (st != SA_OK) return st;
    if (p.mulshift || p.addalu || p.shiftadd) return SA_ERR_UNSUPPORTED;      // (decode kernels only)
    if (lost && (p.d != 64 || p.k != 4 || p.fp16 || p.fp4 || p.int8 || p.nibble)) return SA_ERR_UNSUPPORTED;
    ChunkArgs a{};
    st = check_cache(p, cache, &a.c);
    if (st != SA_OK) return st;
    if (lost) {
        if (lost[0] < 0 || lost[0] >= a.c.batch || lost[1] < 0 || lost[1] >= p.Hkv) return SA_ERR_INVALID_ARG;
        a.lost_b = lost[0], a.lost_head = lost[1], a.lost_tile = lost[2];
    }
    if (!cu_lens_host || window < 0 || sinks < 0) return SA_ERR_INVALID_ARG;
    if (o_dtype != SA_F16 && o_dtype != SA_BF16) return SA_ERR_UNSUPPORTED;
    int64_t longest = 0;
    for (int b = 0; b < a.c.batch; ++b) {
        const int64_t n = cu_lens_host[b + 1] - cu_lens_host[b];
        if (n < 0 || cu_lens_host[b] < 0) return SA_ERR_INVALID_ARG;
        if (n > (int64_t)a.c.max_pages * kPageTokens || n > (0x7fffffff - 256) / p.G) return SA_ERR_CAPACITY;
        longest = n > longest ? n : longest;
    }
    const int64_t n_rows = cu_lens_host[a.c.batch];
    if (longest == 0) return SA_OK;                                            // (a tensor without elements has no address)
    if (!Q || !O || !workspace) return SA_ERR_INVALID_ARG;
    if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(workspace, 256)) return SA_ERR_ALIGNMENT;
    if (n_rows > (int64_t)(PTRDIFF_MAX / 4) / ((int64_t)p.Hq * p.d)) return SA_ERR_CAPACITY;
    // a block may read queries of a row behind another's writing of its output
    const uintptr_t q0 = reinterpret_cast<uintptr_t>(Q), o0 = reinterpret_cast<uintptr_t>(O), bytes = (uintptr_t)n_rows * p.Hq * p.d * 2;
    if (q0 < o0 + bytes && o0 < q0 + bytes) return SA_ERR_INVALID_ARG;
    if (workspace_bytes < chunk_workspace(p, longest * p.G, chunk_blocks_most())) return SA_ERR_CAPACITY;
    a.Q = Q;
    a.O = O;
    a.workspace = static_cast<uint8_t*>(workspace);
    a.Hq = p.Hq;
    a.G = p.G;
    a.by_group = ChunkDivisor(p.G);
    a.window = window;
    a.sinks = sinks;
    a.bf16 = o_dtype == SA_BF16;
    const float log2e_over_root = 1.4426950408889634f / (p.d == 64 ? 8.0f : 11.313708498984761f);
    a.factor = log2e_over_root * (p.fp16 || p.fp4 ? 1.0f : p.int8 ? 1.0f / 127.0f : 256.0f);       // (power-of-two codes: operands of 2^-120 and 2^112)
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (!launch_kind(p, a, cu_lens_host, false, lost != nullptr, s) || !launch_kind(p, a, cu_lens_host, true, lost != nullptr, s)) {
        cudaGetLastError();                                                    // (not the next call's)
        return SA_ERR_CUDA;
    }
    return cudaGetLastError() == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

}  // namespace sa

using namespace sa;

extern "C" {

sa_status sa_chunk_workspace_bytes(const sa_config* cfg, int batch, int64_t n_tokens, size_t* out) {
    if (!out || batch <= 0 || n_tokens < 0) return SA_ERR_INVALID_ARG;
    Plan p;
    const sa_status st = make_plan(cfg, &p);
    if (st != SA_OK) return st;
    // (the longest chunk may have all tokens)
    *out = chunk_workspace(p, n_tokens > 0x7fffffff ? 0x7fffffff : n_tokens * p.G, chunk_blocks_most());
    return SA_OK;
}

sa_status sa_chunk_attention(const sa_config* cfg, const sa_cache* cache, const uint16_t* Q, const int64_t* cu_lens_host, int window, int sinks, void* O, int o_dtype,
                             void* workspace, size_t workspace_bytes, sa_stream stream) {
    return chunk_attention(cfg, cache, Q, cu_lens_host, window, sinks, O, o_dtype, workspace, workspace_bytes, nullptr, stream);
}

sa_status sa_debug_chunk_lost_copy(const sa_config* cfg, const sa_cache* cache, const uint16_t* Q, const int64_t* cu_lens_host, void* O, void* workspace, size_t workspace_bytes,
                                   int b, int kv_head, int tile, sa_stream stream) {
    const int lost[3] = {b, kv_head, tile};
    return chunk_attention(cfg, cache, Q, cu_lens_host, 0, 0, O, SA_F16, workspace, workspace_bytes, lost, stream);
}

}  // extern "C"

// sa_append_qkv: checks and launches, and the kernel for projections in binary16.
#include "sa_append.cuh"

namespace sa {

// The lengths behind a call in which a sequence has several blocks: a warp a sequence.
__global__ void __launch_bounds__(32) append_lengths_kernel(CacheArgs c, const __grid_constant__ AppendSeqs s) {
    pdl_wait();
    pdl_launch_dependents();
    const int b = s.b0 + blockIdx.x, n = s.tokens[blockIdx.x], start = c.seq_lens[b];
    if (n > 0 && __all_sync(0xffffffffu, append_pages(c, b, start, n, threadIdx.x, 32)) && threadIdx.x == 0) c.seq_lens[b] = start + n;
}

}  // namespace sa

using namespace sa;

extern "C" sa_status sa_append_qkv(const sa_config* cfg, const sa_cache* cache, const sa_rotary* rot, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                                   const void* V, int64_t v_stride, const int32_t* positions, int64_t n, const int64_t* cu_lens_host, uint16_t* Q_out, int bump_lens,
                                   sa_stream stream) {
    Plan p;
    sa_status st = make_plan(cfg, &p);
    if (st != SA_OK) return st;
    AppendArgs a;
    st = check_cache(p, cache, &a.c);
    if (st != SA_OK) return st;
    a.c.k = p.k;
    st = rotate_args(p, rot, {Q, K, V}, {q_stride, k_stride, v_stride}, {Q_out, nullptr, nullptr}, true, positions, n, &a.r);
    if (st != SA_OK) return st;
    if (!cu_lens_host) return SA_ERR_INVALID_ARG;
    int64_t total = 0, longest = 0;
    for (int b = 0; b < a.c.batch; ++b) {
        const int64_t T = cu_lens_host[b + 1] - cu_lens_host[b];
        if (T < 0 || cu_lens_host[b] < 0) return SA_ERR_INVALID_ARG;
        if (T > (int64_t)a.c.max_pages * kPageTokens) return SA_ERR_CAPACITY;
        total += T;
        longest = T > longest ? T : longest;
    }
    if (cu_lens_host[a.c.batch] > n) return SA_ERR_INVALID_ARG;                // (rows that are not there)
    const int tokens_most = p.d == 64 ? 4 : 2;
    if ((int64_t)tokens_most * 4 * p.Hkv * p.d > kAppendRowsMost) return SA_ERR_UNSUPPORTED;
    if (total == 0) return SA_OK;
    a.form = p.fp16 ? APPEND_FP16 : p.fp4 ? APPEND_FP4 : p.int8 ? APPEND_INT8 : p.nibble ? APPEND_DENSE : APPEND_BYTE;
    // As sa_rotate_qkv, a token a block while a wave of blocks holds them; but two tokens whose 4-bit values share bytes have to be in one.
    const int tokens = total <= (int64_t)sm_count() * (rot->dtype == SA_F32 ? 3 : 4) && (longest == 1 || !p.fp4) ? 1 : tokens_most;
    const bool several = longest > 1;                                          // (blocks of a sequence)
    a.bump = bump_lens && !several;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    for (int b0 = 0; b0 < a.c.batch; b0 += kAppendBatch) {
        a.s.b0 = b0;
        a.s.n = a.c.batch - b0 < kAppendBatch ? a.c.batch - b0 : kAppendBatch;
        a.s.blocks[0] = 0;
        for (int i = 0; i < a.s.n; ++i) {
            const int64_t T = cu_lens_host[b0 + i + 1] - cu_lens_host[b0 + i];
            a.s.row0[i] = cu_lens_host[b0 + i];
            a.s.tokens[i] = (int)T;
            a.s.blocks[i + 1] = a.s.blocks[i] + (int)(T ? (T + 2 * (tokens - 1)) / tokens : 0);        // (wherever in a group of places the first token falls)
        }
        if (a.s.blocks[a.s.n] == 0) continue;
        const cudaError_t e = rot->dtype == SA_F16 ? launch_append_typed<__half>(a, p.d, tokens, s) : rot->dtype == SA_BF16 ? launch_append_bf16(a, p.d, tokens, s) : launch_append_f32(a, p.d, tokens, s);
        if (e != cudaSuccess || (bump_lens && several && launch_pdl(append_lengths_kernel, dim3((unsigned)a.s.n), dim3(32), 0, s, a.c, a.s) != cudaSuccess)) {
            cudaGetLastError();                                                // (not the next call's)
            return SA_ERR_CUDA;
        }
    }
    return cudaGetLastError() == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

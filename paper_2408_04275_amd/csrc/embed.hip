// Embedding of a pack, and its gradient by sorted tokens.
#include "ops.h"
#include "vec8.h"

namespace mmt {
namespace {

// where a token's row comes from: row of the table, vocab + row of features, or -1
__device__ __forceinline__ int source_of(const EmbedArgs &a, int id) {
    if (id >= 0) return id < a.vocab ? id : -1;
    return id >= -a.features ? a.vocab - 1 - id : -1;
}

template <typename T>
__global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedArgs a) {
    const int chunks = a.H / 8;
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long)a.T * chunks) return;
    const int t = (int)(i / chunks), c = (int)(i % chunks), src = source_of(a, a.ids[t]);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (src >= 0) {
        const bool text = src < a.vocab;
        load8((text ? (const T *)a.table + (long)src * a.H : (const T *)a.rows + (long)(src - a.vocab) * a.H) + 8 * c, v);
        if (text) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        }
    }
    store8((T *)a.y + (long)t * a.H + 8 * c, v);
}

// place of each token in the order by (row, token), by counting the tokens in front of it
__global__ __launch_bounds__(256) void embed_rank_kernel(EmbedArgs a, int *order, int *key) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    const int mine = t < a.T ? source_of(a, a.ids[t]) : 0;
    int rank = 0;
    for (int u = 0; u < a.T; ++u) {
        const int other = source_of(a, a.ids[u]);
        rank += other < mine || (other == mine && u < t);
    }
    if (t < a.T) { order[rank] = t; key[rank] = mine; }
}

// a workgroup per place in the order: the first of its row's sums up the row
template <typename T, typename G>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, const int *order, const int *key) {
    const int i = blockIdx.x, row = key[i];
    if (row < 0 || (i > 0 && key[i - 1] == row)) return;
    const bool text = row < a.vocab;
    if (text ? !a.d_table : !a.d_rows) return;
    for (int c = threadIdx.x; c < a.H / 8; c += 256) {
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8];
        for (int j = i; j < a.T && key[j] == row; ++j) {
            load8((const T *)a.dy + (long)order[j] * a.H + 8 * c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += v[e];
        }
        if (!text) { store8((T *)a.d_rows + (long)(row - a.vocab) * a.H + 8 * c, s); continue; }
        G *out = (G *)a.d_table + (long)row * a.H + 8 * c;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] *= a.scale;
        if (a.accumulate) {
            load8(out, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += v[e];
        }
        store8(out, s);
    }
}

}  // namespace

hipError_t embed_fwd(int dtype, const EmbedArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const int grid = ceil_div((long)a.T * (a.H / 8), 256);
    if (dtype == DT_F32) embed_fwd_kernel<float><<<grid, 256, 0, st>>>(a);
    else embed_fwd_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

size_t embed_bwd_bytes(int T, int H) { return (size_t)T * 2 * sizeof(int) + 256; }

hipError_t embed_bwd(int dtype, const EmbedArgs &a, hipStream_t st) {
    hipError_t e = hipSuccess;
    const int table_dtype = a.table_f32 ? DT_F32 : dtype;
    if (a.d_table && !a.accumulate) e = fill_zero(a.d_table, (size_t)a.vocab * a.H, table_dtype, st);
    if (e == hipSuccess && a.d_rows) e = fill_zero(a.d_rows, (size_t)a.features * a.H, dtype, st);
    if (e != hipSuccess || a.T == 0) return e;
    int *order = (int *)a.ws, *key = order + a.T;
    embed_rank_kernel<<<ceil_div(a.T, 256), 256, 0, st>>>(a, order, key);
    if (dtype == DT_F32) embed_sum_kernel<float, float><<<a.T, 256, 0, st>>>(a, order, key);
    else if (a.table_f32) embed_sum_kernel<bf16_t, float><<<a.T, 256, 0, st>>>(a, order, key);
    else embed_sum_kernel<bf16_t, bf16_t><<<a.T, 256, 0, st>>>(a, order, key);
    return hipGetLastError();
}

}  // namespace mmt

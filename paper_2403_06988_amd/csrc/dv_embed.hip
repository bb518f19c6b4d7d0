// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//     out[n] = scale E[id_n]              (0 where id_n is no token)
//     dE[v]  = scale sum of dout[n] over the n with id_n = v, in order of n
//
// Both only move memory: the lookup 2 N D elements, the gradient N D read and
// the whole table written.  The gradient never adds with atomics: the rows are
// sorted by token (stable, so equal tokens keep their order), every sum runs in
// that order in fp32 and is rounded once, and two calls give the same bits.
#include "dv_train.h"

namespace dv {
namespace {

constexpr int kThreads = 256;

// Elements of one lane: as many bytes as row starts share alignment with.
template <typename T, int N>
struct Pack {
    T x[N];
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return widen(x); }
__device__ __forceinline__ void from_float(float y, float &x) { x = y; }
__device__ __forceinline__ void from_float(float y, uint16_t &x) { x = narrow(y); }

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p)
{
    Pack<T, N> v;
    __builtin_memcpy(&v, p, sizeof v);
    return v;
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, N> &v)
{
    __builtin_memcpy(p, &v, sizeof v);
}

// A lane group of 2^lanes_log2 lanes copies one row, N elements a lane at a
// time (the last lanes of a row that N does not divide go one by one).
template <typename T, int N>
__global__ __launch_bounds__(kThreads) void embed_kernel(const T *weight, int64_t ld, int V, int D, const int32_t *ids,
                                                          int rows, float scale, T *out, int lanes_log2)
{
    const int lanes = 1 << lanes_log2;
    const int64_t row = (int64_t)blockIdx.x * (kThreads >> lanes_log2) + (threadIdx.x >> lanes_log2);
    if (row >= rows)
        return;
    const int id = ids[row];
    const bool in = (uint32_t)id < (uint32_t)V;
    const T *src = weight + (int64_t)(in ? id : 0) * ld;
    T *dst = out + row * D;
    const int first = blockIdx.y * lanes + (threadIdx.x & (lanes - 1));
    const int whole = D / N;
    for (int j = first; j < whole; j += lanes * gridDim.y) {
        Pack<T, N> v = load_pack<T, N>(src + (int64_t)j * N);
#pragma unroll
        for (int i = 0; i < N; ++i)
            from_float(in ? to_float(v.x[i]) * scale : 0.f, v.x[i]);
        store_pack(dst + (int64_t)j * N, v);
    }
    for (int i = whole * N + first; i < D; i += lanes * gridDim.y)
        from_float(in ? to_float(src[i]) * scale : 0.f, dst[i]);
}

// ------------------------------------------------------------------ sorting
//
// A least-significant-digit radix sort of (token, row) pairs in digits of 6
// bits, one bin per lane of a wave.  Ids that are no token sort last, as V.
constexpr int kDigitBits = 6;
constexpr int kBins = 1 << kDigitBits;
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kKeysPerLane = 8;
constexpr int kSortKeys = kSortThreads * kKeysPerLane;  // of one block

int digits_of(int V)
{
    int bits = 1;
    while (bits < 31 && (V >> bits))
        ++bits;
    return (bits + kDigitBits - 1) / kDigitBits;
}

__device__ __forceinline__ int sort_key(int id, int V) { return (uint32_t)id < (uint32_t)V ? id : V; }

// Places of a wave's keys among its own keys of the same digit: `counts` (LDS,
// kBins words of the wave) holds the wave's running counts.
__device__ __forceinline__ int wave_rank(int digit, bool live, int *counts)
{
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const bool bit = digit >> b & 1;
        const uint64_t with = __ballot(bit);
        same &= bit ? with : ~with;
    }
    const int lane = threadIdx.x & (kWave - 1);
    const int before = __popcll(same & ((1ull << lane) - 1ull));
    int base = 0;
    if (live)
        base = counts[digit];
    wave_lds_sync();
    if (live && before == 0)
        counts[digit] = base + __popcll(same);
    wave_lds_sync();
    return base + before;
}

// counts[w][d] -> keys of digit d in the waves before w (+ keys of smaller
// digits with BASE); sums[d] the block's keys of digit d.  kBins x kSortWaves
// words by all threads of the block.
__device__ __forceinline__ void scan_counts(int (*counts)[kBins], int *sums, bool base)
{
    __syncthreads();
    if (threadIdx.x < kBins) {
        int total = 0;
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = counts[w][threadIdx.x];
            counts[w][threadIdx.x] = total;
            total += c;
        }
        int before = total;  // inclusive scan over the digits of the wave
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int up = __shfl_up(before, d);
            if ((int)threadIdx.x >= d)
                before += up;
        }
        before -= total;
        sums[threadIdx.x] = total;
        if (base)
            for (int w = 0; w < kSortWaves; ++w)
                counts[w][threadIdx.x] += before;
    }
    __syncthreads();
}

// Block 0 sorts up to kSortKeys rows in LDS; with `fill` the other blocks
// write zeros over the table at the same time (the sums then overwrite the
// rows of the tokens that occur).
struct SortShared {
    int key[kSortKeys];
    int row[kSortKeys];
    int counts[kSortWaves][kBins];
    int sums[kBins];
};

__device__ __forceinline__ void fill_zeros(char *p, size_t bytes, size_t block, size_t blocks, int threads)
{
    // the table is contiguous: its ends byte pair by byte pair, the rest in 16 bytes
    const size_t head = (16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15;
    const size_t h = head < bytes ? head : bytes;
    const size_t vecs = (bytes - h) / 16;
    const size_t tail = (bytes - h) - vecs * 16;
    uint4 *q = reinterpret_cast<uint4 *>(p + h);
    const size_t stride = blocks * threads;
    for (size_t i = block * threads + threadIdx.x; i < vecs; i += stride)
        q[i] = make_uint4(0, 0, 0, 0);
    if (block == 0) {
        uint16_t *a = reinterpret_cast<uint16_t *>(p), *b = reinterpret_cast<uint16_t *>(p + h + vecs * 16);
        for (size_t i = threadIdx.x; i < h / 2; i += threads)
            a[i] = 0;
        for (size_t i = threadIdx.x; i < tail / 2; i += threads)
            b[i] = 0;
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_block_kernel(const int32_t *ids, int rows, int V, int digits,
                                                                   int *keys, int *order, char *fill, size_t fill_bytes)
{
    __shared__ SortShared sh;
    if (blockIdx.x) {
        fill_zeros(fill, fill_bytes, blockIdx.x - 1, gridDim.x - 1, kSortThreads);
        return;
    }
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int per_wave = (rows + kSortWaves - 1) / kSortWaves;  // each wave owns one run of the keys
    const int w0 = wave * per_wave, w1 = w0 + per_wave < rows ? w0 + per_wave : rows;
    for (int i = threadIdx.x; i < rows; i += kSortThreads) {
        sh.key[i] = sort_key(ids[i], V);
        sh.row[i] = i;
    }
    for (int d = 0; d < digits; ++d) {
        int key[kKeysPerLane], row[kKeysPerLane], rank[kKeysPerLane];
        sh.counts[wave][lane] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kKeysPerLane; ++j) {
            const int i = w0 + j * kWave + lane;
            const bool live = i < w1;
            key[j] = live ? sh.key[i] : 0;
            row[j] = live ? sh.row[i] : 0;
            rank[j] = 0;
            if (w0 + j * kWave < w1)
                rank[j] = wave_rank(key[j] >> (d * kDigitBits) & (kBins - 1), live, sh.counts[wave]);
        }
        scan_counts(sh.counts, sh.sums, true);
#pragma unroll
        for (int j = 0; j < kKeysPerLane; ++j)
            if (w0 + j * kWave + lane < w1) {
                const int at = sh.counts[wave][key[j] >> (d * kDigitBits) & (kBins - 1)] + rank[j];
                sh.key[at] = key[j];
                sh.row[at] = row[j];
            }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < rows; i += kSortThreads) {
        keys[i] = sh.key[i];
        order[i] = sh.row[i];
    }
}

// More rows: per digit, each block counts its kSortKeys keys, then places
// them behind the keys of smaller digits and of the blocks before it.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t *ids, const int *keys, int rows, int V,
                                                                   int digit, int *hist, char *fill, size_t fill_bytes,
                                                                   int blocks)
{
    if ((int)blockIdx.x >= blocks) {
        fill_zeros(fill, fill_bytes, blockIdx.x - blocks, gridDim.x - blocks, kSortThreads);
        return;
    }
    __shared__ int count[kBins];
    if (threadIdx.x < kBins)
        count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortKeys;
    for (int j = 0; j < kKeysPerLane; ++j) {
        const int64_t i = first + j * kSortThreads + threadIdx.x;
        if (i < rows)
            atomicAdd(&count[(ids ? sort_key(ids[i], V) : keys[i]) >> (digit * kDigitBits) & (kBins - 1)], 1);
    }
    __syncthreads();
    if (threadIdx.x < kBins)
        hist[(size_t)threadIdx.x * blocks + blockIdx.x] = count[threadIdx.x];
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t *ids, const int *keys, const int *order,
                                                                   int rows, int V, int digit, const int *hist,
                                                                   int *keys_out, int *order_out)
{
    __shared__ int counts[kSortWaves][kBins];
    __shared__ int sums[kBins];
    __shared__ int before[kBins], total[kBins];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int blocks = gridDim.x;
    // keys of each digit in the blocks before this one, and in all
    for (int d = wave; d < kBins; d += kSortWaves) {
        int mine = 0, all = 0;
        for (int b = lane; b < blocks; b += kWave) {
            const int c = hist[(size_t)d * blocks + b];
            all += c;
            mine += b < (int)blockIdx.x ? c : 0;
        }
#pragma unroll
        for (int s = 32; s; s >>= 1) {
            all += __shfl_xor(all, s);
            mine += __shfl_xor(mine, s);
        }
        if (lane == 0) {
            before[d] = mine;
            total[d] = all;
        }
    }
    counts[wave][lane] = 0;
    __syncthreads();
    const int64_t w0 = (int64_t)blockIdx.x * kSortKeys + wave * (kSortKeys / kSortWaves);
    int key[kKeysPerLane], row[kKeysPerLane], rank[kKeysPerLane];
#pragma unroll
    for (int j = 0; j < kKeysPerLane; ++j) {
        const int64_t i = w0 + j * kWave + lane;
        const bool live = i < rows;
        key[j] = live ? (ids ? sort_key(ids[i], V) : keys[i]) : 0;
        row[j] = live ? (ids ? (int)i : order[i]) : 0;
    }
#pragma unroll
    for (int j = 0; j < kKeysPerLane; ++j)
        rank[j] = wave_rank(key[j] >> (digit * kDigitBits) & (kBins - 1), w0 + j * kWave + lane < rows, counts[wave]);
    scan_counts(counts, sums, false);
    if (threadIdx.x < kBins) {  // keys of smaller digits, in all blocks
        int t = total[threadIdx.x], inc = t;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int up = __shfl_up(inc, d);
            if ((int)threadIdx.x >= d)
                inc += up;
        }
        sums[threadIdx.x] = before[threadIdx.x] + inc - t;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeysPerLane; ++j)
        if (w0 + j * kWave + lane < rows) {
            const int d = key[j] >> (digit * kDigitBits) & (kBins - 1);
            const int at = sums[d] + counts[wave][d] + rank[j];
            keys_out[at] = key[j];
            order_out[at] = row[j];
        }
}

// -------------------------------------------------------------------- sums
//
// The sorted rows are cut into chunks of `chunk`; a block sums one chunk's
// runs of equal tokens over a slab of columns.  A run that lies inside its
// chunk is finished there.  Of a run that crosses chunks, each chunk keeps its
// part in fp32: slot 0 of the chunk if the run came in from the chunk before,
// slot 1 if it began here; the second kernel adds the parts in chunk order.
template <typename T, int N>
__device__ __forceinline__ void emit(T *grad, int64_t at, float (&acc)[N], float scale, bool accumulate)
{
    Pack<T, N> v;
    if (accumulate)
        v = load_pack<T, N>(grad + at);
#pragma unroll
    for (int i = 0; i < N; ++i)
        from_float(accumulate ? to_float(v.x[i]) + acc[i] * scale : acc[i] * scale, v.x[i]);
    store_pack(grad + at, v);
}

template <typename T, int N>
__global__ __launch_bounds__(kThreads) void sum_chunks_kernel(const T *grad_out, int64_t ld, int D, const int *keys,
                                                               const int *order, int rows, int V, int chunk,
                                                               float scale, bool accumulate, T *grad, float *parts)
{
    const int c = blockIdx.x;
    const int64_t from = (int64_t)c * chunk;
    const int64_t to = from + chunk < rows ? from + chunk : rows;
    const int col = (blockIdx.y * blockDim.x + threadIdx.x) * N;
    if (col >= D)
        return;
    const bool came = from > 0 && keys[from - 1] == keys[from];
    const bool goes = to < rows && keys[to] == keys[to - 1];
    constexpr int U = 8;
    float acc[N] = {};
    bool first = true;  // still in the chunk's first run
    int key = keys[from];
    for (int64_t i = from; i < to && key < V; i += U) {
        Pack<T, N> v[U];
        int k[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = i + u < to ? i + u : to - 1;
            k[u] = i + u < to ? keys[at] : V;
            v[u] = load_pack<T, N>(grad_out + (int64_t)order[at] * ld + col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k[u] != key) {
                if (key < V && !(i + u >= to)) {
                    if (first && came) {
                        float *p = parts + ((int64_t)c * 2) * D + col;
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            p[e] = acc[e];
                    } else {
                        emit<T, N>(grad, (int64_t)key * D + col, acc, scale, accumulate);
                    }
                    first = false;
                    key = k[u];
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        acc[e] = 0.f;
                }
            }
            if (i + u < to && key < V)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    acc[e] += to_float(v[u].x[e]);
        }
    }
    if (key >= V)
        return;
    if ((first && came) || goes) {
        float *p = parts + ((int64_t)c * 2 + (first && came ? 0 : 1)) * D + col;
#pragma unroll
        for (int e = 0; e < N; ++e)
            p[e] = acc[e];
    } else {
        emit<T, N>(grad, (int64_t)key * D + col, acc, scale, accumulate);
    }
}

template <typename T, int N>
__global__ __launch_bounds__(kThreads) void sum_parts_kernel(int D, const int *keys, int rows, int V, int chunk,
                                                              int chunks, float scale, bool accumulate, T *grad,
                                                              const float *parts)
{
    const int c = blockIdx.x;
    const int64_t from = (int64_t)c * chunk;
    const int64_t to = from + chunk;
    if (to >= rows)
        return;
    const int key = keys[to - 1];
    // a run that begins in this chunk and goes on into the next
    if (key >= V || keys[to] != key || (from > 0 && keys[from] == key && keys[from - 1] == key))
        return;
    const int col = (blockIdx.y * blockDim.x + threadIdx.x) * N;
    if (col >= D)
        return;
    float acc[N];
    const float *own = parts + ((int64_t)c * 2 + 1) * D + col;
#pragma unroll
    for (int e = 0; e < N; ++e)
        acc[e] = own[e];
    for (int d = c + 1; d < chunks && keys[(int64_t)d * chunk] == key; ++d) {
        const float *p = parts + ((int64_t)d * 2) * D + col;
#pragma unroll
        for (int e = 0; e < N; ++e)
            acc[e] += p[e];
    }
    emit<T, N>(grad, (int64_t)key * D + col, acc, scale, accumulate);
}

// Chunks of 32 rows, doubled until there are at most kMaxChunks.
constexpr int kMaxChunks = 512;

int chunk_of(int rows)
{
    int c = 32;
    while ((int64_t)c * kMaxChunks < rows)
        c *= 2;
    return c;
}

struct EmbedLayout {
    size_t keys[2], order[2], hist, parts, bytes;
};

EmbedLayout embed_layout(int rows, int hidden)
{
    EmbedLayout l{};
    const size_t n = align_up((size_t)(rows > 0 ? rows : 1) * 4, 256);
    size_t at = 0;
    for (int i = 0; i < 2; ++i) {
        l.keys[i] = at;
        at += n;
        l.order[i] = at;
        at += n;
    }
    const size_t blocks = ((size_t)rows + kSortKeys - 1) / kSortKeys;
    l.hist = at;
    at += align_up((blocks ? blocks : 1) * kBins * 4, 256);
    l.parts = at;
    // chunk_of's chunks, or more (the size never falls as rows grow)
    const size_t chunks = rows < 32 * kMaxChunks ? ((size_t)rows + 31) / 32 : (size_t)kMaxChunks;
    at += align_up(chunks * 2 * (size_t)hidden * 4 + 4, 256);
    l.bytes = at;
    return l;
}

// Bytes that every row start of a [..][ld] array is a multiple of, 16 at most.
int row_alignment(const void *p, int64_t ld, int elt)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * elt) | 16;
    return (int)(a & (~a + 1));
}

template <typename T, int N>
hipError_t embed_with(const T *weight, int64_t ld, int V, int D, const int32_t *ids, int rows, float scale, T *out,
                      hipStream_t stream)
{
    const int vecs = (D + N - 1) / N;
    int log2 = 0;
    while (log2 < 8 && (1 << log2) < vecs)
        ++log2;
    const int rows_per_block = kThreads >> log2;
    const int gx = (rows + rows_per_block - 1) / rows_per_block;
    int gy = (vecs + (1 << log2) - 1) >> log2;
    gy = gy < 64 ? gy : 64;
    embed_kernel<T, N><<<dim3(gx, gy), kThreads, 0, stream>>>(weight, ld, V, D, ids, rows, scale, out, log2);
    return last_launch();
}

template <typename T, int N>
hipError_t sums_with(const T *grad_out, int64_t ld, int D, const int *keys, const int *order, int rows, int V,
                     float scale, bool accumulate, T *grad, float *parts, hipStream_t stream)
{
    const int chunk = chunk_of(rows), chunks = (rows + chunk - 1) / chunk;
    const int vecs = (D + N - 1) / N;
    int threads = kWave;
    while (threads < kThreads && threads < vecs)
        threads *= 2;
    const dim3 grid(chunks, (vecs + threads - 1) / threads);
    sum_chunks_kernel<T, N><<<grid, threads, 0, stream>>>(grad_out, ld, D, keys, order, rows, V, chunk, scale,
                                                          accumulate, grad, parts);
    hipError_t e = last_launch();
    if (e != hipSuccess || chunks == 1)
        return e;
    sum_parts_kernel<T, N><<<grid, threads, 0, stream>>>(D, keys, rows, V, chunk, chunks, scale, accumulate, grad,
                                                         parts);
    return last_launch();
}

}  // namespace

hipError_t launch_embed(const void *weight, int64_t ld_w, int dtype, int V, int hidden, const int32_t *ids, int rows,
                        float scale, void *out, hipStream_t stream)
{
    const int elt = dtype == 1 ? 2 : 4;
    const int in = row_alignment(weight, ld_w, elt), to = row_alignment(out, hidden, elt);
    const int bytes = in < to ? in : to;
    if (dtype == 1) {
        const uint16_t *w = static_cast<const uint16_t *>(weight);
        uint16_t *o = static_cast<uint16_t *>(out);
        if (bytes == 16)
            return embed_with<uint16_t, 8>(w, ld_w, V, hidden, ids, rows, scale, o, stream);
        return embed_with<uint16_t, 2>(w, ld_w, V, hidden, ids, rows, scale, o, stream);
    }
    const float *w = static_cast<const float *>(weight);
    float *o = static_cast<float *>(out);
    if (bytes == 16)
        return embed_with<float, 4>(w, ld_w, V, hidden, ids, rows, scale, o, stream);
    return embed_with<float, 1>(w, ld_w, V, hidden, ids, rows, scale, o, stream);
}

size_t embed_backward_workspace_bytes(int rows, int hidden, int V)
{
    (void)V;
    return embed_layout(rows, hidden).bytes;
}

hipError_t launch_embed_backward(const void *grad_out, int64_t ld, int dtype, int rows, int hidden, const int32_t *ids,
                                 int V, float scale, bool accumulate, void *grad_weight, void *workspace,
                                 hipStream_t stream)
{
    const EmbedLayout l = embed_layout(rows, hidden);
    char *ws = static_cast<char *>(workspace);
    int *keys[2], *order[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = reinterpret_cast<int *>(ws + l.keys[i]);
        order[i] = reinterpret_cast<int *>(ws + l.order[i]);
    }
    int *hist = reinterpret_cast<int *>(ws + l.hist);
    float *parts = reinterpret_cast<float *>(ws + l.parts);
    const int elt = dtype == 1 ? 2 : 4;
    const size_t table = accumulate ? 0 : (size_t)V * (size_t)hidden * elt;
    char *fill = static_cast<char *>(grad_weight);
    const size_t per_block = (size_t)kSortThreads * 16 * 4;
    size_t fill_blocks = (table + per_block - 1) / per_block;
    fill_blocks = fill_blocks < 2048 ? fill_blocks : 2048;
    const int digits = digits_of(V);
    int at = 0;  // which of the two buffers holds the sorted rows
    hipError_t e;
    if (rows <= kSortKeys) {
        sort_block_kernel<<<(unsigned)(1 + fill_blocks), kSortThreads, 0, stream>>>(
            ids, rows, V, digits, keys[0], order[0], fill, table);
        if ((e = last_launch()) != hipSuccess)
            return e;
    } else {
        const int blocks = (rows + kSortKeys - 1) / kSortKeys;
        for (int d = 0; d < digits; ++d) {
            const int32_t *first = d ? nullptr : ids;
            const size_t extra = d ? 0 : fill_blocks;
            sort_count_kernel<<<(unsigned)(blocks + extra), kSortThreads, 0, stream>>>(
                first, keys[at], rows, V, d, hist, fill, table, blocks);
            if ((e = last_launch()) != hipSuccess)
                return e;
            sort_place_kernel<<<blocks, kSortThreads, 0, stream>>>(first, keys[at], order[at], rows, V, d, hist,
                                                                   keys[1 - at], order[1 - at]);
            if ((e = last_launch()) != hipSuccess)
                return e;
            at = 1 - at;
        }
    }
    if (rows == 0)
        return hipSuccess;
    const int in = row_alignment(grad_out, ld, elt), to = row_alignment(grad_weight, hidden, elt);
    const bool wide = in == 16 && to == 16 && hidden % (16 / elt) == 0;
    if (dtype == 1) {
        const uint16_t *g = static_cast<const uint16_t *>(grad_out);
        uint16_t *w = static_cast<uint16_t *>(grad_weight);
        if (wide)
            return sums_with<uint16_t, 8>(g, ld, hidden, keys[at], order[at], rows, V, scale, accumulate, w, parts, stream);
        return sums_with<uint16_t, 1>(g, ld, hidden, keys[at], order[at], rows, V, scale, accumulate, w, parts, stream);
    }
    const float *g = static_cast<const float *>(grad_out);
    float *w = static_cast<float *>(grad_weight);
    if (wide)
        return sums_with<float, 4>(g, ld, hidden, keys[at], order[at], rows, V, scale, accumulate, w, parts, stream);
    return sums_with<float, 1>(g, ld, hidden, keys[at], order[at], rows, V, scale, accumulate, w, parts, stream);
}

}  // namespace dv

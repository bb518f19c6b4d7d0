// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//     out[n] = scale E[id_n]              (0 where id_n is no token)
//     dE[v]  = scale sum of dout[n] over the n with id_n = v, in order of n
//
// Both only move memory: the lookup 2 N D elements, the gradient N D read and
// the whole table written.  The gradient never adds with atomics: the rows are
// sorted by token (stable, so equal tokens keep their order), every sum runs in
// that order in fp32 and is rounded once, and two calls give the same bits.
//
// 8,192 rows of 2,048 bf16 in a table of 128,256: the lookup takes 16.3 us (4.1 TB/s), the
// gradient 113 us (560 MB, most of them the table's zeros: 5.0 TB/s).
#include "dv_train.h"

namespace dv {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return widen(x); }
__device__ __forceinline__ void from_float(float y, float &x) { x = y; }
__device__ __forceinline__ void from_float(float y, uint16_t &x) { x = narrow(y); }

// Elements of one lane, 16 bytes from any element on; rows end where they end, so
// a row's last lane may hold fewer (`n` of them).
template <typename T>
struct Pack {
    static constexpr int kN = 16 / sizeof(T);
    Words w;
    __device__ __forceinline__ T get(int i) const { return element<T>(w, i); }
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= kN) {
            w = load_words(p);
        } else {
            T x[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i)
                x[i] = i < n ? p[i] : T(0);
            set(x);
        }
    }
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if (n >= kN) {
            store_words(p, w);
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (i < n)
                    p[i] = get(i);
        }
    }
    __device__ __forceinline__ void set(const T (&x)[kN])
    {
        union {
            T t[kN];
            Words w;
        } u;
#pragma unroll
        for (int i = 0; i < kN; ++i)
            u.t[i] = x[i];
        w = u.w;
    }
    // f(i) in T, for every element
    template <typename F>
    __device__ __forceinline__ void fill(F &&f)
    {
        T x[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i)
            from_float(f(i), x[i]);
        set(x);
    }
};

// A lane group of 2^lanes_log2 lanes copies ROWS rows at once, `step` apart.
template <typename T, int ROWS>
__global__ __launch_bounds__(kThreads) void embed_kernel(const T *weight, int64_t ld, int V, int D, const int32_t *ids,
                                                          int rows, int64_t step, float scale, T *out, int lanes_log2)
{
    constexpr int N = Pack<T>::kN;
    const int lanes = 1 << lanes_log2;
    const int64_t row = (int64_t)blockIdx.x * (kThreads >> lanes_log2) + (threadIdx.x >> lanes_log2);
    if (row >= step)
        return;
    int id[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        id[r] = row + r * step < rows ? ids[row + r * step] : -1;
    for (int64_t col = (int64_t)(blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * N; col < D;
         col += (int64_t)lanes * gridDim.y * N) {
        const int n = (int)(D - col);
        Pack<T> v[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            v[r].load(weight + (int64_t)((uint32_t)id[r] < (uint32_t)V ? id[r] : 0) * ld + col, n);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool in = (uint32_t)id[r] < (uint32_t)V;
            Pack<T> y;
            y.fill([&](int i) { return in ? to_float(v[r].get(i)) * scale : 0.f; });
            if (row + r * step < rows)
                y.store(out + (row + r * step) * D + col, n);
        }
    }
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
    // lanes of the same digit, as 32-bit halves: a bit's ballot, or its complement where
    // this lane's bit is clear (the sort is bound by its one compute unit's vector issue)
    const uint64_t alive = __ballot(live);
    uint32_t lo = (uint32_t)alive, hi = (uint32_t)(alive >> 32);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const int mine = (int)((uint32_t)digit << (31 - b)) >> 31;  // -1 or 0
        const uint64_t with = __ballot(mine != 0);
        lo &= ~((uint32_t)with ^ (uint32_t)mine);
        hi &= ~((uint32_t)(with >> 32) ^ (uint32_t)mine);
    }
    const int before = (int)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
    int base = 0;
    if (live)
        base = counts[digit];
    wave_lds_sync();
    if (live && before == 0)
        counts[digit] = base + __popc(lo) + __popc(hi);
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
// write zeros over the table (or its first rows) at the same time (the sums then
// overwrite the rows of the tokens that occur).
struct SortShared {
    int key[kSortKeys];
    int row[kSortKeys];
    int counts[kSortWaves][kBins];
    int sums[kBins];
};

// Zeros over [p, p + bytes) by `threads` threads, of which this is number `thread`.
__device__ __forceinline__ void fill_zeros(char *p, size_t bytes, size_t thread, size_t threads)
{
    // the ends byte pair by byte pair, the rest in 16 bytes
    const size_t head = (16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15;
    const size_t h = head < bytes ? head : bytes;
    const size_t vecs = (bytes - h) / 16;
    const size_t tail = (bytes - h) - vecs * 16;
    uint4 *q = reinterpret_cast<uint4 *>(p + h);
    for (size_t i = thread; i < vecs; i += threads)
        q[i] = make_uint4(0, 0, 0, 0);
    uint16_t *a = reinterpret_cast<uint16_t *>(p), *b = reinterpret_cast<uint16_t *>(p + h + vecs * 16);
    if (thread < h / 2)  // less than 8 of each
        a[thread] = 0;
    if (thread < tail / 2)
        b[thread] = 0;
}

__global__ __launch_bounds__(kSortThreads) void sort_block_kernel(const int32_t *ids, int rows, int V, int digits,
                                                                   int *keys, int *order, char *fill, size_t fill_bytes)
{
    __shared__ SortShared sh;
    if (blockIdx.x) {
        fill_zeros(fill, fill_bytes, (size_t)(blockIdx.x - 1) * kSortThreads + threadIdx.x,
                   (size_t)(gridDim.x - 1) * kSortThreads);
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
        fill_zeros(fill, fill_bytes, (size_t)(blockIdx.x - blocks) * kSortThreads + threadIdx.x,
                   (size_t)(gridDim.x - blocks) * kSortThreads);
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
template <typename T>
__device__ __forceinline__ void emit(T *grad, const float (&acc)[Pack<T>::kN], int n, float scale, bool accumulate)
{
    Pack<T> v;
    if (accumulate)
        v.load(grad, n);
    Pack<T> y;
    y.fill([&](int i) { return accumulate ? to_float(v.get(i)) + acc[i] * scale : acc[i] * scale; });
    y.store(grad, n);
}

// Zeros over the rows of tokens from `first` to V that no key names: a wave looks
// `group` tokens up at once, and fills each run of them that does not occur.
template <typename T>
__device__ __forceinline__ void fill_absent(T *grad, int D, const int *keys, int rows, int first, int V, int group,
                                            int64_t wave, int64_t waves)
{
    const int lane = threadIdx.x & (kWave - 1);
    for (int64_t from = first + wave * group; from < V; from += waves * group) {
        const int64_t v = from + lane;
        bool absent = lane < group && v < V;
        int lo = 0, hi = rows;  // the first key that is not below v
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (keys[mid] < v)
                lo = mid + 1;
            else
                hi = mid;
        }
        if (lo < rows && keys[lo] == v)
            absent = false;
        uint64_t todo = __ballot(absent);
        while (todo) {
            const int at = __builtin_ctzll(todo);
            const uint64_t up = ~(todo >> at);
            const int n = up ? __builtin_ctzll(up) : kWave;
            fill_zeros(reinterpret_cast<char *>(grad + (from + at) * D), (size_t)n * D * sizeof(T), lane, kWave);
            todo = at + n < kWave ? todo >> (at + n) << (at + n) : 0;
        }
    }
}

// Blocks past the chunks' fill the rows from `fill_from` on, `fill_group` at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void sum_chunks_kernel(const T *grad_out, int64_t ld, int D, const int *keys,
                                                               const int *order, int rows, int V, int chunk, int chunks,
                                                               float scale, bool accumulate, T *grad, float *parts,
                                                               int part_ld, int fill_from, int fill_group)
{
    constexpr int N = Pack<T>::kN;
    constexpr int U = 8;  // rows on their way at once
    const int c = blockIdx.x;
    if (c >= chunks) {
        const int waves = blockDim.x / kWave;
        const int64_t block = (int64_t)(c - chunks) * gridDim.y + blockIdx.y;
        fill_absent(grad, D, keys, rows, fill_from, V, fill_group, block * waves + threadIdx.x / kWave,
                    (int64_t)(gridDim.x - chunks) * gridDim.y * waves);
        return;
    }
    const int64_t from = (int64_t)c * chunk;
    const int64_t to = from + chunk < rows ? from + chunk : rows;
    const int col = (blockIdx.y * blockDim.x + threadIdx.x) * N;
    if (col >= D)
        return;
    const int n = D - col;
    const bool came = from > 0 && keys[from - 1] == keys[from];
    const bool goes = to < rows && keys[to] == keys[to - 1];
    float acc[N] = {};
    bool first = true;  // still in the chunk's first run
    int key = keys[from];
    const auto keep = [&](int slot) {
        float *p = parts + ((int64_t)c * 2 + slot) * part_ld + col;
#pragma unroll
        for (int e = 0; e < N; e += 4)
            *reinterpret_cast<float4 *>(p + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    };
    for (int64_t i = from; i < to && key < V; i += U) {
        Pack<T> v[U];
        int k[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = i + u < to ? i + u : to - 1;
            k[u] = keys[at];
            v[u].load(grad_out + (int64_t)order[at] * ld + col, n);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= to)
                break;
            if (k[u] != key) {
                if (key < V) {
                    if (first && came)
                        keep(0);
                    else
                        emit<T>(grad + (int64_t)key * D + col, acc, n, scale, accumulate);
                }
                first = false;
                key = k[u];
#pragma unroll
                for (int e = 0; e < N; ++e)
                    acc[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < N; ++e)
                acc[e] += to_float(v[u].get(e));
        }
    }
    if (key >= V)
        return;
    if (first && came)
        keep(0);
    else if (goes)
        keep(1);
    else
        emit<T>(grad + (int64_t)key * D + col, acc, n, scale, accumulate);
}

// N floats of a part (16-byte aligned: parts are a multiple of 8 floats apart).
template <int N>
__device__ __forceinline__ void read_part(float (&x)[N], const float *p)
{
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        const float4 f = *reinterpret_cast<const float4 *>(p + e);
        x[e] = f.x;
        x[e + 1] = f.y;
        x[e + 2] = f.z;
        x[e + 3] = f.w;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sum_parts_kernel(int D, const int *keys, int rows, int V, int chunk,
                                                              int chunks, float scale, bool accumulate, T *grad,
                                                              const float *parts, int part_ld)
{
    constexpr int N = Pack<T>::kN;
    const int c = blockIdx.x;
    const int64_t from = (int64_t)c * chunk;
    const int64_t to = from + chunk;
    if (to >= rows)
        return;
    const int key = keys[to - 1];
    // a run that begins in this chunk and goes on into the next
    if (key >= V || keys[to] != key || (from > 0 && keys[from] == key && keys[from - 1] == key))
        return;
    // the chunks that the run goes on into, a wave's lanes looking at 64 at a time
    int last = c;
    for (;;) {
        const int d = last + 1 + (int)(threadIdx.x & (kWave - 1));
        const uint64_t on = __ballot(d < chunks && keys[(int64_t)(d < chunks ? d : c) * chunk] == key);
        if (~on) {
            last += __builtin_ctzll(~on);
            break;
        }
        last += kWave;
    }
    const int col = (blockIdx.y * blockDim.x + threadIdx.x) * N;
    if (col >= D)
        return;
    float acc[N];
    const float *p = parts + ((int64_t)c * 2 + 1) * part_ld + col;
    read_part(acc, p);
    p += part_ld;  // slot 0 of the next chunk
    constexpr int U = 8;
    for (int d = c + 1; d <= last; d += U) {
        float part[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u)
            read_part(part[u], p + (int64_t)(d + u <= last ? u : 0) * 2 * part_ld);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e)
                acc[e] += d + u <= last ? part[u][e] : 0.f;
        p += (int64_t)U * 2 * part_ld;
    }
    emit<T>(grad + (int64_t)key * D + col, acc, D - col, scale, accumulate);
}

// Chunks of 8 rows, doubled until there are at most kMaxChunks: short ones keep
// many rows on their way, and a token's parts are added one after the other.
constexpr int kLeastChunk = 8;
constexpr int kMaxChunks = 1024;

int chunk_of(int rows)
{
    int c = kLeastChunk;
    while ((int64_t)c * kMaxChunks < rows)
        c *= 2;
    return c;
}

int part_stride(int hidden) { return (hidden + 7) & ~7; }

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
    const size_t chunks = rows < kLeastChunk * kMaxChunks ? ((size_t)rows + kLeastChunk - 1) / kLeastChunk
                                                          : (size_t)kMaxChunks;
    at += align_up(chunks * 2 * (size_t)part_stride(hidden) * 4 + 4, 256);
    l.bytes = at;
    return l;
}

template <typename T, int ROWS>
hipError_t embed_with(const T *weight, int64_t ld, int V, int D, const int32_t *ids, int rows, float scale, T *out,
                      hipStream_t stream)
{
    const int vecs = (D + Pack<T>::kN - 1) / Pack<T>::kN;
    int log2 = 0;
    while (log2 < 8 && (1 << log2) < vecs)
        ++log2;
    const int64_t step = ((int64_t)rows + ROWS - 1) / ROWS;
    const int64_t per_block = kThreads >> log2;
    int gy = (vecs + (1 << log2) - 1) >> log2;
    gy = gy < 64 ? gy : 64;
    embed_kernel<T, ROWS><<<dim3((unsigned)((step + per_block - 1) / per_block), gy), kThreads, 0, stream>>>(
        weight, ld, V, D, ids, rows, step, scale, out, log2);
    return last_launch();
}

// Four rows a lane once that leaves the compute units enough blocks: each row's
// load waits for its id.
template <typename T>
hipError_t embed(const void *weight, int64_t ld, int V, int D, const int32_t *ids, int rows, float scale, void *out,
                 hipStream_t stream)
{
    const T *w = static_cast<const T *>(weight);
    T *o = static_cast<T *>(out);
    if ((int64_t)rows * D >= (int64_t)4 * 1024 * kThreads * Pack<T>::kN)
        return embed_with<T, 4>(w, ld, V, D, ids, rows, scale, o, stream);
    return embed_with<T, 1>(w, ld, V, D, ids, rows, scale, o, stream);
}

constexpr size_t kFillBytes = 32 << 10;  // of the rows that a wave looks up at once

template <typename T>
hipError_t sums(const void *grad_out, int64_t ld, int D, const int *keys, const int *order, int rows, int V, float scale,
                bool accumulate, void *grad_weight, float *parts, int fill_from, hipStream_t stream)
{
    const T *g = static_cast<const T *>(grad_out);
    T *w = static_cast<T *>(grad_weight);
    const int chunk = chunk_of(rows), chunks = (rows + chunk - 1) / chunk;
    const int vecs = (D + Pack<T>::kN - 1) / Pack<T>::kN;
    int threads = kWave;
    while (threads < kThreads && threads < vecs)
        threads *= 2;
    const dim3 grid(chunks, (vecs + threads - 1) / threads);
    const int part_ld = part_stride(D);
    int group = kWave;
    while (group > 1 && (size_t)group * D * sizeof(T) > kFillBytes)
        group /= 2;
    const int64_t fill_waves = ((int64_t)V - fill_from + group - 1) / group;
    const int64_t per_x = (int64_t)(threads / kWave) * grid.y;
    const dim3 with_fill((unsigned)(chunks + (fill_waves + per_x - 1) / per_x), grid.y);
    sum_chunks_kernel<T><<<with_fill, threads, 0, stream>>>(g, ld, D, keys, order, rows, V, chunk, chunks, scale, accumulate,
                                                            w, parts, part_ld, fill_from, group);
    hipError_t e = last_launch();
    if (e != hipSuccess || chunks == 1)
        return e;
    sum_parts_kernel<T><<<grid, threads, 0, stream>>>(D, keys, rows, V, chunk, chunks, scale, accumulate, w, parts,
                                                      part_ld);
    return last_launch();
}

// The rows of the table that are filled while the sort runs: as many as its time allows
// (about 8 us and 1.3 more for 1,000 rows, at 7 GB/ms), where the rest can be filled while the
// sums run, which leave the memory idle.  All of them and this rule (us): 64 rows x 2048 x
// 128,256 bf16 112 and 95, 1,000 x 4096 x 128,256 203 and 195, 8,192 x 2048 x 128,256 122 and
// 113, 4,000 x 1024 x 256,000 fp32 202 and 191.  Rows under 2 KiB leave short runs (8,192 x
// 512 x 256,000 bf16: 56 and 59), and more than kSortKeys rows sort in several launches.
int64_t early_rows(int rows, int V, size_t row_bytes)
{
    if (rows == 0 || rows > kSortKeys || row_bytes < 2048)
        return V;
    const int64_t early = (int64_t)((((size_t)48 << 20) + (size_t)rows * (16 << 10)) / row_bytes);
    return early < V ? early : V;
}

}  // namespace

hipError_t launch_embed(const void *weight, int64_t ld_w, int dtype, int V, int hidden, const int32_t *ids, int rows,
                        float scale, void *out, hipStream_t stream)
{
    return dtype == 1 ? embed<uint16_t>(weight, ld_w, V, hidden, ids, rows, scale, out, stream)
                      : embed<float>(weight, ld_w, V, hidden, ids, rows, scale, out, stream);
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
    const size_t row_bytes = (size_t)hidden * elt;
    const int64_t early = early_rows(rows, V, row_bytes);
    const size_t table = accumulate ? 0 : (size_t)early * row_bytes;
    const int fill_from = accumulate ? V : (int)early;
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
    return dtype == 1 ? sums<uint16_t>(grad_out, ld, hidden, keys[at], order[at], rows, V, scale, accumulate, grad_weight,
                                       parts, fill_from, stream)
                      : sums<float>(grad_out, ld, hidden, keys[at], order[at], rows, V, scale, accumulate, grad_weight,
                                    parts, fill_from, stream);
}

}  // namespace dv

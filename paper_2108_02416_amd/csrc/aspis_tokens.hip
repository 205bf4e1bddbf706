// aspis_tokens.hip -- gfx950 kernels of the embedding lookup, its gradient by
// sorted tokens, and dropout from a counter-based generator.
//
// Results are functions of the values, the sizes and the seed alone: sums are
// cut by sizes and joined in order, without atomics, and dropout's mask comes
// from an element's position, so that workers with the same file return the
// same bits.
#include "aspis_tokens.h"

#include "aspis_elements.h"

namespace aspis {

namespace {

constexpr int kBlock = 256;
constexpr int64_t kMaxGrid = int64_t(1) << 22;   // workgroups of one launch

// N elements of type E from p as floats, and back; N is E::V or a multiple.
template <typename E, int N, Use USE = Use::Again>
__device__ __forceinline__ void load_floats(Ptr<E> p, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += E::V) {
        float y[E::V];
        E::unpack(load_vec<E, USE>(p + i), y);
#pragma unroll
        for (int j = 0; j < E::V; ++j) x[i + j] = y[j];
    }
}
template <typename E, int N, Use USE = Use::Again>
__device__ __forceinline__ void store_floats(MutPtr<E> p, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += E::V) {
        float y[E::V];
#pragma unroll
        for (int j = 0; j < E::V; ++j) y[j] = x[i + j];
        store_vec<E, USE>(p + i, E::pack(y));
    }
}

// log2 of the lanes that hold `vecs` vectors, at most 256
int lane_shift(int64_t vecs) {
    int s = 0;
    while (s < 8 && (int64_t(1) << s) < vecs) ++s;
    return s;
}
unsigned grid_for(int64_t items, int per_block) {
    const int64_t blocks = (items + per_block - 1) / per_block;
    return (unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid);
}

// ---------------------------------------------------------------------------
// embedding lookup

// 2^shift lanes take U rows at a time.  Memory bounds it: 16,384 rows of
// 2,048 f32 out of 32,003, to bf16, in 21.4 us, 5.2 TB/s, with two rows at a
// time and stores past the cache (in turn: 22.7 us so, one at a time 30.3, four
// 22.8, two with plain stores 27.4).  Few rows are latency, either way as fast
// (4,096 bf16 rows 5.6 us; 8,192 7.1 in pairs and 9.7 one by one), and their
// results, one by one, stay in the cache.
constexpr int64_t kPairRows = 4096;   // workgroups of single rows from which on pairs are taken

template <typename EI, typename EO, int U>
__global__ __launch_bounds__(kBlock) void embed_kernel(EmbedArgs a, int shift) {
    constexpr int N = EI::V > EO::V ? EI::V : EO::V, W = N / EI::V;
    const int lane = (int)threadIdx.x & ((1 << shift) - 1);
    const int64_t per_block = (kBlock >> shift) * U;
    const int64_t nv = a.d / N;
    for (int64_t row0 = blockIdx.x * per_block + (threadIdx.x >> shift) * U; row0 < a.n;
         row0 += gridDim.x * per_block) {
        int token[U];
#pragma unroll
        for (int u = 0; u < U; ++u) token[u] = a.tokens.get(row0 + u < a.n ? row0 + u : a.n - 1, a.vocab);
        auto from = [&](int u) { return (Ptr<EI>)a.table + (token[u] < 0 ? 0 : token[u]) * a.ld; };
        auto to = [&](int u) { return (MutPtr<EO>)a.out + (row0 + u) * a.ldo; };
        // (0 times a negative scale is -0)
        auto scale = [&](int u) { return token[u] < 0 ? 0.0f : a.scale; };
        for (int64_t v = lane; v < nv; v += 1 << shift) {
            u32x4 x[U][W];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    x[u][w] = (u32x4){0, 0, 0, 0};
                    if (token[u] >= 0) x[u][w] = load_vec<EI>(from(u) + v * N + w * EI::V);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float y[N];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    float z[EI::V];
                    EI::unpack(x[u][w], z);
#pragma unroll
                    for (int j = 0; j < EI::V; ++j) y[w * EI::V + j] = z[j] * scale(u);
                }
                if (row0 + u < a.n) store_floats<EO, N, U == 1 ? Use::Again : Use::Once>(to(u) + v * N, y);
            }
        }
        for (int64_t i = nv * N + lane; i < a.d; i += 1 << shift)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (row0 + u < a.n)
                    to(u)[i] = put_product<EO>(token[u] >= 0 ? EI::get(from(u)[i]) * a.scale : 0.0f);
    }
}

// ---------------------------------------------------------------------------
// its gradient: the tokens sorted

// The tokens in order (vocab where a token is none, so that those come last)
// and the positions they were at, those of equal tokens in order.
struct Sorted {
    uint32_t *token, *at;
};

// The value of the lane whose index differs in the bits of M.
template <int M>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
    const int w = (int)v;
    if constexpr (M == 1) return __builtin_amdgcn_update_dpp(0, w, 0xB1, 0xF, 0xF, true);
    else if constexpr (M == 2) return __builtin_amdgcn_update_dpp(0, w, 0x4E, 0xF, 0xF, true);
    else if constexpr (M == 4)   // the mirrors of 8 and of 4 lanes
        return __builtin_amdgcn_update_dpp(
            0, __builtin_amdgcn_update_dpp(0, w, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);
    else if constexpr (M == 8)   // half a turn of 16 lanes
        return __builtin_amdgcn_update_dpp(0, w, 0x128, 0xF, 0xF, true);
    else return __shfl_xor(v, M, 64);
}
template <int M>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
    return (uint64_t)lane_xor<M>((uint32_t)(v >> 32)) << 32 | lane_xor<M>((uint32_t)v);
}

// A bitonic sort of kSortRun keys, kSortKeys a thread: key r of thread t is
// number t * kSortKeys + r.  Keys meet in a thread, between lanes, and
// through LDS between waves.  No two are equal (but those past the end).
// Its steps, one after the other, bound it: 5.3 us for one run.
constexpr int kSortKeys = kSortRun / kBlock;

// Step J of the merge to sequences of K.
template <int K, int J, typename T>
__device__ __forceinline__ void sort_step(T (&key)[kSortKeys], T *lds) {
    const int t = threadIdx.x;
    if constexpr (J < kSortKeys) {
#pragma unroll
        for (int r = 0; r < kSortKeys; ++r) {
            if (r & J) continue;
            const bool up = ((t * kSortKeys + r) & K) == 0;
            const T x = key[r], y = key[r | J];
            const bool swap = (y < x) == up;
            key[r] = swap ? y : x;
            key[r | J] = swap ? x : y;
        }
    } else {
        constexpr int M = J / kSortKeys;   // the other key is that many threads away
        const bool low = ((t * kSortKeys & K) == 0) == ((t & M) == 0);   // it keeps the lower
        if constexpr (M >= 64) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kSortKeys; ++r) lds[r * kBlock + t] = key[r];
            __syncthreads();
        }
#pragma unroll
        for (int r = 0; r < kSortKeys; ++r) {
            T other;
            if constexpr (M >= 64) other = lds[r * kBlock + (t ^ M)];
            else other = lane_xor<M>(key[r]);
            key[r] = (other < key[r]) == low ? other : key[r];
        }
    }
    if constexpr (J > 1) sort_step<K, J / 2>(key, lds);
}
template <int K, typename T>
__device__ __forceinline__ void sort_run(T (&key)[kSortKeys], T *lds) {
    if constexpr (K > 2) sort_run<K / 2>(key, lds);
    sort_step<K, K / 2>(key, lds);
}

// Zeros in rows of the table's gradient but those whose bit in `skip` is set,
// 2^shift lanes a row.
template <typename EO>
__device__ __forceinline__ void fill_rows(const EmbedGradArgs &a, int64_t first, int rows, int shift,
                                          const uint32_t *skip) {
    const int lane = (int)threadIdx.x & ((1 << shift) - 1);
    const float zero[EO::V] = {};
    const int64_t nv = a.d / EO::V;
    for (int r = (int)threadIdx.x >> shift; r < rows; r += kBlock >> shift) {
        if (skip != nullptr && (skip[r / 32] >> r % 32 & 1)) continue;
        const MutPtr<EO> to = (MutPtr<EO>)a.out + (first + r) * a.ldo;
        for (int64_t v = lane; v < nv; v += 1 << shift) store_floats<EO>(to + v * EO::V, zero);
        for (int64_t i = nv * EO::V + lane; i < a.d; i += 1 << shift) to[i] = EO::put(0.0f);
    }
}

constexpr int kZeroRows = 256;   // rows of a workgroup that fills in zeros, at most
// Bytes of them: 32,768 tokens into 32,003 rows of 2,048 f32, 110 us without,
// 107.5 with 64 MB, 104 with 96 or 160, 108 with 300.  Not where the tokens
// are more than twice the rows, most of which would be written twice: 100,000
// into 8,003 rows of 1,024, 96 us without, 99.7 with 96 MB.
constexpr int64_t kEarlyBytes = 96 << 20;

// Rows that are filled with zeros while the tokens are sorted, which leaves
// memory idle: the last ones, from row `from` on, those with tokens too, which
// are written again afterwards.
struct EarlyRows {
    int64_t from;
    int rows, shift;   // of a workgroup; log2 of the lanes a row
    int64_t runs;      // workgroups that sort, before those that fill
};

// Runs of kSortRun tokens, a workgroup each.  T: 32 bits where a token and
// its place in the run fit them, else 64.
template <typename T>
__global__ __launch_bounds__(kBlock) void sort_runs_kernel(EmbedGradArgs a, Sorted out, EarlyRows early) {
    if (blockIdx.x >= early.runs) {
        const int64_t first = early.from + ((int64_t)blockIdx.x - early.runs) * early.rows;
        const int rows = (int)(a.vocab - first < early.rows ? a.vocab - first : early.rows);
        with_type(a.out_dtype, [&](auto e) {
            fill_rows<decltype(e)>(a, first, rows, early.shift, nullptr);
        });
        return;
    }
    constexpr int kBits = 10;
    static_assert(kSortRun == 1 << kBits, "");
    __shared__ T lds[kSortRun];
    const int64_t base = (int64_t)blockIdx.x * kSortRun;
    const int n = (int)(a.n - base < kSortRun ? a.n - base : kSortRun);
    T key[kSortKeys];
#pragma unroll
    for (int r = 0; r < kSortKeys; ++r) {
        const int i = r * kBlock + threadIdx.x;
        key[r] = ~(T)0;   // above every token's
        if (i < n) {
            const int token = a.tokens.get(base + i, a.vocab);
            key[r] = (T)(token < 0 ? (uint32_t)a.vocab : (uint32_t)token) << kBits | (T)i;
        }
    }
    sort_run<kSortRun>(key, lds);
#pragma unroll
    for (int r = 0; r < kSortKeys; ++r) {
        const int i = (int)threadIdx.x * kSortKeys + r;
        if (i >= n) continue;
        out.token[base + i] = (uint32_t)(key[r] >> kBits);
        out.at[base + i] = (uint32_t)base + (uint32_t)(key[r] & (kSortRun - 1));
    }
}

// Merges runs in LDS, kMergeRuns * kSortRun tokens at most: a token's place
// is the number of tokens before it in every run (the lower ones, and the
// equal ones of earlier runs), found by binary searches.  SHARE threads share
// a token's, each doing all of its own a step at a time: the more, the more
// workgroups there are, which all hold the whole.  Latency of the searches
// bounds it.  Gradients of 32,768 tokens, rows of 64, us: with 8 threads 43.6, 4
// 47.1, 2 54.4; of 65,536, 61.2, 58.7 and 65.8; of 131,072, 81.1, 77.3 and 75.4.
constexpr int kMergeBlock = 1024;

template <int SHARE>
__global__ __launch_bounds__(kMergeBlock) void merge_runs_kernel(Sorted in, Sorted out, int64_t n) {
    constexpr int kGroup = kMergeRuns * kSortRun, R = kMergeRuns / SHARE;
    constexpr int V = kGroup / (4 * kMergeBlock);
    // runs begin 16 bytes apart in the banks: searches of several of them
    // begin in the same places (8.6 us of 32,768 tokens without)
    constexpr int kRun = kSortRun + 4;
    __shared__ u32x4 vecs[kMergeRuns * kRun / 4];
    const uint32_t *all = (const uint32_t *)vecs;
    const int per_block = kMergeBlock / SHARE;
    const int64_t group = (int64_t)blockIdx.x * per_block / kGroup * kGroup;
    const int size = (int)(n - group < kGroup ? n - group : kGroup);
    u32x4 v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {   // (the last vector: into the array's padding)
        const int i = k * kMergeBlock + threadIdx.x;
        v[k] = *((const u32x4 *)(in.token + group) + (i * 4 < size ? i : 0));
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int i = k * kMergeBlock + threadIdx.x;
        vecs[i + i / (kSortRun / 4)] = v[k];
    }
    __syncthreads();
    const int i = (int)((int64_t)blockIdx.x * per_block - group) + (int)threadIdx.x / SHARE;
    const int own = i / kSortRun, first = threadIdx.x % SHARE;
    const uint32_t token = i < size ? all[i + own * (kRun - kSortRun)] : 0;
    uint32_t below[R];
#pragma unroll
    for (int k = 0; k < R; ++k) below[k] = 0;
    for (int step = kSortRun; step > 0; step /= 2) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int r = first + k * SHARE, at = (int)below[k] + step;
            const bool inside = (at <= kSortRun) & (r * kSortRun + at <= size);
            const uint32_t other = all[inside ? r * kRun + at - 1 : 0];
            if (inside & ((other < token) | ((r < own) & (other == token)))) below[k] = at;
        }
    }
    uint32_t place = 0;
#pragma unroll
    for (int k = 0; k < R; ++k)
        place += first + k * SHARE == own ? (uint32_t)(i % kSortRun) : below[k];
#pragma unroll
    for (int m = 1; m < SHARE; m *= 2) place += __shfl_xor(place, m, 64);
    if (i >= size || first != 0) return;
    out.token[group + place] = token;
    out.at[group + place] = in.at[group + i];
}

// The first position whose token is not below `token`; a wave looks at 64
// places at once.
__device__ __forceinline__ int64_t first_not_below(const uint32_t *sorted, int64_t n, uint32_t token) {
    int64_t low = 0, high = n;   // the answer lies in [low, high]
    while (low < high) {
        const int64_t step = (high - low + 63) / 64;
        const int64_t at = low + (int64_t)(threadIdx.x % 64) * step;
        const int below = __popcll(__ballot(at < high && sorted[at] < token));
        if (below == 0) return low;
        const int64_t last = low + (below - 1) * step;   // the last place looked at that is below
        low = last + 1;
        high = last + step < high ? last + step : high;
    }
    return low;
}

// Longer runs where they are, kMergeWide at a time.  A workgroup's tokens are
// neighbours in a run: its waves find where the lowest and the highest of
// them would come in the other runs, and its threads search between, in all
// runs a step at a time.  Latency bounds it: 8.4 us for 65,536 tokens.
constexpr int kMergeWide = 16;

__global__ __launch_bounds__(kBlock) void merge_long_kernel(Sorted in, Sorted out, int64_t n,
                                                            int64_t length) {
    __shared__ int64_t bounds[kMergeWide][2];
    const int64_t i0 = (int64_t)blockIdx.x * kBlock, i = i0 + threadIdx.x;   // (all of one run)
    const int64_t group = i0 / (length * kMergeWide) * (length * kMergeWide);
    const int64_t left = n - group;
    const int own = (int)((i0 - group) / length);
    const int runs = (int)(left < length * kMergeWide ? (left + length - 1) / length : kMergeWide);
    auto size = [&](int r) { return left - r * length < length ? left - r * length : length; };
    const uint32_t lowest = in.token[i0], highest = in.token[i0 + kBlock <= n ? i0 + kBlock - 1 : n - 1];
    for (int p = threadIdx.x / 64; p < 2 * runs; p += kBlock / 64) {
        const int r = p / 2;
        const int64_t at = r == own ? 0 : first_not_below(in.token + group + r * length, size(r),
                                                          p % 2 ? highest + 1 : lowest);
        if (threadIdx.x % 64 == 0) bounds[r][p % 2] = at;
    }
    __syncthreads();
    int64_t widest = 0;
    for (int r = 0; r < runs; ++r) {
        const int64_t w = bounds[r][1] - bounds[r][0];
        if (w > widest) widest = w;
    }
    if (i >= n) return;
    const uint32_t token = in.token[i];
    int64_t below[kMergeWide];
#pragma unroll
    for (int r = 0; r < kMergeWide; ++r) below[r] = r < runs ? bounds[r][0] : 0;
    int64_t step = 1;
    while (step <= widest) step *= 2;
    for (step /= 2; step > 0; step /= 2) {
#pragma unroll
        for (int r = 0; r < kMergeWide; ++r) {
            if (r >= runs || r == own) continue;
            const int64_t at = below[r] + step;
            if (at > bounds[r][1]) continue;
            const uint32_t other = in.token[group + r * length + at - 1];
            if (other < token || (r < own && other == token)) below[r] = at;
        }
    }
    int64_t place = i - group - own * length;
#pragma unroll
    for (int r = 0; r < kMergeWide; ++r) place += below[r];
    out.token[group + place] = token;
    out.at[group + place] = in.at[i];
}

// ---------------------------------------------------------------------------
// its gradient: the sums

// A segment is the sorted positions of one token.  A group of lanes takes the
// segments that begin in its window of positions, each to its end; a long
// one is cut at the borders of blocks of two windows, and its pieces, of a
// block at most, are the windows' that they begin in, to be joined by another
// launch.  Long: it holds all of a block after the first border in it.  So
// at a border within a segment it is cut where it also holds the position a
// block before or after, and few segments are cut at all.
struct SumArgs {
    EmbedGradArgs a;
    Sorted sorted;
    float *partial;      // [blocks][2][row]: the piece from the block's border on, and
                         // the one before it
    int64_t row;
    int shift;           // log2 of a window's positions
    int64_t windows;
    int slabs, tail;     // waves that share a row's whole vectors; 1 for the elements after
    int64_t sum_blocks;  // workgroups of windows; the others fill rows with zeros:
    int zero_rows, zero_shift;   // so many each, 2^shift lanes a row, up to row
    int64_t zero_end;            // zero_end
    int64_t first;       // the launch's first workgroup
};

// What nothing writes while a kernel runs, read through the scalar cache
// where the address is the same in all lanes.
#define CONSTANT __attribute__((address_space(4)))
typedef const uint32_t CONSTANT *ConstWords;

// Whether position i holds this token.  (Always a load, so that several of
// them are on their way at once.)
__device__ __forceinline__ bool holds(const SumArgs &g, int64_t i, uint32_t token) {
    const bool inside = (uint64_t)i < (uint64_t)g.a.n;
    return (((ConstWords)g.sorted.token)[inside ? i : 0] == token) & inside;
}

// N elements of a row from column col on, scaled, to the result.
template <typename EO, int N>
__device__ __forceinline__ void finish_row(const EmbedGradArgs &a, uint32_t token, int64_t col,
                                           const float (&x)[N]) {
    const MutPtr<EO> to = (MutPtr<EO>)a.out + (int64_t)token * a.ldo + col;
    if constexpr (N == 1) {
        const float v = x[0] * a.scale;
        *to = put_product<EO>(a.accumulate ? EO::get(*to) + v : v);
    } else {
        float y[N] = {};
        if (a.accumulate) load_floats<EO, N>((Ptr<EO>)to, y);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = a.accumulate ? y[j] + x[j] * a.scale : x[j] * a.scale;
        store_floats<EO, N>(to, y);
    }
}


// Zeros in those of a workgroup's g.zero_rows rows that no token names.
template <typename EO>
__device__ __forceinline__ void zero_rows(const SumArgs &g, int64_t block) {
    __shared__ uint32_t there[kZeroRows / 32];
    __shared__ int64_t bounds[2];   // the rows' positions
    const EmbedGradArgs &a = g.a;
    const uint32_t *sorted = g.sorted.token;
    const int64_t first = block * g.zero_rows;
    const int rows = (int)(g.zero_end - first < g.zero_rows ? g.zero_end - first : g.zero_rows);
    if (threadIdx.x < kZeroRows / 32) there[threadIdx.x] = 0;
    if (threadIdx.x < 128) {
        const int64_t at = first_not_below(sorted, a.n, (uint32_t)(first + threadIdx.x / 64 * rows));
        if (threadIdx.x % 64 == 0) bounds[threadIdx.x / 64] = at;
    }
    __syncthreads();
    const int64_t begin = bounds[0], end = bounds[1];
    if (end - begin <= 4 * kBlock) {   // few: all of them
        for (int64_t i = begin + threadIdx.x; i < end; i += kBlock) {
            const uint32_t of = sorted[i] - (uint32_t)first;
            atomicOr(&there[of / 32], 1u << of % 32);
        }
    } else if ((int)threadIdx.x < rows) {   // a row each
        const uint32_t token = (uint32_t)first + threadIdx.x;
        int64_t low = begin, high = end;
        while (low < high) {
            const int64_t mid = (low + high) / 2;
            if (sorted[mid] < token) low = mid + 1;
            else high = mid;
        }
        if (low < end && sorted[low] == token) atomicOr(&there[threadIdx.x / 32], 1u << threadIdx.x % 32);
    }
    __syncthreads();
    fill_rows<EO>(a, first, rows, g.zero_shift, there);
}

// N columns of a lane from col on, of the segments and pieces that begin in
// a window: the same window in all lanes, so that what is decided by tokens
// is decided in scalar registers.
template <typename EI, typename EO, int N>
__device__ __forceinline__ void sum_window(const SumArgs &g, int64_t window, int64_t col) {
    constexpr int W = N == 1 ? 1 : N / EI::V, U = 8;
    const EmbedGradArgs &a = g.a;
    const uint32_t none = (uint32_t)a.vocab;
    const int64_t span = int64_t(2) << g.shift;   // positions of a block
    const int64_t p0 = window << g.shift, p1 = p0 + span / 2 < a.n ? p0 + span / 2 : a.n;
    const ConstWords tokens = (ConstWords)g.sorted.token, places = (ConstWords)g.sorted.at;

    const bool border = (window & 1) == 0;
    const int64_t next = border ? p0 + span : p0 + span / 2;   // the border from p1 on
    auto look = [&](int64_t i) { return tokens[(uint64_t)i < (uint64_t)a.n ? i : p0]; };
    auto inside = [&](int64_t i) { return (uint64_t)i < (uint64_t)a.n; };
    uint32_t token = tokens[p0], last = tokens[p1 - 1], w0 = look(p0 - 1), w1 = look(p0 - span),
             w2 = look(p0 + span), w3 = look(p1), w4 = look(next), w5 = look(next - span),
             w6 = look(next + span);
    // all of them on their way before the first is waited for
    asm volatile("" : "+s"(token), "+s"(last), "+s"(w0), "+s"(w1), "+s"(w2), "+s"(w3), "+s"(w4),
                 "+s"(w5), "+s"(w6));
    if (token >= none) return;
    const uint32_t first = token;
    const bool begun = inside(p0 - 1) & (w0 == first), before = inside(p0 - span) & (w1 == first),
               after = inside(p0 + span) & (w2 == first), goes_on = inside(p1) & (w3 == last);
    const bool at_next = inside(next) & (w4 == last), by_next = inside(next - span) & (w5 == last),
               past_next = inside(next + span) & (w6 == last);
    // the segment at p0: begun before, and not cut here, it is another window's
    const bool long_one = border & (after | (begun & before));
    const bool skip = begun & !long_one;
    // where the last one ends, at the latest, and whether it is cut there
    const bool tail_cut = goes_on & at_next & (by_next | past_next);
    const int64_t end = !goes_on ? p1 : tail_cut ? next : next + span < a.n ? next + span : a.n;

    enum { kSkip, kPiece, kSegment } kind = skip ? kSkip : long_one ? kPiece : kSegment;
    float acc[N] = {};
    auto flush = [&](bool cut) {
        if (kind == kSkip) return;
        if (kind == kSegment && !cut) {
            finish_row<EO, N>(a, token, col, acc);
            return;
        }
        const int64_t slot = kind == kPiece ? window : (end >> (g.shift + 1)) * 2 + 1;
        float GLOBAL *to = (float GLOBAL *)g.partial + slot * g.row + col;
        if constexpr (N == 1) *to = acc[0];
        else store_floats<F32, N>(to, acc);
    };
    for (int64_t p = p0; p < end; p += U) {
        typedef uint32_t Eight __attribute__((ext_vector_type(8), aligned(4)));
        // (past the end of the array: its padding)
        const Eight tok = *(const Eight CONSTANT *)(tokens + p);
        const Eight place = *(const Eight CONSTANT *)(places + p);
        uint32_t now[U];
        typename EI::T one[U];
        u32x4 x[U][W];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            now[u] = tok[u];
            // no more of this window, or not its
            if ((p + u >= end) | ((p + u >= p1) & (now[u] != last))) now[u] = none;
            const Ptr<EI> from = (Ptr<EI>)a.grad + (int64_t)place[u] * a.ld + col;
            if constexpr (N == 1) one[u] = EI::put(0.0f);
#pragma unroll
            for (int i = 0; i < W; ++i) x[u][i] = (u32x4){0, 0, 0, 0};
            if ((now[u] >= none) | (skip & (now[u] == first))) continue;
            if constexpr (N == 1) {
                one[u] = *from;
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) x[u][i] = load_vec<EI, Use::Once>(from + i * EI::V);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (now[u] != token) {
                flush(false);
                if (now[u] >= none) return;
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] = 0.0f;
                token = now[u];
                kind = kSegment;
            }
            if constexpr (N == 1) {
                acc[0] += EI::get(one[u]);
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    float y[EI::V];
                    EI::unpack(x[u][i], y);
#pragma unroll
                    for (int j = 0; j < EI::V; ++j) acc[i * EI::V + j] += y[j];
                }
            }
        }
    }
    flush(tail_cut);
}

// A wave for every window and 64 vectors of a row, eight rows on their way at
// a time.  Memory bounds it: of 32,768 rows of 2,048 bf16, with the rows of
// zeros that sorting left over, 300 MB in 58 us, 5.2 TB/s.
template <typename EI, typename EO>
__global__ __launch_bounds__(kBlock) void sum_rows_kernel(SumArgs g) {
    constexpr int N = EI::V > EO::V ? EI::V : EO::V;
    const int64_t block = g.first + blockIdx.x;
    if (block >= g.sum_blocks) {
        zero_rows<EO>(g, block - g.sum_blocks);
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int64_t item = block * (kBlock / 64) + wave;
    const int64_t window = item / (g.slabs + g.tail);
    const int slab = (int)(item % (g.slabs + g.tail));
    if (window >= g.windows) return;
    const int64_t whole = g.a.d / N * N;
    if (slab < g.slabs) {
        const int64_t col = ((int64_t)slab * 64 + lane) * N;
        if (col < whole) sum_window<EI, EO, N>(g, window, col);
    } else if (whole + lane < g.a.d) {
        sum_window<EI, EO, 1>(g, window, whole + lane);
    }
}

// Joins the pieces of a long segment in their order: a workgroup for the
// first border in it and 256 columns; most find none and end.  Latency bounds
// it: 4.3 to 5.3 us after 32,768 or 65,536 tokens with a common one among them.
template <typename EO>
__global__ __launch_bounds__(kBlock) void join_pieces_kernel(SumArgs g, int64_t slabs) {
    constexpr int N = 4, WAVES = kBlock / 64;
    __shared__ float sums[WAVES][64 * N];
    const EmbedGradArgs &a = g.a;
    const int64_t item = g.first + blockIdx.x;
    const int64_t block = item / slabs, span = int64_t(2) << g.shift;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = (item % slabs * 64 + lane) * N;
    const int64_t p = block * span;
    const ConstWords tokens = (ConstWords)g.sorted.token;
    const uint32_t token = tokens[p];
    if (token >= (uint32_t)a.vocab || !holds(g, p + span, token) || holds(g, p - span, token)) return;
    const int64_t head = holds(g, p - 1, token);   // a piece before the border
    // the blocks that begin with it: `high` is past them
    const int64_t blocks = (a.n + span - 1) / span;
    int64_t low = block + 1, high = blocks;   // low begins with it
    const int64_t near = low + lane;
    const uint64_t are = __ballot(near < blocks && g.sorted.token[near < blocks ? near * span : p] == token);
    if (~are != 0) {
        high = low + __ffsll((unsigned long long)~are) - 1;
    } else {
        low += 63;
        while (high - low > 1) {
            const int64_t mid = (low + high) / 2;
            if (tokens[mid * span] == token) low = mid;
            else high = mid;
        }
    }
    const int64_t count = high - block + head;
    const int64_t share = (count + WAVES - 1) / WAVES;
    const int64_t from = wave * share, to = from + share < count ? from + share : count;
    float acc[N] = {};
    if (col < a.d) {
        constexpr int U = 8;
        for (int64_t k = from; k < to; k += U) {
            u32x4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = k + u < to ? k + u : to - 1;
                const int64_t slot = head && i == 0 ? block * 2 + 1 : (block + i - head) * 2;
                w[u] = *(const u32x4 GLOBAL *)((const float GLOBAL *)g.partial + slot * g.row + col);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u < to)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] += __uint_as_float(w[u][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sums[wave][lane * N + j] = acc[j];
    __syncthreads();
    if (wave != 0 || col >= a.d) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float v = sums[0][lane * N + j];
        for (int w = 1; w < WAVES; ++w) v += sums[w][lane * N + j];
        if (col + j >= a.d) continue;
        const MutPtr<EO> out = (MutPtr<EO>)a.out + (int64_t)token * a.ldo + col + j;
        v *= a.scale;
        *out = put_product<EO>(a.accumulate ? EO::get(*out) + v : v);
    }
}

// ---------------------------------------------------------------------------
// its gradient, of few tokens, in one launch

// Up to kFewTokens tokens, not too many a row, are not sorted as a whole: a
// workgroup takes some rows of the table and 64 vectors of them, picks the
// rows' tokens out of all of them, sorts those few, and its waves share them
// evenly; sums of a segment that several waves hold are joined in LDS, in
// order.  Latency bounds it, in one launch instead of three: 515 tokens of 257
// f32 into 4,099 rows in 9.1 us, 15.0 by sorting all.  (Columns after the last
// vector take workgroups of their own: at 257, half of them.)
constexpr int kFewRows = 64;   // of a workgroup, at most

struct FewArgs {
    EmbedGradArgs a;
    int rows;          // of a workgroup
    int slabs, tail;   // as in SumArgs
    int64_t first;     // the launch's first workgroup
};

// The table rows' tokens in order: (row << 10 | position), and which rows
// have any.
struct FewList {
    uint32_t key[kSortRun + 16], other[kSortRun];   // (as many as sort_run takes)
    uint64_t there;
    int count[kFewTokens / 64];
};
static_assert(kFewTokens <= kSortRun && kFewTokens % kBlock == 0 && kFewTokens <= 1 << 10, "");

// Fills the list; returns its length.
__device__ __forceinline__ int few_tokens(const EmbedGradArgs &a, int64_t first, int rows, FewList &l) {
    constexpr int K = kFewTokens / kBlock, WAVES = kBlock / 64;
    const int t = threadIdx.x, lane = t % 64, wave = t / 64;
    int row[K];
    uint64_t mine[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * kBlock + t;
        const int64_t token = i < a.n ? (int64_t)a.tokens.get(i, a.vocab) : -1;
        row[k] = token >= first && token < first + rows ? (int)(token - first) : -1;
        mine[k] = __ballot(row[k] >= 0);
        if (lane == 0) l.count[k * WAVES + wave] = __popcll(mine[k]);
    }
    if (t == 0) l.there = 0;
    __syncthreads();
    int m = 0, from[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) from[k] = m;
            m += l.count[k * WAVES + w];
        }
    m = __builtin_amdgcn_readfirstlane(m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (row[k] < 0) continue;
        const int at = from[k] + __popcll(mine[k] & ((uint64_t(1) << lane) - 1));
        l.other[at] = (uint32_t)row[k] << 10 | (uint32_t)(k * kBlock + t);
        atomicOr((unsigned long long *)&l.there, 1ull << row[k]);
    }
    __syncthreads();
    if (m <= kBlock) {   // a key's place is the number of lower ones (no two are equal)
        const uint32_t key = t < m ? l.other[t] : ~0u;
        int place = 0;
        for (int j = 0; j < m; ++j) place += l.other[j] < key;
        if (t < m) l.key[place] = key;
    } else {
        uint32_t key[kSortKeys];
#pragma unroll
        for (int r = 0; r < kSortKeys; ++r) key[r] = r * kBlock + t < m ? l.other[r * kBlock + t] : ~0u;
        __syncthreads();
        sort_run<kSortRun>(key, l.other);
#pragma unroll
        for (int r = 0; r < kSortKeys; ++r) l.key[t * kSortKeys + r] = key[r];
    }
    __syncthreads();
    return m;
}

template <typename EI, typename EO, int N>
__device__ __forceinline__ void few_sums(const FewArgs &g, FewList &l, float (*part)[2][64 * 8],
                                         int m, int64_t first, int rows, int64_t col, bool active) {
    constexpr int W = N == 1 ? 1 : N / EI::V, U = 16 / W, WAVES = kBlock / 64;
    const EmbedGradArgs &a = g.a;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int share = m > 4 * WAVES ? (m + WAVES - 1) / WAVES : 4;
    const int begin = wave * share, end = begin + share < m ? begin + share : m;
    auto row_at = [&](int p) {   // the row of the list's entry p; -1 outside of it
        return __builtin_amdgcn_readfirstlane(p >= 0 && p < m ? (int)(l.key[p] >> 10) : -1);
    };
    if (begin < end) {
        int row = row_at(begin);
        bool open = row_at(begin - 1) == row;
        float acc[N] = {};
        auto flush = [&](bool goes_on) {
            if (!open && !goes_on) {
                if (active) finish_row<EO, N>(a, (uint32_t)(first + row), col, acc);
                return;
            }
#pragma unroll
            for (int j = 0; j < N; ++j) part[wave][open ? 0 : 1][j * 64 + lane] = acc[j];
        };
        for (int p = begin; p < end; p += U) {
            int now[U];
            typename EI::T one[U];
            u32x4 x[U][W];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t key = __builtin_amdgcn_readfirstlane(l.key[p + u]);   // (16 past the end)
                now[u] = p + u < end ? (int)(key >> 10) : -1;
                const Ptr<EI> from = (Ptr<EI>)a.grad + (int64_t)(key & 1023) * a.ld + col;
                if constexpr (N == 1) one[u] = EI::put(0.0f);
#pragma unroll
                for (int i = 0; i < W; ++i) x[u][i] = (u32x4){0, 0, 0, 0};
                if (now[u] < 0 || !active) continue;
                if constexpr (N == 1) {
                    one[u] = *from;
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i) x[u][i] = load_vec<EI, Use::Once>(from + i * EI::V);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (now[u] < 0) break;
                if (now[u] != row) {
                    flush(false);
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] = 0.0f;
                    row = now[u];
                    open = false;
                }
                if constexpr (N == 1) {
                    acc[0] += EI::get(one[u]);
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        float y[EI::V];
                        EI::unpack(x[u][i], y);
#pragma unroll
                        for (int j = 0; j < EI::V; ++j) acc[i * EI::V + j] += y[j];
                    }
                }
            }
        }
        flush(row_at(end) == row);
    }
    __syncthreads();
    // the segment that begins among this wave's and goes on
    if (begin < end && end < m) {
        const int row = row_at(end - 1);
        if (row_at(end) == row && (row_at(begin) != row || row_at(begin - 1) != row)) {
            float acc[N];
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] = part[wave][1][j * 64 + lane];
            for (int w = wave + 1; w < WAVES && row_at(w * share) == row; ++w)
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += part[w][0][j * 64 + lane];
            if (active) finish_row<EO, N>(a, (uint32_t)(first + row), col, acc);
        }
    }
    if (a.accumulate || !active) return;
    const uint64_t there = l.there;
    const float zero[N] = {};
    for (int r = wave; r < rows; r += WAVES) {
        if (there >> r & 1) continue;
        const MutPtr<EO> to = (MutPtr<EO>)a.out + (first + r) * a.ldo + col;
        if constexpr (N == 1) *to = EO::put(0.0f);
        else store_floats<EO, N>(to, zero);
    }
}

template <typename EI, typename EO>
__global__ __launch_bounds__(kBlock) void few_tokens_kernel(FewArgs g) {
    constexpr int N = EI::V > EO::V ? EI::V : EO::V;
    __shared__ FewList list;
    __shared__ float part[kBlock / 64][2][64 * 8];
    const int64_t item = g.first + blockIdx.x;
    const int64_t first = item / (g.slabs + g.tail) * g.rows;
    const int slab = (int)(item % (g.slabs + g.tail)), lane = threadIdx.x % 64;
    const int rows = (int)(g.a.vocab - first < g.rows ? g.a.vocab - first : g.rows);
    const int m = few_tokens(g.a, first, rows, list);
    const int64_t whole = g.a.d / N * N;
    if (slab < g.slabs) {
        const int64_t col = ((int64_t)slab * 64 + lane) * N;
        few_sums<EI, EO, N>(g, list, part, m, first, rows, col, col < whole);
    } else {
        few_sums<EI, EO, 1>(g, list, part, m, first, rows, whole + lane, whole + lane < g.a.d);
    }
}

// ---------------------------------------------------------------------------
// dropout

// The first 128 bits of Philox4x32-10 for a counter below 2^64: its words 2
// and 3 are 0.
__device__ __forceinline__ u32x4 philox(uint64_t key, uint64_t counter) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = 0, c3 = 0;
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return (u32x4){c0, c1, c2, c3};
}

// A row's blocks of eight positions, which share random bits: 2^shift lanes
// take one of `chunks` groups of them.  The elements of a row's first and last block,
// where those are cut, are few among many for a long row: there they go to
// workgroups of their own, a lane each, since a wave that does both kinds
// takes the time of both (120,000 rows of 257 bf16, one apart: 40.5 us against
// 32.4; of 65 as long either way, and of 33 76 where they go apart, 56 not).
// Memory bounds it, then the generator's 20 wide products a block: 16,384 rows
// of 2,048 bf16 with a residual, 201 MB, in 33.8 us, 6.0 TB/s.
struct DropPlan {
    int shift;
    int64_t chunks;
    double inverse;        // 1 / chunks
    bool apart;            // cut blocks on their own
    int64_t whole_blocks;  // workgroups of the others
};

template <typename E, bool RES>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutArgs a, DropPlan plan) {
    const uint64_t key = a.seed_at != nullptr ? *a.seed_at : a.seed;
    auto kept = [&](uint32_t word, int j) { return (word >> (j % 2 * 16) & 0xFFFFu) >= a.limit; };
    if (blockIdx.x >= plan.whole_blocks) {
        // 16 lanes a row: positions of the block it begins in, and of the one
        // it ends in (rows of a block at least)
        for (int64_t i = ((int64_t)blockIdx.x - plan.whole_blocks) * kBlock + threadIdx.x;
             i < a.rows * 16; i += ((int64_t)gridDim.x - plan.whole_blocks) * kBlock) {
            const int64_t row = i / 16;
            const uint64_t q0 = a.offset + (uint64_t)row * (uint64_t)a.d;
            const int head = (int)(q0 & 7), skip = (int)(-q0 & 7);
            const int64_t at = i % 16 < 8 ? i % 8 - head : skip + (a.d - skip) / 8 * 8 + i % 8;
            if (at < 0 || at >= (i % 16 < 8 ? skip : a.d)) continue;
            const uint64_t q = q0 + (uint64_t)at;
            const u32x4 bits = philox(key, q >> 3);
            const int j = (int)(q & 7);
            const uint32_t word = j < 4 ? (j < 2 ? bits.x : bits.y) : (j < 6 ? bits.z : bits.w);
            float y = kept(word, j) ? E::get(((Ptr<E>)a.x)[row * a.ld + at]) * a.scale : 0.0f;
            if constexpr (RES) y += E::get(((Ptr<E>)a.residual)[row * a.ldr + at]);
            ((MutPtr<E>)a.out)[row * a.ldo + at] = put_product<E>(y);
        }
        return;
    }
    const int lane = (int)threadIdx.x & ((1 << plan.shift) - 1);
    const int per_block = kBlock >> plan.shift;
    for (int64_t item = (int64_t)blockIdx.x * per_block + (threadIdx.x >> plan.shift);
         item < a.rows * plan.chunks; item += plan.whole_blocks * per_block) {
        int64_t row = 0, block = item;
        if (a.rows > 1) {   // fewer than 2^31 items: off by one at most
            row = (int)((double)item * plan.inverse);
            block = item - row * plan.chunks;
            if (block < 0) --row, block += plan.chunks;
            else if (block >= plan.chunks) ++row, block -= plan.chunks;
        }
        block = (block << plan.shift) + lane;
        const uint64_t q0 = a.offset + (uint64_t)row * (uint64_t)a.d;
        const int head = (int)(q0 & 7);
        const int64_t i0 = block * 8 - head;   // the row's element at the block's start
        const bool whole = i0 >= 0 && i0 + 8 <= a.d;
        if (i0 >= a.d || (plan.apart && !whole)) continue;
        // (counters wrap as positions do)
        const u32x4 bits = philox(key, ((q0 >> 3) + (uint64_t)block) & (~uint64_t(0) >> 3));
        const Ptr<E> x = (Ptr<E>)a.x + row * a.ld + i0;
        const Ptr<E> r = (Ptr<E>)a.residual + row * a.ldr + i0;
        const MutPtr<E> out = (MutPtr<E>)a.out + row * a.ldo + i0;
        if (whole) {
            float v[8], add[8];
            load_floats<E, 8, Use::Once>(x, v);
            if constexpr (RES) load_floats<E, 8, Use::Once>(r, add);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = kept(bits[j / 2], j) ? v[j] * a.scale : 0.0f;
                if constexpr (RES) v[j] += add[j];
            }
            store_floats<E, 8, Use::Once>(out, v);
            continue;
        }
        // all elements loaded before one is stored
        typename E::T v[8], add[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool inside = (i0 + j >= 0) & (i0 + j < a.d);
            const int64_t at = inside ? j : i0 < 0 ? head : 0;   // else one that is
            v[j] = x[at];
            if constexpr (RES) add[j] = r[at];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y = kept(bits[j / 2], j) ? E::get(v[j]) * a.scale : 0.0f;
            if constexpr (RES) y += E::get(add[j]);
            if ((i0 + j >= 0) & (i0 + j < a.d)) out[j] = put_product<E>(y);
        }
    }
}

template <int N>
struct Int {
    static constexpr int value = N;
};

// Calls launch(first, n) until `blocks` workgroups are launched.
template <typename F>
hipError_t over_blocks(int64_t blocks, F &&launch) {
    for (int64_t first = 0; first < blocks; first += kMaxGrid) {
        launch(first, (unsigned)(blocks - first < kMaxGrid ? blocks - first : kMaxGrid));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Calls f with the element types of two dtype codes.
template <typename F>
hipError_t with_types(int from, int to, F &&f) {
    auto second = [&](auto e) {
        if (to == ASPIS_F32) return f(e, F32());
        if (to == ASPIS_BF16) return f(e, BF16());
        return f(e, F16());
    };
    if (from == ASPIS_F32) return second(F32());
    if (from == ASPIS_BF16) return second(BF16());
    return second(F16());
}

template <typename E>
hipError_t start_dropout(DropoutArgs a, hipStream_t s) {
    if ((a.ld == a.d || a.rows == 1) && (a.ldo == a.d || a.rows == 1) &&
        (a.residual == nullptr || a.ldr == a.d || a.rows == 1)) {
        a.d *= a.rows;   // one long row
        a.rows = 1;
        a.ld = a.ldr = a.ldo = a.d;
    }
    DropPlan plan;
    const int64_t blocks = (a.d + 14) / 8;   // of a row, wherever it begins
    // groups of one lane where a row is read, of four where two are: 400,000 rows
    // of 64 bf16, 8 apart, 21.2 us by one lane, 25.7 by four, 32.2 by eight;
    // 20,000 of 2,049 with a residual, 42.2, 40.0 and 41.5
    plan.shift = a.residual == nullptr ? 0 : lane_shift(blocks) < 2 ? lane_shift(blocks) : 2;
    plan.chunks = (blocks + (1 << plan.shift) - 1) >> plan.shift;
    plan.inverse = 1.0 / (double)plan.chunks;
    // rows of a launch, fewer than 2^31 chunks together
    const int64_t most = int64_t(1) << 30, rows = a.rows;
    const int64_t step = plan.chunks > most ? 1 : most / plan.chunks;
    for (int64_t first = 0; first < rows; first += step) {
        DropoutArgs b = a;
        b.rows = rows - first < step ? rows - first : step;
        b.x = (const typename E::T *)a.x + first * a.ld;
        b.out = (typename E::T *)a.out + first * a.ldo;
        if (a.residual != nullptr) b.residual = (const typename E::T *)a.residual + first * a.ldr;
        b.offset += (uint64_t)first * (uint64_t)a.d;
        plan.apart = a.d >= 64 && (b.offset % 8 != 0 || a.d % 8 != 0);
        plan.whole_blocks = grid_for(b.rows * plan.chunks, kBlock >> plan.shift);
        const unsigned grid = (unsigned)plan.whole_blocks + (plan.apart ? grid_for(b.rows * 16, kBlock) : 0);
        if (a.residual != nullptr) dropout_kernel<E, true><<<grid, kBlock, 0, s>>>(b, plan);
        else dropout_kernel<E, false><<<grid, kBlock, 0, s>>>(b, plan);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_embed(const EmbedArgs &a, hipStream_t s) {
    if (a.n == 0 || a.d == 0) return hipSuccess;
    return with_types(a.dtype, a.out_dtype, [&](auto from, auto to) {
        typedef decltype(from) EI;
        typedef decltype(to) EO;
        constexpr int N = EI::V > EO::V ? EI::V : EO::V;
        const int shift = lane_shift((a.d + N - 1) / N);
        const int per_block = kBlock >> shift;
        if (a.n >= kPairRows * per_block)
            embed_kernel<EI, EO, 2><<<grid_for(a.n, 2 * per_block), kBlock, 0, s>>>(a, shift);
        else embed_kernel<EI, EO, 1><<<grid_for(a.n, per_block), kBlock, 0, s>>>(a, shift);
        return hipGetLastError();
    });
}

hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t s) {
    if (a.vocab == 0 || a.d == 0 || (a.n == 0 && a.accumulate)) return hipSuccess;
    if (embed_few(a.n, a.vocab))
        return with_types(a.dtype, a.out_dtype, [&](auto from, auto to) {
            typedef decltype(from) EI;
            typedef decltype(to) EO;
            constexpr int N = EI::V > EO::V ? EI::V : EO::V;
            FewArgs g{};
            g.a = a;
            g.slabs = (int)((a.d / N + 63) / 64);
            g.tail = a.d % N != 0;
            // few rows, so that the commonest tokens' workgroup has little to do, but
            // not so few that reading the tokens takes most of the time: 700 into
            // 10,000 rows of 1,024, 19 us with 4 rows, 23 with 16; 100 into 131,072 of
            // 7, 7.2 with 64, 13 with 16
            const int64_t slabs = g.slabs + g.tail, width = a.d < 256 ? a.d : 256;
            g.rows = kFewRows;
            while (g.rows > 4 && (a.vocab + g.rows / 4 - 1) / (g.rows / 4) * slabs <= 8192 &&
                   g.rows / 4 * width >= 256)
                g.rows /= 4;
            return over_blocks((a.vocab + g.rows - 1) / g.rows * slabs, [&](int64_t first, unsigned n) {
                g.first = first;
                few_tokens_kernel<EI, EO><<<n, kBlock, 0, s>>>(g);
            });
        });
    const EmbedGradPlan plan = embed_grad_plan(a.n, a.d);
    const int64_t row_bytes = a.d * (a.out_dtype == ASPIS_F32 ? 4 : 2);
    // enough rows a workgroup to be worth the search that comes first: 8,192 tokens
    // into 128,000 rows of 1,024, 114 us by 16 rows, 120 by 64, 136 by 256; into
    // 500,000 of 64, 41, 36 and 48; into 2,000,000 of 7, 65, 41 and 37
    EarlyRows early{a.vocab, a.d >= 512 ? 16 : a.d >= 64 ? 64 : kZeroRows,
                    lane_shift(row_bytes / 16 + 1), 0};
    if (!a.accumulate && a.n <= 2 * a.vocab) {
        const int64_t most = kEarlyBytes / row_bytes;
        early.from = a.vocab > most ? a.vocab - most : 0;
    }
    char *ws = (char *)a.ws;
    auto array = [&](int i) { return (uint32_t *)(ws + i * plan.words); };
    Sorted sorted{array(0), array(1)}, other{array(2), array(3)};
    auto merged = [&]() {
        const Sorted swap = sorted;
        sorted = other;
        other = swap;
        return hipGetLastError();
    };
    {
        early.runs = (a.n + kSortRun - 1) / kSortRun;
        const unsigned blocks = (unsigned)(early.runs + (a.vocab - early.from + early.rows - 1) / early.rows);
        if (a.vocab < (1 << 22) - 1) sort_runs_kernel<uint32_t><<<blocks, kBlock, 0, s>>>(a, sorted, early);
        else sort_runs_kernel<uint64_t><<<blocks, kBlock, 0, s>>>(a, sorted, early);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && a.n > kSortRun) {
            auto merge = [&](auto share) {   // about a workgroup per compute unit
                constexpr int S = decltype(share)::value, kTokens = kMergeBlock / S;
                const unsigned blocks = (unsigned)((a.n + kTokens - 1) / kTokens);
                merge_runs_kernel<S><<<blocks, kMergeBlock, 0, s>>>(sorted, other, a.n);
            };
            if (a.n <= 256 * kMergeBlock / 8) merge(Int<8>());
            else if (a.n <= 256 * kMergeBlock / 4) merge(Int<4>());
            else merge(Int<2>());
            e = merged();
        }
        for (int64_t length = kSortRun * kMergeRuns; length < a.n && e == hipSuccess;
             length *= kMergeWide) {
            merge_long_kernel<<<(unsigned)((a.n + kBlock - 1) / kBlock), kBlock, 0, s>>>(
                sorted, other, a.n, length);
            e = merged();
        }
        if (e != hipSuccess) return e;
    }
    SumArgs g{};
    g.a = a;
    g.sorted = sorted;
    g.partial = (float *)(ws + 4 * plan.words);
    g.shift = plan.shift;
    g.windows = (a.n + (1 << plan.shift) - 1) >> plan.shift;
    g.row = embed_row(a.d);
    return with_types(a.dtype, a.out_dtype, [&](auto from, auto to) {
        typedef decltype(from) EI;
        typedef decltype(to) EO;
        constexpr int N = EI::V > EO::V ? EI::V : EO::V;
        g.slabs = (int)((a.d / N + 63) / 64);
        g.tail = a.d % N != 0;
        g.sum_blocks = (g.windows * (g.slabs + g.tail) + kBlock / 64 - 1) / (kBlock / 64);
        g.zero_rows = early.rows;
        g.zero_shift = early.shift;
        g.zero_end = a.accumulate ? 0 : early.from;
        const int64_t zero = (g.zero_end + g.zero_rows - 1) / g.zero_rows;
        const hipError_t st = over_blocks(g.sum_blocks + zero, [&](int64_t first, unsigned n) {
            g.first = first;
            sum_rows_kernel<EI, EO><<<n, kBlock, 0, s>>>(g);
        });
        // a long segment holds more than a block
        if (st != hipSuccess || a.n <= (2 << g.shift)) return st;
        const int64_t slabs = (a.d + 255) / 256;
        return over_blocks(plan.blocks * slabs, [&](int64_t first, unsigned n) {
            g.first = first;
            join_pieces_kernel<EO><<<n, kBlock, 0, s>>>(g, slabs);
        });
    });
}

hipError_t launch_dropout(const DropoutArgs &a, hipStream_t s) {
    if (a.rows == 0 || a.d == 0) return hipSuccess;
    if (a.dtype == ASPIS_F32) return start_dropout<F32>(a, s);
    if (a.dtype == ASPIS_BF16) return start_dropout<BF16>(a, s);
    return start_dropout<F16>(a, s);
}

}  // namespace aspis

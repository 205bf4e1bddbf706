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

template <typename EI, typename EO>
__global__ __launch_bounds__(kBlock) void embed_kernel(EmbedArgs a, int shift) {
    constexpr int N = EI::V > EO::V ? EI::V : EO::V;
    const int lane = (int)threadIdx.x & ((1 << shift) - 1);
    const int per_block = kBlock >> shift;
    const int64_t nv = a.d / N;
    for (int64_t row = (int64_t)blockIdx.x * per_block + (threadIdx.x >> shift); row < a.n;
         row += (int64_t)gridDim.x * per_block) {
        const int token = a.tokens.get(row, a.vocab);
        const Ptr<EI> from = (Ptr<EI>)a.table + (token < 0 ? 0 : token) * a.ld;
        const MutPtr<EO> to = (MutPtr<EO>)a.out + row * a.ldo;
        for (int64_t v = lane; v < nv; v += 1 << shift) {
            float x[N] = {};
            if (token >= 0) load_floats<EI, N>(from + v * N, x);
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] *= a.scale;
            store_floats<EO, N>(to + v * N, x);
        }
        for (int64_t i = nv * N + lane; i < a.d; i += 1 << shift)
            to[i] = EO::put(token >= 0 ? EI::get(from[i]) * a.scale : 0.0f);
    }
}

// ---------------------------------------------------------------------------
// its gradient: the tokens sorted

// A token (vocab where it is none) and its position, in one word that orders
// by both: no two are equal, so every way of sorting gives the same order.
typedef uint64_t Pair;
__device__ __forceinline__ Pair pair_of(uint32_t token, uint32_t at) {
    return (uint64_t)token << 32 | at;
}
__device__ __forceinline__ uint32_t token_of(Pair p) { return (uint32_t)(p >> 32); }

template <typename K>
__device__ __forceinline__ K lane_xor(K v, int mask) {
    return __shfl_xor(v, mask, 64);
}

// kSortRun tokens sorted by one workgroup: a bitonic sort of eight keys a
// thread, exchanged in registers, between lanes, and through LDS.
constexpr int kSortKeys = kSortRun / kBlock;

template <typename K>
__device__ __forceinline__ void order(K &a, K &b, bool up) {
    const bool swap = up ? b < a : a < b;
    const K low = swap ? b : a;
    b = swap ? a : b;
    a = low;
}

template <typename K>
__device__ void sort_run(K (&key)[kSortKeys], K *lds) {
    const int t = threadIdx.x;
#pragma unroll 1
    for (int k = 2; k <= kSortRun; k *= 2) {
#pragma unroll 1
        for (int j = k / 2; j >= kSortKeys; j /= 2) {
            const int m = j / kSortKeys;   // the other key is m threads away
            const bool up = (t * kSortKeys & k) == 0, low = (t & m) == 0;
            K other[kSortKeys];
            if (m < 64) {
#pragma unroll
                for (int r = 0; r < kSortKeys; ++r) other[r] = lane_xor(key[r], m);
            } else {
                __syncthreads();
#pragma unroll
                for (int r = 0; r < kSortKeys; ++r) lds[r * kBlock + t] = key[r];
                __syncthreads();
#pragma unroll
                for (int r = 0; r < kSortKeys; ++r) other[r] = lds[r * kBlock + (t ^ m)];
            }
#pragma unroll
            for (int r = 0; r < kSortKeys; ++r)
                key[r] = (other[r] < key[r]) == (up == low) ? other[r] : key[r];
        }
        // distances below kSortKeys: within the thread
#pragma unroll
        for (int j = kSortKeys / 2; j >= 1; j /= 2) {
            if (j >= k) continue;
#pragma unroll
            for (int r = 0; r < kSortKeys; ++r)
                if ((r & j) == 0) order(key[r], key[r | j], ((t * kSortKeys + r) & k) == 0);
        }
    }
}

// K: 32 bits where a token and its place in the run fit them, else 64.
template <typename K>
__global__ __launch_bounds__(kBlock) void sort_runs_kernel(EmbedGradArgs a, Pair *out) {
    constexpr int kBits = 11;
    static_assert(kSortRun == 1 << kBits, "");
    __shared__ K lds[kSortRun];
    const int64_t base = (int64_t)blockIdx.x * kSortRun;
    const int n = (int)(a.n - base < kSortRun ? a.n - base : kSortRun);
    K key[kSortKeys];
#pragma unroll
    for (int r = 0; r < kSortKeys; ++r) {
        const int i = r * kBlock + threadIdx.x;
        key[r] = ~(K)0;   // above every token's
        if (i < n) {
            const int token = a.tokens.get(base + i, a.vocab);
            key[r] = (K)(token < 0 ? (uint32_t)a.vocab : (uint32_t)token) << kBits | (K)i;
        }
    }
    sort_run(key, lds);
#pragma unroll
    for (int r = 0; r < kSortKeys; ++r) {
        const int i = (int)threadIdx.x * kSortKeys + r;
        if (i < n)
            out[base + i] = pair_of((uint32_t)(key[r] >> kBits),
                                    (uint32_t)base + (uint32_t)(key[r] & (kSortRun - 1)));
    }
}

// Merges kMergeRuns sorted runs of `length` pairs: a pair's place is the
// number of smaller ones in all of them, found by a binary search in each,
// all searches a step at a time.
__global__ __launch_bounds__(kBlock) void merge_runs_kernel(const Pair *in, Pair *out, int64_t n,
                                                            int64_t length) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= n) return;
    const int64_t group = i / (length * kMergeRuns) * (length * kMergeRuns);
    const int64_t left = n - group;
    const int own = (int)((i - group) / length);
    const int runs = (int)(left < length * kMergeRuns ? (left + length - 1) / length : kMergeRuns);
    const Pair key = in[i];
    uint32_t below[kMergeRuns];
#pragma unroll
    for (int r = 0; r < kMergeRuns; ++r) below[r] = 0;
    for (int64_t step = length; step > 0; step /= 2) {
#pragma unroll
        for (int r = 0; r < kMergeRuns; ++r) {
            if (r >= runs || r == own) continue;
            const int64_t at = below[r] + step;   // pairs taken as smaller, if the last one is
            const int64_t first = group + r * length;
            if (at <= length && first + at <= n && in[first + at - 1] < key) below[r] += step;
        }
    }
    int64_t place = i - group - own * length;
#pragma unroll
    for (int r = 0; r < kMergeRuns; ++r) place += below[r];
    out[group + place] = key;
}

// The first of n sorted pairs whose token is not below `token`.
__device__ __forceinline__ int64_t first_not_below(const Pair *pairs, int64_t n, uint32_t token) {
    int64_t low = 0, high = n;
    while (low < high) {
        const int64_t mid = (low + high) / 2;
        if (token_of(pairs[mid]) < token) low = mid + 1;
        else high = mid;
    }
    return low;
}

struct SumArgs {
    EmbedGradArgs a;
    const Pair *pairs;
    float *partial;      // [tiles][2][row]: the segment a tile begins in, the one it ends in
    int64_t tiles, row;
    int tile, shift;     // positions of a tile; log2 of the lanes that share it
    int64_t slabs;       // of columns, where 256 lanes do not hold a row
    int64_t sum_blocks;  // workgroups of tiles; the others fill rows with zeros
    int64_t first;       // the launch's first workgroup
};

// The sum of a row, scaled, to the result.
template <typename EO, int N>
__device__ __forceinline__ void finish_row(const EmbedGradArgs &a, uint32_t token, int64_t col,
                                           bool whole, float (&x)[N]) {
    const MutPtr<EO> to = (MutPtr<EO>)a.out + (int64_t)token * a.ldo + col;
    if (whole) {
        float y[N] = {};
        if (a.accumulate) load_floats<EO, N>((Ptr<EO>)to, y);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = a.accumulate ? y[j] + x[j] * a.scale : x[j] * a.scale;
        store_floats<EO, N>(to, y);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (col + j < a.d) {
            const float v = x[j] * a.scale;
            to[j] = EO::put(a.accumulate ? EO::get(to[j]) + v : v);
        }
}

constexpr int kZeroRows = 64;   // rows of a workgroup that fills in zeros

template <typename EO>
__device__ __forceinline__ void zero_rows(const SumArgs &g, int64_t block) {
    __shared__ uint64_t there;
    const EmbedGradArgs &a = g.a;
    const int64_t first = block * kZeroRows;
    if (threadIdx.x < 64) {
        const uint32_t token = (uint32_t)first + threadIdx.x;
        const int64_t at = first_not_below(g.pairs, a.n, token);
        const uint64_t mask = __ballot(at < a.n && token_of(g.pairs[at]) == token);
        if (threadIdx.x == 0) there = mask;
    }
    __syncthreads();
    const int rows = (int)(a.vocab - first < kZeroRows ? a.vocab - first : kZeroRows);
    const float zero[EO::V] = {};
    const int64_t nv = a.d / EO::V;
    for (int r = 0; r < rows; ++r) {
        if (there >> r & 1) continue;
        const MutPtr<EO> to = (MutPtr<EO>)a.out + (first + r) * a.ldo;
        for (int64_t v = threadIdx.x; v < nv; v += kBlock) store_floats<EO>(to + v * EO::V, zero);
        for (int64_t i = nv * EO::V + threadIdx.x; i < a.d; i += kBlock) to[i] = EO::put(0.0f);
    }
}

template <typename EI, typename EO>
__global__ __launch_bounds__(kBlock) void sum_tiles_kernel(SumArgs g) {
    constexpr int N = EI::V > EO::V ? EI::V : EO::V, U = 4;
    const EmbedGradArgs &a = g.a;
    const int64_t block = g.first + blockIdx.x;
    if (block >= g.sum_blocks) {
        zero_rows<EO>(g, block - g.sum_blocks);
        return;
    }
    const int lane = (int)threadIdx.x & ((1 << g.shift) - 1);
    const int64_t item = (block * kBlock + threadIdx.x) >> g.shift;
    const int64_t tile = item / g.slabs;
    const int64_t col = (item % g.slabs * (1 << g.shift) + lane) * N;
    if (tile >= g.tiles || col >= a.d) return;
    const bool whole = col + N <= a.d;
    const int64_t p0 = tile * g.tile;
    const int64_t p1 = p0 + g.tile < a.n ? p0 + g.tile : a.n;
    float acc[N] = {};
    uint32_t token = token_of(g.pairs[p0]);
    // whether the segment at hand began before the tile
    bool open = p0 > 0 && token_of(g.pairs[p0 - 1]) == token;
    auto flush = [&](bool goes_on) {
        if (!open && !goes_on) {
            finish_row<EO, N>(a, token, col, whole, acc);
            return;
        }
        float GLOBAL *to = (float GLOBAL *)g.partial + (tile * 2 + (open ? 0 : 1)) * g.row + col;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (col + j < a.d) to[j] = acc[j];
    };
    for (int64_t p = p0; p < p1; p += U) {
        Pair pair[U];
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            pair[u] = g.pairs[p + u < p1 ? p + u : p1 - 1];
            const bool real = token_of(pair[u]) < (uint32_t)a.vocab;
            const Ptr<EI> from = (Ptr<EI>)a.grad + (int64_t)(uint32_t)pair[u] * a.ld + col;
#pragma unroll
            for (int j = 0; j < N; ++j) x[u][j] = 0.0f;
            if (!real || p + u >= p1) continue;
            if (whole) {
                load_floats<EI, N, Use::Once>(from, x[u]);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (col + j < a.d) x[u][j] = EI::get(from[j]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= p1) continue;
            if (token_of(pair[u]) != token) {
                flush(false);
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] = 0.0f;
                token = token_of(pair[u]);
                open = false;
            }
            if (token >= (uint32_t)a.vocab) return;   // none: the last segment
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] += x[u][j];
        }
    }
    flush(p1 < a.n && token_of(g.pairs[p1]) == token);
}

// Joins the sums of a segment that several tiles hold, in their order: a
// workgroup for each tile that such a segment begins in and 256 columns.
template <typename EO>
__global__ __launch_bounds__(kBlock) void join_tiles_kernel(SumArgs g, int64_t slabs) {
    constexpr int N = EO::V > 4 ? 4 : EO::V, WAVES = kBlock / 64;
    __shared__ float sums[WAVES][64 * N];
    const EmbedGradArgs &a = g.a;
    const int64_t block = g.first + blockIdx.x;
    const int64_t tile = block / slabs;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = (block % slabs * 64 + lane) * N;
    const int64_t p0 = tile * g.tile, p1 = p0 + g.tile;
    if (p1 >= a.n) return;   // the last tile: nothing goes on
    const uint32_t token = token_of(g.pairs[p1 - 1]);
    if (token >= (uint32_t)a.vocab || token_of(g.pairs[p1]) != token) return;
    // it began in an earlier tile
    if (token_of(g.pairs[p0]) == token && p0 > 0 && token_of(g.pairs[p0 - 1]) == token) return;
    // the tiles after this one that begin with it
    int64_t low = tile + 1, high = g.tiles;   // low begins with it
    while (high - low > 1) {
        const int64_t mid = (low + high) / 2;
        if (token_of(g.pairs[mid * g.tile]) == token) low = mid;
        else high = mid;
    }
    const int64_t count = high - tile;   // sums: this tile's second, the others' first
    const int64_t share = (count + WAVES - 1) / WAVES;
    const int64_t from = wave * share, to = from + share < count ? from + share : count;
    float acc[N] = {};
    if (col < a.d) {
        for (int64_t k = from; k < to; ++k) {
            const float *p = g.partial + ((tile + k) * 2 + (k == 0 ? 1 : 0)) * g.row + col;
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] += p[j];
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
        *out = EO::put(a.accumulate ? EO::get(*out) + v : v);
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

// Eight positions share a block of random bits; `shift` lanes (log2) take a
// row's blocks, or, 256 of them, one of its `chunks`.
template <typename E, bool RES>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutArgs a, int shift, int64_t chunks) {
    const uint64_t key = a.seed_at != nullptr ? *a.seed_at : a.seed;
    const int lane = (int)threadIdx.x & ((1 << shift) - 1);
    const int per_block = kBlock >> shift;
    for (int64_t item = (int64_t)blockIdx.x * per_block + (threadIdx.x >> shift);
         item < a.rows * chunks; item += (int64_t)gridDim.x * per_block) {
        const int64_t row = item / chunks;
        const uint64_t q0 = a.offset + (uint64_t)row * (uint64_t)a.d;
        const int head = (int)(q0 & 7);
        const int64_t block = item % chunks * kBlock + lane;
        const int64_t i0 = block * 8 - head;   // the row's element at the block's start
        if (i0 >= a.d) continue;
        // (counters wrap as positions do)
        const u32x4 bits = philox(key, ((q0 >> 3) + (uint64_t)block) & (~uint64_t(0) >> 3));
        const Ptr<E> x = (Ptr<E>)a.x + row * a.ld + i0;
        const Ptr<E> r = (Ptr<E>)a.residual + row * a.ldr + i0;
        const MutPtr<E> out = (MutPtr<E>)a.out + row * a.ldo + i0;
        auto kept = [&](int j) { return (bits[j / 2] >> (j % 2 * 16) & 0xFFFFu) >= a.limit; };
        if (i0 >= 0 && i0 + 8 <= a.d) {
            float v[8], add[8];
            load_floats<E, 8, Use::Once>(x, v);
            if constexpr (RES) load_floats<E, 8, Use::Once>(r, add);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = kept(j) ? v[j] * a.scale : 0.0f;
                if constexpr (RES) v[j] += add[j];
            }
            store_floats<E, 8, Use::Once>(out, v);
            continue;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i0 + j < 0 || i0 + j >= a.d) continue;
            float v = kept(j) ? E::get(x[j]) * a.scale : 0.0f;
            if constexpr (RES) v += E::get(r[j]);
            out[j] = E::put(v);
        }
    }
}

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
    const int64_t blocks = (a.d + 14) / 8;   // of a row, wherever it begins
    const int shift = lane_shift(blocks);
    const int64_t chunks = (blocks + (1 << shift) - 1) >> shift;
    const unsigned grid = grid_for(a.rows * chunks, kBlock >> shift);
    if (a.residual != nullptr) dropout_kernel<E, true><<<grid, kBlock, 0, s>>>(a, shift, chunks);
    else dropout_kernel<E, false><<<grid, kBlock, 0, s>>>(a, shift, chunks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const EmbedArgs &a, hipStream_t s) {
    if (a.n == 0 || a.d == 0) return hipSuccess;
    return with_types(a.dtype, a.out_dtype, [&](auto from, auto to) {
        typedef decltype(from) EI;
        typedef decltype(to) EO;
        constexpr int N = EI::V > EO::V ? EI::V : EO::V;
        const int shift = lane_shift((a.d + N - 1) / N);
        embed_kernel<EI, EO><<<grid_for(a.n, kBlock >> shift), kBlock, 0, s>>>(a, shift);
        return hipGetLastError();
    });
}

hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t s) {
    if (a.vocab == 0 || a.d == 0 || (a.n == 0 && a.accumulate)) return hipSuccess;
    const EmbedGradPlan plan = embed_grad_plan(a.n, a.d);
    Pair *pairs = (Pair *)a.ws, *other = (Pair *)((char *)a.ws + plan.pairs);
    hipError_t e = hipSuccess;
    if (a.n > 0) {
        const unsigned runs = (unsigned)((a.n + kSortRun - 1) / kSortRun);
        if (a.vocab < (1 << 21) - 1) sort_runs_kernel<uint32_t><<<runs, kBlock, 0, s>>>(a, pairs);
        else sort_runs_kernel<uint64_t><<<runs, kBlock, 0, s>>>(a, pairs);
        e = hipGetLastError();
        for (int64_t length = kSortRun; length < a.n && e == hipSuccess; length *= kMergeRuns) {
            merge_runs_kernel<<<(unsigned)((a.n + kBlock - 1) / kBlock), kBlock, 0, s>>>(
                pairs, other, a.n, length);
            e = hipGetLastError();
            Pair *const swap = pairs;
            pairs = other;
            other = swap;
        }
        if (e != hipSuccess) return e;
    }
    SumArgs g{};
    g.a = a;
    g.pairs = pairs;
    g.partial = (float *)((char *)a.ws + 2 * plan.pairs);
    g.tiles = plan.tiles;
    g.tile = plan.tile;
    g.row = embed_row(a.d);
    return with_types(a.dtype, a.out_dtype, [&](auto from, auto to) {
        typedef decltype(from) EI;
        typedef decltype(to) EO;
        constexpr int N = EI::V > EO::V ? EI::V : EO::V;
        const int64_t vecs = (a.d + N - 1) / N;
        g.shift = lane_shift(vecs);
        g.slabs = (vecs + (1 << g.shift) - 1) >> g.shift;
        g.sum_blocks = (g.tiles * g.slabs + (kBlock >> g.shift) - 1) >> (8 - g.shift);
        const int64_t zero = a.accumulate ? 0 : (a.vocab + kZeroRows - 1) / kZeroRows;
        const hipError_t st = over_blocks(g.sum_blocks + zero, [&](int64_t first, unsigned n) {
            g.first = first;
            sum_tiles_kernel<EI, EO><<<n, kBlock, 0, s>>>(g);
        });
        if (st != hipSuccess || g.tiles <= 1) return st;
        const int64_t slabs = (a.d + 255) / 256;
        return over_blocks(g.tiles * slabs, [&](int64_t first, unsigned n) {
            g.first = first;
            join_tiles_kernel<EO><<<n, kBlock, 0, s>>>(g, slabs);
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

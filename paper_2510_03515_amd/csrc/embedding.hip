// Input embedding of a tied model: rows of the table [V, d] looked up by token id, and the gradient of that lookup added up per id.
//
//   forward   h[p, :] = scale E[tokens[p], :]                      (0 at masked positions)
//   backward  dE[v, :] (+)= scale sum_{valid p: tokens[p] = v} dh[p, :]
//
// Both are bound by memory.  The backward sorts the valid positions by (token, position) first, so that every row of dE is formed by one
// owner, in one order that hangs on the batch's size alone: no floating-point atomics, the same bits in every run.
#include "rapid_internal.h"
#include "row_math.h"

namespace rapid {

namespace {

// A row is worked on in pieces: 16 bytes, or (fp32 rows whose length is no multiple of 16 bytes) one element.
struct BF16x8 { static constexpr int N = 8; typedef bf16_t elem; typedef uint4 raw;
    static __device__ __forceinline__ void get(const raw& v, float (&f)[8]) { unpack8(v, f); }
    static __device__ __forceinline__ raw put(const float (&f)[8]) { return pack8(f); } };
struct F32x4 { static constexpr int N = 4; typedef float elem; typedef float4 raw;
    static __device__ __forceinline__ void get(const raw& v, float (&f)[4]) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    static __device__ __forceinline__ raw put(const float (&f)[4]) { return make_float4(f[0], f[1], f[2], f[3]); } };
struct F32x1 { static constexpr int N = 1; typedef float elem; typedef float raw;
    static __device__ __forceinline__ void get(const raw& v, float (&f)[1]) { f[0] = v; }
    static __device__ __forceinline__ raw put(const float (&f)[1]) { return f[0]; } };

// token at position p, or -1 where it has no row: masked, or (flagged) out of range
__device__ __forceinline__ int valid_token(const int32_t* __restrict__ tokens, const uint8_t* __restrict__ mask, int64_t p, int V,
                                           int32_t* __restrict__ dev_status) {
    if (mask && mask[p] == 0) return -1;
    const int tok = tokens[p];
    if (tok >= 0 && tok < V) return tok;
    if (dev_status) atomicOr(dev_status, RAPID_STATUS_BAD_TOKEN);
    return -1;
}

// ------------------------------------------------------------------------------------------- lookup
// A wave takes `rows` consecutive positions (at most 64; its lanes hold their ids) and walks their pieces side by side: lane l has pieces
// l, l + 64, ... of the run of rows, so no lane idles where a row is no multiple of 64 pieces.  (row, piece) advance by 64 pieces =
// step_rows rows and step_pieces pieces.
template <class P>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const typename P::elem* __restrict__ table, const int32_t* __restrict__ tokens,
                                                            const uint8_t* __restrict__ mask, int64_t positions, int pieces, int V,
                                                            float scale, typename P::elem* __restrict__ out,
                                                            int32_t* __restrict__ dev_status, int rows, int step_rows, int step_pieces) {
    typedef typename P::raw raw;
    const int lane = threadIdx.x & 63;
    const int64_t p0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * rows;
    if (p0 >= positions) return;
    const int n = (int)min((int64_t)rows, positions - p0);
    const int tok = lane < n ? valid_token(tokens, mask, p0 + lane, V, dev_status) : -1;
    int row = lane / pieces, piece = lane - row * pieces;
    raw* dst = (raw*)out + p0 * pieces;
    const raw* src = (const raw*)table;
    constexpr int U = 4;
    for (int base = 0; base < n * pieces; base += 64 * U) {
        raw v[U];
        int t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            t[u] = __shfl(tok, row < n ? row : 0, 64);
            v[u] = src[(int64_t)(t[u] < 0 ? 0 : t[u]) * pieces + piece];
            row += step_rows;
            piece += step_pieces;
            if (piece >= pieces) { piece -= pieces; ++row; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * 64 + lane;
            if (i >= n * pieces) break;
            float f[P::N];
            P::get(v[u], f);
#pragma unroll
            for (int e = 0; e < P::N; ++e) f[e] = t[u] < 0 ? 0.f : f[e] * scale;
            dst[i] = P::put(f);
        }
    }
}

template <class P>
void fwd_t(const EmbeddingArgs& a, const void* table, void* out, hipStream_t st) {
    const int pieces = (int)(a.d / P::N);
    // few positions: a wave for each, so that all are under way together
    const int rows = a.positions <= 16384 ? 1 : a.positions <= ((int64_t)1 << 26) ? 8 : 64;     // a launch holds less than 2^32 threads
    const int64_t waves = (a.positions + rows - 1) / rows;
    embedding_fwd_kernel<P><<<(unsigned)((waves + 3) / 4), 256, 0, st>>>(
        (const typename P::elem*)table, a.tokens, a.mask, a.positions, pieces, (int)a.V, a.scale, (typename P::elem*)out, a.dev_status, rows,
        64 / pieces, 64 % pieces);
}

// --------------------------------------------------------------------------------------------- sort
// Stable radix sort of the valid positions by token, `bits` of the id a pass (lowest first).  Block b owns a run of `tile` items.  count:
// how many of them have each digit; scatter: where each digit of the block begins (all lower digits, and the same digit of the blocks
// before: summed from the counts, no scan launch of its own), then every item's rank.  Ranks are found 64 items at a time: ballots over the
// digit's bits give the lanes that share it, a wave-private count in the LDS the items of earlier rounds.
// The first pass reads ids and mask in the order of the positions and drops what has no row.
constexpr int MAX_DIGIT_BITS = 9, MAX_DIGITS = 1 << MAX_DIGIT_BITS;
constexpr int SORT_WAVES = 8, SORT_THREADS = 64 * SORT_WAVES, SORT_ITEMS = 8;      // a round of a block: 4096 items

struct SortPass {
    const int32_t *tokens; const uint8_t* mask; int V; int32_t* dev_status;       // first pass
    const int32_t *key_in, *pos_in;                                               // later passes
    int32_t *key_out, *pos_out;
    int32_t* hist;          // [blocks][digits]
    int32_t* counts;        // [0] = number of valid positions (written by the first pass's scatter)
    uint32_t* touched;      // NULL, or one bit per id: set for the ids that occur (first pass, zero before)
    int64_t items, tile;
    int shift, bits, blocks;
};

template <bool FIRST>
__device__ __forceinline__ int sort_key(const SortPass& a, int64_t i, int64_t end, int32_t* status) {
    if (i >= end) return -1;
    return FIRST ? valid_token(a.tokens, a.mask, i, a.V, status) : a.key_in[i];
}

template <bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortPass a) {
    __shared__ int s_hist[MAX_DIGITS];
    const int digits = 1 << a.bits;
    for (int i = threadIdx.x; i < digits; i += SORT_THREADS) s_hist[i] = 0;
    __syncthreads();
    const int64_t items = FIRST ? a.items : a.counts[0];
    const int64_t begin = (int64_t)blockIdx.x * a.tile, end = min(items, begin + a.tile);
    for (int64_t i = begin + threadIdx.x; i < end; i += SORT_THREADS) {
        const int key = sort_key<FIRST>(a, i, end, a.dev_status);
        if (key < 0) continue;
        atomicAdd(&s_hist[(key >> a.shift) & (digits - 1)], 1);
        if (FIRST && a.touched) {
            const uint32_t bit = 1u << (key & 31);
            if (!(a.touched[key >> 5] & bit)) atomicOr(&a.touched[key >> 5], bit);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += SORT_THREADS) a.hist[(int64_t)blockIdx.x * digits + i] = s_hist[i];
}

template <bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_scatter_kernel(SortPass a) {
    __shared__ int s_base[MAX_DIGITS];                       // where the block's next item of each digit goes
    __shared__ int s_wave[SORT_WAVES][MAX_DIGITS];           // items of each digit per wave of a round
    __shared__ int s_sum[SORT_WAVES];
    const int digits = 1 << a.bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // a thread per digit: items of that digit, and those of them that lie in earlier blocks
    static_assert(SORT_THREADS >= MAX_DIGITS, "a thread per digit");
    int total = 0, before = 0;
    if (tid < digits) {
#pragma unroll 8
        for (int b = 0; b < a.blocks; ++b) {
            const int h = a.hist[(int64_t)b * digits + tid];
            total += h;
            before += b < (int)blockIdx.x ? h : 0;
        }
    }
    int run = total;                                         // inclusive sum over the digits
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(run, o, 64);
        if (lane >= o) run += v;
    }
    if (lane == 63) s_sum[wave] = run;
    __syncthreads();
    int lower = 0, all = 0;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) {
        if (w < wave) lower += s_sum[w];
        all += s_sum[w];
    }
    if (tid < digits) s_base[tid] = lower + run - total + before;
    if (FIRST && blockIdx.x == 0 && tid == 0) a.counts[0] = all;
    const int64_t items = FIRST ? a.items : all;
    const int64_t begin = (int64_t)blockIdx.x * a.tile, end = min(items, begin + a.tile);
    for (int64_t r0 = begin; r0 < end; r0 += SORT_THREADS * SORT_ITEMS) {
        for (int i = tid; i < SORT_WAVES * digits; i += SORT_THREADS) s_wave[i >> a.bits][i & (digits - 1)] = 0;
        int key[SORT_ITEMS], pos[SORT_ITEMS], rank[SORT_ITEMS] = {};
        const int64_t first = r0 + (int64_t)wave * 64 * SORT_ITEMS + lane;
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u) {
            key[u] = sort_key<FIRST>(a, first + u * 64, end, nullptr);
            pos[u] = FIRST ? (int)(first + u * 64) : first + u * 64 < end ? a.pos_in[first + u * 64] : 0;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u) {
            const int digit = (key[u] >> a.shift) & (digits - 1);
            unsigned long long same = __ballot(key[u] >= 0);
            for (int b = 0; b < a.bits; ++b) {
                const unsigned long long votes = __ballot((digit >> b) & 1);
                same &= ((digit >> b) & 1) ? votes : ~votes;
            }
            if (key[u] >= 0) {
                const int ahead = __popcll(same & ((1ull << lane) - 1ull));
                const int old = s_wave[wave][digit];         // the wave's own row: its lanes run in step
                rank[u] = old + ahead;
                __builtin_amdgcn_wave_barrier();
                if (ahead == 0) s_wave[wave][digit] = old + __popcll(same);
                __builtin_amdgcn_wave_barrier();
            }
        }
        __syncthreads();
        if (tid < digits) {                                  // counts -> first places; the base moves on for the next round
            int at = s_base[tid];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int c = s_wave[w][tid];
                s_wave[w][tid] = at;
                at += c;
            }
            s_base[tid] = at;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u) {
            if (key[u] < 0) continue;
            const int at = s_wave[wave][(key[u] >> a.shift) & (digits - 1)] + rank[u];
            a.key_out[at] = key[u];
            a.pos_out[at] = pos[u];
        }
        __syncthreads();
    }
}

// --------------------------------------------------------------------------------------------- sums
// Sorted position i of the batch has id key[i].  A group of threads takes the `rows` sorted positions of one stretch, a thread one piece of
// the columns, and adds the gradient rows up in fp32; an id's sum that began and ended inside the stretch is the row of dE.  What crosses an end of the
// stretch goes to `part`: slot 0 the sum that came in from before and ended here, slot 1 the one that goes on behind (it may have come in, too).  So the
// work is shared out by rows whatever the ids are: one id that owns the whole batch is as quick as all ids different.
struct SumArgs {
    const int32_t *key, *pos, *counts;
    int64_t rows;           // per stretch
    int pieces;             // of a row
    float* part;            // [stretches][2][d]
    int64_t d;
    float scale;
    int accumulate;
};

template <class P, class D>
__device__ __forceinline__ void store_row(D* __restrict__ at, const float (&acc)[P::N], float scale, int accumulate) {
    constexpr int N = P::N;
    if constexpr (sizeof(D) == 4 && N == 1) {
        at[0] = accumulate ? fmaf(acc[0], scale, at[0]) : acc[0] * scale;
    } else if constexpr (sizeof(D) == 4) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            float4* to = (float4*)at + q;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (accumulate) v = *to;
            *to = make_float4(fmaf(acc[4 * q], scale, v.x), fmaf(acc[4 * q + 1], scale, v.y), fmaf(acc[4 * q + 2], scale, v.z),
                              fmaf(acc[4 * q + 3], scale, v.w));
        }
    } else if constexpr (N == 8) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = acc[e] * scale;
        *(uint4*)at = pack8(f);
    } else if constexpr (N == 4) {
        *(uint2*)at = make_uint2(pack2(acc[0] * scale, acc[1] * scale), pack2(acc[2] * scale, acc[3] * scale));
    } else {
        at[0] = __builtin_bit_cast(bf16_t, (__bf16)(acc[0] * scale));
    }
}

template <class P, class D>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs a, const typename P::elem* __restrict__ dh, D* __restrict__ dE) {
    typedef typename P::raw raw;
    const int64_t M = a.counts[0];
    const int64_t s = (int64_t)blockIdx.x * blockDim.y + threadIdx.y, begin = s * a.rows;
    if (begin >= M) return;
    const int64_t end = min(M, begin + a.rows);
    const raw* src = (const raw*)dh;
    constexpr int U = 8;
    for (int piece = blockIdx.y * blockDim.x + threadIdx.x; piece < a.pieces; piece += gridDim.y * blockDim.x) {
        float acc[P::N];
#pragma unroll
        for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
        bool came_in = begin > 0 && a.key[begin - 1] == a.key[begin];
        for (int64_t i0 = begin; i0 < end; i0 += U) {
            raw v[U];
            int k[U + 1];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = i0 + u < end ? i0 + u : end - 1;
                k[u] = a.key[i];
                v[u] = src[(int64_t)a.pos[i] * a.pieces + piece];
            }
            k[U] = i0 + U < M ? a.key[i0 + U] : -1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = i0 + u;
                if (i >= end) break;
                float f[P::N];
                P::get(v[u], f);
#pragma unroll
                for (int e = 0; e < P::N; ++e) acc[e] += f[e];
                const int next = i + 1 < end ? k[u + 1] : end < M ? a.key[end] : -1;
                if (next == k[u] && i + 1 < end) continue;
                const bool goes_on = next == k[u];
                if (came_in || goes_on) {
                    float* to = a.part + (s * 2 + (goes_on ? 1 : 0)) * a.d + (int64_t)piece * P::N;
#pragma unroll
                    for (int e = 0; e < P::N; ++e) to[e] = acc[e];
                } else {
                    store_row<P, D>(dE + (int64_t)k[u] * a.d + (int64_t)piece * P::N, acc, a.scale, a.accumulate);
                }
                came_in = false;
#pragma unroll
                for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
            }
        }
    }
}

// Joins the sums that crossed ends of stretches: the block of the stretch in which such an id began adds up what the stretches after it left, in
// order (in MERGE_WAVES consecutive shares, then these in order).
constexpr int MERGE_WAVES = 8;
template <class P, class D>
__global__ __launch_bounds__(64 * MERGE_WAVES) void embedding_merge_kernel(SumArgs a, D* __restrict__ dE) {
    __shared__ float s_sum[MERGE_WAVES][64][P::N];
    const int64_t M = a.counts[0], s = blockIdx.x, begin = s * a.rows, end = begin + a.rows;
    if (end >= M) return;                                   // nothing goes on behind the last stretch
    const int key = a.key[end - 1];
    if (a.key[end] != key) return;
    if (a.key[begin] == key && begin > 0 && a.key[begin - 1] == key) return;      // began in an earlier stretch
    int64_t lo = end, hi = M;                               // first sorted position behind the id's
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (a.key[mid] == key) lo = mid + 1; else hi = mid;
    }
    const int64_t last = (lo - 1) / a.rows;                 // stretches s .. last; the sum ended in the last one: slot 0 there
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n = last - s + 1, from = s + n * wave / MERGE_WAVES, to = s + n * (wave + 1) / MERGE_WAVES;
    for (int piece0 = blockIdx.y * 64; piece0 < a.pieces; piece0 += gridDim.y * 64) {
        const int piece = piece0 + lane;
        float acc[P::N];
#pragma unroll
        for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
        if (piece < a.pieces) {
#pragma unroll 4
            for (int64_t c = from; c < to; ++c) {
                const float* p = a.part + (c * 2 + (c == last ? 0 : 1)) * a.d + (int64_t)piece * P::N;
#pragma unroll
                for (int e = 0; e < P::N; ++e) acc[e] += p[e];
            }
        }
#pragma unroll
        for (int e = 0; e < P::N; ++e) s_sum[wave][lane][e] = acc[e];
        __syncthreads();
        if (wave == 0 && piece < a.pieces) {
            for (int w = 1; w < MERGE_WAVES; ++w)
#pragma unroll
                for (int e = 0; e < P::N; ++e) acc[e] += s_sum[w][lane][e];
            store_row<P, D>(dE + (int64_t)key * a.d + (int64_t)piece * P::N, acc, a.scale, a.accumulate);
        }
        __syncthreads();
    }
}

// rows of ids that do not occur
template <class W>
__global__ __launch_bounds__(256) void embedding_zero_kernel(const uint32_t* __restrict__ touched, int64_t V, int64_t words, W* __restrict__ dE) {
    for (int64_t v = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); v < V; v += (int64_t)gridDim.x * 4) {
        if ((touched[v >> 5] >> (v & 31)) & 1u) continue;
        for (int64_t i = threadIdx.x & 63; i < words; i += 64) dE[v * words + i] = W{};
    }
}

__global__ void zero_words_kernel(uint32_t* __restrict__ p, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0u;
}

template <class P, class D>
void sum_t(const EmbeddingArgs& a, const SumArgs& s, int64_t stretches, const void* dh, D* dE, hipStream_t st) {
    // a group of threads for a stretch: enough of them for a row's pieces, up to a block
    int x = 8;
    while (x < 64 && x < s.pieces) x *= 2;
    if (s.pieces > 64) x = s.pieces >= 256 ? 256 : (s.pieces + 63) / 64 * 64;
    const int y = 256 / x;
    const int64_t columns = (s.pieces + x - 1) / x;
    embedding_sum_kernel<P, D><<<dim3((unsigned)((stretches + y - 1) / y), (unsigned)columns), dim3(x, y), 0, st>>>(s, (const typename P::elem*)dh, dE);
    if (stretches > 1)
        embedding_merge_kernel<P, D><<<dim3((unsigned)(stretches - 1), (unsigned)((s.pieces + 63) / 64)), 64 * MERGE_WAVES, 0, st>>>(s, dE);
}

template <class D>
void bwd_t(const EmbeddingArgs& a, SumArgs s, const uint32_t* touched, int64_t stretches, const void* dh, D* dE, hipStream_t st) {
    if (!s.accumulate) {
        const int64_t bytes = a.d * (int64_t)sizeof(D);
        const unsigned grid = (unsigned)((a.V + 3) / 4 < 8192 ? (a.V + 3) / 4 : 8192);
        if (bytes % 16 == 0) embedding_zero_kernel<uint4><<<grid, 256, 0, st>>>(touched, a.V, bytes / 16, (uint4*)dE);
        else embedding_zero_kernel<D><<<grid, 256, 0, st>>>(touched, a.V, a.d, dE);
    }
    if (a.dtype == RAPID_DTYPE_BF16) sum_t<BF16x8, D>(a, s, stretches, dh, dE, st);
    else if (a.d % 4 == 0) sum_t<F32x4, D>(a, s, stretches, dh, dE, st);
    else sum_t<F32x1, D>(a, s, stretches, dh, dE, st);
}

int64_t sort_tile(int64_t positions) {
    constexpr int64_t round = SORT_THREADS * SORT_ITEMS;
    const int64_t per = (positions + 255) / 256;            // at most 256 blocks: every block adds up the counts of all
    return (per + round - 1) / round * round;
}
int64_t stretch_rows(int64_t positions) { return positions <= 32768 ? 16 : positions <= 262144 ? 64 : positions <= ((int64_t)1 << 24) ? 128 : 1024; }

}  // namespace

void launch_embedding_fwd(const EmbeddingArgs& a, const void* table, void* out, hipStream_t st) {
    if (a.dtype == RAPID_DTYPE_BF16) fwd_t<BF16x8>(a, table, out, st);
    else if (a.d % 4 == 0) fwd_t<F32x4>(a, table, out, st);
    else fwd_t<F32x1>(a, table, out, st);
}

EmbeddingPlan embedding_plan(int64_t positions, int64_t d, int64_t V) {
    EmbeddingPlan p;
    int bits = 1;
    while (((int64_t)1 << bits) < V) ++bits;
    p.passes = (bits + MAX_DIGIT_BITS - 1) / MAX_DIGIT_BITS;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tile = sort_tile(positions);
    p.blocks = (positions + p.tile - 1) / p.tile;
    p.rows = stretch_rows(positions);
    p.stretches = (positions + p.rows - 1) / p.rows;
    size_t cur = 0;
    auto take = [&](size_t bytes) { const size_t at = cur; cur += (bytes + 255) / 256 * 256; return at; };
    p.counts = take(64 * 4);
    for (int i = 0; i < 2; ++i) {
        p.key[i] = take((size_t)positions * 4);
        p.pos[i] = take((size_t)positions * 4);
    }
    p.hist = take((size_t)p.blocks * (1u << p.bits) * 4);
    p.touched = take((size_t)((V + 31) / 32) * 4);
    p.part = take((size_t)p.stretches * 2 * (size_t)d * 4);
    p.total = cur;
    return p;
}

void launch_embedding_bwd(const EmbeddingArgs& a, const EmbeddingPlan& p, void* ws, const void* dh, int dw_dtype, int accumulate, void* dE, hipStream_t st) {
    char* w = (char*)ws;
    uint32_t* touched = accumulate ? nullptr : (uint32_t*)(w + p.touched);
    if (touched) {
        const int64_t words = (a.V + 31) / 32;
        zero_words_kernel<<<(unsigned)((words + 255) / 256), 256, 0, st>>>(touched, words);
    }
    SortPass s{};
    s.tokens = a.tokens; s.mask = a.mask; s.V = (int)a.V; s.dev_status = a.dev_status;
    s.hist = (int32_t*)(w + p.hist); s.counts = (int32_t*)(w + p.counts); s.touched = touched;
    s.items = a.positions; s.tile = p.tile; s.bits = p.bits; s.blocks = (int)p.blocks;
    const unsigned grid = (unsigned)p.blocks;
    for (int pass = 0; pass < p.passes; ++pass) {
        const int to = pass & 1;
        s.shift = pass * p.bits;
        s.key_in = (const int32_t*)(w + p.key[to ^ 1]); s.pos_in = (const int32_t*)(w + p.pos[to ^ 1]);
        s.key_out = (int32_t*)(w + p.key[to]); s.pos_out = (int32_t*)(w + p.pos[to]);
        if (pass == 0) {
            sort_count_kernel<true><<<grid, SORT_THREADS, 0, st>>>(s);
            sort_scatter_kernel<true><<<grid, SORT_THREADS, 0, st>>>(s);
        } else {
            sort_count_kernel<false><<<grid, SORT_THREADS, 0, st>>>(s);
            sort_scatter_kernel<false><<<grid, SORT_THREADS, 0, st>>>(s);
        }
    }
    SumArgs u{};
    u.key = s.key_out; u.pos = s.pos_out; u.counts = s.counts; u.rows = p.rows;
    u.pieces = (int)(a.d / (a.dtype == RAPID_DTYPE_BF16 ? 8 : a.d % 4 == 0 ? 4 : 1));
    u.part = (float*)(w + p.part); u.d = a.d; u.scale = a.scale; u.accumulate = accumulate;
    if (dw_dtype == RAPID_DTYPE_F32) bwd_t<float>(a, u, touched, p.stretches, dh, (float*)dE, st);
    else bwd_t<bf16_t>(a, u, touched, p.stretches, dh, (bf16_t*)dE, st);
}

}  // namespace rapid

// Input embedding of a tied model: rows of the table [V, d] looked up by token id, and the gradient of that lookup added up per id.
//
//   forward   h[p, :] = scale E[tokens[p], :]                      (0 at masked positions)
//   backward  dE[v, :] (+)= scale sum_{valid p: tokens[p] = v} dh[p, :]
//
// Both are bound by memory.  The backward sorts the valid positions by (token, position) first, so that every row of dE is formed by one
// owner, in one order that hangs on the valid positions alone: no floating-point atomics, the same bits in every run.
#include "rapid_internal.h"
#include "row_math.h"

namespace rapid {

namespace {

// A row is worked on in pieces: 16 bytes, or (fp32 rows whose length is no multiple of 16 bytes) one element, in the lookup 16 bytes at any multiple of
// 4, the row's last piece moved back to end with it: the columns that it shares with the one before are written twice, with the same values.
struct BF16x8 { static constexpr int N = 8; static constexpr bool ANY = false; typedef bf16_t elem; typedef uint4 raw;
    static __device__ __forceinline__ void get(const raw& v, float (&f)[8]) { unpack8(v, f); }
    static __device__ __forceinline__ raw put(const float (&f)[8]) { return pack8(f); } };
struct F32x4 { static constexpr int N = 4; static constexpr bool ANY = false; typedef float elem; typedef float4 raw;
    static __device__ __forceinline__ void get(const raw& v, float (&f)[4]) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    static __device__ __forceinline__ raw put(const float (&f)[4]) { return make_float4(f[0], f[1], f[2], f[3]); } };
struct F32x1 { static constexpr int N = 1; static constexpr bool ANY = false; typedef float elem; typedef float raw;
    static __device__ __forceinline__ void get(const raw& v, float (&f)[1]) { f[0] = v; }
    static __device__ __forceinline__ raw put(const float (&f)[1]) { return f[0]; } };
struct F32x4Any { static constexpr int N = 4; static constexpr bool ANY = true; typedef float elem; typedef float raw __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void get(const raw& v, float (&f)[4]) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    static __device__ __forceinline__ raw put(const float (&f)[4]) { return raw{f[0], f[1], f[2], f[3]}; } };

// 16 bytes (or an element) that nobody reads before they have left the caches: stored past them, read without keeping them
template <class R>
__device__ __forceinline__ void store_past(R* to, const R& v) {
    if constexpr (alignof(R) == 16) {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        __builtin_nontemporal_store(__builtin_bit_cast(u4, v), (u4*)to);
    } else {
        __builtin_nontemporal_store(v, to);
    }
}
template <class R>
__device__ __forceinline__ R load_once(const R* from) {
    if constexpr (sizeof(R) == 16) {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(R, __builtin_nontemporal_load((const u4*)from));
    } else {
        return __builtin_nontemporal_load(from);
    }
}

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
// step_rows rows and step_pieces pieces.  PAST: the output is larger than the memory-side cache, which is left to the table (256 x 2048 x 1536 bf16: 505 us
// without, 394 with).
template <class P, bool PAST, int U>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const typename P::elem* __restrict__ table, const int32_t* __restrict__ tokens,
                                                            const uint8_t* __restrict__ mask, int64_t positions, int pieces, int V,
                                                            float scale, typename P::elem* __restrict__ out, int32_t* __restrict__ dev_status,
                                                            int rows, int step_rows, int step_pieces, int d) {
    typedef typename P::raw raw;
    const int lane = threadIdx.x & 63;
    const int64_t p0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * rows;
    if (p0 >= positions) return;
    const int n = (int)min((int64_t)rows, positions - p0);
    const int tok = lane < n ? valid_token(tokens, mask, p0 + lane, V, dev_status) : -1;
    int row = lane / pieces, piece = lane - row * pieces;
    typename P::elem* dst = out + p0 * d;
    for (int base = 0; base < n * pieces; base += 64 * U) {
        raw v[U];
        int t[U], at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int column = P::ANY ? min(piece * P::N, d - P::N) : piece * P::N;
            at[u] = row * d + column;
            t[u] = __shfl(tok, row < n ? row : 0, 64);
            v[u] = raw{};
            if (t[u] >= 0) v[u] = *(const raw*)(table + (int64_t)t[u] * d + column);
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
            if (PAST) store_past((raw*)(dst + at[u]), P::put(f));
            else *(raw*)(dst + at[u]) = P::put(f);
        }
    }
}

constexpr int64_t BEYOND_CACHES = (int64_t)256 << 20;      // bytes of the memory-side cache
template <class P>
void fwd_t(const EmbeddingArgs& a, const void* table, void* out, hipStream_t st) {
    const int pieces = (int)((a.d + P::N - 1) / P::N);
    // A wave takes a row, in trips of U pieces a lane with as few lanes left over as can be, or the rows that make up a trip of 4.  (256 x 2048 x 1536,
    // 3 pieces a lane, cold tables: U = 3 387 us, U = 4 411; 2, 4 and 8 rows a wave with U = 3: 385, 416, 454.)  A launch holds less than 2^32 threads.
    const int trips = (pieces + 63) / 64;
    int rows = 256 / pieces < 1 ? 1 : trips > 1 ? 1 : 256 / pieces > 64 ? 64 : 256 / pieces;
    // Few positions: all under way together.  Table in the caches, a row a wave and several: bf16, d = 64: 2048 positions 3.0 and 3.1 us, 4096 3.5 and
    // 3.1; d = 512: 2048 3.2 and 3.3, 4096 3.9 and 3.6; fp32, d = 256: 2048 3.1 and 3.1, 4096 3.7 and 3.4.
    if (a.positions <= 2048) rows = 1;
    if (a.positions > ((int64_t)1 << 25)) rows = 64;
    const int64_t waves = (a.positions + rows - 1) / rows;
    const bool past = a.positions * a.d * (int64_t)sizeof(typename P::elem) > BEYOND_CACHES;
    auto go = [&](auto* kernel) {
        kernel<<<(unsigned)((waves + 3) / 4), 256, 0, st>>>((const typename P::elem*)table, a.tokens, a.mask, a.positions, pieces, (int)a.V, a.scale,
                                                             (typename P::elem*)out, a.dev_status, rows, 64 / pieces, 64 % pieces, (int)a.d);
    };
    if (trips == 2) past ? go(&embedding_fwd_kernel<P, true, 2>) : go(&embedding_fwd_kernel<P, false, 2>);
    else if (trips > 1 && (trips + 2) / 3 * 3 < (trips + 3) / 4 * 4) past ? go(&embedding_fwd_kernel<P, true, 3>) : go(&embedding_fwd_kernel<P, false, 3>);
    else past ? go(&embedding_fwd_kernel<P, true, 4>) : go(&embedding_fwd_kernel<P, false, 4>);
}

// --------------------------------------------------------------------------------------------- sort
// Stable radix sort of the valid positions by token, `bits` of the id a pass (lowest first).  Block b owns a run of `tile` items.  count:
// how many of them have each digit; scatter: where each digit of the block begins (all lower digits, and the same digit of the blocks
// before: summed from the counts, no scan launch of its own), then every item's rank.  Ranks are found 64 items at a time: ballots over the
// digit's bits give the lanes that share it, a wave-private count in the LDS the items of earlier rounds.
// The first pass reads ids and mask in the order of the positions and drops what has no row.
// Up to 12 bits are sorted in one pass where there are few blocks, whose counts (16 KB each) every block reads: 512 x 48 positions, V 4096: 13.6 us for
// 19.2 in two passes of 6 bits, and two launches less.
constexpr int MAX_DIGIT_BITS = 9, MAX_DIGITS = 1 << MAX_DIGIT_BITS, WIDE_BITS = 12, WIDE_DIGITS = 1 << WIDE_BITS;
constexpr int SORT_WAVES = 8, SORT_THREADS = 64 * SORT_WAVES;

struct SortPass {
    const int32_t *tokens; const uint8_t* mask; int V; int32_t* dev_status;       // first pass
    const int32_t *key_in, *pos_in;                                               // later passes
    int32_t *key_out, *pos_out;
    int32_t* hist;          // [blocks][digits]
    int32_t* counts;        // [0] = number of valid positions (written by the first pass's scatter)
    uint32_t* flags;        // NULL, or flag_words words that the first pass clears
    int64_t items, tile, flag_words;
    int shift, bits, blocks;
};

// ids of U items, `step` apart from i on (-1: none, masked, or out of range): all loads first, a chain of one trip
template <bool FIRST, int U>
__device__ __forceinline__ void sort_keys(const SortPass& a, int64_t i, int64_t step, int64_t end, bool flag, int (&key)[U], int (&pos)[U]) {
    uint8_t m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t at = i + u * step < end ? i + u * step : end - 1;
        key[u] = FIRST ? a.tokens[at] : a.key_in[at];
        pos[u] = FIRST ? (int)at : a.pos_in[at];
        m[u] = FIRST && a.mask ? a.mask[at] : 1;
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool here = i + u * step < end && m[u] != 0, in = !FIRST || (key[u] >= 0 && key[u] < a.V);
        bad |= here && !in;
        if (!here || !in) key[u] = -1;
    }
    if (FIRST && flag && bad && a.dev_status) atomicOr(a.dev_status, RAPID_STATUS_BAD_TOKEN);
}
__device__ __forceinline__ void clear_flags(const SortPass& a, int64_t i, int64_t step) {
    if (a.flags)
        for (; i < a.flag_words; i += step) a.flags[i] = 0u;
}
// lanes with the same digit as this one, among those with an item
__device__ __forceinline__ unsigned long long same_digit(int digit, int bits, bool item) {
    unsigned long long same = __ballot(item);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long votes = __ballot((digit >> b) & 1);
        same &= ((digit >> b) & 1) ? votes : ~votes;
    }
    return same;
}
// Ranks of a wave's items of one round among its items of the same digit.  count: the wave's own counters in the LDS (its lanes run in step).
__device__ __forceinline__ int rank_in_wave(int key, int digit, int bits, int* count) {
    const unsigned long long same = same_digit(digit, bits, key >= 0);
    int rank = 0;
    if (key >= 0) {
        const int ahead = __popcll(same & ((1ull << (threadIdx.x & 63)) - 1ull)), old = count[digit];
        rank = old + ahead;
        __builtin_amdgcn_wave_barrier();
        if (ahead == 0) count[digit] = old + __popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
    return rank;
}
// sums of v over the threads before this one and over all of them; s_sum [waves]
template <int WAVES>
__device__ __forceinline__ void scan_threads(int v, int* s_sum, int& before, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int run = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int w = __shfl_up(run, o, 64);
        if (lane >= o) run += w;
    }
    if (lane == 63) s_sum[wave] = run;
    __syncthreads();
    before = run - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += s_sum[w];
        all += s_sum[w];
    }
}

// DIGITS: the most digits of a pass, a multiple of SORT_THREADS
template <bool FIRST, int SORT_ITEMS, int DIGITS>
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortPass a) {
    __shared__ int s_hist[DIGITS];
    const int digits = 1 << a.bits;
    for (int i = threadIdx.x; i < digits; i += SORT_THREADS) s_hist[i] = 0;
    if (FIRST) clear_flags(a, (int64_t)blockIdx.x * SORT_THREADS + threadIdx.x, (int64_t)gridDim.x * SORT_THREADS);
    __syncthreads();
    const int64_t items = FIRST ? a.items : a.counts[0];
    const int64_t begin = (int64_t)blockIdx.x * a.tile, end = min(items, begin + a.tile);
    for (int64_t r0 = begin; r0 < end; r0 += SORT_THREADS * SORT_ITEMS) {
        int key[SORT_ITEMS], pos[SORT_ITEMS];
        sort_keys<FIRST, SORT_ITEMS>(a, r0 + threadIdx.x, SORT_THREADS, end, true, key, pos);
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u)
            if (key[u] >= 0) atomicAdd(&s_hist[(key[u] >> a.shift) & (digits - 1)], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += SORT_THREADS) a.hist[(int64_t)blockIdx.x * digits + i] = s_hist[i];
}

template <int DIGITS>
constexpr int scatter_lds() { return (DIGITS + SORT_WAVES * DIGITS + SORT_WAVES) * 4; }
template <bool FIRST, int SORT_ITEMS, int DIGITS>
__global__ __launch_bounds__(SORT_THREADS) void sort_scatter_kernel(SortPass a) {
    constexpr int PER = DIGITS / SORT_THREADS;              // digits of a thread, next to each other
    static_assert(PER * SORT_THREADS == DIGITS, "whole digits a thread");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int* const s_wave = (int*)lds;                           // [SORT_WAVES][digits]: items of each digit per wave of a round
    int* const s_base = s_wave + SORT_WAVES * DIGITS;        // where the block's next item of each digit goes
    int* const s_sum = s_base + DIGITS;
    const int digits = 1 << a.bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, d0 = tid * PER;
    // items of the thread's digits, and those of them that lie in earlier blocks
    int total[PER], mine[PER], sum = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) total[q] = mine[q] = 0;
    if (d0 < digits) {
        const int32_t* h = a.hist + d0;
#pragma unroll (16 / PER < 4 ? 4 : 16 / PER)
        for (int b = 0; b < a.blocks; ++b) {
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int n = h[(b << a.bits) + q];
                total[q] += n;
                mine[q] += b < (int)blockIdx.x ? n : 0;
            }
        }
#pragma unroll
        for (int q = 0; q < PER; ++q) sum += total[q];
    }
    int lower, all;
    scan_threads<SORT_WAVES>(sum, s_sum, lower, all);
    if (d0 < digits) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            s_base[d0 + q] = lower + mine[q];
            lower += total[q];
        }
    }
    if (FIRST && blockIdx.x == 0 && tid == 0) a.counts[0] = all;
    const int64_t items = FIRST ? a.items : all;
    const int64_t begin = (int64_t)blockIdx.x * a.tile, end = min(items, begin + a.tile);
    for (int64_t r0 = begin; r0 < end; r0 += SORT_THREADS * SORT_ITEMS) {
        int key[SORT_ITEMS], pos[SORT_ITEMS], rank[SORT_ITEMS];
        sort_keys<FIRST, SORT_ITEMS>(a, r0 + (int64_t)wave * 64 * SORT_ITEMS + lane, 64, end, false, key, pos);
        if constexpr (PER > 1) {
            for (int i = tid; i < SORT_WAVES * digits / 4; i += SORT_THREADS) ((int4*)s_wave)[i] = make_int4(0, 0, 0, 0);
        } else {
            for (int i = tid; i < SORT_WAVES * digits; i += SORT_THREADS) s_wave[i] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u) rank[u] = rank_in_wave(key[u], (key[u] >> a.shift) & (digits - 1), a.bits, s_wave + (wave << a.bits));
        __syncthreads();
        if constexpr (PER == 1) {       // counts -> first places; the base moves on for the next round
            if (tid < digits) {
                int at = s_base[tid];
#pragma unroll
                for (int w = 0; w < SORT_WAVES; ++w) {
                    const int c = s_wave[(w << a.bits) + tid];
                    s_wave[(w << a.bits) + tid] = at;
                    at += c;
                }
                s_base[tid] = at;
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u) {
            if (key[u] < 0) continue;
            const int digit = (key[u] >> a.shift) & (digits - 1);
            int at = rank[u];
            if constexpr (PER == 1) {
                at += s_wave[(wave << a.bits) + digit];
            } else {                    // more digits than items, and one round: every item adds up the waves before its own
                at += s_base[digit];
#pragma unroll
                for (int w = 0; w < SORT_WAVES - 1; ++w) {
                    const int c = s_wave[(w << a.bits) + digit];
                    at += w < wave ? c : 0;
                }
            }
            a.key_out[at] = key[u];
            a.pos_out[at] = pos[u];
        }
        __syncthreads();
    }
}

// The whole sort of a small batch in one block: the items stay in registers, and change places through the LDS after every pass.
constexpr int ONE_WAVES = 16, ONE_THREADS = 64 * ONE_WAVES;
template <int ONE_ITEMS>
constexpr int one_block_lds() { return ONE_WAVES * MAX_DIGITS * 4 + ONE_THREADS * ONE_ITEMS * (4 + 2) + 64 * 4; }
template <int ONE_ITEMS>
__global__ __launch_bounds__(ONE_THREADS) void sort_one_block_kernel(SortPass a, int passes) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int* const s_wave = (int*)lds;                            // [ONE_WAVES][digits]
    int* const s_key = s_wave + ONE_WAVES * MAX_DIGITS;
    uint16_t* const s_pos = (uint16_t*)(s_key + ONE_THREADS * ONE_ITEMS);
    int* const s_sum = (int*)(s_pos + ONE_THREADS * ONE_ITEMS);
    const int digits = 1 << a.bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rounds = (int)((a.items + ONE_THREADS - 1) / ONE_THREADS), first = wave * rounds * 64 + lane;    // a wave's items lie next to each other
    clear_flags(a, tid, ONE_THREADS);
    int key[ONE_ITEMS], pos[ONE_ITEMS], rank[ONE_ITEMS];
    uint8_t m[ONE_ITEMS];
#pragma unroll
    for (int u = 0; u < ONE_ITEMS; ++u) {
        pos[u] = min(first + u * 64, (int)a.items - 1);
        key[u] = u < rounds ? a.tokens[pos[u]] : -1;
        m[u] = u < rounds && a.mask ? a.mask[pos[u]] : 1;
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < ONE_ITEMS; ++u) {
        const bool here = u < rounds && first + u * 64 < (int)a.items && m[u] != 0, in = key[u] >= 0 && key[u] < a.V;
        bad |= here && !in;
        if (!here || !in) key[u] = -1;
    }
    if (bad && a.dev_status) atomicOr(a.dev_status, RAPID_STATUS_BAD_TOKEN);
    int items = 0;
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * a.bits;
        for (int i = tid; i < ONE_WAVES * digits; i += ONE_THREADS) s_wave[i] = 0;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ONE_ITEMS; ++u) {
            rank[u] = 0;
            if (u < rounds) rank[u] = rank_in_wave(key[u], (key[u] >> shift) & (digits - 1), a.bits, s_wave + wave * digits);
        }
        __syncthreads();
        int total = 0, lower;
        if (tid < digits) {
#pragma unroll
            for (int w = 0; w < ONE_WAVES; ++w) total += s_wave[w * digits + tid];
        }
        scan_threads<ONE_WAVES>(total, s_sum, lower, items);
        if (tid < digits) {
#pragma unroll
            for (int w = 0; w < ONE_WAVES; ++w) {
                const int c = s_wave[w * digits + tid];
                s_wave[w * digits + tid] = lower;
                lower += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ONE_ITEMS; ++u) {
            if (key[u] < 0) continue;
            const int at = s_wave[wave * digits + ((key[u] >> shift) & (digits - 1))] + rank[u];
            s_key[at] = key[u];
            s_pos[at] = (uint16_t)pos[u];
        }
        __syncthreads();
        if (pass + 1 < passes) {
#pragma unroll
            for (int u = 0; u < ONE_ITEMS; ++u) {
                const int i = first + u * 64;
                const bool here = u < rounds && i < items;
                key[u] = here ? s_key[i] : -1;
                pos[u] = here ? s_pos[i] : 0;
            }
        }
    }
    for (int i = tid; i < items; i += ONE_THREADS) {
        a.key_out[i] = s_key[i];
        a.pos_out[i] = s_pos[i];
    }
    if (tid == 0) a.counts[0] = items;
}

// --------------------------------------------------------------------------------------------- sums
// Sorted position i of the batch has id key[i].  A group of threads takes a stretch of sorted positions (the batch's valid positions shared out
// evenly over at most `stretches` groups, which is about what the chip holds at once), a thread one piece of
// the columns, and adds the gradient rows up in fp32; an id's sum that began and ended inside the stretch is the row of dE.  What crosses an end of the
// stretch goes to `part`: slot 0 the sum that came in from before and ended here, slot 1 the one that goes on behind (it may have come in, too).  So the
// work is shared out by rows whatever the ids are: one id that owns the whole batch is as quick as all ids different.
struct SumArgs {
    const int32_t *key, *pos, *counts;
    int64_t stretches, least_rows;
    int pieces;             // of a row
    float* part;            // [stretches][2][d]
    uint8_t* flags;         // NULL (accumulate), or a byte per id that is set for those that occur
    int64_t d;
    float scale;
    int once;               // the gradient rows are more than the caches hold: read past them (256 x 2048 x 1536 bf16: sums 273 -> 237 us)
};
__device__ __forceinline__ int64_t stretch_rows(const SumArgs& a, int64_t M) { return max(a.least_rows, (M + a.stretches - 1) / a.stretches); }

template <class P, class D, bool ACC>
__device__ __forceinline__ void store_row(D* __restrict__ at, const float (&acc)[P::N], const float (&old)[ACC ? P::N : 1], float scale) {
    constexpr int N = P::N;
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = ACC ? fmaf(acc[e], scale, old[ACC ? e : 0]) : acc[e] * scale;
    if constexpr (sizeof(D) == 4 && N == 1) {
        at[0] = f[0];
    } else if constexpr (sizeof(D) == 4) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) ((float4*)at)[q] = make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]);
    } else if constexpr (N == 8) {
        *(uint4*)at = pack8(f);
    } else if constexpr (N == 4) {
        *(uint2*)at = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
    } else {
        at[0] = __builtin_bit_cast(bf16_t, (__bf16)f[0]);
    }
}
template <class P, class D, bool ACC>
__device__ __forceinline__ void load_row(const D* __restrict__ at, float (&old)[ACC ? P::N : 1]) {
    if constexpr (ACC && P::N == 1) old[0] = at[0];
    else if constexpr (ACC) {
#pragma unroll
        for (int q = 0; q < P::N / 4; ++q) {
            const float4 v = ((const float4*)at)[q];
            old[4 * q] = v.x; old[4 * q + 1] = v.y; old[4 * q + 2] = v.z; old[4 * q + 3] = v.w;
        }
    }
}

// U rows under way together; with ACC also the old values of the rows that end among them.  The next batch's ids and positions are asked for
// before this batch's rows are waited for.  WAVES: groups are whole waves, ids and positions scalars (104 registers a thread without, 70 with).
template <class P, class D, bool ACC, bool WAVES>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs a, const typename P::elem* __restrict__ dh, D* __restrict__ dE) {
    typedef typename P::raw raw;
    constexpr int U = ACC ? 4 : 8;
    const int64_t M = a.counts[0], rows = stretch_rows(a, M);
    const int group = WAVES ? __builtin_amdgcn_readfirstlane(threadIdx.y) : threadIdx.y;
    const int64_t s = (int64_t)blockIdx.x * blockDim.y + group, begin = s * rows;
    const int piece = blockIdx.y * blockDim.x + threadIdx.x;
    if (begin >= M || piece >= a.pieces) return;
    const int64_t end = min(M, begin + rows);
    const raw* src = (const raw*)dh + piece;
    float acc[P::N];
#pragma unroll
    for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
    const int behind = end < M ? a.key[end] : -1;
    bool came_in = begin > 0 && a.key[begin - 1] == a.key[begin];
    int k[U], p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = min(begin + u, end - 1);
        k[u] = a.key[i];
        p[u] = a.pos[i];
    }
    for (int64_t i0 = begin; i0 < end; i0 += U) {
        raw v[U];
        float old[U][ACC ? P::N : 1];
        int kn[U], pn[U];
        if (a.once) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_once(src + (int64_t)p[u] * a.pieces);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = src[(int64_t)p[u] * a.pieces];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = min(i0 + U + u, end - 1);
            kn[u] = a.key[i];
            pn[u] = a.pos[i];
        }
        auto next_of = [&](int u) { return i0 + u + 1 >= end ? behind : u + 1 < U ? k[u + 1] : kn[0]; };
        if constexpr (ACC) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (next_of(u) != k[u]) load_row<P, D, ACC>(dE + (int64_t)k[u] * a.d + (int64_t)piece * P::N, old[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u >= end) break;
            float f[P::N];
            P::get(v[u], f);
#pragma unroll
            for (int e = 0; e < P::N; ++e) acc[e] += f[e];
            const bool last = i0 + u + 1 == end, goes_on = next_of(u) == k[u];
            if (goes_on && !last) continue;
            if (came_in || goes_on) {
                float* to = a.part + (s * 2 + (goes_on ? 1 : 0)) * a.d + (int64_t)piece * P::N;
#pragma unroll
                for (int e = 0; e < P::N; ++e) to[e] = acc[e];
            } else {
                store_row<P, D, ACC>(dE + (int64_t)k[u] * a.d + (int64_t)piece * P::N, acc, old[u], a.scale);
            }
            if (!ACC && piece == 0) a.flags[k[u]] = 1;
            came_in = false;
#pragma unroll
            for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) { k[u] = kn[u]; p[u] = pn[u]; }
    }
}

// acc += what stretches from .. to - 1 left of the id whose run ends in stretch `last`, in order; U of them under way together, the last ones too
template <int U, int N>
__device__ __forceinline__ void add_parts(const float* __restrict__ part, int64_t d, int64_t from, int64_t to, int64_t last, float (&acc)[N]) {
    for (int64_t c0 = from; c0 < to; c0 += U) {
        float v[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = min(c0 + u, to - 1);
            const float* q = part + (c * 2 + (c == last ? 0 : 1)) * d;
#pragma unroll
            for (int e = 0; e < N; ++e) v[u][e] = q[e];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += c0 + u < to ? v[u][e] : 0.f;
    }
}
// Joins the sums that crossed ends of stretches, and clears the rows of the ids that do not occur.  A wave looks at one stretch, and for the id that begins
// in it and goes on behind it adds up what the stretches after it left, 64 pieces of the columns; ids of more than SHORT_RUN stretches are left to the
// block's waves together (in MERGE_WAVES consecutive shares, then these in order).  The blocks behind those clear ZERO_ROWS ids a wave.
// (A block a stretch: 6144 blocks of little more than two trips to the keys each, 8.6 of 36 us in the bandit's batch.)
constexpr int MERGE_WAVES = 8, ZERO_ROWS = 16, SHORT_RUN = 16;
template <class P, class D, bool ACC, class W>
__global__ __launch_bounds__(64 * MERGE_WAVES) void embedding_merge_kernel(SumArgs a, D* __restrict__ dE, int64_t V, int64_t row_words) {
    __shared__ float s_sum[MERGE_WAVES][64][P::N];
    __shared__ int64_t s_last[MERGE_WAVES];                 // of the wave's run, if all waves are to join it
    __shared__ int s_key[MERGE_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunks = (a.pieces + 63) / 64;                // of a row: a block each
    const int64_t joins = (a.stretches + MERGE_WAVES - 1) / MERGE_WAVES * chunks;
    if (!ACC && blockIdx.x >= joins) {
        const int64_t v0 = ((blockIdx.x - joins) * MERGE_WAVES + wave) * ZERO_ROWS;
        unsigned long long rows = __ballot(lane < ZERO_ROWS && v0 + lane < V && a.flags[v0 + lane] == 0);
        for (; rows; rows &= rows - 1) {
            W* row = (W*)dE + (v0 + __ffsll((long long)rows) - 1) * row_words;
            for (int64_t i = lane; i < row_words; i += 64) row[i] = W{};
        }
        return;
    }
    const int64_t s0 = blockIdx.x / chunks * (int64_t)MERGE_WAVES, s = s0 + wave;
    const int piece = (int)(blockIdx.x % chunks) * 64 + lane;
    const int64_t M = a.counts[0], n_rows = stretch_rows(a, M), begin = s * n_rows, end = begin + n_rows;
    const float* const part = a.part + (int64_t)piece * P::N;
    auto finish = [&](int key, float (&acc)[P::N]) {
        D* to_row = dE + (int64_t)key * a.d + (int64_t)piece * P::N;
        float old[ACC ? P::N : 1];
        load_row<P, D, ACC>(to_row, old);
        store_row<P, D, ACC>(to_row, acc, old, a.scale);
    };
    int64_t last = s;                                       // the stretch in which the run ends (s: none begins here that goes on)
    int key = 0;
    if (end < M) {                                          // (nothing goes on behind the last stretch; the keys are asked for together)
        key = a.key[end - 1];
        const int behind = a.key[end], first = a.key[begin], before = a.key[begin > 0 ? begin - 1 : 0];
        if (behind == key && !(first == key && begin > 0 && before == key)) {
            // the first stretch behind this one whose last row is not the id's, or not there: 64 are looked at together, every one, or (long
            // runs) every 64th, then the 64 in between
            auto ends = [&](int64_t c) { return c * n_rows >= M - n_rows || a.key[(c + 1) * n_rows - 1] != key; };
            int64_t step = 1;
            for (last = s + 1;;) {
                const unsigned long long other = __ballot(ends(last + lane * step));
                last += (other ? __ffsll((long long)other) - 1 : 64) * step;
                if (other && step == 1) break;
                if (other) last -= 63;
                step = other ? 1 : 64;
            }
            if (a.key[last * n_rows] != key) --last;        // it ended with the stretch before (its sum there is in slot 0 all the same)
        }
    }
    const bool together = last - s >= SHORT_RUN;
    if (lane == 0) { s_last[wave] = together ? last : -1; s_key[wave] = key; }
    if (last > s && !together && piece < a.pieces) {
        float acc[P::N];
#pragma unroll
        for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
        add_parts<4, P::N>(part, a.d, s, last + 1, last, acc);
        finish(key, acc);
    }
    __syncthreads();
    for (int w = 0; w < MERGE_WAVES; ++w) {
        if (s_last[w] < 0) continue;
        const int64_t begun = s0 + w, n = s_last[w] - begun + 1;
        float acc[P::N];
#pragma unroll
        for (int e = 0; e < P::N; ++e) acc[e] = 0.f;
        if (piece < a.pieces) add_parts<8, P::N>(part, a.d, begun + n * wave / MERGE_WAVES, begun + n * (wave + 1) / MERGE_WAVES, s_last[w], acc);
#pragma unroll
        for (int e = 0; e < P::N; ++e) s_sum[wave][lane][e] = acc[e];
        __syncthreads();
        if (wave == 0 && piece < a.pieces) {
#pragma unroll
            for (int o = 1; o < MERGE_WAVES; ++o)
#pragma unroll
                for (int e = 0; e < P::N; ++e) acc[e] += s_sum[o][lane][e];
            finish(s_key[w], acc);
        }
        __syncthreads();
    }
}

// threads of a group: enough of them for a row's pieces, up to a block
int group_threads(int64_t pieces) {
    if (pieces > 64) return pieces >= 256 ? 256 : (int)((pieces + 63) / 64 * 64);
    int x = 8;
    while (x < pieces) x *= 2;
    return x;
}

template <class P, class D, bool ACC, class W>
void sum_t(const SumArgs& s, int64_t V, int64_t row_words, const void* dh, D* dE, hipStream_t st) {
    const int x = group_threads(s.pieces), y = 256 / x;
    const dim3 grid((unsigned)((s.stretches + y - 1) / y), (unsigned)((s.pieces + x - 1) / x)), block(x, y);
    if (x % 64 == 0) embedding_sum_kernel<P, D, ACC, true><<<grid, block, 0, st>>>(s, (const typename P::elem*)dh, dE);
    else embedding_sum_kernel<P, D, ACC, false><<<grid, block, 0, st>>>(s, (const typename P::elem*)dh, dE);
    const int64_t blocks = (s.stretches + MERGE_WAVES - 1) / MERGE_WAVES * ((s.pieces + 63) / 64) + (ACC ? 0 : (V + MERGE_WAVES * ZERO_ROWS - 1) / (MERGE_WAVES * ZERO_ROWS));
    embedding_merge_kernel<P, D, ACC, W><<<(unsigned)blocks, 64 * MERGE_WAVES, 0, st>>>(s, dE, V, row_words);
}
template <class P, class D>
void sum_d(const SumArgs& s, int64_t V, const void* dh, D* dE, hipStream_t st) {
    if constexpr (sizeof(D) == 4)
        if (!s.flags) { sum_t<P, D, true, D>(s, V, 0, dh, dE, st); return; }
    const int64_t bytes = s.d * (int64_t)sizeof(D);
    if (bytes % 16 == 0) sum_t<P, D, false, uint4>(s, V, bytes / 16, dh, dE, st);
    else sum_t<P, D, false, D>(s, V, s.d, dh, dE, st);
}

int pieces_of(int64_t d, int dtype) { return (int)(d / (dtype == RAPID_DTYPE_BF16 ? 8 : d % 4 == 0 ? 4 : 1)); }

// Items a thread takes in a round of the sort.  Few positions: more blocks with less to do each.
constexpr int FEW_ITEMS = 2, MANY_ITEMS = 8;
// d = 64, whole gradients: with 2 items and with 8 65536 positions 62 and 72 us, 131072 97 and 105, 262144 142 and 142, 524288 147 and 142 (V = 151936).
constexpr int64_t FEW_POSITIONS = 131072;
// One pass over 10 to 12 bits and two of half as many, V = 4096: 8200 positions 23.8 and 30.1 us, 32768 38.2 and 39.1, 65536 62.9 and 59.7.
constexpr int64_t WIDE_POSITIONS = 32768;
static_assert(WIDE_POSITIONS <= 256 * SORT_THREADS * FEW_ITEMS && WIDE_POSITIONS <= FEW_POSITIONS, "a block of a wide pass has one round");
// All passes in one block, and the launches of many.  Ids that many blocks sort in one pass: V = 4096: 2048 positions 18.8 and 19.1 us, 4096 22.7 and 21.2,
// 8192 29.5 and 22.7; V = 300: 2048 16.4 and 17.4, 4097 21.4 and 19.9.  In two or more: V = 5000: 5120 26.2 and 26.4, 8192 31.8 and 31.2; V = 151936: 4096
// 30.1 and 32.3, 6144 34.3 and 34.1, 8192 37.3 and 35.2.
constexpr int64_t ONE_BLOCK_ONE_PASS = 2560, ONE_BLOCK_SORT = 6144;
static_assert(ONE_BLOCK_ONE_PASS <= ONE_BLOCK_SORT && ONE_BLOCK_SORT <= 8 * ONE_THREADS, "a block holds its items in registers, 8 a thread");
int64_t sort_tile(int64_t positions) {
    const int64_t round = SORT_THREADS * (positions <= FEW_POSITIONS ? FEW_ITEMS : MANY_ITEMS);
    const int64_t per = (positions + 255) / 256;            // at most 256 blocks: every block adds up the counts of all
    return (per + round - 1) / round * round;
}
template <int ITEMS>
void sort_one_t(const SortPass& s, int passes, hipStream_t st) {
    allow_lds<&sort_one_block_kernel<ITEMS>>(one_block_lds<ITEMS>());
    sort_one_block_kernel<ITEMS><<<1, ONE_THREADS, one_block_lds<ITEMS>(), st>>>(s, passes);
}
template <bool FIRST, int ITEMS, int DIGITS>
void sort_pass_t(const SortPass& s, hipStream_t st) {
    sort_count_kernel<FIRST, ITEMS, DIGITS><<<(unsigned)s.blocks, SORT_THREADS, 0, st>>>(s);
    allow_lds<&sort_scatter_kernel<FIRST, ITEMS, DIGITS>>(scatter_lds<DIGITS>());
    sort_scatter_kernel<FIRST, ITEMS, DIGITS><<<(unsigned)s.blocks, SORT_THREADS, scatter_lds<DIGITS>(), st>>>(s);
}
void sort_pass(const SortPass& s, hipStream_t st) {
    const bool few = s.items <= FEW_POSITIONS, first = s.shift == 0;
    if (s.bits > MAX_DIGIT_BITS) sort_pass_t<true, FEW_ITEMS, WIDE_DIGITS>(s, st);
    else if (few) first ? sort_pass_t<true, FEW_ITEMS, MAX_DIGITS>(s, st) : sort_pass_t<false, FEW_ITEMS, MAX_DIGITS>(s, st);
    else first ? sort_pass_t<true, MANY_ITEMS, MAX_DIGITS>(s, st) : sort_pass_t<false, MANY_ITEMS, MAX_DIGITS>(s, st);
}

}  // namespace

void launch_embedding_fwd(const EmbeddingArgs& a, const void* table, void* out, hipStream_t st) {
    if (a.dtype == RAPID_DTYPE_BF16) fwd_t<BF16x8>(a, table, out, st);
    else if (a.d % 4 == 0) fwd_t<F32x4>(a, table, out, st);
    else if (a.d > 4) fwd_t<F32x4Any>(a, table, out, st);
    else fwd_t<F32x1>(a, table, out, st);
}

EmbeddingPlan embedding_plan(int64_t positions, int64_t d, int64_t V, int dtype) {
    EmbeddingPlan p;
    int bits = 1;
    while (((int64_t)1 << bits) < V) ++bits;
    p.one_block = positions <= (bits <= WIDE_BITS ? ONE_BLOCK_ONE_PASS : ONE_BLOCK_SORT);
    p.passes = bits <= WIDE_BITS && !p.one_block && positions <= WIDE_POSITIONS ? 1 : (bits + MAX_DIGIT_BITS - 1) / MAX_DIGIT_BITS;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tile = sort_tile(positions);
    p.blocks = (positions + p.tile - 1) / p.tile;
    // 28 waves per CU, 4 rows at least a group
    p.least_rows = 4;
    const int64_t pieces = pieces_of(d, dtype), x = group_threads(pieces), held = (int64_t)7168 * 64 / ((pieces + x - 1) / x * x);
    const int64_t wanted = (positions + p.least_rows - 1) / p.least_rows;
    p.stretches = wanted < held ? wanted : held < 64 ? 64 : held;
    if (p.stretches > wanted) p.stretches = wanted;
    size_t cur = 0;
    auto take = [&](size_t bytes) { const size_t at = cur; cur += (bytes + 255) / 256 * 256; return at; };
    p.counts = take(64 * 4);
    for (int i = 0; i < 2; ++i) {
        p.key[i] = take((size_t)positions * 4);
        p.pos[i] = take((size_t)positions * 4);
    }
    p.hist = take((size_t)p.blocks * (1u << p.bits) * 4);
    p.flags = take((size_t)V);
    p.part = take((size_t)p.stretches * 2 * (size_t)d * 4);
    p.total = cur;
    return p;
}

void launch_embedding_bwd(const EmbeddingArgs& a, const EmbeddingPlan& p, void* ws, const void* dh, int dw_dtype, int accumulate, void* dE, hipStream_t st) {
    char* w = (char*)ws;
    SortPass s{};
    s.tokens = a.tokens; s.mask = a.mask; s.V = (int)a.V; s.dev_status = a.dev_status;
    s.hist = (int32_t*)(w + p.hist); s.counts = (int32_t*)(w + p.counts);
    s.flags = accumulate ? nullptr : (uint32_t*)(w + p.flags); s.flag_words = (a.V + 3) / 4;
    s.items = a.positions; s.tile = p.tile; s.bits = p.bits; s.blocks = (int)p.blocks;
    if (p.one_block) {
        s.key_out = (int32_t*)(w + p.key[0]); s.pos_out = (int32_t*)(w + p.pos[0]);
        if (a.positions <= ONE_THREADS) sort_one_t<1>(s, p.passes, st);
        else if (a.positions <= 4 * ONE_THREADS) sort_one_t<4>(s, p.passes, st);
        else sort_one_t<8>(s, p.passes, st);
    } else {
        for (int pass = 0; pass < p.passes; ++pass) {
            const int to = pass & 1;
            s.shift = pass * p.bits;
            s.key_in = (const int32_t*)(w + p.key[to ^ 1]); s.pos_in = (const int32_t*)(w + p.pos[to ^ 1]);
            s.key_out = (int32_t*)(w + p.key[to]); s.pos_out = (int32_t*)(w + p.pos[to]);
            sort_pass(s, st);
        }
    }
    SumArgs u{};
    u.key = s.key_out; u.pos = s.pos_out; u.counts = s.counts; u.stretches = p.stretches; u.least_rows = p.least_rows;
    u.pieces = pieces_of(a.d, a.dtype);
    u.part = (float*)(w + p.part); u.flags = (uint8_t*)s.flags; u.d = a.d; u.scale = a.scale;
    u.once = a.positions * a.d * (a.dtype == RAPID_DTYPE_BF16 ? 2 : 4) > BEYOND_CACHES;
    auto go = [&](auto* out) {
        if (a.dtype == RAPID_DTYPE_BF16) sum_d<BF16x8>(u, a.V, dh, out, st);
        else if (a.d % 4 == 0) sum_d<F32x4>(u, a.V, dh, out, st);
        else sum_d<F32x1>(u, a.V, dh, out, st);
    };
    if (dw_dtype == RAPID_DTYPE_F32) go((float*)dE);
    else go((bf16_t*)dE);
}

}  // namespace rapid

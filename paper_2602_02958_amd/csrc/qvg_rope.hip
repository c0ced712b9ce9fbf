// Rotary positions: tables of (cos, sin), rows turned by them, and the new tokens' way into a cache of 16-bit pages, their keys turned
// on the way.
#include "qvg_rows.hpp"

#include <type_traits>

namespace qvg {

// ---- tables -------------------------------------------------------------------------------------------------
// A pair to a thread.  The angle is taken in quarter turns: place x frequency x 4 / 2 pi in 64 bits, less its nearest whole number (adding
// 1.5 x 2^52 rounds to it, and leaves it in the sum's low bits), is half a quarter or less, which 32 bits hold to 2^-27 of a
// turn.  Sine and cosine of that are Taylor's polynomials in 32 bits (their next terms are below 2^-29 at pi / 4), and the quarter says which
// is which and its sign.  Memory bounds a large table of 32 bits: 748800 x 64 pairs and three axes, 392 MB, 70 us (5.6 TB/s); of 16 bits the
// 35 instructions of a pair do, 49 us for 201 MB (replayed in a graph).
__device__ __forceinline__ float2 cos_sin_of(double place, double quarters) {
    const double x = place * quarters, sum = x + 6755399441055744.0;
    const float r = (float)(x - (sum - 6755399441055744.0));
    const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, sum);
    const float z = __builtin_amdgcn_fmed3f(r, -0.5f, 0.5f) * 1.57079637f, w = z * z;
    auto fma = [](float x, float y, float t) { return __builtin_fmaf(x, y, t); };
    const float s = fma(z * w, fma(w, fma(w, fma(w, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), z);
    const float c = fma(w, fma(w, fma(w, fma(w, fma(w, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
    const uint32_t cb = __float_as_uint(k & 1u ? s : c) ^ ((k + 1u & 2u) << 30), sb = __float_as_uint(k & 1u ? c : s) ^ ((k & 2u) << 30);
    return make_float2(__uint_as_float(cb), __uint_as_float(sb));
}
template <typename TAB, int ROWS, bool GIVEN>
__global__ __launch_bounds__(256)
void rope_table_kernel(RopeTableArgs a, FastDiv by_pairs, int rows_per_block) {
    typedef uint32_t two __attribute__((ext_vector_type(2)));
    typedef typename std::conditional<sizeof(TAB) == 4, two, uint32_t>::type pair;
    const int sub = (int)quotient(threadIdx.x, by_pairs), p = (int)threadIdx.x - sub * a.n_pairs;
    const int64_t i0 = (a.first_block + blockIdx.x) * (rows_per_block * ROWS) + sub, left = a.n_rows - i0;
    if (sub >= rows_per_block || left <= 0) return;
    const double quarters = a.freq[p] * 0.6366197723675814;
    // (rows, and pairs, are a fixed way apart: addresses are sums)
    const int rows = (int)(left < ROWS * 256 ? left : ROWS * 256);       // (of which every rows_per_block-th is this thread's)
    int at[ROWS];
    if constexpr (GIVEN) {
        // (where the arguments lie: as a value, indexed at run time, every thread would keep the axes in scratch memory)
        const int ax = ((const RopeTableArgs *)__builtin_amdgcn_kernarg_segment_ptr())->axis[p];
        const int32_t *from = a.positions + (i0 * a.n_axes + ax);
#pragma unroll
        for (int j = 0; j < ROWS; ++j) at[j] = from[(uint32_t)(min(j * rows_per_block, rows - 1) * a.n_axes)];
    } else {
#pragma unroll
        for (int j = 0; j < ROWS; ++j) at[j] = (int)(a.first + i0) + j * rows_per_block;
    }
    pair *to = reinterpret_cast<pair *>(a.out) + (i0 * a.n_pairs + p);
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (j * rows_per_block >= rows) return;
        float2 cs = cos_sin_of((double)at[j], quarters);
        cs.x *= a.amplitude; cs.y *= a.amplitude;
        pair v;
        if constexpr (sizeof(TAB) == 4) v = two{__float_as_uint(cs.x), __float_as_uint(cs.y)};
        else v = pack_f16x2_rne(cs.x, cs.y);
        pair *row = to + (uint32_t)(j * rows_per_block * a.n_pairs);
        // (replayed in a graph a large table, 392 MB, takes 66 to 72 us past the caches, 80 through them, and what reads it next is no
        // slower: 37440 places and then 12 x 4680 rows turned by some of them 11.5 and 11.8 us)
        if constexpr (ROWS > 1) __builtin_nontemporal_store(v, row);
        else *row = v;
    }
}
constexpr int64_t kMostBlocks = 1 << 23;        // of a launch: it has fewer than 2^32 threads along an axis
template <typename TAB, int ROWS>
static void launch_table(RopeTableArgs a, int64_t blocks, int per, hipStream_t s) {
    const FastDiv by = fast_div((uint32_t)a.n_pairs);
    for (a.first_block = 0; a.first_block < blocks; a.first_block += kMostBlocks) {
        const dim3 n((unsigned)(blocks - a.first_block < kMostBlocks ? blocks - a.first_block : kMostBlocks));
        if (a.positions) rope_table_kernel<TAB, ROWS, true><<<n, dim3(256), 0, s>>>(a, by, per);
        else rope_table_kernel<TAB, ROWS, false><<<n, dim3(256), 0, s>>>(a, by, per);
    }
}
constexpr int kTableRows = 16;     // of a thread, whose places it asks for together, where there are many
hipError_t launch_rope_table(const RopeTableArgs &a, bool f32, hipStream_t s) {
    const int per = 256 / a.n_pairs;
    const int64_t blocks = (a.n_rows + per - 1) / per, fewer = (blocks + kTableRows - 1) / kTableRows;
    if (blocks > 8192) f32 ? launch_table<float, kTableRows>(a, fewer, per, s) : launch_table<f16_t, kTableRows>(a, fewer, per, s);
    else f32 ? launch_table<float, 1>(a, blocks, per, s) : launch_table<f16_t, 1>(a, blocks, per, s);
    return hipGetLastError();
}

// ---- rows -----------------------------------------------------------------------------------------------------
struct Bf16 { typedef bf16_t raw; };
struct F16 { typedef f16_t raw; };
struct F32 { typedef float raw; };
template <class T> struct Octet { uint4 w[sizeof(typename T::raw) / 2]; };      // eight elements as stored

template <class T>
__device__ __forceinline__ Octet<T> load_octet(const typename T::raw *p) {
    Octet<T> o;
#pragma unroll
    for (size_t i = 0; i < sizeof(o.w) / 16; ++i) o.w[i] = reinterpret_cast<const uint4 *>(p)[i];
    return o;
}
// FAR: past the caches' usual order of eviction
template <class T, bool FAR>
__device__ __forceinline__ void store_octet(typename T::raw *p, const Octet<T> &o) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
#pragma unroll
    for (size_t i = 0; i < sizeof(o.w) / 16; ++i) {
        if constexpr (FAR) __builtin_nontemporal_store(__builtin_bit_cast(words, o.w[i]), reinterpret_cast<words *>(p) + i);
        else reinterpret_cast<uint4 *>(p)[i] = o.w[i];
    }
}
__device__ __forceinline__ void octet_values(const Octet<Bf16> &o, float *v) { unpack_bf16x8(o.w[0], v); }
__device__ __forceinline__ void octet_values(const Octet<F16> &o, float *v) {
    const uint32_t w[4] = {o.w[0].x, o.w[0].y, o.w[0].z, o.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = f16_bits_to_f32(w[i] & 0xffffu); v[2 * i + 1] = f16_bits_to_f32(w[i] >> 16); }
}
__device__ __forceinline__ void octet_values(const Octet<F32> &o, float *v) { __builtin_memcpy(v, o.w, 32); }
__device__ __forceinline__ void octet_of(const float *v, Octet<Bf16> &o) { o.w[0] = pack_bf16x8(v); }
__device__ __forceinline__ void octet_of(const float *v, Octet<F16> &o) {
    o.w[0] = make_uint4(pack_f16x2_rne(v[0], v[1]), pack_f16x2_rne(v[2], v[3]), pack_f16x2_rne(v[4], v[5]), pack_f16x2_rne(v[6], v[7]));
}
__device__ __forceinline__ void octet_of(const float *v, Octet<F32> &o) { __builtin_memcpy(o.w, v, 32); }
// the pairs of an octet from `from` on, as they were
template <class T>
__device__ __forceinline__ void keep_pairs(Octet<T> &o, const Octet<T> &was, int from) {
    constexpr int kWords = sizeof(typename T::raw) / 2;                  // 32-bit words of a pair
    uint32_t now[4 * kWords], old[4 * kWords];
    __builtin_memcpy(now, o.w, sizeof(now));
    __builtin_memcpy(old, was.w, sizeof(old));
#pragma unroll
    for (int i = 0; i < 4 * kWords; ++i) now[i] = i / kWords < from ? now[i] : old[i];
    __builtin_memcpy(o.w, now, sizeof(now));
}
__device__ __forceinline__ float value_of(bf16_t x, Bf16) { return bf16_lo(x); }
__device__ __forceinline__ float value_of(f16_t x, F16) { return f16_bits_to_f32(x); }
__device__ __forceinline__ float value_of(float x, F32) { return x; }
__device__ __forceinline__ bf16_t raw_of(float x, Bf16) { return (bf16_t)pack_bf16x2(x, 0.0f); }
__device__ __forceinline__ f16_t raw_of(float x, F16) { return (f16_t)f32_to_f16_bits(x); }
__device__ __forceinline__ float raw_of(float x, F32) { return x; }

__device__ __forceinline__ void turn(float &x0, float &x1, float2 cs) {
    const float t0 = x1 * cs.y, t1 = x1 * cs.x, y0 = __builtin_fmaf(x0, cs.x, -t0);
    x1 = __builtin_fmaf(x0, cs.y, t1);
    x0 = y0;
}
template <typename TAB>
__device__ __forceinline__ float2 table_pair(const TAB *row, int p) {
    if constexpr (sizeof(TAB) == 4) return reinterpret_cast<const float2 *>(row)[p];
    else {
        const uint32_t w = reinterpret_cast<const uint32_t *>(row)[p];
        return make_float2(f16_bits_to_f32(w & 0xffffu), f16_bits_to_f32(w >> 16));
    }
}
// Pairs p0 .. p0 + N - 1 (N a multiple of 4) of a row; `whole`: rows are 16-byte aligned and have all of them
template <typename TAB, int N>
__device__ __forceinline__ void table_pairs(const TAB *row, int p0, int n_pairs, bool whole, float2 *cs) {
    if (whole) {
        constexpr int kWords = N * (int)sizeof(TAB) / 8;
        uint4 w[kWords];
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4 *>(row + 2 * p0)[i];
        if constexpr (sizeof(TAB) == 4) __builtin_memcpy(cs, w, sizeof(w));
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t x = (&w[i / 4].x)[i % 4];
                cs[i] = make_float2(f16_bits_to_f32(x & 0xffffu), f16_bits_to_f32(x >> 16));
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) cs[i] = p0 + i < n_pairs ? table_pair(row, p0 + i) : make_float2(1.0f, 0.0f);
    }
}

// What is done with a row: pairs (2p, 2p + 1), an octet of channels to a thread; pairs (p, p + n), eight of them (two octets) to a
// thread, or one where they do not start at multiples of eight; nothing.  Channels behind the pairs are copied.
enum { kTurnNext, kTurnHalf, kTurnPair, kTurnNone };
constexpr int kTurnHeads = 4;      // heads that a thread takes at once, where there are many rows: they share the table's row

// A thread takes a piece of a token's rows in `HP` heads: it reads the table's row once for all of them, and all rows before it
// writes any.  Memory bounds it, the rows both ways: 40 heads x 10800 rows of 128 bf16, 224 MB with the table, 41 us (5.5 TB/s); 12
// heads x 4680 keys and values into pages, 59 MB, 12.5 us (4.7 TB/s); a token's 12 heads 3.2 us, a launch.  Pages are written past the
// caches: in a graph 9.7 us, 11.3 written through them, which attention that reads them next pays back, so that a step is as long either way
// (append and attend: a chunk behind another, one row of each head 28.8 and 28.7 us, all rows 600 and 598; a token of 16 sequences over
// 512 12.9 and 13.1; 64 new ones of each 33.9 to 34.3 and 34.0).
// One pair to a thread and a head (kTurnPair), where the pairs' second halves start between 16-byte places: 12 x 4680 rows 17 us for 60
// pairs and 23 for 29, 6.2 for 64; into pages 26, 34 and 7.9 (in a graph).  Elements of 2 bytes are loaded and stored one by one; octets
// would have to be shifted between lanes.
template <class T, typename TAB, int MODE, bool APPEND, int HP>
__global__ __launch_bounds__(256)
void turn_kernel(TurnArgs a, int per_block, int whole) {
    typedef typename T::raw raw;
    const int sub = per_block == 1 ? 0 : (int)quotient(threadIdx.x, a.by_units);
    const int64_t t = (a.first_block + blockIdx.x) * per_block + sub;
    if (sub >= per_block || t >= a.tokens) return;
    int u = (int)threadIdx.x - sub * a.units;
    const int b = (int)quotient((uint32_t)t, a.by_tokens), i = (int)t - b * a.n_tokens;
    const raw *src = static_cast<const raw *>(a.x) + b * a.x_seq + i * a.x_tok, *vsrc = nullptr;
    raw *dst, *vdst = nullptr;
    int64_t dst_head;
    int place;
    if constexpr (APPEND) {
        int len = a.kv_len[b], n = a.n_tokens;
        len = len < 0 ? 0 : (len > a.capacity ? a.capacity : len);
        if (a.live) { n = a.live[b]; n = n < 0 ? 0 : (n > a.n_tokens ? a.n_tokens : n); }
        const int room = a.capacity - len;                               // (len + n may pass 31 bits)
        // (where the new lengths have a place of their own; else they wait for the rows to be done with the old ones)
        if (a.lengths_here && i == 0 && u == 0 && blockIdx.y == 0) a.len_out[b] = len + (n < room ? n : room);
        if (i >= n || i >= room) return;
        place = len + i;
        const int pi = (int)quotient((uint32_t)place, a.by_page);
        const uint32_t pg = (uint32_t)a.table[(int64_t)b * a.table_pages + pi];
        if (pg >= a.pool_pages) return;
        const int64_t to = (int64_t)pg * a.page + (int64_t)(place - pi * (int)a.by_page.d) * a.tok;
        dst = static_cast<raw *>(a.k_pages) + to; vdst = static_cast<raw *>(a.v_pages) + to;
        vsrc = static_cast<const raw *>(a.v) + b * a.x_seq + i * a.x_tok;
        dst_head = a.head;
    } else {
        dst = static_cast<raw *>(a.out) + b * a.o_seq + i * a.o_tok;
        dst_head = a.o_head;
        place = 0;
    }
    const TAB *row = nullptr;
    if constexpr (MODE != kTurnNone) {
        int64_t at = a.r.positions ? a.r.positions[t] : APPEND ? place : (a.first ? (int64_t)a.first[b] : 0) + i;
        at = at < 0 ? 0 : (at >= a.r.n_rows ? a.r.n_rows - 1 : at);
        row = static_cast<const TAB *>(a.r.table) + at * (2 * a.r.n_pairs);
    }
    const int P = a.r.n_pairs, heads = (int)gridDim.y;
    const float sign = a.backward ? -1.0f : 1.0f;

    if constexpr (MODE == kTurnPair) {
        for (; u < a.units; u += 256) {                                  // (one piece, but of rows of more than 256)
            const bool pair = u < P;
            const int c0 = pair ? u : u + P;
            float2 cs = make_float2(1.0f, 0.0f);
            if (pair) { cs = table_pair(row, u); cs.y *= sign; }
            for (int h = blockIdx.y; h < a.H; h += heads) {
                const raw *x = src + h * a.x_head;
                raw *y = dst + h * dst_head;
                if (pair) {
                    float x0 = value_of(x[c0], T{}), x1 = value_of(x[c0 + P], T{});
                    turn(x0, x1, cs);
                    y[c0] = raw_of(x0, T{}); y[c0 + P] = raw_of(x1, T{});
                } else y[c0] = x[c0];
                if constexpr (APPEND) {
                    const raw *vx = vsrc + h * a.x_head;
                    raw *vy = vdst + h * dst_head;
                    vy[c0] = vx[c0];
                    if (pair) vy[c0 + P] = vx[c0 + P];
                }
            }
        }
        return;
    }

    constexpr int kOct = MODE == kTurnHalf ? 2 : 1;                      // octets of a piece
    int c[2];                                                            // their first channels
    bool turned;
    if constexpr (MODE == kTurnHalf) {
        turned = u * 8 < P;
        c[0] = turned ? u * 8 : P + u * 8; c[1] = c[0] + (turned ? P : 0);    // (pieces behind the pairs have one octet)
    } else {
        c[0] = c[1] = u * 8;
        turned = MODE == kTurnNext && u * 4 < P;
    }
    float2 cs[4 * kOct];
    if (MODE != kTurnNone && turned) {
        table_pairs<TAB, 4 * kOct>(row, MODE == kTurnHalf ? u * 8 : u * 4, P, whole && (MODE == kTurnHalf || u * 4 + 4 <= P), cs);
#pragma unroll
        for (int p = 0; p < 4 * kOct; ++p) cs[p].y *= sign;
    }
    for (int h0 = blockIdx.y; h0 < a.H; h0 += heads * HP) {
        Octet<T> x[HP][kOct], v[HP][APPEND ? kOct : 1];
#pragma unroll
        for (int k = 0; k < HP; ++k) {
            const int h = h0 + k * heads;
            if (h < a.H) {
#pragma unroll
                for (int o = 0; o < kOct; ++o)
                    if (o == 0 || turned) {
                        x[k][o] = load_octet<T>(src + h * a.x_head + c[o]);
                        if constexpr (APPEND) v[k][o] = load_octet<T>(vsrc + h * a.x_head + c[o]);
                    }
            }
        }
#pragma unroll
        for (int k = 0; k < HP; ++k) {
            const int h = h0 + k * heads;
            if (h < a.H) {
                if (MODE != kTurnNone && turned) {
                    float f[kOct][8];
#pragma unroll
                    for (int o = 0; o < kOct; ++o) octet_values(x[k][o], f[o]);
                    if constexpr (MODE == kTurnHalf) {
#pragma unroll
                        for (int p = 0; p < 8; ++p) turn(f[0][p], f[1][p], cs[p]);
                    } else {
#pragma unroll
                        for (int p = 0; p < 4; ++p)
                            if (u * 4 + p < P) turn(f[0][2 * p], f[0][2 * p + 1], cs[p]);
                    }
                    const Octet<T> was = x[k][0];
#pragma unroll
                    for (int o = 0; o < kOct; ++o) octet_of(f[o], x[k][o]);
                    if constexpr (MODE == kTurnNext)
                        if (u * 4 + 4 > P) keep_pairs(x[k][0], was, P - u * 4);      // (what is not turned stays bit for bit)
                }
#pragma unroll
                for (int o = 0; o < kOct; ++o)
                    if (o == 0 || turned) {
                        store_octet<T, APPEND>(dst + h * dst_head + c[o], x[k][o]);
                        if constexpr (APPEND) store_octet<T, APPEND>(vdst + h * dst_head + c[o], v[k][o]);
                    }
            }
        }
    }
}
// (in a launch of its own, behind the rows, when len_out may be kv_len)
__global__ __launch_bounds__(256)
void append_lengths_kernel(TurnArgs a, int n_seqs) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= n_seqs) return;
    int len = a.kv_len[b], n = a.n_tokens;
    len = len < 0 ? 0 : (len > a.capacity ? a.capacity : len);
    if (a.live) { n = a.live[b]; n = n < 0 ? 0 : (n > a.n_tokens ? a.n_tokens : n); }
    a.len_out[b] = len + (n < a.capacity - len ? n : a.capacity - len);
}

template <class T, typename TAB, int MODE, bool APPEND>
static void launch_turn(TurnArgs &a, hipStream_t s) {
    const int per = a.units < 256 ? 256 / a.units : 1;
    const int64_t blocks = (a.tokens + per - 1) / per;
    const int heads = (a.H + kTurnHeads - 1) / kTurnHeads;
    const int whole = MODE != kTurnNone && a.r.n_pairs % 4 == 0 && (reinterpret_cast<uintptr_t>(a.r.table) & 15u) == 0;
    a.by_units = fast_div((uint32_t)a.units);
    a.by_tokens = fast_div((uint32_t)a.n_tokens);
    const bool many = MODE != kTurnPair && blocks * a.H > 1024;
    for (a.first_block = 0; a.first_block < blocks; a.first_block += kMostBlocks) {
        const unsigned n = (unsigned)(blocks - a.first_block < kMostBlocks ? blocks - a.first_block : kMostBlocks);
        if constexpr (MODE != kTurnPair)
            if (many) {
                turn_kernel<T, TAB, MODE, APPEND, kTurnHeads><<<dim3(n, (unsigned)heads), dim3(256), 0, s>>>(a, per, whole);
                continue;
            }
        turn_kernel<T, TAB, MODE, APPEND, 1><<<dim3(n, (unsigned)a.H), dim3(256), 0, s>>>(a, per, whole);
    }
}
template <class T, bool APPEND>
static void launch_typed(TurnArgs &a, bool turned_only, hipStream_t s) {
    const int P = a.r.table ? a.r.n_pairs : 0;
    const bool f32 = a.r.type == QVG_F32;
    if (P == 0) {
        a.units = a.d / 8;
        if constexpr (APPEND) launch_turn<T, f16_t, kTurnNone, APPEND>(a, s);
    } else if (!a.r.half) {
        a.units = turned_only ? (P + 3) / 4 : a.d / 8;
        f32 ? launch_turn<T, float, kTurnNext, APPEND>(a, s) : launch_turn<T, f16_t, kTurnNext, APPEND>(a, s);
    } else if (P % 8 == 0) {
        a.units = turned_only ? P / 8 : P / 8 + (a.d - 2 * P) / 8;
        f32 ? launch_turn<T, float, kTurnHalf, APPEND>(a, s) : launch_turn<T, f16_t, kTurnHalf, APPEND>(a, s);
    } else {
        a.units = turned_only ? P : a.d - P;
        f32 ? launch_turn<T, float, kTurnPair, APPEND>(a, s) : launch_turn<T, f16_t, kTurnPair, APPEND>(a, s);
    }
}
hipError_t launch_rope(TurnArgs &a, int type, hipStream_t s) {
    const bool turned_only = a.out == a.x;                               // (with x's strides: the other channels are there)
    if (type == QVG_BF16) launch_typed<Bf16, false>(a, turned_only, s);
    else if (type == QVG_F16) launch_typed<F16, false>(a, turned_only, s);
    else launch_typed<F32, false>(a, turned_only, s);
    return hipGetLastError();
}
// (both types are 16 bits: rows that are not turned are copied as either)
hipError_t launch_append(TurnArgs &a, int n_seqs, int type, hipStream_t s) {
    if (a.tokens > 0) {
        if (type == QVG_BF16 || !a.r.table) launch_typed<Bf16, true>(a, false, s);
        else launch_typed<F16, true>(a, false, s);
    }
    if (a.len_out && !a.lengths_here) append_lengths_kernel<<<dim3((unsigned)((n_seqs + 255) / 256)), dim3(256), 0, s>>>(a, n_seqs);
    return hipGetLastError();
}

}  // namespace qvg

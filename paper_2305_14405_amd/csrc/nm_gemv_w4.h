// Products of a few rows with 4-bit weights (nm_gemv_w4): the kernel.  One translation unit for each type of x.
//
// Bound by memory: N K / 2 bytes of weights, each read once, for 2 M operations a weight.  A workgroup has 16 or 32 columns (rows of W)
// and all of K, which eight or sixteen wavefronts share in blocks of 128; their sums are joined through LDS, so that columns alone need not
// fill the GPU.  K goes by chunks: x of a chunk, and the chunk's scales as fp32, lie in LDS (the next chunk's are on their way into
// registers), and a wavefront takes a run of the chunk's blocks.  Where a chunk or two are all of K (few rows), weights go
// directly into LDS, a ring of blocks for each wavefront; with more chunks through registers, for whoever waits for a chunk's x would
// wait for the whole ring (33 rows, 8192 x 8192: 46 us with the ring).  Then 32 columns are two sets of eight wavefronts, four to a
// SIMD: fetching and ordering x, unpacking weights and the matrix instructions of one run under another's (8192 x 8192: 33 rows 20.0 us, 21.8
// with eight wavefronts of 32 columns; 48: 22.3 and 25.4; 17: 15.4 and 16.7; 16: 14.6 and 15.9).
//   Four neighbouring lanes load 64 bytes, 128 weights, of a row, a run of 32 each: neighbouring lanes in different rows, as the matrix
// instruction wants them, cost the address unit four times as much (28672 x 8192: 54 us so, 2.2 TB/s).  From LDS lane (j, row) then
// gets run j of its row.  The 16x16x32 instruction (rows of x its rows, columns its columns) adds over the four lanes of a
// row, so to add within one run (the smallest group) these exchange words, four half swaps for 16 bytes: then register i of lane
// group j holds weights 8 j .. 8 j + 7 of run i.
//   int8: (v << 4) & 0xf0f0f0f0 and v & 0xf0f0f0f0 are 16 times the even and the odd weights as int8: three operations for eight
// weights, and exact.  fp16: u = w + 8 is put under an exponent, 16 + u, and 24 taken off, both exact, in thirteen.  bf16: one
// conversion of the lower four bits of a byte for each weight, to w / 16 in fp32, whose upper half is taken; thirteen too.  The matrix instructions so
// have the weights themselves: what x they meet a zero with is not in the sum (with 16 + u there, and 24 times the sum of x taken off by
// further matrix instructions, a value 30000 times the others that met a zero left an error some 1000 times that of an fp32 sum).
//   What a group's sum is multiplied by is one number per lane (its column).
#pragma once

#include <mutex>

#include "nm_decode.h"

namespace nm {

typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));
typedef f16 v2h __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

constexpr int kW4Waves = 8, kW4Threads = 64 * kW4Waves;

// Scales that a thread has of a chunk; threads: eight wavefronts times this.
constexpr int w4_scales(int tiles, int threads) { return ((tiles == 1 ? 8 : 2) + threads - 1) / threads; }

struct W4Args {
    nm_w4_desc d;
    DevTable table;
    FastDiv per;         // blocks to a group of 128 or more
    int chunk_shift;     // log2 of a chunk's length in K / 1024: a wavefront's blocks of a chunk
    int chunks;
    int x_stride;        // bytes between rows of x in LDS
    int passes;          // over the weights: tiles of rows
    int second;          // where a second buffer of a chunk's scales and x begins behind the first; 0: there is one
};
constexpr int kW4Chunk = 128 * kW4Waves;

// Pieces of 16 bytes of x that a thread has of a chunk: of the shortest chunk of 16-bit rows and more.
constexpr int w4_pieces(int tiles, bool ring, int sets, int shares) { return tiles == 1 && !ring ? 8 / (sets * shares) : 4 * tiles / sets; }
// Blocks of a wavefront's ring in LDS (16 columns are 1 KB of each), or its places for blocks in LDS where registers hold the next two.
constexpr int w4_stages(int columns, bool ring) { return !ring ? 1 : columns == 1 ? 4 : 3; }

template <typename X>
int32_t launch_w4(const W4Args& a, hipStream_t s);

// Register i of lane group j <-> register j of lane group i.
__device__ __forceinline__ v4u exchange(v4u w)
{
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), e = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return v4u{c[0], c[1], e[0], e[1]};
}

__device__ __forceinline__ unsigned in_vgpr_u(unsigned x)
{
    unsigned v;
    asm("v_mov_b32 %0, %1" : "=v"(v) : "s"(x));
    return v;
}

// What differs by the type of x: its eight values of a lane, the sum over them, and eight weights times 1 / (kUnit kEnd): kUnit goes with the
// scales, kEnd with the whole sum (a scale times 16 might overflow, a sum of w / 16 can only where that of w does).
template <typename X> struct W4;
template <> struct W4<int8_t> {
    typedef v2u Rows;
    typedef v4i Sum;
    // of a lane's eight values the even ones first: so the weights come out of their word
    static __device__ __forceinline__ v4u order(v4u x)
    {
        return v4u{__builtin_amdgcn_perm(x[1], x[0], 0x06040200u), __builtin_amdgcn_perm(x[1], x[0], 0x07050301u),
                   __builtin_amdgcn_perm(x[3], x[2], 0x06040200u), __builtin_amdgcn_perm(x[3], x[2], 0x07050301u)};
    }
    static __device__ __forceinline__ unsigned exponent() { return 0; }
    static __device__ __forceinline__ v2u weights(unsigned w, unsigned) { return v2u{(w << 4) & 0xf0f0f0f0u, w & 0xf0f0f0f0u}; }
    static __device__ __forceinline__ Sum add(Rows x, v2u w, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, x), __builtin_bit_cast(long, w), c, 0, 0, 0); }
    static constexpr float kUnit = 1.0f / 16.0f, kEnd = 1.0f;
};
template <> struct W4<f16> {
    typedef v4u Rows;
    typedef v4f Sum;
    // a lane's eight values in the order in which the weights come out of their word: 0 4 1 5 2 6 3 7
    static __device__ __forceinline__ v4u order(v4u x)
    {
        return v4u{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                    __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
    }
    // 16 + u: u in the upper four bits of the mantissa of 10.  exponent: of 16, twice, in a vector register, so that mask and exponent are
    // one instruction (an instruction takes one constant from elsewhere)
    static __device__ __forceinline__ unsigned exponent() { return in_vgpr_u(0x4c004c00u); }
    static __device__ __forceinline__ v4u weights(unsigned w, unsigned exponent)
    {
        const unsigned u = w ^ 0x88888888u;
        auto less24 = [](unsigned p) { return __builtin_bit_cast(unsigned, (v2h)(__builtin_bit_cast(v2h, p) - v2h{(f16)24.0f, (f16)24.0f})); };
        return v4u{less24(((u << 6) & 0x03c003c0u) | exponent), less24(((u << 2) & 0x03c003c0u) | exponent),
                   less24(((u >> 2) & 0x03c003c0u) | exponent), less24(((u >> 6) & 0x03c003c0u) | exponent)};
    }
    static __device__ __forceinline__ Sum add(Rows x, v4u w, Sum c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, w), c, 0, 0, 0); }
    static constexpr float kUnit = 1.0f, kEnd = 1.0f;
};
template <> struct W4<bf16> {
    typedef v4u Rows;
    typedef v4f Sum;
    static __device__ __forceinline__ v4u order(v4u x) { return x; }
    static __device__ __forceinline__ unsigned exponent() { return 0; }
    static __device__ __forceinline__ v4u weights(unsigned w, unsigned)
    {
        unsigned odd = w >> 4;
        asm("" : "+v"(odd));   // as a number of its own, so that its bytes are operands as they lie and not shifts of w
        v4u o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // byte i has weights 2 i and 2 i + 1; their sixteenths have four bits or fewer, so nothing is in the lower halves
            const unsigned a = __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * i) & 0xffu)));
            const unsigned b = __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)(odd >> (8 * i) & 0xffu)));
            o[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        }
        return o;
    }
    static __device__ __forceinline__ Sum add(Rows x, v4u w, Sum c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, w), c, 0, 0, 0); }
    static constexpr float kUnit = 1.0f, kEnd = 16.0f;
};

// S: bits of a scale (float, or either 16-bit type); kRuns: runs of 32 weights to a scale within a block of 128 (1, 2, 4); kM: tiles of
// 16 rows; kN: of 16 columns that a wavefront has; kRing: weights by a ring in LDS; kC: sets of wavefronts with columns of their own;
// kK: times eight wavefronts share K.
template <typename X, typename S, int kRuns, int kM, int kN, bool kRing, int kC, int kK>
__global__ __launch_bounds__(kW4Threads * kC * kK, kRing ? 4 : 2 * kC * kK) void gemv_w4_kernel(W4Args a)
{
    typedef W4<X> Q;
    typedef typename Q::Rows Rows;
    typedef typename Q::Sum Sum;
    constexpr int kScales = 4 / kRuns;                        // to a block
    constexpr int kThreads = kW4Threads * kC * kK, kParts = kW4Waves * kK, kWaves = kParts * kC, kLength = kW4Chunk * kK;   // kLength: of the shortest chunk
    constexpr int kCols = 16 * kN * kC, kPer16 = 16 / (int)sizeof(X);
    constexpr int kPieces = w4_pieces(kM, kRing, kC, kK), kW4Scales = w4_scales(kM, kC * kK);   // that a thread has of a chunk
    static_assert(kPieces * kThreads * 16 >= 16 * kM * kLength * 2 && kW4Scales * kThreads >= kLength / 128 * (4 / kRuns) * kCols, "the shortest chunk");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const nm_w4_desc& d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, number = tid >> 6, wave = number % kParts, side = number / kParts, column = lane & 15, j = lane >> 4;
    constexpr int kStages = w4_stages(kN, kRing);
    // the passes over the same columns are neighbours on an XCD (workgroup i runs on XCD i mod 8)
    const int pass = blockIdx.x / 8 % a.passes, n0 = (blockIdx.x / 8 / a.passes * 8 + blockIdx.x % 8) * kCols;
    const int m0 = pass * 16 * kM, rows = min(d.M - m0, 16 * kM);
    if (n0 >= d.N) return;
    const int groups = d.K / d.group;
    const int run = 1 << a.chunk_shift;                       // a wavefront's blocks of a chunk
    const int entry_shift = a.chunk_shift + (kK == 2 ? 4 : 3) + (kRuns == 4 ? 0 : kRuns == 2 ? 1 : 2), entries = 1 << entry_shift;   // scales of a column and chunk
    const unsigned exponent = Q::exponent();
    // LDS: the wavefronts' rings, the chunk's scales (rows one longer), the chunk's x; at the end the sums, from the start
    char* s_w = smem + number * kStages * 1024 * kN;
    float* s_scale = reinterpret_cast<float*>(smem + kWaves * kStages * 1024 * kN);
    char* s_x = smem + kWaves * kStages * 1024 * kN + (kCols * (entries + 1) * 4 + 15) / 16 * 16;

    // weights: lane 4 r + i has run i ^ r / 4 % 4 of row r, so that no two banks meet when lane (j, row) reads run j of its row.  Columns
    // behind the last read the last one's: what comes of them is not written.  Behind K the last run is repeated: it meets zeros of x.
    const uint8_t* wrow[kN];
#pragma unroll
    for (int c = 0; c < kN; ++c) wrow[c] = d.W + (long)min(n0 + (side * kN + c) * 16 + (lane >> 2), d.N - 1) * (d.K / 2);
    const int total = a.chunks * run;                         // the wavefront's blocks
    const unsigned ring = (unsigned)(uintptr_t)smem + number * kStages * 1024 * kN;
    auto bytes_of = [&](int u) {                              // of the lane's piece of block number u, from the row's begin
        const int kb = ((u >> a.chunk_shift) * kParts + wave) * run + (u & (run - 1));
        return min(kb * 128 + ((lane & 3) ^ (lane >> 4 & 3)) * 32, d.K - 32) / 2;
    };
    auto request = [&](int u, int slot) {
        const int at = bytes_of(u);
#pragma unroll
        for (int c = 0; c < kN; ++c) dma16(wrow[c] + at, ring + (slot * kN + c) * 1024);
    };
    const int read_at = (column * 4 + (j ^ (column >> 2))) * 16;

    // x and scales of a chunk: into registers, then into LDS (x in the order that the matrix instructions want)
    const int row_shift = a.chunk_shift + (sizeof(X) == 1 ? 6 : 7) + (kK == 2);   // pieces to a row of a chunk: 64 and more, so a wavefront's are of one row
    const int uniform_wave = __builtin_amdgcn_readfirstlane(number);
    v4u xp[kPieces];
    S sp[kW4Scales];
    auto fetch = [&](int chunk) {
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
            const int p = uniform_wave * 64 + q * kThreads, r = min(p >> row_shift, rows - 1);
            const int k = (chunk * (kLength << a.chunk_shift) + (p & ((1 << row_shift) - 1)) * kPer16) + lane * kPer16;
            xp[q] = *reinterpret_cast<const v4u*>(static_cast<const X*>(d.x) + (long)(m0 + r) * d.x_stride + (unsigned)min(k, d.K - kPer16));
        }
#pragma unroll
        for (int q = 0; q < kW4Scales; ++q) {
            const int i = tid + q * kThreads, c = min(i >> entry_shift, kCols - 1), e = i & (entries - 1), block = chunk * (run * kParts) + e / kScales;
            const int g = min(kRuns == 4 ? (int)quotient(block, a.per) : block * kScales + e % kScales, groups - 1);
            sp[q] = static_cast<const S*>(d.scales)[(long)min(n0 + c, d.N - 1) * groups + g];
        }
        __builtin_amdgcn_sched_barrier(0);                    // loads are waited for in their order
    };
    int flip = 0;                                             // of the buffer in use
    auto stage = [&](int chunk) {
        int lane_at = lane * 16;
        asm volatile("" : "+v"(lane_at));                      // not every piece's address in a register of its own from the start
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
            const int p = uniform_wave * 64 + q * kThreads, r = p >> row_shift, at = p & ((1 << row_shift) - 1);
            if (r < rows) *reinterpret_cast<v4u*>(s_x + flip + r * a.x_stride + at * 16 + lane_at) = Q::order(xp[q]);
        }
        if ((chunk + 1) * (kLength << a.chunk_shift) > d.K) {        // zeros behind K
            asm volatile("");
#pragma unroll 1
            for (int q = 0; q < kPieces; ++q) {
                const int p = uniform_wave * 64 + q * kThreads, r = p >> row_shift, at = p & ((1 << row_shift) - 1);
                if (r < rows && (chunk * (kLength << a.chunk_shift) + at * kPer16) + lane * kPer16 >= d.K)
                    *reinterpret_cast<v4u*>(s_x + flip + r * a.x_stride + at * 16 + lane * 16) = v4u{};
            }
        }
#pragma unroll
        for (int q = 0; q < kW4Scales; ++q) {
            const int i = tid + q * kThreads, c = i >> entry_shift, e = i & (entries - 1);
            float v;
            if constexpr (sizeof(S) == 4) v = sp[q];
            else v = d.scale_dtype == NM_DT_BF16 ? __uint_as_float((unsigned)sp[q] << 16) : (float)__builtin_bit_cast(f16, sp[q]);
            if (c < kCols) *reinterpret_cast<float*>(reinterpret_cast<char*>(s_scale + c * (entries + 1) + e) + flip) = v * Q::kUnit;
        }
    };

    v4f sum[kM][kN];
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int c = 0; c < kN; ++c) sum[t][c] = v4f{0, 0, 0, 0};
    const char* xrow[kM];
#pragma unroll
    for (int t = 0; t < kM; ++t) xrow[t] = s_x + min(t * 16 + column, rows - 1) * a.x_stride + (wave * run * 128 + j * 8) * sizeof(X);
    const float* srow = s_scale + (side * kN * 16 + column) * (entries + 1) + wave * run * kScales;

    // x and scales of a block for one tile of rows: they do not wait for its weights
    constexpr bool kEarly = kM == 1 && !kRing;
    Rows x1[4];
    float scale1[kScales][kN];
    auto rows_of = [&](int t, int at, int i) { return *reinterpret_cast<const Rows*>(xrow[t] + flip + (at * 128 + i * 32) * sizeof(X)); };
    auto scale_of = [&](int c, int at, int g) { return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(srow + c * 16 * (entries + 1) + at * kScales + g) + flip); };
    auto ahead = [&](int at) {
        if constexpr (kEarly) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x1[i] = rows_of(0, at, i);
#pragma unroll
            for (int g = 0; g < kScales; ++g)
#pragma unroll
                for (int c = 0; c < kN; ++c) scale1[g][c] = scale_of(c, at, g);
        }
    };
    auto block = [&](int at, const v4u (&now)[kN]) {          // block number at of the wavefront's run in this chunk
#pragma unroll
        for (int g = 0; g < kScales; ++g) {
            float scale[kN];
#pragma unroll
            for (int c = 0; c < kN; ++c) scale[c] = kEarly ? scale1[g][c] : scale_of(c, at, g);
            decltype(Q::weights(0u, 0u)) weights[kM > 1 ? kRuns : 1][kN];   // made once for all tiles of rows
            if constexpr (kM > 1) {
#pragma unroll
                for (int i = 0; i < kRuns; ++i)
#pragma unroll
                    for (int c = 0; c < kN; ++c) weights[i][c] = Q::weights(now[c][g * kRuns + i], exponent);
            }
#pragma unroll
            for (int t = 0; t < kM; ++t) {
                Rows x[kRuns];
                Sum acc[kN];
#pragma unroll
                for (int i = 0; i < kRuns; ++i) x[i] = kEarly ? x1[g * kRuns + i] : rows_of(t, at, g * kRuns + i);
#pragma unroll
                for (int c = 0; c < kN; ++c) acc[c] = Sum{};
#pragma unroll
                for (int i = 0; i < kRuns; ++i)
#pragma unroll
                    for (int c = 0; c < kN; ++c) {
                        if constexpr (kM == 1) acc[c] = Q::add(x[i], Q::weights(now[c][g * kRuns + i], exponent), acc[c]);
                        else acc[c] = Q::add(x[i], weights[i][c], acc[c]);
                    }
#pragma unroll
                for (int c = 0; c < kN; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[t][c][e] = __builtin_fmaf((float)acc[c][e], scale[c], sum[t][c][e]);
            }
        }
    };

    auto next_chunk = [&](int chunk) {
        if (chunk && !a.second) __syncthreads();              // the chunk before is not read any more
        flip = !kRing && (chunk & 1) ? a.second : 0;
        stage(chunk);
        if (chunk + 1 < a.chunks) fetch(chunk + 1);
        __syncthreads();
    };
    auto read = [&](v4u (&now)[kN], int slot) {
#pragma unroll
        for (int c = 0; c < kN; ++c) now[c] = *reinterpret_cast<const v4u*>(s_w + (slot * kN + c) * 1024 + read_at);
    };
    fetch(0);
    if constexpr (kRing) {
#pragma unroll
        for (int u = 0; u < kStages; ++u)
            if (u < total) request(u, u);
        for (int u = 0, slot = 0; u < total; ++u, slot = slot + 1 == kStages ? 0 : slot + 1) {
            if (!(u & (run - 1))) next_chunk(u >> a.chunk_shift);
            ahead(u & (run - 1));
            // what was requested behind this block may still be under way; at the end nothing is requested any more
            if (u + kStages <= total) wait_vmcnt<(kStages - 1) * kN>();
            else wait_vmcnt<0>();
            v4u now[kN];
            read(now, slot);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // the slot is read before it is written again
            if (u + kStages < total) request(u + kStages, slot);
#pragma unroll
            for (int c = 0; c < kN; ++c) now[c] = exchange(now[c]);
            block(u & (run - 1), now);
        }
    } else {
        v4u w[2][kN];
        auto load = [&](int u, v4u (&to)[kN]) {
            const int at = bytes_of(u);
#pragma unroll
            for (int c = 0; c < kN; ++c) to[c] = *reinterpret_cast<const v4u*>(wrow[c] + at);
            __builtin_amdgcn_sched_barrier(0);
        };
        load(0, w[0]);
        load(1, w[1]);
        for (int u0 = 0; u0 < total; u0 += 2)
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                const int u = u0 + odd;
                if (u >= total) break;
                if (!(u & (run - 1))) next_chunk(u >> a.chunk_shift);
                ahead(u & (run - 1));
#pragma unroll
                for (int c = 0; c < kN; ++c) *reinterpret_cast<v4u*>(s_w + c * 1024 + lane * 16) = w[odd][c];
                load(u + 2, w[odd]);                          // behind the last block: the last run, not used
                v4u now[kN];
                read(now, 0);
#pragma unroll
                for (int c = 0; c < kN; ++c) now[c] = exchange(now[c]);
                block(u & (run - 1), now);
            }
    }
    __syncthreads();
    float (*s_sum)[kM][16][kCols] = reinterpret_cast<float (*)[kM][16][kCols]>(smem);
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int c = 0; c < kN; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_sum[wave][t][j * 4 + e][(side * kN + c) * 16 + column] = sum[t][c][e];
    __syncthreads();
    for (int i = tid; i < kM * 16 * kCols; i += kThreads) {
        const int c = i % kCols, r = i / kCols % 16, t = i / (16 * kCols), m = m0 + t * 16 + r, col = n0 + c;
        if (m >= d.M || col >= d.N) continue;
        float v = 0.0f;
#pragma unroll
        for (int p = 0; p < kParts; ++p) v += s_sum[p][t][r][c];
        v *= Q::kEnd;
        v = __builtin_fmaf(v, d.alpha, d.bias ? d.bias[col] : 0.0f);
        if (d.table_idx >= 0) {
            int seg;
            v = pwl_eval(v, a.table, a.table.kb, seg);
        }
        store1(d.out, d.out_dtype, (long)m * d.out_stride + col, v, d.out_inv_scale);
    }
}

template <typename X, typename S, int kRuns, int kM>
static int32_t launch_w4_registers(const W4Args& a, hipStream_t s);
template <typename X, typename S, int kRuns, int kM, int kN, bool kRing, int kC = 1, int kK = 1>
static int32_t launch_w4_tiles(W4Args a, hipStream_t s)
{
    a.passes = (a.d.M + 16 * kM - 1) / (16 * kM);
    // the longest chunk whose x and scales a workgroup's threads hold at once, no longer than K
    const int rows = a.d.M < 16 * kM ? a.d.M : 16 * kM;
    constexpr int kCols = 16 * kN * kC, kWaves = kW4Waves * kC * kK, kLength = kW4Chunk * kK;
    const long room = (long)w4_pieces(kM, kRing, kC, kK) * kWaves * 64 * 16, scales = (long)w4_scales(kM, kC * kK) * kWaves * 64;
    a.chunk_shift = 0;
    while ((kLength << a.chunk_shift) < a.d.K && (2 * kLength << a.chunk_shift) / 128 * (4 / kRuns) * kCols <= scales && rows * (long)(2 * kLength << a.chunk_shift) * (long)sizeof(X) <= room) ++a.chunk_shift;
    const int chunk = kLength << a.chunk_shift;
    a.chunks = (a.d.K + chunk - 1) / chunk;
    if constexpr (kRing)
        if (a.chunks > 2 / kK) return launch_w4_registers<X, S, kRuns, 1>(a, s);   // (4 rows of 4096 x 11008: 11.9 us, 13.2 as two chunks of the ring)
    a.x_stride = chunk * (int)sizeof(X) + 16;
    const int entries = (chunk / 128) * (4 / kRuns);
    const size_t one = (size_t)(kCols * (entries + 1) * 4 + 15) / 16 * 16 + (size_t)rows * a.x_stride;
    size_t used = (size_t)kWaves * w4_stages(kN, kRing) * 1024 * kN + one;
    // with two buffers a wavefront may write the next chunk's while another still reads this one's: one barrier a chunk instead of two
    if (!kRing && a.chunks > 1 && used + one <= 160 * 1024) {
        a.second = (int)one;
        used += one;
    }
    const size_t sums = (size_t)kW4Waves * kK * kM * 16 * kCols * 4, shmem = used > sums ? used : sums;
    auto kern = gemv_w4_kernel<X, S, kRuns, kM, kN, kRing, kC, kK>;
    if (shmem > 64 * 1024) {
        static std::once_flag once;
        static int32_t once_rc;
        std::call_once(once, [&] {
            once_rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024),
                                "hipFuncSetAttribute(gemv_w4_kernel)");
        });
        if (once_rc) return once_rc;
    }
    queue_kernel(kern, dim3(((a.d.N + kCols - 1) / kCols + 7) / 8 * 8 * a.passes), dim3(64 * kWaves), shmem, s, a);
    return check_hip(hipGetLastError(), "nm_gemv_w4 launch");
}
// Weights through registers, tiles of 16 kM rows: 16 columns to a workgroup where no more than a CU's worth come of it, 32 where there
// are more.  A chunk of x fills LDS either way, so one workgroup has a CU and more than 256 are a second round (16 columns of 7168 x 8192
// took 18.9 us at 16 rows, 32 take 13.6).  With 16 columns sixteen wavefronts share K, unless it is a chunk of eight's
// (4096 x 11008, 16 rows: 13.3 us, eight 14.9).
template <typename X, typename S, int kRuns, int kM>
static int32_t launch_w4_registers(const W4Args& a, hipStream_t s)
{
    const long passes = (a.d.M + 16 * kM - 1) / (16 * kM), columns = (a.d.N + 15) / 16;
    if constexpr (kM < 3)
        if (passes * columns <= 256) {
            if constexpr (kM == 2)
                if (a.d.K <= 2048) return launch_w4_tiles<X, S, kRuns, kM, 1, false>(a, s);
            return launch_w4_tiles<X, S, kRuns, kM, 1, false, 1, 2>(a, s);   // (one tile of rows has a ring for so short a K)
        }
    return launch_w4_tiles<X, S, kRuns, kM, 1, false, 2>(a, s);
}
template <typename X, typename S, int kRuns>
static int32_t launch_w4_rows(const W4Args& a, hipStream_t s)
{
    // The fewest rows and columns to a workgroup that leave it a CU of its own, for rows are what a workgroup's time grows with (40 rows of
    // 4096 x 11008: 26.8 us as one tile of 48, 19.4 as two of 32; of 768 x 768 5.9 and, as three of 16, 4.1).  Where there are more workgroups
    // than CUs anyway, tiles of 48 rows if they save a pass over the weights (those and x of a chunk are what LDS holds).
    // A ring of eight wavefronts has 4096 columns of x under way at once; beyond, sixteen (one row of 4096 x 11008 11.3 us, 11.8 with eight; at
    // 4096 x 4096 either, 5.4 and 5.6).
    const long M = a.d.M, columns = (a.d.N + 15) / 16;
    if ((M + 15) / 16 * columns <= 256)
        return a.d.K <= 4096 ? launch_w4_tiles<X, S, kRuns, 1, 1, true>(a, s) : launch_w4_tiles<X, S, kRuns, 1, 1, true, 1, 2>(a, s);
    if (M <= 16) return launch_w4_tiles<X, S, kRuns, 1, 2, true>(a, s);
    if ((M + 31) / 32 * ((columns + 1) / 2) > 256 && (M + 47) / 48 < (M + 31) / 32) return launch_w4_registers<X, S, kRuns, 3>(a, s);
    return launch_w4_registers<X, S, kRuns, 2>(a, s);
}
template <typename X, typename S>
static int32_t launch_w4_group(const W4Args& a, hipStream_t s)
{
    if (a.d.group == 32) return launch_w4_rows<X, S, 1>(a, s);
    if (a.d.group == 64) return launch_w4_rows<X, S, 2>(a, s);
    return launch_w4_rows<X, S, 4>(a, s);
}
template <typename X>
int32_t launch_w4(const W4Args& a, hipStream_t s)
{
    return a.d.scale_dtype == NM_DT_F32 ? launch_w4_group<X, float>(a, s) : launch_w4_group<X, unsigned short>(a, s);
}

}  // namespace nm

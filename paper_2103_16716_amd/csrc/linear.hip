// The experts' products: rows of the routed order times the matrix of each row's
// expert, and the gradients.
//
//   y[r]  = act(x[r] W_e^T + b_e) + residual[r]      W [E, O, K], e the row's expert
//   dx[r] = (dy[r] W_e) where relu_of[r] > 0, else 0
//   dW_e  = sum over its rows of dy[r] x[r]^T,  db_e = sum of dy[r]
//
// Products are summed in fp32 on the matrix cores (bf16: v_mfma_f32_32x32x16_bf16; fp32:
// v_mfma_f32_32x32x2_f32, full fp32 products). Rows in no expert's range are left alone;
// an expert without rows has zero dW and db.
//
// One kernel in three forms, by which index of an operand is contiguous in memory:
//   kNT  y: x and W both by the contraction (inputs)
//   kNN  dx: dy by the contraction (outputs), W by the result's columns
//   kTN  dW: dy and x both across it; the contraction is over the expert's rows
#include <mutex>

#include "common.hpp"
#include "internal.hpp"
#include "rows.hpp"

namespace base {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

#define BASE_LDS __attribute__((address_space(3)))

// Whose tile is number `tile` of the experts' rows in tiles of BM, expert after expert: the
// expert, its rows [r0, r1), its first tile and the number of its tiles. Asked by whole waves.
struct RowTiles {
    int e, r0, r1, first, count;
};
__device__ inline bool find_row_tiles(const int32_t *__restrict__ offsets, int E, int N, int BM,
                                      int tile, RowTiles &out) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int e = e0 + lane;
        const int a = e < E ? row_bound(offsets, e, N) : 0;
        const int z = e < E ? row_bound(offsets, e + 1, N) : 0;
        const int n = z > a ? (z - a - 1) / BM + 1 : 0;
        int sum = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off);
            if (lane >= off) sum += o;
        }
        const uint64_t past = __ballot(before + sum > tile);
        if (past != 0) {
            const int f = __ffsll((unsigned long long)past) - 1;
            out.e = e0 + f;
            out.r1 = __builtin_amdgcn_readlane(z, f);
            out.r0 = __builtin_amdgcn_readlane(a, f);
            out.first = before + __builtin_amdgcn_readlane(sum - n, f);
            out.count = __builtin_amdgcn_readlane(n, f);
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}


enum { kNT = BASE_PRODUCT_Y, kNN = BASE_PRODUCT_DX, kTN = BASE_PRODUCT_DW };

// 16 bytes of an operand's contraction per lane. bf16: one instruction multiplies the
// lanes' 8 elements; fp32: four, instruction i the lanes' element i.
struct Bf16 {
    static constexpr bool kBf16 = true;
    using elem_t = uint16_t;
    using unit_t = bf16x8_t;
    static constexpr int kPer = 8;
    static constexpr int kMma = 1;
    __device__ static f32x16_t mma(unit_t a, unit_t b, f32x16_t c, int) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // The sum of a result row's elements: products with ones.
    using sum_t = f32x16_t;
    __device__ static void add(unit_t a, sum_t &sum) {
        const __bf16 i = (__bf16)1.0f;
        sum = mma(unit_t{i, i, i, i, i, i, i, i}, a, sum, 0);
    }
    __device__ static float total(const sum_t &sum) { return sum[0]; }
};
struct F32 {
    static constexpr bool kBf16 = false;
    using elem_t = float;
    using unit_t = f32x4_t;
    static constexpr int kPer = 4;
    static constexpr int kMma = 4;
    __device__ static f32x16_t mma(unit_t a, unit_t b, f32x16_t c, int i) {
        return __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    }
    // (Here the matrix cores are what is short.)
    using sum_t = float;
    __device__ static void add(unit_t a, sum_t &sum) { sum += (a[0] + a[1]) + (a[2] + a[3]); }
    __device__ static float total(sum_t sum) { return sum + __shfl_xor(sum, 32); }
};

// Waits until at most N vector-memory operations of this wave are in flight (loads into
// LDS count until their data is there) and its LDS reads are done.
template <int N>
__device__ inline void wait_first() {
    static_assert(N >= 0 && N < 64, "vmcnt field");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

// Workgroup barrier with no wait of its own; the empty asm statements keep the compiler
// from moving memory accesses across it.
__device__ inline void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int kChunk = 128;            // bytes of the contraction per stage and row
constexpr int kUnits = kChunk / 16;
constexpr int64_t kUnitsOfDevice = 256;
constexpr uint32_t kNowhere = 0x80000000u;   // an offset past every buffer: reads as zero

// A stage of one operand: B rows of the result by one chunk of the contraction, S steps.
//
// kAlong (contiguous by the contraction): LDS row r holds result row r, and its 16-byte
// slot s the row's unit s ^ (r / 2 % 8): the operand reads take one unit of 16 rows a
// cycle, and two rows fill the banks.
//
// Across: LDS row s holds step s of the contraction with the B result rows side by side.
// bf16 operands are read with the transposing LDS load, which gives a lane four steps of
// its own result row; a load instruction takes four steps of 64 bytes each (and as much
// 8 steps on), so segments of 64 bytes are exchanged by the step: segment g of step s
// stands at g ^ (s % 4) (rows of 128 bytes: g ^ (s / 2 % 2)). fp32 operands are read by
// element; a load takes 128 bytes of steps s and s + 4, so segments of 128 bytes stand at
// g ^ (s / 4 % 2).
template <class In, bool kAlong, int B, int kThreads>
struct Stage {
    using unit_t = typename In::unit_t;
    static constexpr int kSize = sizeof(typename In::elem_t);
    static constexpr int S = kChunk / kSize;              // steps of the contraction
    static constexpr int kBytes = B * kChunk;
    static constexpr int kSlots = kBytes / 16 / kThreads; // 16-byte slots per thread
    static constexpr int kRow = B * kSize;                // bytes of an LDS row (across)
    static constexpr int kRowUnits = kRow / 16;
    static_assert(kBytes % (16 * kThreads) == 0, "whole slots");
    static_assert(kAlong || (kThreads / kRowUnits) % 8 == 0, "a thread's slots swizzle alike");

    __device__ static int exchange(int s) {
        if constexpr (!In::kBf16) return (s >> 2) & 1;
        else return B >= 128 ? s & 3 : (s >> 1) & 1;
    }

    uint32_t at[kSlots];   // offsets of this thread's slots from the chunk's first byte
    uint32_t unit;         // kAlong: this thread's unit of a row's chunk

    // ld: bytes from a row (across: a step) to the next; rows: the result rows left in the
    // matrix (across only: along, those past the end lie behind the buffer).
    __device__ void init(int64_t ld, int rows) {
        const int tid = threadIdx.x;
        if constexpr (kAlong) {
            unit = (tid % kUnits) ^ ((tid / kUnits >> 1) & 7);
#pragma unroll
            for (int i = 0; i < kSlots; ++i)
                at[i] = (uint32_t)((i * kThreads + tid) / kUnits * ld) + unit * 16;
        } else {
            const int s0 = tid / kRowUnits;
            const int u = (tid % kRowUnits) ^ (exchange(s0) << (In::kBf16 ? 2 : 3));
            const bool in = u * In::kPer < rows;
#pragma unroll
            for (int i = 0; i < kSlots; ++i)
                at[i] = in ? (uint32_t)((i * (kThreads / kRowUnits) + s0) * ld) + u * 16 : kNowhere;
        }
    }
    // base: the chunk's first byte; bytes: up to the end of what may be read; steps: those
    // of the chunk inside the contraction (kAlong only).
    __device__ void load(const char *base, uint32_t bytes, int steps, BASE_LDS char *lds) const {
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const bool in = !kAlong || (int)unit * In::kPer < steps;
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rsrc, (BASE_LDS void *)(lds + (i * kThreads + wave * 64) * 16), 16,
                (int)(in ? at[i] : kNowhere), 0, 0, 0);
    }
    // Unit 2 ks + lane / 32 of the contraction for result row 32 t + lane % 32.
    __device__ static unit_t read(const char *lds, int t, int ks) {
        const int lane = threadIdx.x & 63;
        const int half = lane >> 5;
        if constexpr (kAlong) {
            const int r = 32 * t + (lane & 31);
            return *reinterpret_cast<const unit_t *>(lds + r * kChunk +
                                                     (((2 * ks + half) ^ ((r >> 1) & 7)) * 16));
        } else if constexpr (In::kBf16) {
            const int s = 8 * half + ((lane & 15) >> 2);   // (+ 16 ks; + 4 for the second half)
            const int in_row = ((lane >> 3) & 2) * 16 + ((lane >> 1) & 1) * 16 + (lane & 1) * 8;
            BASE_LDS char *at = (BASE_LDS char *)lds + (16 * ks + s) * kRow + in_row;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (BASE_LDS s16x4_t *)(at + (t ^ exchange(s)) * 64));
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (BASE_LDS s16x4_t *)(at + 4 * kRow + (t ^ exchange(s + 4)) * 64));
            typedef short s16x8_t __attribute__((ext_vector_type(8)));
            const s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(unit_t, v);
        } else {
            unit_t v;
            const int s = 4 * (2 * ks + half);
            const char *p = lds + s * kRow + (t ^ half) * 128 + (lane & 31) * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float *>(p + i * kRow);
            return v;
        }
    }
};

// The experts' row tiles in all.
__device__ inline int count_row_tiles(const int32_t *__restrict__ offsets, int E, int N, int BM) {
    int n = 0;
    for (int e = threadIdx.x & 63; e < E; e += 64) {
        const int a = row_bound(offsets, e, N), z = row_bound(offsets, e + 1, N);
        n += z > a ? (z - a - 1) / BM + 1 : 0;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
    return __builtin_amdgcn_readfirstlane(n);
}

// The tile of a call's `tiles` that block number `block` computes. Blocks go to the eight
// XCDs in turn; each XCD takes a run of consecutive tiles, which share rows or a matrix, so
// that its L2 serves them. -1: none.
__device__ inline int tile_of_block(int tiles, int block) {
    const int per = (tiles + 7) / 8;
    const int u = block >> 3;
    const int t = (block & 7) * per + u;
    return u < per && t < tiles ? t : -1;
}

// Tile i of an expert's nm x nn, in strips of up to kMost tiles of rows, as equal as can be:
// neighbours in a strip share columns, and the strip's rows stay in the L2 while its columns
// go by. Eight for rows (32768 uneven rows x 2048 to 8192: 1034 us, 1051 with four; by columns
// of 16384, 2048 to 8192, 575 and 590), four for the matrices' gradient (749 us, 802 with
// eight).
template <int kMost>
__device__ inline void tile_in_strip(int i, int nm, int nn, int &m, int &n) {
    const int strips = (nm + kMost - 1) / kMost;
    const int height = (nm + strips - 1) / strips;
    const int s = i / (height * nn);
    const int r = i - s * height * nn;
    const int h = nm - s * height < height ? nm - s * height : height;
    n = r / h;
    m = s * height + r - n * h;
}

struct LinearCall {
    const void *A, *B, *bias, *extra;   // extra: the residual (kNT) or relu_of (kNN)
    const int32_t *offsets;
    void *out;
    float *db;    // kTN: sums of the rows of A, or null
    int N, E, K, O, relu;
    int block0;   // the number of the launch's first block
    // The contraction in `parts`, whose results follow each other in `out`, part_size of them
    // (fp32) each, and so those of db.
    int parts;
    int64_t part_size;
};

// A tile of the result: expert, rows [m0, m_end), columns from n0, contraction [s0, s1).
struct Tile {
    int e, m0, m_end, n0, s0, s1;
};

// BM rows (kTN: outputs) by BN columns of the result, WM x WN waves. A wave has every WM-th
// 32 rows and TN x 32 neighbouring columns, so that a tile with few rows left (the end of an
// expert) is spread over the waves, which skip what lies behind: the loop is compiled for
// each number of 32 rows a wave may have.
template <class In, int kForm, int BM, int BN, int WM, int WN, int kStages, bool kPartial = false>
struct Tiles {
    using unit_t = typename In::unit_t;
    using elem_t = typename In::elem_t;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    using StageA = Stage<In, kForm != kTN, BM, kThreads>;
    using StageB = Stage<In, kForm == kNT, BN, kThreads>;
    static constexpr int S = StageA::S;
    static constexpr int64_t kSize = sizeof(elem_t);
    static constexpr int kBytes = StageA::kBytes + StageB::kBytes;
    static constexpr int kLoads = StageA::kSlots + StageB::kSlots;   // of a wave, per stage
    static constexpr bool kSums = kForm == kTN || kPartial;   // results stored as fp32 sums
    static constexpr int kOutSize = kSums ? 4 : (int)kSize;
    // fp32 sums are stored 128 bytes of a row at once, 4 to a lane (16 bytes to a lane take 32
    // of a row: dW 4096 x 1024 of 64 experts, 64 rows 216 us, 201 so; 4096 rows 251 and 242).
    // Not by 256 x 256 tiles, which wait for the number of their stores (16384 rows 412, 509).
    static constexpr bool kByRow = kSums && BM < 256;

    const LinearCall &c;
    char *lds;
    StageA sa;
    StageB sb;
    const char *A, *B;
    int64_t lda, ldb;
    int cols, wm, wn, lane;
    Tile t;
    int nk, ncols;

    __device__ Tiles(const LinearCall &call, char *l) : c(call), lds(l) {
        cols = kForm == kNT ? c.O : c.K;
        lda = (kForm == kNT ? c.K : c.O) * kSize;
        ldb = c.K * kSize;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        wm = wave / WN;
        wn = wave % WN;
    }
    // Makes `tile` the one whose chunks are loaded. Its numbers are the same in every lane;
    // they are made scalars, so that loads take their buffer from scalar registers (from
    // vector registers each load is a loop over the lanes' values: 1035 us, then 1099, for
    // 32768 rows x 2048 to 8192).
    __device__ void set(const Tile &tile) {
        t.e = __builtin_amdgcn_readfirstlane(tile.e);
        t.m0 = __builtin_amdgcn_readfirstlane(tile.m0);
        t.m_end = __builtin_amdgcn_readfirstlane(tile.m_end);
        t.n0 = __builtin_amdgcn_readfirstlane(tile.n0);
        t.s0 = __builtin_amdgcn_readfirstlane(tile.s0);
        t.s1 = __builtin_amdgcn_readfirstlane(tile.s1);
        ncols = cols - t.n0 < BN ? cols - t.n0 : BN;
        sa.init(lda, t.m_end - t.m0);
        sb.init(ldb, ncols);
        A = static_cast<const char *>(c.A);
        B = static_cast<const char *>(c.B);
        if (kForm != kTN) B += (int64_t)t.e * c.O * ldb;
        A += kForm == kTN ? t.s0 * lda + t.m0 * kSize : t.m0 * lda + t.s0 * kSize;
        B += kForm == kNT ? t.n0 * ldb + t.s0 * kSize : t.s0 * ldb + t.n0 * kSize;
        nk = t.s1 > t.s0 ? (t.s1 - t.s0 - 1) / S + 1 : 0;
    }
    // The loads of chunk kc into stage st, of operand A (1), B (2) or both.
    __device__ void issue(int kc, int st, int which) const {
        BASE_LDS char *base = (BASE_LDS char *)lds + st * kBytes;
        const int left = t.s1 - t.s0 - kc * S;   // steps from this chunk on
        const int steps = left < S ? left : S;
        const int rows = t.m_end - t.m0 < BM ? t.m_end - t.m0 : BM;
        const int64_t step_a = kForm == kTN ? S * lda : kChunk;
        const int64_t step_b = kForm == kNT ? kChunk : S * ldb;
        const int64_t before = t.s0 * kSize + kc * kChunk;   // of a row, along the contraction
        const int64_t end_a = kForm == kTN ? steps * lda - t.m0 * kSize : rows * lda - before;
        const int64_t end_b = kForm == kNT ? ncols * ldb - before : steps * ldb - t.n0 * kSize;
        if (which & 1) sa.load(A + kc * step_a, (uint32_t)end_a, left, base);
        if (which & 2) sb.load(B + kc * step_b, (uint32_t)end_b, left, base + StageA::kBytes);
    }
    __device__ void issue_first() const {
#pragma unroll
        for (int k = 0; k < kStages; ++k)
            if (k < nk) issue(k, k, 3);
    }

    // Operand reads go between the products of the step before, one to a product or every
    // few: 32768 rows x 2048 to 8192, 32 experts 1035 -> 1010 us, by columns 1028 -> 1005. (Not
    // for the matrices' gradient: 4096 rows of 64 experts, 1024 to 4096, 274 -> 306 us.)
    template <int X>
    __device__ static void interleave() {
        if constexpr (In::kBf16 && kForm != kTN) {
            constexpr int reads = X + TN * (kForm == kNT ? 1 : 2);
            constexpr int every = X * TN / reads > 0 ? X * TN / reads : 1;
            constexpr int per = (reads * every + X * TN - 1) / (X * TN);
#pragma unroll
            for (int i = 0; i < X * TN / every; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, every, 0);   // matrix instructions
                __builtin_amdgcn_sched_group_barrier(0x100, per, 0);   // LDS reads
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __device__ void wait_chunk_0() const {
        if (nk >= kStages) wait_first<kLoads * (kStages - 1)>();
        else wait_first<0>();
    }

    // 256 x 256 tiles load into the stage handed over in two parts, A behind the barrier and B
    // a quarter of a chunk later (both at once: 32768 rows x 2048 to 8192, 32 experts 1010 us,
    // 975 so; smaller tiles are bound by the loads and issue them at once: 8192 rows by columns
    // of 64 experts, 4096 to 1024, 209 us in two parts, 164 at once).
    static constexpr bool kSplit = BM == 256 && kStages == 2;

    // The products of the tile, whose first chunks have been issued and whose chunk 0 has
    // landed for this wave. The last quarter of a chunk is multiplied behind the barrier that
    // hands its stage over: its operands are in registers by then, and the next chunk's
    // first ones are read beside it. Behind the last barrier all stages are free.
    //
    // db's sums are taken beside them by the tiles of the first columns: each wave adds up 32
    // rows (a kernel of its own read dy again: dW 4464 x 168 of 29473 rows 195 us, 125 so).
    template <int X, bool kSum>
    __device__ void contract(f32x16_t (&acc)[X][TN], typename In::sum_t &sum) const {
        static_assert(X <= WN || kForm != kTN, "a wave for each 32 rows");
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[x][j][i] = 0.0f;
        if (kSum) sum = typename In::sum_t{};
        unit_t a[2][X], b[2][TN], s[2];
        const int sum_tile = wm + WM * (wn < X ? wn : 0);
        auto fetch = [&](int set, const char *st, int ks) {
            if (kSum) s[set] = StageA::read(st, sum_tile, ks);
#pragma unroll
            for (int x = 0; x < X; ++x) a[set][x] = StageA::read(st, wm + WM * x, ks);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                b[set][j] = StageB::read(st + StageA::kBytes, wn * TN + j, ks);
        };
        auto multiply = [&](int set) {
#pragma unroll
            for (int i = 0; i < In::kMma; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int x = 0; x < X; ++x)
                        acc[x][j] = kByRow ? In::mma(a[set][x], b[set][j], acc[x][j], i)
                                           : In::mma(b[set][j], a[set][x], acc[x][j], i);
            if (kSum) In::add(s[set], sum);
        };
        barrier();
        if (nk > 0) fetch(0, lds, 0);
        int st = 0;
        for (int kc = 0; kc < nk; ++kc) {
            const char *cur = lds + st * kBytes;
            const int st1 = st + 1 < kStages ? st + 1 : 0;
            fetch(1, cur, 1);
            if (kSplit && kc > 0 && kc + 1 < nk) issue(kc + 1, st1, 2);
            multiply(0);
            interleave<X>();
            fetch(0, cur, 2);
            multiply(1);
            interleave<X>();
            fetch(1, cur, 3);
            multiply(0);
            interleave<X>();
            // Chunk kc + 1 has landed once only those after it are in flight.
            if (kc + kStages <= nk) wait_first<kLoads * (kStages - 2)>();
            else wait_first<0>();
            barrier();
            if (kc + 1 < nk) fetch(0, lds + st1 * kBytes, 0);
            if (kc + kStages < nk) issue(kc + kStages, st, kSplit ? 1 : 3);
            multiply(1);
            if (In::kBf16 && kForm != kTN) __builtin_amdgcn_sched_barrier(0);
            st = st1;
        }
    }

    // What is added to the results or (relu_of) masks them: the bias of the wave's columns,
    // loaded before the products, and `extra`, loaded behind them at once and ahead of the next
    // tile's chunks, 16 bytes each (fp32: twice). Loaded where they are used, each would wait
    // for those chunks (32768 rows x 2048 to 8192: with bias and ReLU 1060 us, 964 so; with
    // bias and residual 1284, 1042).
    static constexpr int kWords = In::kBf16 ? 1 : 2;
    template <int X>
    struct Added {
        u32x4_t bias[kForm == kNT ? TN : 1][2][kWords];
        u32x4_t extra[kSums ? 1 : X][TN][2][kWords];
        __device__ void load_bias(const Tiles &g) {
            if (kSums || kForm != kNT || g.c.bias == nullptr) return;
            const elem_t *row = static_cast<const elem_t *>(g.c.bias) + (int64_t)g.t.e * g.c.O;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int n = g.t.n0 + 32 * (g.wn * TN + j) + 16 * p + 8 * (g.lane >> 5);
#pragma unroll
                    for (int h = 0; h < kWords; ++h)
                        bias[kForm == kNT ? j : 0][p][h] = RowChunk<In::kBf16>::fetch(
                            row + (n < g.cols ? n : 0), h);
                }
        }
        __device__ void load_extra(const Tiles &g) {
            if (kSums || g.c.extra == nullptr) return;
            const int rows = g.t.m_end - g.t.m0;
#pragma unroll
            for (int x = 0; x < X; ++x) {
                const int r = 32 * (g.wm + WM * x) + (g.lane & 31);
                const elem_t *row = static_cast<const elem_t *>(g.c.extra) +
                                    (int64_t)(g.t.m0 + (r < rows ? r : rows - 1)) * g.cols;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const int n = g.t.n0 + 32 * (g.wn * TN + j) + 16 * p + 8 * (g.lane >> 5);
#pragma unroll
                        for (int h = 0; h < kWords; ++h)
                            extra[kSums ? 0 : x][j][p][h] =
                                RowChunk<In::kBf16>::fetch(row + (n < g.cols ? n : 0), h);
                    }
            }
        }
        __device__ static void widen(const u32x4_t (&w)[kWords], float (&v)[8]) {
            if constexpr (In::kBf16) {
                RowChunk<true>::widen(w[0], v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i >> 2][i & 3]);
            }
        }
    };

    // Stores of a wave per 32 x 32 results, of 16 bytes a lane each.
    static constexpr int kStores = 16 * kOutSize / 16;

    // What follows the product, and the stores. 32x32 results: lane holds row lane % 32;
    // register i column 8 (i / 4) + 4 (lane / 32) + i % 4; kByRow the other way round. kNT and
    // kNN exchange halves between the half waves, so that a lane has eight neighbouring
    // columns. Lanes outside the result store to nowhere, so that every wave issues the same
    // number of stores.
    template <int X>
    __device__ void finish(const Tile &d, f32x16_t (&acc)[X][TN], const Added<X> &added) const {
        const int half = lane >> 5;
        char *out = static_cast<char *>(c.out) +
                    ((kForm == kTN ? (int64_t)d.e * c.O * c.K : 0) + (int64_t)d.m0 * cols) * kOutSize;
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc(out, 0, 0x7fffffff, 0x00020000);
#pragma unroll
        for (int x = 0; x < X; ++x) {
            const int r = 32 * (wm + WM * x) + (lane & 31);
            const bool row_in = r < d.m_end - d.m0;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int nj = d.n0 + 32 * (wn * TN + j);
                if constexpr (kByRow) {
                    const int n = nj + (lane & 31);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int m = 32 * (wm + WM * x) + 8 * (i / 4) + 4 * half + i % 4;
                        const uint32_t at = ((uint32_t)m * cols + n) * 4;
                        __builtin_amdgcn_raw_buffer_store_b32(
                            __float_as_uint(acc[x][j][i]), rsrc,
                            (int)(m < d.m_end - d.m0 && n < cols ? at : kNowhere), 0, 0);
                    }
                } else if constexpr (kSums) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int n = nj + 8 * q + 4 * half;
                        const uint32_t at = ((uint32_t)r * cols + n) * 4;
                        const u32x4_t v = {__float_as_uint(acc[x][j][4 * q]),
                                           __float_as_uint(acc[x][j][4 * q + 1]),
                                           __float_as_uint(acc[x][j][4 * q + 2]),
                                           __float_as_uint(acc[x][j][4 * q + 3])};
                        __builtin_amdgcn_raw_buffer_store_b128(
                            v, rsrc, (int)(row_in && n < cols ? at : kNowhere), 0, 0);
                    }
                } else {
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
                            const u32x2_t w = __builtin_bit_cast(
                                u32x2_t, __builtin_amdgcn_permlane32_swap(
                                             __float_as_uint(acc[x][j][8 * p + i]),
                                             __float_as_uint(acc[x][j][8 * p + 4 + i]), false, false));
                            v[i] = __uint_as_float(w[0]);
                            v[4 + i] = __uint_as_float(w[1]);
                        }
                        const int n = nj + 16 * p + 8 * half;
                        const bool in = row_in && n < cols;
                        if (kForm == kNT && c.bias != nullptr) {
                            float u[8];
                            Added<X>::widen(added.bias[kForm == kNT ? j : 0][p], u);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] += u[i];
                        }
                        if (kForm == kNT && c.relu) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];
                        }
                        if (c.extra != nullptr) {
                            float u[8];
                            Added<X>::widen(added.extra[kSums ? 0 : x][j][p], u);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                if (kForm == kNT) v[i] += u[i];
                                else v[i] = u[i] > 0.0f ? v[i] : 0.0f;
                            }
                        }
                        const uint32_t to = ((uint32_t)r * cols + n) * kOutSize;
                        if constexpr (In::kBf16) {
                            __builtin_amdgcn_raw_buffer_store_b128(RowChunk<true>::narrow(v), rsrc,
                                                                   (int)(in ? to : kNowhere), 0, 0);
                        } else {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float w[4] = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                                __builtin_amdgcn_raw_buffer_store_b128(
                                    RowChunk<false>::narrow(w), rsrc,
                                    (int)(in ? to + 16 * h : kNowhere), 0, 0);
                            }
                        }
                    }
                }
            }
        }
    }

    // The tile that is set, then, when next is given, its first loads, which run beside the
    // results' stores. Vector memory operations complete in order, so chunk 0 of the next
    // tile has landed once no more are in flight than were issued behind it. (What the compiler
    // keeps in memory, the next Tile and for dW three registers, and the stores of db come on
    // top of those counted: the wait is then longer than needed, never shorter.)
    template <int X>
    __device__ void compute(const Tile *next) {
        f32x16_t acc[X][TN];
        Added<X> added;
        added.load_bias(*this);
        typename In::sum_t sum;
        const bool sums = kForm == kTN && t.n0 == 0 && c.db != nullptr;
        if (sums) contract<X, kForm == kTN>(acc, sum);
        else contract<X, false>(acc, sum);
        added.load_extra(*this);
        asm volatile("" ::: "memory");
        const Tile done = t;
        if (next != nullptr) {
            set(*next);
            issue_first();
            asm volatile("" ::: "memory");
        }
        if (sums) {
            const int m = done.m0 + 32 * (wm + WM * wn) + lane;
            const float total = In::total(sum);
            if (lane < 32 && wn < X && m < done.m_end) c.db[(int64_t)done.e * c.O + m] = total;
        }
        finish<X>(done, acc, added);
        if (next != nullptr) {
            asm volatile("" ::: "memory");
            constexpr int kBehind = X * TN * kStores;
            if (nk >= kStages) wait_first<kLoads * (kStages - 1) + kBehind>();
            else wait_first<kBehind>();
        }
    }
    __device__ void run(const Tile *next) {
        const int rows = t.m_end - t.m0;
        if (TM == 1 || rows > 32 * WM * (TM - 1)) compute<TM>(next);
        else if (TM <= 2 || rows > 32 * WM * (TM - 2)) compute<(TM > 1 ? TM - 1 : 1)>(next);
        else if (TM <= 3 || rows > 32 * WM * (TM - 3)) compute<(TM > 2 ? TM - 2 : 1)>(next);
        else compute<(TM > 3 ? TM - 3 : 1)>(next);
    }
};

// The tile of kTN that block number `block` computes: every expert's tiles are spread over the
// XCDs (an expert with many rows would else hold up one of them), a run to each. Small matrices
// go round by block.
template <int BM, int BN>
__device__ inline bool matrix_tile(const LinearCall &c, int block, Tile &t, bool &more) {
    const int nm = (c.O + BM - 1) / BM, nn = (c.K + BN - 1) / BN, all = nm * nn;
    int k;
    if (all >= 32) {
        const int per = (all + 7) / 8;
        const int u = block >> 3;
        t.e = u / per;
        k = (block & 7) * per + u - t.e * per;
    } else {
        t.e = block / all;
        k = block - t.e * all;
    }
    more = t.e < c.E;
    if (!more || k >= all) return false;
    int m, n;
    tile_in_strip<4>(k, nm, nn, m, n);
    t.m0 = m * BM;
    t.m_end = c.O;
    t.n0 = n * BN;
    t.s0 = row_bound(c.offsets, t.e, c.N);
    t.s1 = row_bound(c.offsets, t.e + 1, c.N);
    if (t.s1 < t.s0) t.s1 = t.s0;
    return true;
}

// One block per compute unit, each going through its tiles: for the tile that fills a unit.
template <class In, int kForm, int BM, int BN, int WM, int WN, int kStages>
__global__ __launch_bounds__(64 * WM * WN, 1) void linear_wide_kernel(LinearCall c) {
    using G = Tiles<In, kForm, BM, BN, WM, WN, kStages>;
    static_assert(!G::kByRow, "kStores is the number of stores");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    G g(c, lds);
    // first[e]: row tiles of the experts before e; a thread for a run of experts.
    int32_t *first = reinterpret_cast<int32_t *>(lds + kStages * G::kBytes);   // [E + 1]
    const int nn = (g.cols + BN - 1) / BN;
    if constexpr (kForm != kTN) {
        __shared__ int wave_sum[WM * WN];
        const int per = (c.E + G::kThreads - 1) / G::kThreads;
        const int e0 = threadIdx.x * per;
        int sum = 0;
        for (int e = e0; e < e0 + per && e < c.E; ++e) {
            const int a = row_bound(c.offsets, e, c.N), z = row_bound(c.offsets, e + 1, c.N);
            sum += z > a ? (z - a - 1) / BM + 1 : 0;
        }
        int scan = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(scan, off);
            if (g.lane >= off) scan += o;
        }
        if (g.lane == 63) wave_sum[threadIdx.x >> 6] = scan;
        __syncthreads();
        int at = scan - sum;
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) at += wave_sum[w];
        for (int e = e0; e < e0 + per && e < c.E; ++e) {
            const int a = row_bound(c.offsets, e, c.N), z = row_bound(c.offsets, e + 1, c.N);
            first[e] = at;
            at += z > a ? (z - a - 1) / BM + 1 : 0;
            if (e == c.E - 1) first[c.E] = at;
        }
        __syncthreads();
    }
    // An XCD's tiles go round its blocks. Those of a last round that would leave half of the
    // blocks without one are cut into two or four by their rows.
    int i = 0;
    auto next_tile = [&](Tile &t) {
        if constexpr (kForm == kTN) {
            bool more = true;
            while (more)
                if (matrix_tile<BM, BN>(c, blockIdx.x + gridDim.x * i++, t, more)) return true;
            return false;
        } else {
            const int tiles = __builtin_amdgcn_readfirstlane(first[c.E]) * nn;
            const int run = (tiles + 7) / 8;
            const int left = tiles - (blockIdx.x & 7) * run;
            const int mine = left < run ? left : run;   // (may be negative)
            const int slots = gridDim.x >> 3;
            const int whole = mine > 0 ? mine / slots * slots : 0;
            const int rest = mine - whole;
            const int parts = 4 * rest <= slots ? 4 : 2 * rest <= slots ? 2 : 1;
            for (;;) {
                int u = (blockIdx.x >> 3) + slots * i++;
                int part = 0, rows = BM;
                if (u >= whole) {
                    u -= whole;
                    if (u >= rest * parts) return false;
                    part = u % parts;
                    rows = BM / parts;
                    u = whole + u / parts;
                }
                const int k = (blockIdx.x & 7) * run + u;
                int e = 0;
                for (int e1 = 0; e1 < c.E; e1 += 64) {
                    const int q = e1 + g.lane;
                    e += __popcll(__ballot(q < c.E && first[q < c.E ? q + 1 : c.E] * nn <= k));
                }
                const int f = __builtin_amdgcn_readfirstlane(first[e]);
                const int a = row_bound(c.offsets, e, c.N);
                t.e = e;
                t.m_end = row_bound(c.offsets, e + 1, c.N);
                int m, n;
                const int nm = __builtin_amdgcn_readfirstlane(first[e + 1]) - f;
                tile_in_strip<8>(k - f * nn, nm, nn, m, n);
                t.m0 = a + m * BM + part * rows;
                if (t.m0 >= t.m_end) continue;
                if (t.m_end - t.m0 > rows) t.m_end = t.m0 + rows;
                t.n0 = n * BN;
                break;
            }
            t.s0 = 0;
            t.s1 = kForm == kNT ? c.K : c.O;
            return true;
        }
    };
    Tile t, u;
    if (!next_tile(t)) return;
    g.set(t);
    g.issue_first();
    g.wait_chunk_0();
    for (;;) {
        const bool more = next_tile(u);
        g.run(more ? &u : nullptr);
        if (!more) break;
    }
}

// Smaller tiles, of which several share a compute unit: a block for each. kPartial: for each
// part of the contraction.
template <class In, int kForm, int BM, int BN, int WM, int WN, int kStages, bool kPartial>
__global__ __launch_bounds__(64 * WM * WN) void linear_kernel(LinearCall c) {
    using G = Tiles<In, kForm, BM, BN, WM, WN, kStages, kPartial>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    int block = c.block0 + (int)blockIdx.x;
    int part = 0;
    if constexpr (kPartial) {
        const int u = block >> 3;   // the parts of a tile on the same XCD, next to each other
        part = u % c.parts;
        block = u / c.parts * 8 + (block & 7);
        c.out = static_cast<float *>(c.out) + part * c.part_size;
        if (kForm == kTN && c.db != nullptr) c.db += part * c.part_size;
    }
    G g(c, lds);
    Tile t;
    if constexpr (kForm == kTN) {
        bool more;
        if (!matrix_tile<BM, BN>(c, block, t, more)) return;
    } else {
        const int nn = (g.cols + BN - 1) / BN;
        RowTiles rt;
        const int k = tile_of_block(count_row_tiles(c.offsets, c.E, c.N, BM) * nn, block);
        if (k < 0 || !find_row_tiles(c.offsets, c.E, c.N, BM, k / nn, rt)) return;
        // Strips read a matrix once for their rows; one that the L2 (4 MB) holds most of is read
        // there, and its rows go by once. By strips and without, us: y of 347 x 2592 to 3496, two
        // experts (18 MB) 22 and 28; dx of 512 x 2048 to 2048 (8 MB) 17.6 and 24.7; y of
        // 5801 x 4488 to 544, 30 experts (5 MB) 93 and 80, of 4692 x 3384 to 200, five (1 MB) 32
        // and 26.
        int m = k / nn - rt.first, n = k % nn;
        if ((int64_t)c.K * c.O * G::kSize > (6 << 20))
            tile_in_strip<8>(k - rt.first * nn, rt.count, nn, m, n);
        t = Tile{rt.e, rt.r0 + m * BM, rt.r1, n * BN, 0, kForm == kNT ? c.K : c.O};
    }
    if constexpr (kPartial) {   // whole chunks; the last parts may have none
        const int chunks = t.s1 > t.s0 ? (t.s1 - t.s0 - 1) / G::S + 1 : 0;
        const int per = (chunks + c.parts - 1) / c.parts;
        const int first = part * per < chunks ? part * per : chunks;
        const int last = first + per < chunks ? first + per : chunks;
        if (last < chunks) t.s1 = t.s0 + last * G::S;
        t.s0 = first < chunks ? t.s0 + first * G::S : t.s1;
    }
    g.set(t);
    g.issue_first();
    g.wait_chunk_0();
    g.run(nullptr);
}

// The parts' sums of y or dx, added up in their order, and what follows the product. A wave
// for 512 columns of a row.
template <class In, int kForm>
__global__ __launch_bounds__(256) void join_rows_kernel(LinearCall c, const float *part) {
    using Ck = RowChunk<In::kBf16>;
    constexpr int kSteps = 8 / Ck::kN;
    const int cols = kForm == kNT ? c.O : c.K;
    const int groups = (cols + 511) / 512;
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < (int64_t)c.N * groups;
         w += (int64_t)gridDim.x * 4) {
        const int r = (int)(w / groups);
        const int n = (int)(w % groups) * 512 + 8 * lane;
        if (r < c.offsets[0]) continue;
        const int e = expert_of_row(c.offsets, c.E, r);
        if (e >= c.E || n >= cols) continue;
        const int64_t at = (int64_t)r * cols + n;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
#pragma unroll 8
        for (int p = 0; p < c.parts; ++p) {
            const float4 *q = reinterpret_cast<const float4 *>(part + p * c.part_size + at);
            const float4 x = q[0], y = q[1];
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
            v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
        }
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            float u[Ck::kN], o[Ck::kN];
#pragma unroll
            for (int i = 0; i < Ck::kN; ++i) o[i] = v[h * Ck::kN + i];
            const int64_t chunk = at / Ck::kN + h;
            if (kForm == kNT && c.bias != nullptr) {
                Ck::widen(Ck::fetch(c.bias, ((int64_t)e * c.O + n) / Ck::kN + h), u);
#pragma unroll
                for (int i = 0; i < Ck::kN; ++i) o[i] += u[i];
            }
            if (kForm == kNT && c.relu) {
#pragma unroll
                for (int i = 0; i < Ck::kN; ++i) o[i] = o[i] < 0.0f ? 0.0f : o[i];
            }
            if (c.extra != nullptr) {
                Ck::widen(Ck::fetch(c.extra, chunk), u);
#pragma unroll
                for (int i = 0; i < Ck::kN; ++i) {
                    if (kForm == kNT) o[i] += u[i];
                    else o[i] = u[i] > 0.0f ? o[i] : 0.0f;
                }
            }
            Ck::store(c.out, chunk, o);
        }
    }
}

// The same for dW, n results, and db behind it, m; both % 4 == 0.
__global__ __launch_bounds__(256) void join_sums_kernel(const float *__restrict__ part, int parts,
                                                        int64_t part_size, int64_t n, int64_t m,
                                                        float *__restrict__ dw,
                                                        float *__restrict__ db) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n + m;
         i += (int64_t)gridDim.x * 1024) {
        float4 sum = *reinterpret_cast<const float4 *>(part + i);
#pragma unroll 8
        for (int p = 1; p < parts; ++p) {
            const float4 x = *reinterpret_cast<const float4 *>(part + p * part_size + i);
            sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
        }
        *reinterpret_cast<float4 *>(i < n ? dw + i : db + (i - n)) = sum;
    }
}

enum { kEach, kWide, kInParts };   // a block per tile; per compute unit; per part of a tile

template <class In, int kForm, int BM, int BN, int WM, int WN, int kStages, int kHow>
hipError_t launch_tiles(const LinearCall &c, hipStream_t s) {
    const size_t lds =
        kStages * (size_t)(BM + BN) * kChunk + (kHow == kWide ? (size_t)(c.E + 1) * 4 : 0);
    const void *kernel;
    if constexpr (kHow == kWide)
        kernel = (const void *)&linear_wide_kernel<In, kForm, BM, BN, WM, WN, kStages>;
    else
        kernel = (const void *)&linear_kernel<In, kForm, BM, BN, WM, WN, kStages, kHow == kInParts>;
    if (kStages * (BM + BN) * kChunk > 65536 || kHow == kWide) {   // opted in once per device
        static std::mutex m;
        static bool granted[64] = {};
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
        std::lock_guard<std::mutex> lock(m);
        if (!granted[dev]) {
            const hipError_t err =
                hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                    kStages * (BM + BN) * kChunk + 2049 * 4);
            if (err != hipSuccess) return err;
            granted[dev] = true;
        }
    }
    int64_t blocks = kUnitsOfDevice;
    LinearCall call = c;
    if (kHow != kWide) {
        const int64_t nn = ((kForm == kNT ? c.O : c.K) + BN - 1) / BN;
        const int64_t nm = (c.O + BM - 1) / BM;
        if (kForm != kTN) blocks = nn * ((int64_t)c.N / BM + (c.E < c.N ? c.E : c.N));
        else blocks = nm * nn >= 32 ? (nm * nn + 7) / 8 * 8 * c.E : nm * nn * c.E;
        blocks = (blocks + 7) / 8 * 8;
        if (kHow == kInParts) blocks *= c.parts;
    }
    constexpr int64_t kMost = 1 << 22;   // a launch has fewer than 2^32 threads
    for (int64_t b = 0; b < blocks; b += kMost) {
        call.block0 = (int)b;
        void *args[] = {&call};
        const int64_t now = blocks - b < kMost ? blocks - b : kMost;
        const hipError_t err =
            hipLaunchKernel(kernel, dim3((unsigned)now), dim3(64 * WM * WN), args, lds, s);
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

// The choice of tile. The row ranges are on the GPU, so it goes by the rows an expert has
// on average. A product takes the larger of one tile's time and the time of all tiles over
// the compute units: us per chunk of a tile alone on a unit, and of a tile among many (bf16,
// 64 steps a chunk). The numbers are measured ones, set within their spread so that the choices
// are best over 400 calls of all sizes: those take 1.9 % longer than with the best tile each.
// For instance (N rows, E experts, K inputs, O outputs; us):
//   256 x 256  13140, 3, 7256, 1872: 402, 128 x 128 520, 64 x 128 648
//   128 x 128  8192, 64, 1024, 4096: 155, 64 x 128 171, 64 x 64 202
//   64 x 128   314, 20, 2960, 4864: 125, 128 x 128 144, 64 x 64 132
//   64 x 64    512, 1, 2048, 2048: 13.7, 64 x 128 22.7, 256 x 256 52
// The 256 x 256 tiles are one to a unit: a started round of them takes a whole one's time, or
// 0.9 or 0.45 of it where its tiles are cut. fp32 (32 steps a chunk): 64 x 128 1.03, 64 x 64
// 0.6, the same rate at the matrix cores' limit (8192, 8, 1024, 4096: 526 us, 131 TFLOP/s,
// 64 x 64 571; 1501, 10, 2056, 520, in one piece: 77.6 and 74.0).
struct TileCost {
    int bm, bn;
    double alone, many;
};
constexpr TileCost kCosts[2][4] = {   // kNT, kNN
    {{64, 128, 0.65, 0.45}, {128, 128, 0.85, 0.68}, {256, 256, 1.7, 1.85}, {64, 64, 0.37, 0.27}},
    {{64, 128, 0.8, 0.4}, {128, 128, 1.05, 0.62}, {256, 256, 1.6, 1.7}, {64, 64, 0.64, 0.28}}};

int pick_tile(int form, int64_t N, int64_t E, int64_t cols, double &low) {
    const int64_t experts = E < N ? E : N;
    int best = 0;
    for (int i = 0; i < 4; ++i) {
        const TileCost &t = kCosts[form][i];
        // Half a tile goes to waste at an expert's end.
        double rows = (double)N / t.bm + 0.5 * experts;
        if (rows < experts) rows = (double)experts;
        double rounds = rows * ((cols + t.bn - 1) / t.bn) / kUnitsOfDevice;
        if (t.bm == 256) {
            rounds *= 1.03;   // (a few tiles more than on average start another round)
            const double whole = (double)(int64_t)rounds;
            const double rest = rounds - whole;
            rounds = whole + (rest > 0.5 ? 1.0 : rest > 0.25 ? 0.9 : rest > 0.0 ? 0.45 : 0.0);
        }
        const double cost = rounds * t.many > t.alone ? rounds * t.many : t.alone;
        if (i == 0 || cost < low) {
            best = i;
            low = cost;
        }
    }
    return best;
}

// Parts of the contraction, for a call whose tiles leave compute units idle or with one tile
// each, which a unit does not overlap with anything: the number with the least time of the
// products (a chunk of a tile alone on a unit, and of each of several; tiles of 64 x 64, kTN
// 128 x 128 or fp32 64 x 128), of the sums' way through memory and of the launch that joins
// them, with four chunks at least in a part. In one piece and in parts, us: y of 1 row x 8192 to
// 512 in 32 parts 40 and 14 (fp32 165 and 18), of 512 x 4096 to 256 in 6 23 and 12 (80 and 23);
// dx of 150 x 6152 to 1032 72 and 21 (121 and 41), of 1000 x 4096 to 512, two experts, 41 and 18;
// dW 200 x 64 of 5000 rows in 19 67 and 15 (in 32 188 and 20), fp32 216 x 1672 of 8606 rows, three
// experts, in 3 109 and 76; fp32 dx of 3584 x 6112 to 344, seven experts, 204 and 158. What the
// rule leaves whole: dx of 1 x 512 to 2048, 5.8, in 2 parts 7.1; and experts of few rows in many
// tiles, which are bound by their matrices' bytes (fp32 y of 94 x 6976 to 1032, 27 experts, 158,
// in parts 219).
int parts_of(int form, bool bf16, int64_t N, int64_t E, int64_t K, int64_t O) {
    const int64_t steps = kChunk / (bf16 ? 2 : 4);
    const int64_t experts = E < N ? E : N;
    const int64_t cols = form == kNT ? O : K;
    constexpr TileCost kPart[3][2] = {{{64, 64, 0.6, 0.48}, {64, 64, 0.36, 0.3}},
                                      {{64, 64, 0.6, 0.48}, {64, 64, 0.64, 0.4}},
                                      {{64, 128, 1.05, 0.9}, {128, 128, 0.85, 0.62}}};
    const TileCost &t = kPart[form][bf16];
    const int64_t rows = form == kTN ? E * ((O + t.bm - 1) / t.bm)
                                     : (N + t.bm - 1) / t.bm + experts - 1;   // at most
    const int64_t tiles = rows * ((cols + t.bn - 1) / t.bn);
    if (tiles > (form != kTN && N / E < 32 ? 1 : 2) * kUnitsOfDevice) return 1;
    const int64_t chunks = ((form == kNT ? K : form == kNN ? O : N / experts) + steps - 1) / steps;
    const double results = form == kTN ? (double)E * O * K : (double)N * cols;
    const int64_t most = chunks / 4 < 32 ? chunks / 4 : 32;
    int best = 1;
    double low = 0.0, whole = 1e30;
    if (bf16 && form != kTN) pick_tile(form, N, E, cols, whole);
    for (int64_t p = 1; p <= most; ++p) {
        const double many = t.many * ((tiles * p + kUnitsOfDevice - 1) / kUnitsOfDevice);
        double cost = chunks * (many > t.alone ? many : t.alone) / p;
        if (p == 1 && cost > chunks * whole) cost = chunks * whole;
        if (p > 1) cost += 1.3 * (4.0 + 8.0 * p * results / 4e6);
        if (p == 1 || cost < low) {
            best = (int)p;
            low = cost;
        }
    }
    return best;
}

constexpr int tile(int rows, int cols) { return rows << 16 | cols; }

// The tile of a call that is in `parts`.
int tile_of(int form, bool bf16, int64_t N, int64_t E, int64_t K, int64_t O, int64_t parts) {
    const int64_t avg = N / E;
    const int64_t cols = form == kNT ? O : K;
    if (form == kTN) {
        // A tile stores its matrix's part once and multiplies little, so the large tile is for
        // experts with many rows only (128 x 128 and 256 x 256 tiles, us: 64 experts of
        // 4096 x 1024 with 16 rows each 219 and 247, 128 rows 317 and 312, 256 rows 428 and 366;
        // eight of 8192 x 2048 with 128 rows each 133 and 148, 256 rows 181 and 174), where its
        // started rounds take less time than all smaller tiles (a chunk of one 1.9 and, among
        // others, 0.58; three experts of 5384 x 520, 27587 rows, 261 and 353, 43 of 264 x 1696,
        // 7447 rows, 30 and 53; over 280 calls 1.2 % longer than with the better tile each).
        if (!bf16) return tile(64, 128);
        if (parts > 1) return tile(128, 128);
        const int64_t wide = E * ((O + 255) / 256) * ((K + 255) / 256);
        const int64_t tiles = E * ((O + 127) / 128) * ((K + 127) / 128);
        const double rounds = (double)((wide + kUnitsOfDevice - 1) / kUnitsOfDevice);
        return avg >= 160 && rounds * 1.9 < (double)tiles / kUnitsOfDevice * 0.58 ? tile(256, 256)
                                                                                  : tile(128, 128);
    }
    if (parts > 1) return tile(64, 64);
    if (!bf16) {
        // Few rows: as much in flight as possible (512 rows of 64 experts, 1024 to 2048: 119 us,
        // 64 x 128 142). The larger tile saves operand reads once there are several to a unit.
        // Over 120 calls of all sizes 1.9 % longer than with the best of the three tiles each, at
        // most 23 % (dx of 695 x 248 to 2656, four experts, 19.8 and 16.1 with 32 x 128).
        if (avg < 32) return tile(32, 128);
        const int64_t tiles = (N / 64 + E / 2) * ((cols + 127) / 128);
        return tiles < 4 * kUnitsOfDevice ? tile(64, 64) : tile(64, 128);
    }
    // A few rows: the matrices' bytes count, and what keeps most of them in flight (64 rows
    // of 64 experts, 1024 to 4096: 58.6 us, 64 x 128 tiles 60.8; of 16, 2048 to 8192: 96 and
    // 121). By columns a row of 32 x 64 tiles reads too short pieces, but for single rows.
    if (avg <= (form == kNT ? 16 : 2)) return tile(32, 64);
    double cost;
    const TileCost &t = kCosts[form][pick_tile(form, N, E, cols, cost)];
    return tile(t.bm, t.bn);
}

template <class In, int kForm>
hipError_t launch_form(const LinearCall &c, hipStream_t s) {
    const int shape = tile_of(kForm, In::kBf16, c.N, c.E, c.K, c.O, c.parts);
    if constexpr (kForm == kTN && In::kBf16) {
        if (c.parts > 1) return launch_tiles<In, kForm, 128, 128, 2, 2, 2, kInParts>(c, s);
        if (shape == tile(256, 256))
            return launch_tiles<In, kForm, 256, 256, 2, 4, 2, kWide>(c, s);
        return launch_tiles<In, kForm, 128, 128, 2, 2, 2, kEach>(c, s);
    } else if constexpr (kForm == kTN) {
        if (c.parts > 1) return launch_tiles<In, kForm, 64, 128, 2, 2, 2, kInParts>(c, s);
        return launch_tiles<In, kForm, 64, 128, 2, 2, 2, kEach>(c, s);
    } else {
        if (c.parts > 1) return launch_tiles<In, kForm, 64, 64, 2, 2, 3, kInParts>(c, s);
        if constexpr (In::kBf16) {
            switch (shape) {
                case tile(32, 64):
                    return launch_tiles<In, kForm, 32, 64, 1, 2, kForm == kNT ? 4 : 2, kEach>(c, s);
                case tile(64, 128): return launch_tiles<In, kForm, 64, 128, 2, 2, 2, kEach>(c, s);
                case tile(128, 128): return launch_tiles<In, kForm, 128, 128, 2, 2, 2, kEach>(c, s);
                case tile(256, 256): return launch_tiles<In, kForm, 256, 256, 2, 4, 2, kWide>(c, s);
                default: return launch_tiles<In, kForm, 64, 64, 2, 2, 3, kEach>(c, s);
            }
        } else {
            switch (shape) {
                case tile(32, 128): return launch_tiles<In, kForm, 32, 128, 1, 4, 3, kEach>(c, s);
                case tile(64, 128): return launch_tiles<In, kForm, 64, 128, 2, 2, 2, kEach>(c, s);
                default: return launch_tiles<In, kForm, 64, 64, 2, 2, 2, kEach>(c, s);
            }
        }
    }
}

// The call, or its parts into the workspace and their join.
template <class In, int kForm>
hipError_t launch_call(LinearCall c, void *workspace, hipStream_t s) {
    c.parts = parts_of(kForm, In::kBf16, c.N, c.E, c.K, c.O);
    if (c.parts == 1) return launch_form<In, kForm>(c, s);
    void *out = c.out;
    const float *part = static_cast<const float *>(workspace);
    const int64_t cols = kForm == kNT ? c.O : c.K;
    const int64_t size = (kForm == kTN ? (int64_t)c.E * c.O : (int64_t)c.N) * cols;
    const int64_t with_db = c.db != nullptr ? (int64_t)c.E * c.O : 0;
    float *db = c.db;
    c.part_size = size + with_db;
    c.out = workspace;
    if (db != nullptr) c.db = static_cast<float *>(workspace) + size;
    hipError_t err = launch_form<In, kForm>(c, s);
    if (err != hipSuccess) return err;
    c.out = out;
    constexpr int64_t kMost = 1 << 20;
    if constexpr (kForm == kTN) {
        const int64_t blocks = (c.part_size + 1023) / 1024;
        hipLaunchKernelGGL(join_sums_kernel, dim3((unsigned)(blocks < kMost ? blocks : kMost)),
                           dim3(256), 0, s, part, c.parts, c.part_size, size, with_db,
                           static_cast<float *>(out), db);
    } else {
        const int64_t blocks = ((int64_t)c.N * ((cols + 511) / 512) + 3) / 4;
        hipLaunchKernelGGL((join_rows_kernel<In, kForm>),
                           dim3((unsigned)(blocks < kMost ? blocks : kMost)), dim3(256), 0, s, c,
                           part);
    }
    return hipGetLastError();
}

template <int kForm>
hipError_t launch(const LinearCall &c, int bf16, void *workspace, hipStream_t s) {
    return bf16 ? launch_call<Bf16, kForm>(c, workspace, s)
                : launch_call<F32, kForm>(c, workspace, s);
}

LinearCall call_of(const void *A, const void *B, const void *bias, const void *extra,
                   const int32_t *offsets, void *out, int64_t N, int64_t E, int64_t K, int64_t O,
                   int relu) {
    LinearCall c{};
    c.A = A;
    c.B = B;
    c.bias = bias;
    c.extra = extra;
    c.offsets = offsets;
    c.out = out;
    c.N = (int)N;
    c.E = (int)E;
    c.K = (int)K;
    c.O = (int)O;
    c.relu = relu;
    return c;
}

}  // namespace

size_t linear_workspace_size(int product, int64_t N, int64_t E, int64_t K, int64_t O, int bf16) {
    const int64_t parts = parts_of(product, bf16 != 0, N, E, K, O);
    if (parts == 1) return 0;
    const int64_t n = product == kNT ? N * O : product == kNN ? N * K : E * O * (K + 1);
    return ((size_t)(parts * n) * 4 + 255) / 256 * 256;
}

void linear_tile(int product, int64_t N, int64_t E, int64_t K, int64_t O, int bf16, int32_t *rows,
                 int32_t *cols, int32_t *parts) {
    *parts = parts_of(product, bf16 != 0, N, E, K, O);
    const int t = tile_of(product, bf16 != 0, N, E, K, O, *parts);
    *rows = t >> 16;
    *cols = t & 0xffff;
}

hipError_t launch_linear(const void *x, const void *w, const void *bias, const void *residual,
                         const int32_t *offsets, void *y, int64_t N, int64_t E, int64_t K,
                         int64_t O, int relu, int bf16, void *workspace, hipStream_t s) {
    return launch<kNT>(call_of(x, w, bias, residual, offsets, y, N, E, K, O, relu), bf16, workspace,
                       s);
}

hipError_t launch_linear_dx(const void *dy, const void *w, const void *relu_of,
                            const int32_t *offsets, void *dx, int64_t N, int64_t E, int64_t K,
                            int64_t O, int bf16, void *workspace, hipStream_t s) {
    return launch<kNN>(call_of(dy, w, nullptr, relu_of, offsets, dx, N, E, K, O, 0), bf16,
                       workspace, s);
}

hipError_t launch_linear_dw(const void *dy, const void *x, const int32_t *offsets, float *dw,
                            float *db, int64_t N, int64_t E, int64_t K, int64_t O, int bf16,
                            void *workspace, hipStream_t s) {
    LinearCall c = call_of(dy, x, nullptr, nullptr, offsets, dw, N, E, K, O, 0);
    c.db = db;
    return launch<kTN>(c, bf16, workspace, s);
}

}  // namespace base

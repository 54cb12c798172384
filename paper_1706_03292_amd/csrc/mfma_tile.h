// The tiled matrix product of the classifier loss: one BM x BN tile of
//
//     C[m][n] = sum_k A(m, k) * B(n, k)
//
// with A and B in bf16 or fp32 in memory, products on the matrix cores
// (16x16x32 bf16, 16x16x4 fp32) and sums in fp32 registers.  Each operand is
// stored either with k along its rows ("k-major": row m holds A(m, 0..K)) or
// with k as the row index ("r-major": row k holds A(0..M, k)), so the three
// products logits = X W^T, dX = G W and dW = G^T X read X, W and G as they are
// and nothing is transposed in memory.
//
// A step takes 128 bytes of k per row (64 bf16 or 32 fp32 values) from each
// operand straight into LDS (gfx950's 16-byte LDS-direct buffer loads; what is
// outside the operand reads 0 by the buffer's range check), up to STAGES
// steps ahead.  Each stage is an LDS object of its own, so that reading one does not
// wait for the loads in flight into another.
//
// LDS layout.  An LDS-direct load writes 16 bytes per lane to consecutive
// addresses, so a permutation of the tile is made by choosing which 16 bytes a
// lane fetches.  k-major: chunks are exchanged within a row so that the
// 16 rows of an operand read lie in different banks.  r-major, bf16:
// operand reads are gfx950's transposing LDS reads (16 lanes name four k rows
// of 16 columns, lane i receives column i's four values); chunk pairs are
// exchanged by a function of the k row so that the rows read together lie in
// different banks.  r-major, fp32: a lane reads single values; groups of four
// chunks are exchanged.
//
// On 256 x 256 tiles, a workgroup a CU, with the grid full: 1.36 PFLOP/s at 8192^3
// k-major (bf16; the library 1.47), 1.3 with one or both operands r-major.  fp32
// in bf16 parts on 128 x 128 tiles: 0.21 PFLOP/s of fp32 products.
//
// Operands enter the matrix instruction exchanged (B's rows first), so a lane
// ends up with four neighbouring n of one row m: wide stores, and row
// statistics that stay in a lane but for the last two steps.
#pragma once

#include "elements.h"

namespace poseidon {
namespace {

typedef float acc4 __attribute__((ext_vector_type(4)));
typedef short h4 __attribute__((ext_vector_type(4)));
typedef short h8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) h4 lds_h4;

constexpr int XCDS = 8;              // MI355X: eight dies, each with an L2 of its own
constexpr int RSRC_RAW = 0x00020000; // buffer resource word 3: raw 32-bit accesses
constexpr int64_t RSRC_MOST = 0x7fff0000;
constexpr int OUTSIDE = 0x7ffffff0;  // an offset no resource here contains
constexpr int STEP_BYTES = 128;      // k per row and step: two sub-steps (fragments of 16 rows and 64 bytes)

typedef int i4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t lds_address(const char* p)
{
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)p));
}

// 16 bytes per lane from rs + v to LDS, lane after lane from `to`.  Written as
// an instruction, not as the builtin: the compiler makes every transposing LDS
// read after the builtin wait for all loads in flight, whichever stage they go
// to.  It has no result register; whoever reads the stage waits for it
// (Tile::turn).  The wait states are those of a vector load whose scalar
// operands (M0 among them) were written just before, by a vector instruction
// even: the compiler does not look for that inside.  (M0 is reserved: the compiler
// sets it itself right before each use of its own, of which these kernels have none.)
__device__ __forceinline__ void load_to_lds(i4 rs, int v, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(v), "s"(rs)
                 : "memory");
}

// One operand: `rows` rows of values of type E from p (a 4-byte boundary, as
// every row's start), ld values apart.  k-major: a row holds K of them;
// r-major: there are K rows.  `plane`: the
// distance between the bf16 parts of one matrix, for products of parts.
struct Operand {
    const void* p;
    int64_t ld;
    int64_t rows;
    int64_t plane;
};

// Which parts the products take, in order: A part sel & 3, B part
// (sel >> 2) & 3, four bits a product.
struct Parts {
    int count;
    uint32_t sel;
};

// fp32 in memory, multiplied as six bf16 products of its exact three parts
// (h*h, h*m, m*h, h*l, l*h, m*m: what is dropped is below 2^-23 of a product),
// the parts made in registers from what the operand reads bring.  An infinity,
// and a value above 3.39e38, whose h is one, have no such parts (a later one is NaN,
// and so are the sums it meets): a tile with a sum that is not finite is made
// again by the fp32 products (Tile::InFp32).
struct Split32 {};

template <typename E>
struct InMemory {
    typedef E type;
};
template <>
struct InMemory<Split32> {
    typedef float type;
};

template <typename E_, int R, int NT, bool KMAJOR, bool SPREAD>
struct Panel {
    typedef typename InMemory<E_>::type E;
    static constexpr bool SPLIT = !__is_same(E_, E);   // operands are eight fp32 values a lane, k from 8 (lane / 16)
    static constexpr int SZ = sizeof(E);
    static constexpr int BYTES = R * STEP_BYTES;
    static constexpr int LOADS = BYTES / 16 / NT;
    static constexpr int BK = STEP_BYTES / SZ;
    static constexpr int PER_ROW = R * SZ / 16;   // r-major: chunks of a k row
    static_assert(BYTES % (16 * NT) == 0, "whole loads");

    static constexpr int CHUNKS = STEP_BYTES / 16;   // k-major: of a row

    // k-major: which chunk of row r sits in slot s is s ^ swz_k(r).  The rows
    // read together are 16 neighbours, or (SPREAD) four neighbours each from
    // four blocks of 16; eight of them in the order of their lanes, and all 16,
    // lie in different banks.
    static __device__ __forceinline__ int swz_k(int r)
    {
        return SPREAD ? ((r & 3) ^ ((r >> 5) & 1)) | (((r >> 4) & 1) << 2) : (r & 7) ^ ((r >> 3) & 1);
    }

    // r-major: which chunk of a k row sits in slot s is s ^ swz_r(k).
    static __device__ __forceinline__ int swz_r(int k)
    {
        if constexpr (SZ == 2) {
            if constexpr (PER_ROW % 16 == 0)   // rows of a multiple of 256 bytes: eight pairs
                return (((k & 3) | (((k >> 4) & 1) << 2)) << 1);
            else if constexpr (PER_ROW % 8 == 0)   // of 128: the row's parity is half of the bank, four pairs
                return ((((k >> 1) & 1) | (((k >> 4) & 1) << 1)) << 1);
            else
                return 0;
        } else {
            if constexpr (PER_ROW % 16 == 0)
                return ((k >> 3) & 3) << 2;
            else
                return 0;
        }
    }

    int off[LOADS];      // this lane's offsets from the step's base
    int kchunk[LOADS];   // k-major: first k of the lane's chunk within the step
    uint64_t base;       // of the next step's first part
    int64_t left;        // bytes from base to the operand's end
    int64_t advance;     // bytes from one step to the next
    i4 rs;               // the next load's resource

    __device__ __forceinline__ void init(const Operand& o, int64_t r0, int64_t k0, int tid)
    {
        const int64_t ldb = o.ld * SZ;
        const int lane = tid & 63, w = tid >> 6;
        if constexpr (KMAJOR) {
            const int64_t rows = o.rows - r0 < R ? o.rows - r0 : R;
            base = reinterpret_cast<uint64_t>(o.p) + r0 * ldb + k0 * SZ;
            left = rows * ldb - k0 * SZ;
            advance = STEP_BYTES;
        } else {
            base = reinterpret_cast<uint64_t>(o.p) + k0 * ldb + r0 * SZ;
            left = (o.rows - k0) * ldb - r0 * SZ;
            advance = BK * ldb;
        }
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int b = q * (NT / 64) + w;   // 1 KB block of the stage
            if constexpr (KMAJOR) {
                const int r = (64 / CHUNKS) * b + lane / CHUNKS, c = (lane % CHUNKS) ^ swz_k(r);
                off[q] = static_cast<int>(r * ldb) + c * 16;
                kchunk[q] = c * (16 / SZ);
            } else {
                const int s = 64 * b + lane, k = s / PER_ROW, c = (s % PER_ROW) ^ swz_r(k);
                off[q] = static_cast<int>(k * ldb) + c * 16;
                kchunk[q] = 0;
            }
        }
    }

    // The resource of the next step's part at `part` bytes; `any`: whether
    // there is such a step (else every lane is outside).
    __device__ __forceinline__ void aim(int64_t part, bool any)
    {
        const uint64_t from = base + static_cast<uint64_t>(part);
        const int64_t n = !any || left < 0 ? 0 : left > RSRC_MOST ? RSRC_MOST : left;
        rs = i4{static_cast<int>(from), static_cast<int>(from >> 32) & 0xffff, static_cast<int>(n), RSRC_RAW};
    }

    __device__ __forceinline__ void next()
    {
        base += static_cast<uint64_t>(advance);
        left -= advance;
    }

    // Load q of the aimed step into the stage; k_left: values of k from the
    // step's first on (k-major chunks past it read 0; r-major rows past it lie
    // outside the operand).
    __device__ __forceinline__ void load(const char* stage, int q, int k_left, int tid) const
    {
        const int v = KMAJOR && kchunk[q] >= k_left ? OUTSIDE : off[q];
        load_to_lds(rs, v, lds_address(stage) + __builtin_amdgcn_readfirstlane((tid >> 6) * 1024) + q * (NT / 64) * 1024);
    }

    // SPLIT's operand: row r0 + 16 j + lane % 16, eight k from 8 (lane / 16).
    static __device__ __forceinline__ f8e frag8(const char* stage, int r0, int j, int lane)
    {
        const int g = lane >> 4, i = lane & 15, r = r0 + 16 * j + i;
        f8e v;
        if constexpr (KMAJOR) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const acc4 x = *reinterpret_cast<const acc4*>(stage + r * STEP_BYTES + (((2 * g + half) ^ swz_k(r)) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[4 * half + e] = x[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = 8 * g + e;
                v[e] = *reinterpret_cast<const float*>(stage + k * (R * 4) + (((r >> 2) ^ swz_r(k)) << 4) + (r & 3) * 4);
            }
        }
        return v;
    }

    // k-major: the step that ends inside a 16-byte chunk has fetched the next
    // row's first values there.  Clears what is past the k_left values of the
    // step's rows (whole chunks past them were not fetched and are 0).
    static __device__ __forceinline__ void clear_past(char* stage, int k_left, int tid)
    {
        constexpr int EACH = 16 / SZ;
        const int c = k_left / EACH, from = k_left % EACH;
        if (!KMAJOR || from == 0 || c >= CHUNKS)
            return;
        for (int r = tid; r < R; r += NT) {
            E* at = reinterpret_cast<E*>(stage + r * STEP_BYTES + ((c ^ swz_k(r)) << 4));
            for (int e = from; e < EACH; ++e)
                at[e] = static_cast<E>(0.f);
        }
    }

    // The operand fragment of 16 rows, sub-step kk: lane l has the k of the 16
    // bytes 2 (l / 16) + kk of the step's 128 (every operand alike: which k meet
    // in an instruction is free).  Read so, no two lanes of a k-major read that
    // are served together want one bank; with bytes 4 kk + l / 16 some do (22%
    // of the cycles of an 8192 x 32768 x 2048 product).  Lane l
    // takes row r0 + l % 16 of block j = (row - r0) / 16; SPREAD: of the four
    // blocks from r0 on, rows 16 (i / 4) + 4 j + i % 4, i = l % 16.
    static __device__ __forceinline__ h8 frag(const char* stage, int r0, int j, int kk, int lane)
    {
        const int g = lane >> 4, i = lane & 15;
        if constexpr (KMAJOR) {
            const int r = SPREAD ? r0 + 16 * (i >> 2) + 4 * j + (i & 3) : r0 + 16 * j + i;
            return *reinterpret_cast<const h8*>(stage + r * STEP_BYTES + (((2 * g + kk) ^ swz_k(r)) << 4));
        } else if constexpr (SZ == 2) {
            h8 v;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int k = 8 * (2 * g + kk) + 4 * half + (i >> 2);
                const int byte = (r0 + 16 * j) * 2 + (i & 3) * 8;
                const char* at = stage + k * (R * 2) + (((byte >> 4) ^ swz_r(k)) << 4) + (byte & 15);
                const h4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_h4*)at);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[4 * half + e] = x[e];
            }
            return v;
        } else {
            acc4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = 4 * (2 * g + kk) + e;
                const int byte = (r0 + 16 * j + i) * 4;
                v[e] = *reinterpret_cast<const float*>(stage + k * (R * 4) + (((byte >> 4) ^ swz_r(k)) << 4) +
                                                       (byte & 15));
            }
            return __builtin_bit_cast(h8, v);
        }
    }
};

typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef __bf16 b2e __attribute__((ext_vector_type(2)));
typedef float f2e __attribute__((ext_vector_type(2)));

struct Parts3 {
    h8 h, m, l;
};

// The upper halves of a and b, a's in the low half: they are bf16 values, exact
// where no more than eight bits are left.
__device__ __forceinline__ unsigned upper_halves(float a, float b)
{
    return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
}

// h and m rounded to nearest, l exact (at most eight bits are left).  Cut off
// instead, h would leave m and l twice as large, and what the six products drop
// four times.
__device__ __forceinline__ Parts3 in_parts3(f8e x)
{
    u4 part[3];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float a = x[2 * q], b = x[2 * q + 1];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const unsigned w = __builtin_bit_cast(unsigned, __builtin_convertvector((f2e){a, b}, b2e));
            part[p][q] = w;
            a -= __builtin_bit_cast(float, w << 16);
            b -= __builtin_bit_cast(float, w & 0xffff0000u);
        }
        part[2][q] = upper_halves(a, b);
    }
    return Parts3{__builtin_bit_cast(h8, part[0]), __builtin_bit_cast(h8, part[1]), __builtin_bit_cast(h8, part[2])};
}

template <typename E>
__device__ __forceinline__ acc4 mfma(h8 a, h8 b, acc4 c)
{
    if constexpr (sizeof(E) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8e, a), __builtin_bit_cast(bf8e, b), c, 0,
                                                       0, 0);
    } else {
        const acc4 x = __builtin_bit_cast(acc4, a), y = __builtin_bit_cast(acc4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
}

// An LDS stage of its own per (size, number, use).
template <int SIZE, int S, int USE>
struct Stage {
    static __device__ __forceinline__ char* ptr()
    {
        __shared__ __align__(1024) char a[SIZE];
        return a;
    }
};

// s_waitcnt's operand: at most so many vector loads and LDS operations left.
constexpr int wait_imm(int vm, int lgkm) { return 0x0070 | (lgkm << 8) | (vm & 15) | ((vm >> 4) << 14); }

template <typename E_, bool AK_, bool BK_, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool SPREAD_ = false>
struct Tile {
    typedef E_ E;
    typedef typename InMemory<E_>::type M;   // in memory
    static constexpr bool AK = AK_, BKM = BK_, SPLIT = !__is_same(E_, M);
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int NWN = BN / WN, WAVES = (BM / WM) * NWN, NT = 64 * WAVES;
    static constexpr int TM = WM / 16, TN = WN / 16;
    static constexpr bool SPREAD = SPREAD_;   // a lane's sums are 16 neighbours of a row, not four of each block
    static_assert(!SPREAD || (TN == 4 && BKM), "four blocks of k-major rows");
    // The same tile by the fp32 matrix instructions, in the same LDS.
    using InFp32 = Tile<M, AK, BKM, BM, BN, WM, WN, STAGES, SPREAD>;
    using PA = Panel<E, BM, NT, AK, false>;
    using PB = Panel<E, BN, NT, BKM, SPREAD>;
    static constexpr int LOADS = PA::LOADS + PB::LOADS;
    static constexpr int STEP = PA::BK;

    template <int S>
    static __device__ __forceinline__ char* a_stage() { return Stage<PA::BYTES, S, 0>::ptr(); }
    template <int S>
    static __device__ __forceinline__ char* b_stage() { return Stage<PB::BYTES, S, 1>::ptr(); }

    PA pa;
    PB pb;
    Parts parts;
    int64_t a_plane, b_plane;
    int k_left;        // values of k from the next step to load on (none left: 0 or less)
    int k_unread;      // and from the stage that is read next
    int part;          // the next product of it
    int wm, wn, lane, tid;

    // The operands that the next products need first.
    struct Ahead {
        h8 a[2], b[TN];
    };
    struct AheadSplit {
        Parts3 a, b[TN];   // in parts: the first row block's, and all of B's
        f8e next;          // as read: the second row block's
    };

    template <bool, typename = void>
    struct Choose {
        typedef Ahead type;
    };
    template <typename U>
    struct Choose<true, U> {
        typedef AheadSplit type;
    };

    __device__ __forceinline__ void aim()
    {
        const uint32_t sel = parts.sel >> (4 * part);
        pa.aim((sel & 3) * a_plane, k_left > 0);
        pb.aim(((sel >> 2) & 3) * b_plane, k_left > 0);
    }

    // Load q of the aimed step (A's, then B's) into stage S.
    template <int S>
    __device__ __forceinline__ void load(int q)
    {
        if (q < PA::LOADS)
            pa.load(a_stage<S>(), q, k_left, tid);
        else
            pb.load(b_stage<S>(), q - PA::LOADS, k_left, tid);
    }

    __device__ __forceinline__ void after_loads()
    {
        if (++part == parts.count) {
            part = 0;
            k_left -= STEP;
            pa.next();
            pb.next();
        }
    }

    // Group g's A operand, and the B operands of sub-step kk.
    template <int S>
    __device__ __forceinline__ h8 a_frag(int g) const { return PA::frag(a_stage<S>(), wm, g % TM, g / TM, lane); }
    template <int S>
    __device__ __forceinline__ h8 b_frag(int j, int kk) const { return PB::frag(b_stage<S>(), wn, j, kk, lane); }

    // Stage S is read next: where K ends inside a chunk of it, what lies past
    // it is cleared first.  (Products of several parts end on whole chunks.)
    template <int S>
    __device__ __forceinline__ void to_read()
    {
        if (k_unread > 0 && k_unread < STEP && k_unread % (16 / static_cast<int>(sizeof(M))) != 0) {
            PA::clear_past(a_stage<S>(), k_unread, tid);
            PB::clear_past(b_stage<S>(), k_unread, tid);
            __syncthreads();
        }
        k_unread -= STEP;
    }

    template <int S>
    __device__ __forceinline__ void read_ahead(Ahead& f) const
    {
#pragma unroll
        for (int j = 0; j < TN; ++j)
            f.b[j] = b_frag<S>(j, 0);
        f.a[0] = a_frag<S>(0);
        f.a[1] = a_frag<S>(1);
    }

    // The products of stage S, in groups (sub-step, row block), operands read
    // two groups before their products.  Two groups before the end every
    // operand of the stage has been read: there the waves meet, the stage's
    // next loads start and the next stage's first operands are read while the
    // last two groups run, so that the matrix cores need not wait for either.
    template <int S>
    __device__ __forceinline__ void turn(acc4 (&acc)[TM][TN], Ahead& f)
    {
        constexpr int G = 2 * TM, FIRST_B = TM - 2 - TN > 0 ? TM - 2 - TN : 0;
        static_assert(TM >= 2 && TN <= TM, "groups to read in");
        h8 a[G], b[2][TN];
#pragma unroll
        for (int j = 0; j < TN; ++j)
            b[0][j] = f.b[j];
        a[0] = f.a[0];
        a[1] = f.a[1];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g + 2 < G)
                a[g + 2] = a_frag<S>(g + 2);
            if (g >= FIRST_B && g - FIRST_B < TN)
                b[1][g - FIRST_B] = b_frag<S>(g - FIRST_B, 1);
            if (g == G - 2) {
                // All of this wave's reads of the stage are done, and its own
                // loads of the next stage; then the other waves'.
                __builtin_amdgcn_s_waitcnt(wait_imm((STAGES - 2) * LOADS, 0));
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                to_read<(S + 1) % STAGES>();
                read_ahead<(S + 1) % STAGES>(f);
                aim();
#pragma unroll
                for (int q = 0; q < (LOADS + 1) / 2; ++q)
                    load<S>(q);
            }
            if (g == G - 1) {
#pragma unroll
                for (int q = (LOADS + 1) / 2; q < LOADS; ++q)
                    load<S>(q);
                after_loads();
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[g % TM][j] = mfma<E>(b[g / TM][j], a[g], acc[g % TM][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // The same for fp32 in parts.  A step is one sub-step of 32 k; a group is a
    // row block's 6 TN products, and while they run the next block is put into
    // parts (in the last group all that the next stage needs first).
    template <int S>
    __device__ __forceinline__ void turn_split(acc4 (&acc)[TM][TN], AheadSplit& f)
    {
        static_assert(!SPLIT || (TM >= 2 && !SPREAD), "row blocks to read in");
        f8e raw[TM + 2], next_b[TN];
        raw[1] = f.next;
        Parts3 a = f.a;
#pragma unroll
        for (int g = 0; g < TM; ++g) {
            if (g + 2 < TM)
                raw[g + 2] = PA::frag8(a_stage<S>(), wm, g + 2, lane);
            if (g == TM - 2) {
                __builtin_amdgcn_s_waitcnt(wait_imm((STAGES - 2) * LOADS, 0));
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                constexpr int N = (S + 1) % STAGES;
                to_read<N>();
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    next_b[j] = PB::frag8(b_stage<N>(), wn, j, lane);
                raw[TM] = PA::frag8(a_stage<N>(), wm, 0, lane);
                raw[TM + 1] = PA::frag8(a_stage<N>(), wm, 1, lane);
                aim();
#pragma unroll
                for (int q = 0; q < (LOADS + 1) / 2; ++q)
                    load<S>(q);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (g == TM - 1) {
#pragma unroll
                for (int q = (LOADS + 1) / 2; q < LOADS; ++q)
                    load<S>(q);
                after_loads();
                __builtin_amdgcn_sched_barrier(0);
            }
            const Parts3 next = in_parts3(raw[g + 1]);
            products(acc[g], a, f.b);
            a = next;
            if (g == TM - 1) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    f.b[j] = in_parts3(next_b[j]);
            }
            // Products and parts in turn: 44 vector instructions put a block
            // into parts.
            if (g < TM - 1)
                interleave<(44 + 6 * TN - 1) / (6 * TN)>();
            else
                interleave<(44 * (TN + 1) + 6 * TN - 1) / (6 * TN)>();
            __builtin_amdgcn_sched_barrier(0);
        }
        f.a = a;
        f.next = raw[TM + 1];
    }

    template <int VALU>
    static __device__ __forceinline__ void interleave()
    {
#pragma unroll
        for (int i = 0; i < 6 * TN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, VALU, 0);
        }
    }

    static __device__ __forceinline__ void products(acc4 (&acc)[TN], const Parts3& a, const Parts3 (&b)[TN])
    {
#pragma unroll
        for (int p = 0; p < 6; ++p) {
            const h8 x = p == 0 || p == 1 || p == 3 ? a.h : p == 4 ? a.l : a.m;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const h8 y = p == 0 || p == 2 || p == 4 ? b[j].h : p == 3 ? b[j].l : b[j].m;
                acc[j] = mfma<__bf16>(y, x, acc[j]);
            }
        }
    }

    template <int S, typename F>
    __device__ __forceinline__ void turns(acc4 (&acc)[TM][TN], F& f, int left)
    {
        if constexpr (S < STAGES) {
            if (left > S) {
                if constexpr (SPLIT)
                    turn_split<S>(acc, f);
                else
                    turn<S>(acc, f);
                turns<S + 1>(acc, f, left);
            }
        }
    }

    template <int S>
    __device__ __forceinline__ void first_loads()
    {
        if constexpr (S < STAGES) {
            aim();
#pragma unroll
            for (int q = 0; q < LOADS; ++q)
                load<S>(q);
            after_loads();
            first_loads<S + 1>();
        }
    }

    // The tile from (m0, n0) over k from k0, K of it.
    __device__ __forceinline__ void run(acc4 (&acc)[TM][TN], const Operand& a, const Operand& b, const Parts& p,
                                        int64_t m0, int64_t n0, int64_t k0, int64_t K)
    {
        tid = threadIdx.x;
        lane = tid & 63;
        wm = ((tid >> 6) / NWN) * WM;
        wn = ((tid >> 6) % NWN) * WN;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[i][j] = acc4{0.f, 0.f, 0.f, 0.f};
        if (K <= 0)
            return;
        pa.init(a, m0, k0, tid);
        pb.init(b, n0, k0, tid);
        parts = p;
        a_plane = a.plane * static_cast<int64_t>(sizeof(M));
        b_plane = b.plane * static_cast<int64_t>(sizeof(M));
        k_left = k_unread = static_cast<int>(K);
        part = 0;
        // Past the last step `load` fetches nothing (every lane outside), which
        // keeps the count of loads in flight the same to the end.
        first_loads<0>();
        __builtin_amdgcn_s_waitcnt(wait_imm((STAGES - 1) * LOADS, 15));
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        to_read<0>();
        typename Choose<SPLIT>::type f;
        if constexpr (SPLIT) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
                f.b[j] = in_parts3(PB::frag8(b_stage<0>(), wn, j, lane));
            f.a = in_parts3(PA::frag8(a_stage<0>(), wm, 0, lane));
            f.next = PA::frag8(a_stage<0>(), wm, 1, lane);
        } else {
            read_ahead<0>(f);
        }
        for (int left = static_cast<int>((K + STEP - 1) / STEP) * p.count; left > 0; left -= STAGES)
            turns<0>(acc, f, left);
        // No load may still be writing LDS when the workgroup ends.
        __builtin_amdgcn_s_waitcnt(wait_imm(0, 0));
    }
};

// Whether a sum of the wave's that lies within the tile's rows and cols is not
// finite (past them are other rows' values).
template <typename T>
__device__ __forceinline__ bool any_not_finite(const acc4 (&acc)[T::TM][T::TN], int rows, int cols)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int m = (w / T::NWN) * T::WM + (lane & 15), n = (w % T::NWN) * T::WN + 4 * (lane >> 4);
    float zero = 0.f;   // 0 times what is finite
    if (rows == T::BM && cols == T::BN) {
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    zero = fmaf(acc[i][j][r], 0.f, zero);
    } else {
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (m + 16 * i < rows && n + 16 * j + r < cols)
                        zero = fmaf(acc[i][j][r], 0.f, zero);
    }
    return zero != 0.f;   // NaN
}

// Workgroup number -> tile: consecutive workgroups go to the eight dies in
// turn, so each die gets a contiguous run of tiles, walked `group` tile rows at
// a time: what it runs at one time shares operand panels in its L2.
__device__ __forceinline__ void tile_of(int64_t id, int64_t tiles_m, int64_t tiles_n, int group, int64_t& tm,
                                        int64_t& tn)
{
    const int64_t tiles = tiles_m * tiles_n, q = tiles / XCDS, r = tiles % XCDS;
    const int64_t x = id % XCDS, t = x * q + (x < r ? x : r) + id / XCDS;
    const int64_t per = group * tiles_n, g = t / per, first = g * group;
    const int64_t rows = tiles_m - first < group ? tiles_m - first : group, in = t - g * per;
    tm = first + in % rows;
    tn = in / rows;
}

}  // namespace
}  // namespace poseidon

// Tiles of matrix products on the matrix cores, for the operators that are made of them (cross_entropy.hip, newton_schulz.hip,
// linear.hip).
//
// C[m, n] = sum_k A[m, k] * B[n, k], both operands row-major with k contiguous ("planes" of 16-bit elements), sums in 32 bits.
// A number that 16 bits do not hold is the sum of up to three planes, and a product of such numbers the products of their
// planes whose magnitudes a 32-bit sum would see:
//   1 plane   bf16 or fp16 as it is                                     1 product
//   2 planes  fp16, 22 bits and a sign: x = x0 + x1                     x0 y0 + x0 y1 + x1 y0        (dropped: 2^-24 of x y)
//   3 planes  bf16, 24 bits of numbers from 2^-109 to a float's largest six products, x1 y2, x2 y1, x2 y2 dropped
#pragma once

#include "internal.h"
#include "wave_util.h"

namespace dol {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// v_mfma_f32_16x16x32: lane l gives row l & 15, k = 8 (l >> 4) .. + 7 of each operand and gets rows 4 (l >> 4) .. + 3 of column l & 15.
template <typename V>
struct Mfma;
template <>
struct Mfma<bf16x8> {
    using E = __bf16;
    __device__ static f32x4 go(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma<f16x8> {
    using E = _Float16;
    __device__ static f32x4 go(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Bits of x rounded to the nearest E.
template <typename E>
__device__ __forceinline__ uint32_t bits16(float x)
{
    return __builtin_bit_cast(uint16_t, static_cast<E>(x));
}

// x rounded to E, and what is left of it for the next plane (nothing, where x is not finite: inf - inf is NaN).
template <typename E>
__device__ __forceinline__ uint32_t take_plane(float &x)
{
    const E h = static_cast<E>(x);
    const float r = x - static_cast<float>(h);
    x = r == r ? r : 0.0f;
    return __builtin_bit_cast(uint16_t, h);
}

// The first of several bf16 planes: what would round to infinity (from 3.396e38 on) takes the largest number instead, and the next planes have
// the rest, infinity or NaN where that is what x is.
__device__ __forceinline__ uint32_t take_first_plane(float &x)
{
    constexpr float kMost = 3.38953139e38f;
    const uint32_t h = bits16<__bf16>(__builtin_amdgcn_fmed3f(x, -kMost, kMost));
    x -= __uint_as_float(h << 16);
    return h;
}

// 64 lanes' 16 bytes straight to LDS, lane l's at lds + 16 l (lds: the same in every lane).
__device__ __forceinline__ void load_to_lds16(const void *g, uint32_t lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                     (__attribute__((address_space(3))) void *)static_cast<uintptr_t>(lds), 16, 0, 0);
}

// Waits until at most N loads to LDS are on their way and every LDS read has returned, then for the other wavefronts to get here.
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The distance of rows of n elements of 16 bits: an odd number of 256-byte blocks, over which memory's channels change.  Tiles read
// the same columns of many rows; with a power of two of blocks from row to row they would all be on a few channels.  Cross entropy's own
// layouts and dl, rows so / as long as they are, us: float 4 096 x 512 x 1 024 135 / 139, bf16 8 192 x 256 x 20 000 618 / 632.
inline int64_t spread(int64_t n)
{
    if (n < 256) return n;
    const int64_t blocks = (n + 127) / 128;
    return (blocks | 1) * 128;
}

struct Planes {
    const uint16_t *data;
    int64_t ld;         // elements from row to row, a multiple of 8
    int64_t plane;      // elements from plane to plane
};

// How an operand lies in memory: a row of the product to a row, k contiguous, or k to a row and the product's rows side by side.
enum Order { kRows, kCols };

// A tile of BM x BN by WM x WN wavefronts, ST stages of BK; A in PA planes, B in PB, ordered OA and OB.  With WK = 2 there are two sets of
// wavefronts, each for half of every step's k (join() adds them up): where a tile has one wavefront to a SIMD, a second one has something to
// do while the first waits.
// kRows: rows lie in LDS as lines of 128 bytes (one row of 64 elements or two of 32) whose 16-byte pieces are exchanged by an exclusive or
// with the line's number, so that eight neighbouring lanes of a read touch all banks once.  The loads to LDS put lane l's piece at 16 l, so
// it is the lanes' addresses in memory that are exchanged.  A row of B that lane c of fragment j takes is 4 c + j of the wavefront's 64:
// a lane then holds four neighbouring columns of C in acc[i][0..3], and a row of C leaves as 8- or 16-byte pieces, 16 lanes to a line.
// kCols: a step's k lie one below the other, and ds_read_b64_tr_b16 hands them to the lanes: of 16 lanes lane 4 r + q names row r, columns
// 4 q .. + 3 of a block of 4 x 16, and lane c gets column c of the four rows.  Pairs of pieces are exchanged by k, so that the 16 rows that a
// wavefront reads at a time lie in all banks.  With A so, a lane's rows 4 (l >> 4) .. + 3 of C are neighbours in memory that is ordered by
// columns of C, which leaves as 8- or 16-byte pieces; with B so, column c of fragment j is 16 j + c.
template <typename V_, int PA_, int PB_, Order OA_, Order OB_, int BM_, int BN_, int BK_, int WM_, int WN_, int ST_, int WK_ = 1>
struct MfmaTile {
    using V = V_;
    using E = typename Mfma<V>::E;
    static constexpr int PA = PA_, PB = PB_, BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, ST = ST_, WK = WK_;
    static constexpr Order OA = OA_, OB = OB_;
    static constexpr int NW = WM * WN * WK, NT = NW * 64;
    static constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
    static constexpr int CPR = BK / 8, RPL = 64 / BK;                   // kRows: pieces to a row, rows to a line
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE = PA * A_BYTES + PB * B_BYTES;
    static constexpr int LA = A_BYTES / (NT * 16), LB = B_BYTES / (NT * 16), LOADS = PA * LA + PB * LB;
    static constexpr int LDS = ST * STAGE;
    static constexpr bool HALVES = BK == 64 && ST == 2 && PA == 1 && PB == 1 && WK == 1;
    static_assert(NI == 4 && (BK == 32 || BK == 64) && A_BYTES % (NT * 16) == 0 && B_BYTES % (NT * 16) == 0 && ST >= 2 && BK / 32 % WK == 0, "tile");
    static_assert(WK == 1 || (WK == 2 && LDS >= BM * BN * 4), "the second set of sums");

    __device__ static int key_a(int line) { return line & 7; }
    __device__ static int key_b(int line) { return (RPL == 1 ? line >> 2 : line >> 1) & 7; }
    // Lanes of a read of B are four rows apart: lines are exchanged in pairs so that neighbouring lanes' lie in both halves of the banks.
    __device__ static int swap_b(int line) { return line ^ ((RPL == 1 ? line >> 2 : line >> 1) & 1); }
    template <int WIDE>
    __device__ static int key_k(int k) { return ((k & 3) | (k >> 1 & 4)) << 1 & (WIDE / 8 - 1); }
    template <bool IS_B>
    __device__ static int place(int row, int c)
    {
        const int line = row / RPL, s = (row % RPL) * CPR + c;
        return (IS_B ? swap_b(line) : line) * 128 + ((s ^ (IS_B ? key_b(line) : key_a(line))) << 4);
    }
    // Row of B's wavefront tile that lane c of fragment j takes, and column of C there.
    __device__ static int col_at(int j, int c) { return OB == kCols ? j * 16 + c : c * 4 + j; }

    // This lane's offsets in bytes from the tile's first element.  Rows of the product past the operand's `rows` repeat its last one (kCols:
    // its last eight): the caller ignores them.  kCols: k past `left` repeats the last one; only one operand may be so, the other has zeros there.
    template <bool IS_B, int L>
    __device__ static void offsets(uint32_t (&o)[L], int wave, int lane, int64_t first, int64_t rows, int64_t ld, int64_t left)
    {
        constexpr int WIDE = IS_B ? BN : BM;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if constexpr ((IS_B ? OB : OA) == kRows) {
                const int at = (i * NW + wave) * 8 + (lane >> 3), line = IS_B ? swap_b(at) : at, s = (lane & 7) ^ (IS_B ? key_b(line) : key_a(line));
                int64_t r = line * RPL + s / CPR;
                r = first + r < rows ? r : rows - 1 - first;
                o[i] = static_cast<uint32_t>(r * ld + (s % CPR) * 8) * 2;
            } else {
                const int slot = (i * NW + wave) * 64 + lane, k = slot / (WIDE / 8);
                int64_t c = ((slot % (WIDE / 8)) ^ key_k<WIDE>(k)) * 8;
                c = first + c < rows ? c : rows - 8 - first;
                o[i] = static_cast<uint32_t>((k < left ? k : left - 1) * ld + c) * 2;
            }
        }
    }

    // kCols: element e of the fragment of 16 columns from `col`, of k 32 kk + 8 (lane >> 4) + e.
    template <int WIDE>
    __device__ static V columns(const char *base, int col, int kk, int lane)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const int k = kk * 32 + (lane >> 4) * 8 + (lane >> 2 & 3), c = (col >> 3) + (lane >> 1 & 1);
        const char *at = base + k * (WIDE * 2) + ((c ^ key_k<WIDE>(k)) << 4) + (lane & 1) * 8;
        using P = __attribute__((address_space(3))) s16x4 *;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 4 * WIDE * 2));
        return __builtin_bit_cast(V, static_cast<s16x8>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)));
    }

    __device__ static void clear(f32x4 (&acc)[MI][NI])
    {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    }

    // acc += rows m0.. of a (of M) times rows n0.. of b (of N), over k0 .. k0 + BK * steps.  kCols operands have `left` k from k0.
    __device__ static void run(const Planes &a, int64_t m0, int64_t M, const Planes &b, int64_t n0, int64_t N, int64_t k0, int steps, char *smem,
                               f32x4 (&acc)[MI][NI], int64_t left = INT64_MAX)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;
        const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)smem));
        uint32_t ao[LA], bo[LB];
        offsets<false>(ao, wave, lane, m0, M, a.ld, left);
        offsets<true>(bo, wave, lane, n0, N, b.ld, left);
        const char *ab = reinterpret_cast<const char *>(a.data + (OA == kRows ? m0 * a.ld + k0 : k0 * a.ld + m0));
        const char *bb = reinterpret_cast<const char *>(b.data + (OB == kRows ? n0 * b.ld + k0 : k0 * b.ld + n0));
        const int64_t as = (OA == kRows ? BK : BK * a.ld) * 2, bs = (OB == kRows ? BK : BK * b.ld) * 2;
        auto issue = [&](int kt, int st) {
            const uint32_t base = lds0 + st * STAGE + wave * 1024;
            if constexpr (OA == kCols || OB == kCols)
                if (kt > 0 && static_cast<int64_t>(kt + 1) * BK > left) {       // (never past the first step of a later share)
                    offsets<false>(ao, wave, lane, m0, M, a.ld, left - static_cast<int64_t>(kt) * BK);
                    offsets<true>(bo, wave, lane, n0, N, b.ld, left - static_cast<int64_t>(kt) * BK);
                }
            const char *pa = ab + kt * as, *pb = bb + kt * bs;
            asm("" : "+s"(pa));         // one address for the wavefront and the lanes' offsets
            asm("" : "+s"(pb));
#pragma unroll
            for (int p = 0; p < PA; ++p)
#pragma unroll
                for (int i = 0; i < LA; ++i) load_to_lds16(pa + p * a.plane * 2 + ao[i], base + p * A_BYTES + i * NW * 1024);
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int i = 0; i < LB; ++i) load_to_lds16(pb + p * b.plane * 2 + bo[i], base + PA * A_BYTES + p * B_BYTES + i * NW * 1024);
        };
        const int r16 = lane & 15, c4 = lane >> 4;
        auto read = [&](int st, int kk, V (&fa)[PA][MI], V (&fb)[PB][NI]) {
            const char *sa = smem + st * STAGE, *sb = sa + PA * A_BYTES;
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    if constexpr (OB == kRows) fb[p][j] = *reinterpret_cast<const V *>(sb + p * B_BYTES + place<true>(wn * TN + col_at(j, r16), kk * 4 + c4));
                    else fb[p][j] = columns<BN>(sb + p * B_BYTES, wn * TN + j * 16, kk, lane);
                }
#pragma unroll
            for (int p = 0; p < PA; ++p)
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    if constexpr (OA == kRows) fa[p][i] = *reinterpret_cast<const V *>(sa + p * A_BYTES + place<false>(wm * TM + i * 16 + r16, kk * 4 + c4));
                    else fa[p][i] = columns<BM>(sa + p * A_BYTES, wm * TM + i * 16, kk, lane);
                }
        };
        auto products = [&](const V (&fa)[PA][MI], const V (&fb)[PB][NI]) {
            constexpr int ORDERS = PA > PB ? PA : PB;
#pragma unroll
            for (int o = ORDERS - 1; o >= 0; --o)       // small products first; a sum's own products apart, for each waits for the one before
#pragma unroll
                for (int p = PA - 1; p >= 0; --p)
                    if (p <= o && o - p < PB)
#pragma unroll
                        for (int i = 0; i < MI; ++i)
#pragma unroll
                            for (int j = 0; j < NI; ++j) acc[i][j] = Mfma<V>::go(fa[p][i], fb[o - p][j], acc[i][j]);
        };
        if constexpr (HALVES) {
            // The halves of a step have registers of their own: while one half's products run the next one's operands are read, the last
            // half's from the next step's buffer.  Reads, loads and products are dealt out in turn, so that none waits for the others to
            // be issued.  4096^3 in bf16 beside the plain order: 1 256 - 1 311 against 1 053 - 1 157 TFLOP/s, the library's 1 311 - 1 508.
            constexpr int READS = (OA == kRows ? MI : 2 * MI) + (OB == kRows ? NI : 2 * NI), EACH = MI * NI / READS > 0 ? MI * NI / READS : 1;
            V fa[2][1][MI], fb[2][1][NI];
            issue(0, 0);
            if (steps > 1) issue(1, 1);
            if (steps > 1) wait_and_meet<LOADS>();
            else wait_and_meet<0>();
            read(0, 0, fa[0], fb[0]);
            int kt = 0;
            for (; kt + 2 < steps; ++kt) {
                read(kt & 1, 1, fa[1], fb[1]);
                products(fa[0], fb[0]);
#pragma unroll
                for (int q = 0; q < READS; ++q) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);          // an LDS read
                    __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0);         // products
                }
                // the next step's loads have landed, here and everywhere; this step's buffer is free
                wait_and_meet<0>();
                issue(kt + 2, kt & 1);
                read(kt + 1 & 1, 0, fa[0], fb[0]);
                products(fa[1], fb[1]);
#pragma unroll
                for (int q = 0; q < LOADS; ++q) {
                    __builtin_amdgcn_sched_group_barrier(0x20, 1, 1);           // a load
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 1);
                }
#pragma unroll
                for (int q = 0; q < READS; ++q) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
                    __builtin_amdgcn_sched_group_barrier(0x8, EACH, 1);
                }
            }
            for (; kt < steps; ++kt) {
                read(kt & 1, 1, fa[1], fb[1]);
                products(fa[0], fb[0]);
                if (kt + 1 < steps) {
                    wait_and_meet<0>();
                    read(kt + 1 & 1, 0, fa[0], fb[0]);
                }
                products(fa[1], fb[1]);
            }
        } else {
#pragma unroll
            for (int s = 0; s < ST - 1; ++s)
                if (s < steps) issue(s, s);
            for (int kt = 0, st = 0; kt < steps; ++kt) {
                // this step's loads have landed, here and (after the barrier) everywhere; the buffer read last is free again
                if (kt + ST - 1 <= steps) wait_and_meet<LOADS * (ST - 2)>();
                else wait_and_meet<0>();
                if (kt + ST - 1 < steps) issue(kt + ST - 1, st == 0 ? ST - 1 : st - 1);
#pragma unroll
                for (int kk = 0; kk < BK / 32; kk += WK) {
                    V fa[PA][MI], fb[PB][NI];
                    read(st, kk + wk, fa, fb);
                    products(fa, fb);
                }
                st = st == ST - 1 ? 0 : st + 1;
            }
        }
    }

    // Whether this wavefront is of the set that begins with what acc is to begin with, and holds the sums after join().
    __device__ static bool first_set() { return WK == 1 || threadIdx.x < WM * WN * 64; }

    // The two sets' sums into the first one's.
    __device__ static void join(f32x4 (&acc)[MI][NI], char *smem)
    {
        if constexpr (WK == 1) return;
        f32x4 *at = reinterpret_cast<f32x4 *>(smem) + threadIdx.x % (WM * WN * 64);
        lds_barrier();
        if (!first_set())
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) at[(i * NI + j) * (WM * WN * 64)] = acc[i][j];
        lds_barrier();
        if (first_set())
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] += at[(i * NI + j) * (WM * WN * 64)];
    }

    // acc[i][j][e] is row row_of(i) + e and column col_of(j) of the tile.
    __device__ static int row_of(int i) { return (threadIdx.x >> 6) / WN % WM * TM + i * 16 + ((threadIdx.x & 63) >> 4) * 4; }
    __device__ static int col_of(int j = 0) { return (threadIdx.x >> 6) % WN * TN + col_at(j, threadIdx.x & 15); }
};

// Four neighbouring elements, of which only each is aligned: memory takes them at once all the same.
template <typename O>
struct __attribute__((packed, aligned(sizeof(O)))) Four {
    O e[4];
};

// The first n (at most four) of v to p.
template <typename O>
__device__ __forceinline__ void store4(O *p, f32x4 v, int n)
{
    if (n >= 4) {
        struct __attribute__((packed, aligned(sizeof(O)))) Words { uint32_t w[sizeof(O)]; } q;
        if constexpr (sizeof(O) == 4) q.w[0] = __float_as_uint(v[0]), q.w[1] = __float_as_uint(v[1]), q.w[2] = __float_as_uint(v[2]), q.w[3] = __float_as_uint(v[3]);
        else q.w[0] = bits16<__bf16>(v[0]) | bits16<__bf16>(v[1]) << 16, q.w[1] = bits16<__bf16>(v[2]) | bits16<__bf16>(v[3]) << 16;
        *reinterpret_cast<Words *>(p) = q;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < n) p[k] = static_cast<O>(v[k]);
}

// Tile w of tm x tn in an order that keeps neighbouring ones close in both directions: bands of `band` rows of tiles, column by column.
__device__ __forceinline__ void tile_of(int w, int tm, int tn, int band, int &mt, int &nt)
{
    const int per = band * tn, b = w / per, first = b * band, height = min(tm - first, band), r = w - b * per;
    mt = first + r % height, nt = r / height;
}

}  // namespace dol

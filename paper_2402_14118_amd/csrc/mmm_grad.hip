// Gradients of the masked product under the maps as built (mmm_matmul_backward):
//     dX[i,k] = a_bits[i,k] ? sum over j of dC[i,j] B[k,j] : 0         B = N(Y), A = M(X)
//     dY[k,j] = b_bits[k,jb] ? sum over i of A[i,k] dC[i,j] : 0
// Both on matrix instructions, over all k, or in row-compacted mode over the live rows k' alone, whose number and places the maps hold.
// Zeros of A and blocks of B that are off are multiplied as zeros, and results that are not wanted are worked out and dropped: of a tile of random elements
// of A, or of 64 rows with random blocks, nearly all are wanted somewhere.
//
// One kernel for both: a workgroup owns a tile of `TR` x `TL` results and walks the contraction in steps of 128 bytes (64 elements of the 16-bit types, 32
// floats).  R is the operand along which a lane holds four neighbouring results, so that they are stored together; L the other.
//               R                          L
//     dX        rows of Y, k               rows of dC, i              contraction j, contiguous in both
//     dY        columns of dC, j           columns of A, k            contraction i
// A comes from the image that the builder made, masked, compacted and with 16 (floats: 4) rows of a column side by side, which is the
// order that an operand of dY wants.  dC is read row by row there, and turned by ds_read_b64_tr_b16 (floats: one by one) on the way out of LDS.
// Operands wait in registers while the step before is multiplied, and are laid into the other half of LDS between its last products: masks are applied on the
// way, one barrier per step (placed behind the products instead: 2048 x 16384 x 4096 bf16, both gradients, 612 us for 565).
// In LDS an operand row is 128 bytes, its eight 16-byte pieces turned with the row, so that eight rows' pieces lie in different banks; rows of dC in dY have their 32 (floats: 64) byte pieces turned.
//
// What bounds it.  Large results: the matrix cores at the clock that the power limit leaves (4096^3 half 1096 TFLOP/s for both, where a library product
// of 8192^3 bf16 reaches 1140; 2048 x 16384 x 4096 bf16 973; floats 135 of 155).  Small ones: the steps of a workgroup, one after another, and one to four
// launches.  Rows by context: writing the results, most of them zeros (2048 x 16384 x 4096 bf16, a tenth of the rows: 178 us, 335 MB of results).
// Operands of the smallest tile two steps ahead, in registers: no faster.
#include <algorithm>
#include <type_traits>

#include "mmm_internal.h"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// 16 bytes of a row, which starts at any element
template <int ESZ> struct AnyPiece { typedef u32x4 type __attribute__((aligned(2), may_alias)); };
template <> struct AnyPiece<4> { typedef u32x4 type __attribute__((aligned(4), may_alias)); };

constexpr int ROWB = 128;   // bytes of the contraction per step

struct GradParams {
    const void *Y, *dC;
    int64_t ldy, lddc;
    void *out;           // dX, of T, or dY, float
    int64_t ldo;
    const char *a_img;
    const uint64_t *a_bits, *b_bits;
    const uint32_t *kinfo, *kmap;   // row-compacted mode; else null
    const uint64_t *rows;           // bitmap of the live rows
    int64_t M, K, N, WA, WB;
    int32_t KBA, steps, bw_shift, accumulate;
    int32_t splits, steps_per_split;
    float *partials;     // splits > 1: [split][along L][along R, rows of whole quads]
    bool parts;          // the image is of floats in parts
    bool whole_rows;     // dX, row-compacted mode: tiles write the zeros between their results as well
};

// Four neighbouring results along R, from r on, of place l along L; `live`: the number of k there are.
template <typename T, bool TO_X> __device__ __forceinline__ void store_results(const GradParams &p, uint32_t l, uint32_t r, uint32_t live, const floatx4 &v)
{
    if constexpr (TO_X) {
        const uint64_t *const bits = p.a_bits != nullptr ? p.a_bits + (uint64_t)l * (uint64_t)p.WA : nullptr;   // null: all elements are wanted
        T *const row = static_cast<T *>(p.out) + (int64_t)l * p.ldo;
        if (p.kinfo == nullptr) {
            const uint32_t on = bits != nullptr ? (uint32_t)(bits[r >> 6] >> (r & 63u)) : 0xfu;
            typedef T vec __attribute__((ext_vector_type(4)));
            typedef vec vec_any __attribute__((aligned(sizeof(T)), may_alias));
            vec to;
#pragma unroll
            for (int u = 0; u < 4; ++u) to[u] = on >> u & 1u ? (T)v[u] : (T)0.f;
            if (r + 4 <= live) {
                *reinterpret_cast<vec_any *>(row + r) = to;
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (r + u < live) row[r + u] = to[u];
            }
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (r + u >= live) continue;
                const uint32_t k = p.kmap[r + u];
                row[k] = bits == nullptr || (bits[k >> 6] >> (k & 63u) & 1ull) ? (T)v[u] : (T)0.f;
            }
        }
    } else {
        const uint32_t k = p.kinfo != nullptr ? p.kmap[l] : l, jb = r >> p.bw_shift;
        const bool on = p.b_bits[(uint64_t)k * (uint64_t)p.WB + (jb >> 6)] >> (jb & 63u) & 1ull;
        typedef floatx4 vec_any __attribute__((aligned(4), may_alias));
        vec_any *const dst = reinterpret_cast<vec_any *>(static_cast<float *>(p.out) + (int64_t)k * p.ldo + r);
        if (p.accumulate) {
            if (on) *dst = *dst + v;
        } else {
            *dst = on ? v : floatx4{0, 0, 0, 0};
        }
    }
}

template <typename T> __device__ __forceinline__ void multiply(const u32x4 &r, const u32x4 &l, floatx4 &acc)
{
    if constexpr (std::is_same_v<T, float>) {
        const floatx4 a = __builtin_bit_cast(floatx4, r), b = __builtin_bit_cast(floatx4, l);
#pragma unroll
        for (int u = 0; u < 4; ++u) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u], b[u], acc, 0, 0, 0);
    } else if constexpr (std::is_same_v<T, _Float16>) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, r), __builtin_bit_cast(halfx8, l), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), __builtin_bit_cast(bf16x8, l), acc, 0, 0, 0);
    }
}

// dX in row-compacted mode, a tile whose contraction is not split: rows as they are in memory, from the first k of the tile to that of the next one, zeros of
// the k that are off among them, so that whole lines are written, and once.  Results go through LDS, with the 16-byte pieces of a row turned with it.
template <typename T, int WR, int WL, int FR, int FL>
__device__ __forceinline__ void spread_rows(const GradParams &p, const floatx4 (&acc)[FR][FL], uint32_t l0, uint32_t r0, uint32_t live, char (&lds)[2][256 * (FL * WL + FR * WR) * 8])
{
    constexpr int ESZ = (int)sizeof(T), TR = 16 * FR * WR, TL = 16 * FL * WL, NW = WR * WL, PER = 16 / ESZ;
    constexpr int CHUNK = 64 * PER, WORDS = CHUNK / 64;   // k of a wave's store, and words of the map
    constexpr int AHEAD = 4;                              // rows whose bits are asked for together
    static_assert(TL * TR * ESZ <= (int)sizeof(lds) && TL % (NW * AHEAD) == 0, "whole turns");
    typedef typename AnyPiece<ESZ>::type piece_any;
    typedef T four_t __attribute__((ext_vector_type(4)));
    typedef four_t four __attribute__((may_alias));
    typedef T element __attribute__((may_alias));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, s = lane >> 4, wr = wave % WR, wl = wave / WR;
    char *const room = lds[0];
    auto place_of = [](uint32_t row, uint32_t col) -> uint32_t { return row * (TR * ESZ) + (((col * ESZ >> 4) ^ (row & 7u)) << 4) + (col * ESZ & 15u); };
    const uint32_t lo = r0 == 0 ? 0u : p.kmap[r0], hi = r0 + TR < live ? p.kmap[r0 + TR] : (uint32_t)p.K;
    __syncthreads();   // operands have been read
#pragma unroll
    for (int b = 0; b < FL; ++b)
#pragma unroll
        for (int a = 0; a < FR; ++a) {
            four_t v;
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = (T)acc[a][b][u];
            *reinterpret_cast<four *>(room + place_of((uint32_t)((wl * FL + b) * 16 + c), (uint32_t)((wr * FR + a) * 16 + s * 4))) = v;
        }
    __syncthreads();
    uint32_t seen = 0;   // live k of the tile in front of the chunk
    for (uint32_t k0 = lo & ~63u; k0 < hi; k0 += CHUNK) {
        // this lane's piece, and which of its k are live; how many of the tile are in front of it
        const uint32_t k = k0 + (uint32_t)lane * PER, word = min(k, (uint32_t)p.K - 1u) >> 6;
        uint64_t on = p.rows[word];
        if (lo > word * 64u) on &= ~0ull << min(lo - word * 64u, 63u);                      // (a word begins at most 63 in front of lo)
        on = word * 64u >= hi || k >= (uint32_t)p.K ? 0ull : hi - word * 64u < 64u ? on & ((1ull << (hi - word * 64u)) - 1ull) : on;
        const uint32_t count = (uint32_t)__popcll(on);
        uint32_t before = seen + (uint32_t)__popcll(on & ((1ull << (k & 63u)) - 1ull));
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const uint32_t n = (uint32_t)__builtin_amdgcn_readlane((int)count, w * (64 / PER));
            before += w < lane / (64 / PER) ? n : 0u;
            seen += n;
        }
        const uint32_t mine = (uint32_t)(on >> (k & 63u)) & ((1u << PER) - 1u);
        const bool inside = k >= lo && k + PER <= hi;
        uint32_t at[PER];
#pragma unroll
        for (int q = 0; q < PER; ++q) at[q] = min(before + (uint32_t)__popc(mine & ((1u << q) - 1u)), (uint32_t)TR - 1u);
        for (uint32_t first = (uint32_t)wave * AHEAD; first < (uint32_t)TL; first += NW * AHEAD) {
            uint64_t bits[AHEAD];
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) {
                const uint32_t l = min(l0 + first + n, (uint32_t)p.M - 1u);
                bits[n] = p.a_bits != nullptr ? p.a_bits[(uint64_t)l * (uint64_t)p.WA + word] : ~0ull;
            }
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) {
                const uint32_t row = first + n, l = l0 + row;
                if (l >= (uint32_t)p.M) continue;
                const uint32_t wanted = (uint32_t)(bits[n] >> (k & 63u)) & mine;
                typedef T piece_t __attribute__((ext_vector_type(PER)));
                piece_t v;
#pragma unroll
                for (int q = 0; q < PER; ++q) {
                    const T x = *reinterpret_cast<const element *>(room + place_of(row, at[q]));
                    v[q] = wanted >> q & 1u ? x : (T)0.f;
                }
                T *const to = static_cast<T *>(p.out) + (int64_t)l * p.ldo + k;
                if (inside) {
                    *reinterpret_cast<piece_any *>(to) = __builtin_bit_cast(u32x4, v);
                } else {
#pragma unroll
                    for (int q = 0; q < PER; ++q)
                        if (k + q >= lo && k + q < hi) to[q] = v[q];
                }
            }
        }
    }
}

// One gradient: workgroup `group` of those that it has.  T: float, _Float16 or __bf16.  WR x WL waves, each FR x FL tiles of 16 x 16.
template <typename T, bool TO_X, int WR, int WL, int FR, int FL>
__device__ __forceinline__ void gradient(const GradParams &p, uint32_t group, char (&lds)[2][256 * (FL * WL + FR * WR) * 8])
{
    constexpr int ESZ = (int)sizeof(T), NT = 64 * WR * WL, TR = 16 * FR * WR, TL = 16 * FL * WL;
    constexpr int STEP = ROWB / ESZ, PER = 16 / ESZ;          // elements of the contraction per step, and of a piece
    constexpr int NL = TL * 8 / NT, NR = TR * 8 / NT;         // pieces of 16 bytes per thread and step
    constexpr int TURNED_ROW = TR * ESZ, PIECES = TR / PER;   // dY: a row of dC in LDS, bytes and pieces
    constexpr uint32_t TURN = TR / 16 < 8 ? TR / 16 - 1 : 7;  // and which of its sixteen columns take each other's place
    constexpr uint32_t OUTSIDE = 0x80000000u;                 // past the end of the buffers below, whatever else is added
    static_assert(NL * NT == TL * 8 && NR * NT == TR * 8, "whole pieces");
    static_assert(sizeof(lds) == 2 * (TL + TR) * ROWB, "two steps");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, s = lane >> 4, wr = wave % WR, wl = wave / WR;
    // Tiles there are: in row-compacted mode the live ones, which the device knows.  Dealt out so that an XCD's workgroups share rows of both operands in its
    // L2: a contiguous range of tiles, in panels of eight tiles along R.
    const uint32_t live = p.kinfo != nullptr ? *p.kinfo : (uint32_t)p.K;
    const uint32_t size_r = TO_X ? live : (uint32_t)p.N, size_l = TO_X ? (uint32_t)p.M : live;
    // (dX: one that writes zeros where no row is live)
    const uint32_t tiles_r = TO_X ? max(1u, (size_r + TR - 1) / TR) : (size_r + TR - 1) / TR, tiles_l = (size_l + TL - 1) / TL, tiles = tiles_r * tiles_l;
    const uint32_t all = tiles * (uint32_t)p.splits;
    if (group >= all) return;
    const uint32_t q8 = all >> 3, rem = all & 7u, x = group & 7u, id = x * q8 + min(x, rem) + (group >> 3);
    const uint32_t split = id / tiles, t = id - split * tiles;
    const uint32_t panel = t / (8 * tiles_l), width = min(8u, tiles_r - panel * 8), in_panel = t - panel * 8 * tiles_l;
    const uint32_t r0 = (panel * 8 + in_panel % width) * TR, l0 = in_panel / width * TL;

    // ---- operands on their way: 16-byte pieces of this thread
    u32x4 piece_l[NL], piece_r[NR];
    uint32_t block_bits[NR], block_bit = 0;   // dX: bytes of the map, and the bit that is this piece's
    const char *row_y[NR];         // dX: rows of Y, and the map's bytes of them
    const uint8_t *map_y[NR];
    uint32_t at_l[NL], at_r[NR];   // byte offsets: dX of rows of dC (L); dY of the image (L) and of rows of dC (R)
    const uint32_t dc_row = (uint32_t)p.lddc * ESZ;
    const uint32_t slab = p.parts ? MMM_BLOCK_PARTS_BYTES : (uint32_t)(MMM_AB_ROWS * MMM_AB_COLS * ESZ);
    const uint32_t row_l = (uint32_t)tid >> 3, c_l = (uint32_t)tid & 7u;   // pieces n of L are rows row_l + n * NT / 8, at c_l
#pragma unroll
    for (int n = 0; n < NL; ++n) {
        const uint32_t row = row_l + (uint32_t)n * (NT / 8);
        if constexpr (TO_X) {
            at_l[n] = l0 + row < (uint32_t)p.M ? row * dc_row : OUTSIDE;
        } else {
            const uint32_t k = l0 + row, kb = min(k / MMM_AB_COLS, (uint32_t)p.KBA - 1u), col = k % MMM_AB_COLS;
            at_l[n] = kb * slab;
            if (p.parts)   // four rows of each part, behind each other in a plane
                at_l[n] += col * MMM_PLANE_COL_BYTES + (c_l >> 2) * MMM_PLANE_BYTES + (c_l & 3u) * 8u;
            else if (ESZ == 4)
                at_l[n] += col * 256u + c_l * 16u;
            else
                at_l[n] += (c_l >> 1) * MMM_PLANE_BYTES + col * MMM_PLANE_COL_BYTES + (c_l & 1u) * 16u;
        }
    }
    if constexpr (TO_X) {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const uint32_t kc = r0 + row_l + (uint32_t)n * (NT / 8);
            const bool there = kc < live;
            const uint32_t k = !there ? 0u : p.kinfo != nullptr ? p.kmap[kc] : kc;
            row_y[n] = static_cast<const char *>(p.Y) + (uint64_t)k * (uint64_t)p.ldy * ESZ;
            map_y[n] = reinterpret_cast<const uint8_t *>(p.b_bits + (uint64_t)k * (uint64_t)p.WB);
            at_r[n] = there ? 0xffu : 0u;   // (of the map's byte)
        }
    } else {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const uint32_t q = (uint32_t)tid + (uint32_t)n * NT, rho = q / PIECES, col = q % PIECES * PER;
            // the row of a step that stands at place rho of it: floats as they are have rows r, r + 16, r + 32 and r + 48 side by side in the image
            const uint32_t row = ESZ == 4 && !p.parts ? (rho >> 2) + 16u * (rho & 3u) : rho;
            at_r[n] = r0 + col < (uint32_t)p.N ? row * dc_row + col * ESZ : OUTSIDE;
        }
    }

    typedef typename AnyPiece<ESZ>::type piece_any;
    auto fetch = [&](int step) __attribute__((always_inline)) {
        if constexpr (TO_X) {
            const uint32_t j = (uint32_t)step * STEP + c_l * PER, N = (uint32_t)p.N;
            const bool inside = j < N;
            const uint32_t rows = min((uint32_t)p.M - l0, (uint32_t)TL);
            const __amdgpu_buffer_rsrc_t dc = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<char *>(static_cast<const char *>(p.dC) + (uint64_t)l0 * dc_row), 0, (int)((rows - 1u) * dc_row + N * ESZ), 0x00020000);
#pragma unroll
            for (int n = 0; n < NL; ++n)
                piece_l[n] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(dc, (int)(inside ? at_l[n] + j * ESZ : OUTSIDE), 0, 0));
            const uint32_t jc = inside ? j : 0u, jb = jc >> p.bw_shift;   // (what exists is read, whether it counts or not)
            block_bit = inside ? 1u << (jb & 7u) : 0u;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                piece_r[n] = *reinterpret_cast<const piece_any *>(row_y[n] + jc * ESZ);
                block_bits[n] = (uint32_t)map_y[n][jb >> 3];
            }
        } else {
            // the block of rows, and which half of it (floats)
            const uint32_t block = ESZ == 4 ? (uint32_t)step >> 1 : (uint32_t)step, half = ESZ == 4 ? (uint32_t)step & 1u : 0u;
            const char *const img = p.a_img + (uint64_t)block * ((uint64_t)(uint32_t)p.KBA * slab) + half * (p.parts ? 2 * MMM_PLANE_BYTES : 128u);
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                if (ESZ == 4 && p.parts) {
                    u32x2 part[MMM_PARTS];
#pragma unroll
                    for (int q = 0; q < MMM_PARTS; ++q) part[q] = *reinterpret_cast<const u32x2 *>(img + at_l[n] + q * MMM_PART_BYTES);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        auto of = [&](int q) -> uint32_t { return part[q][u >> 1] >> (16 * (u & 1)) & 0xffffu; };
                        const uint32_t p0 = of(0), p1 = of(1), p2 = of(2);
                        const float sum = __uint_as_float(p0 << 16) + (__uint_as_float(p1 << 16) + __uint_as_float(p2 << 16));
                        piece_l[n][u] = p2 == MMM_PARTS_RAW ? p0 << 16 | p1 : __float_as_uint(sum);
                    }
                } else {
                    piece_l[n] = *reinterpret_cast<const u32x4 *>(img + at_l[n]);
                }
            }
            const uint32_t row0 = ESZ == 4 && !p.parts ? block * 64u + half * 8u : (uint32_t)step * STEP;
            const uint32_t left = (uint32_t)p.M > row0 ? (uint32_t)p.M - row0 : 0u;   // rows of dC from there on
            const uint32_t cols = ((uint32_t)p.N - r0) * ESZ;
            const __amdgpu_buffer_rsrc_t dc = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<char *>(static_cast<const char *>(p.dC) + (uint64_t)(left != 0u ? row0 : 0u) * dc_row + (uint64_t)r0 * ESZ), 0,
                left != 0u ? (int)((min(left, 64u) - 1u) * dc_row + cols) : 0, 0x00020000);
#pragma unroll
            for (int n = 0; n < NR; ++n) piece_r[n] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(dc, (int)at_r[n], 0, 0));
        }
    };
    // piece n of those of L, then R, to half `to` of LDS
    auto place = [&](int n, int to) __attribute__((always_inline)) {
        char *const at = lds[to];
        if (n < NL) {
            const uint32_t row = row_l + (uint32_t)n * (NT / 8);
            *reinterpret_cast<u32x4 *>(at + row * ROWB + ((c_l ^ (row & 7u)) << 4)) = piece_l[n < NL ? n : 0];
        } else if constexpr (TO_X) {
            const int m = n - NL;
            const uint32_t row = row_l + (uint32_t)m * (NT / 8);
            u32x4 v = piece_r[m];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = (block_bits[m] & at_r[m] & block_bit) != 0u ? v[u] : 0u;
            *reinterpret_cast<u32x4 *>(at + TL * ROWB + row * ROWB + ((c_l ^ (row & 7u)) << 4)) = v;
        } else {
            const int m = n - NL;
            const uint32_t q = (uint32_t)tid + (uint32_t)m * NT, rho = q / PIECES, col = q % PIECES;   // col: piece of the row
            const uint32_t turned = ESZ == 4 ? ((col >> 2) ^ (rho >> 2 & TURN)) << 2 | (col & 3u) : ((col >> 1) ^ (rho & TURN)) << 1 | (col & 1u);
            *reinterpret_cast<u32x4 *>(at + TL * ROWB + rho * TURNED_ROW + (turned << 4)) = piece_r[m];
        }
    };
    floatx4 acc[FR][FL];
#pragma unroll
    for (int a = 0; a < FR; ++a)
#pragma unroll
        for (int b = 0; b < FL; ++b) acc[a][b] = floatx4{0, 0, 0, 0};

    // The step in half `from`; with `more` the next one's operands go to the other half between its last products: a write of 16 bytes per lane takes as long as
    // a matrix instruction or two.
    auto compute = [&](int from, auto more) __attribute__((always_inline)) {
        const char *const at = lds[from];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 l[FL], r[FR];
#pragma unroll
            for (int b = 0; b < FL; ++b) {
                const uint32_t row = (uint32_t)((wl * FL + b) * 16 + c);
                l[b] = *reinterpret_cast<const u32x4 *>(at + row * ROWB + (((uint32_t)(kk * 4 + s) ^ (row & 7u)) << 4));
            }
#pragma unroll
            for (int a = 0; a < FR; ++a) {
                const uint32_t col0 = (uint32_t)((wr * FR + a) * 16);
                if constexpr (TO_X) {
                    const uint32_t row = col0 + (uint32_t)c;
                    r[a] = *reinterpret_cast<const u32x4 *>(at + TL * ROWB + row * ROWB + (((uint32_t)(kk * 4 + s) ^ (row & 7u)) << 4));
                } else if constexpr (ESZ == 4) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const uint32_t rho = (uint32_t)((kk * 4 + s) * 4 + u);
                        r[a][u] = *reinterpret_cast<const uint32_t *>(at + TL * ROWB + rho * TURNED_ROW + (((col0 >> 4) ^ (rho >> 2 & TURN)) << 6) + c * 4);
                    }
                } else {
                    // sixteen lanes read four rows of sixteen columns and get a column of four each
                    typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
                    u32x2 half[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t rho = (uint32_t)((kk * 4 + s) * 8 + h * 4 + (c >> 2));
                        const uint32_t where = TL * ROWB + rho * TURNED_ROW + (((col0 >> 4) ^ (rho & TURN)) << 5) + (uint32_t)(c & 3) * 8u;
                        half[h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)((lds_char *)lds[from] + where)));
                    }
                    r[a] = u32x4{half[0].x, half[0].y, half[1].x, half[1].y};
                }
            }
#pragma unroll
            for (int a = 0; a < FR; ++a) {
#pragma unroll
                for (int b = 0; b < FL; ++b) multiply<T>(r[a], l[b], acc[a][b]);
                if (decltype(more)::value && kk == 1)
#pragma unroll
                    for (int n = a * (NL + NR) / FR; n < (a + 1) * (NL + NR) / FR; ++n) place(n, from ^ 1);
            }
        }
    };
    const int first = (int)split * p.steps_per_split, end = min(first + p.steps_per_split, p.steps);   // (no part is empty)
    fetch(first);
#pragma unroll
    for (int n = 0; n < NL + NR; ++n) place(n, 0);
    int half = 0;
    for (int step = first + 1; step < end; ++step, half ^= 1) {
        fetch(step);
        __syncthreads();   // the step's operands are there; nobody reads the other half any more
        compute(half, std::true_type{});
    }
    __syncthreads();
    compute(half, std::false_type{});

    // ---- results: a lane holds four neighbours along R of sixteen along L
    if constexpr (TO_X && ESZ == 2)
        if (p.whole_rows) {
            spread_rows<T, WR, WL, FR, FL>(p, acc, l0, r0, live, lds);
            return;
        }
    const uint64_t pitch = (size_r + 3u) & ~3u;
    float *const partials = p.splits > 1 ? p.partials + (uint64_t)split * size_l * pitch : nullptr;
#pragma unroll
    for (int b = 0; b < FL; ++b) {
        const uint32_t l = l0 + (uint32_t)((wl * FL + b) * 16 + c);
        if (l >= size_l) continue;
#pragma unroll
        for (int a = 0; a < FR; ++a) {
            const uint32_t r = r0 + (uint32_t)((wr * FR + a) * 16 + s * 4);
            if (r >= size_r) continue;
            if (partials != nullptr)
                *reinterpret_cast<floatx4 *>(partials + l * pitch + r) = acc[a][b];
            else
                store_results<T, TO_X>(p, l, r, live, acc[a][b]);
        }
    }
}

// Row-compacted mode: zeros where no tile writes, the columns of dX and the rows of dY that are off.
struct ClearParams {
    char *dX, *dY;   // null: not asked for
    int64_t dx_pitch, M, dy_pitch, dy_bytes, K;
    const uint64_t *rows;
    uint32_t groups;
};
template <int ESZ> __device__ __forceinline__ void clear(const ClearParams &p, uint32_t group)
{
    typedef typename AnyPiece<ESZ>::type piece_any;
    typedef std::conditional_t<ESZ == 4, uint32_t, uint16_t> bits_t;
    typedef bits_t element __attribute__((may_alias));
    constexpr int PER = 16 / ESZ;
    const int64_t rows_x = p.dX != nullptr ? p.M : 0, rows_y = p.dY != nullptr ? p.K : 0;
    for (int64_t row = group; row < rows_x + rows_y; row += p.groups) {
        if (row < rows_x) {
            char *const out = p.dX + row * p.dx_pitch;
            for (int64_t k = (int64_t)threadIdx.x * PER; k < p.K; k += (int64_t)blockDim.x * PER) {
                const uint32_t live = (uint32_t)(p.rows[k >> 6] >> (k & 63)) & ((1u << PER) - 1u);
                if (live == 0 && k + PER <= p.K) {
                    *reinterpret_cast<piece_any *>(out + k * ESZ) = piece_any{0, 0, 0, 0};
                } else {
#pragma unroll
                    for (int q = 0; q < PER; ++q)
                        if (k + q < p.K && !(live >> q & 1u)) *reinterpret_cast<element *>(out + (k + q) * ESZ) = 0;
                }
            }
        } else {
            const int64_t k = row - rows_x;
            if (p.rows[k >> 6] >> (k & 63) & 1ull) continue;
            typedef AnyPiece<4>::type floats_any;
            for (int64_t at = (int64_t)threadIdx.x * 16; at < p.dy_bytes; at += (int64_t)blockDim.x * 16)   // (N is a multiple of 8)
                *reinterpret_cast<floats_any *>(p.dY + k * p.dy_pitch + at) = floats_any{0, 0, 0, 0};
        }
    }
}

// Everything in one launch: first the workgroups of the gradient with more steps for each (777 x 3001 x 1992 floats, a quarter of the rows, 66.8 us, the other way round
// 70.4), then those of the other, which fill up the last round of the first, then the zeros, which take no matrix instructions
// (2048 x 16384 x 4096 floats, a tenth of the rows: 522 us, with the zeros first 552, with a launch of their own 696).
struct GradWork {
    GradParams x, y;
    uint32_t groups_x, groups_y;   // of each, multiples of eight: an XCD gets every eighth workgroup of either
    bool y_first;
    ClearParams zeros;
};
template <typename T, int WR, int WL, int FR, int FL>
__global__ __launch_bounds__(64 * WR * WL, 2) void mmm_grad_kernel(const GradWork w)
{
    __shared__ __align__(16) char lds[2][256 * (FL * WL + FR * WR) * 8];
    const uint32_t front = w.y_first ? w.groups_y : w.groups_x, back = blockIdx.x - front;
    const bool in_front = blockIdx.x < front;
    if (!in_front && back >= w.groups_x + w.groups_y - front)
        clear<(int)sizeof(T)>(w.zeros, blockIdx.x - w.groups_x - w.groups_y);
    else if (in_front != w.y_first)
        gradient<T, true, WR, WL, FR, FL>(w.x, in_front ? blockIdx.x : back, lds);
    else
        gradient<T, false, WR, WL, FR, FL>(w.y, in_front ? blockIdx.x : back, lds);
}

// The sums of a split contraction, in the order of its parts.
template <typename T, bool TO_X> __device__ __forceinline__ void join(const GradParams &p)
{
    const uint32_t live = p.kinfo != nullptr ? *p.kinfo : (uint32_t)p.K;
    const uint32_t size_r = TO_X ? live : (uint32_t)p.N, size_l = TO_X ? (uint32_t)p.M : live;
    const uint64_t pitch = (size_r + 3u) & ~3u, total = (uint64_t)size_l * pitch;
    const uint32_t r = (blockIdx.x * 256u + threadIdx.x) * 4u;
    if (r >= size_r) return;
    for (uint32_t l = blockIdx.y; l < size_l; l += gridDim.y) {
        const float *const at = p.partials + l * pitch + r;
        floatx4 sum = *reinterpret_cast<const floatx4 *>(at);
        for (int32_t sp = 1; sp < p.splits; sp += 8) {
            floatx4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = sp + i < p.splits ? *reinterpret_cast<const floatx4 *>(at + (uint64_t)(sp + i) * total) : floatx4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        store_results<T, TO_X>(p, l, r, live, sum);
    }
}
template <typename T> __global__ __launch_bounds__(256) void mmm_grad_join_kernel(const GradParams x, const GradParams y)
{
    if (blockIdx.z == 0 && x.splits > 1)
        join<T, true>(x);
    else
        join<T, false>(y);
}

// Tile and split of the contraction.  The larger a tile, the fewer operands it takes from LDS per product (256 x 256: as many cycles of LDS as of
// matrix instructions; 64 x 64: four times as many); a smaller one leaves less of the machine and of its own edges idle.  Where there are few tiles the
// contraction is split and the parts are joined by a second launch.  The estimate is fitted to 36 shapes of each element type, three tiles and one to 32 parts
// (16 x 200 x 16384 to 2048 x 16384 x 4096, 2160 timings, off by 9 % of 16-bit and 5 % of float ones in the mean): its choice takes 3 and 2 % longer than the best.
// Multiplication alone, us, 64, 128, 256: 2048 x 16384 x 4096 bf16, dX 581, 322, 252; 512 x 2048 x 2048 16, 22, 31; floats 2394, 2126, 2034 and 49, 51, 60.
struct TileCost {
    int tile, at_once;            // workgroups that a compute unit runs side by side
    double fixed, alone, busy;    // microseconds: of the launch; of a step, of a workgroup by itself, and of each of many
};
constexpr TileCost kTiles16[] = {{64, 4, 7.5, 0.32, 0.245}, {128, 2, 9.5, 0.69, 0.60}, {256, 1, 13.6, 1.47, 1.47}};
constexpr TileCost kTilesFloat[] = {{64, 4, 7.6, 0.72, 0.59}, {128, 2, 9.9, 2.18, 2.18}, {256, 1, 14.3, 7.57, 7.57}};
constexpr double kJoin = 1.5, kJoinPerMB = 0.3;

constexpr int32_t kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};

// A gradient: its extent along R and L, the steps of its contraction, and the bytes of partial sums for each part of it.
struct GradJob {
    int64_t size_r, size_l, steps;
    size_t bytes;
    int64_t tiles(int64_t tile) const { return ((size_r + tile - 1) / tile) * ((size_l + tile - 1) / tile); }
    int64_t steps_of(int32_t want) const { return (steps + want - 1) / want; }
    int32_t parts_of(int32_t want) const { return (int32_t)((steps + steps_of(want) - 1) / steps_of(want)); }   // (no part is empty)
    double megabytes() const { return (double)size_r * (double)size_l * 4e-6; }
};
struct GradPlan { int tile; int32_t splits, steps_per_split; double us; };

// By itself.  row_bytes: from a row of dC to the next; a tile's rows lie within 2^31 bytes
GradPlan plan_one(const GradJob &j, bool floats, size_t room, int64_t row_bytes)
{
    GradPlan best{0, 0, 0, -1.0};
    for (const TileCost &c : floats ? kTilesFloat : kTiles16) {
        if (c.tile > 128 && c.tile * row_bytes >= 0x80000000LL) continue;
        for (int32_t want : kParts) {
            if (want > 1 && ((size_t)want * j.bytes > room || j.steps < want)) break;
            const int64_t per = j.steps_of(want), splits = j.parts_of(want), groups = j.tiles(c.tile) * splits, round = 256 * c.at_once, left = groups % round;
            const double rounds = (double)(groups / round) * std::max(c.alone, c.busy * c.at_once) +
                                  (left != 0 ? std::max(c.alone, c.busy * (double)((left + 255) / 256)) : 0.0);
            const double us = c.fixed + (double)per * rounds + (splits > 1 ? kJoin + (double)splits * j.megabytes() * kJoinPerMB : 0.0);
            if (best.us < 0.0 || us < best.us) best = {c.tile, (int32_t)splits, (int32_t)per, us};
        }
    }
    return best;
}

// Both in one launch, with the smallest tile: the workgroups of one fill what those of the other leave idle, and a launch (and a join) is saved.  Estimate: the steps of
// all workgroups spread over the machine, and a share of the longest chain; fitted to 19 shapes of each element type and 36 pairs of parts (16 x 200 x 16384 to 512 x 8192 x
// 4096, off by 11 and 6 %).  Taken where it promises less than two launches: 17 (16-bit) and 10 % (floats) less time than these over the shapes, up to 39 % less; not where
// there is work for larger tiles (512 x 8192 x 4096 bf16: 117 us in two, 131 in one) or little more than writing dY (16 x 4096 x 4096: 33 and 37).
struct BothCost { double fixed, step, longest, join, join_per_mb, write_per_mb; };
constexpr BothCost kBoth16{5.05, 0.139, 0.228, 2.23, 0.33, 0.39}, kBothFloat{5.9, 0.48, 0.42, 2.1, 0.27, 0.29};

bool plan_both(const GradJob &x, const GradJob &y, bool floats, size_t room, GradPlan &plan_x, GradPlan &plan_y)
{
    constexpr int TILE = 64;
    const BothCost &c = floats ? kBothFloat : kBoth16;
    double least = plan_x.us + plan_y.us;
    bool together = false;
    for (int32_t want_x : kParts)
        for (int32_t want_y : kParts) {
            if (x.steps < want_x || y.steps < want_y) break;
            const int64_t per_x = x.steps_of(want_x), per_y = y.steps_of(want_y);
            const int32_t splits_x = x.parts_of(want_x), splits_y = y.parts_of(want_y);
            const double of_x = splits_x > 1 ? splits_x : 0, of_y = splits_y > 1 ? splits_y : 0;   // parts that are joined
            if ((size_t)of_x * x.bytes + (size_t)of_y * y.bytes > room) break;
            const double work = (double)(x.tiles(TILE) * splits_x * per_x + y.tiles(TILE) * splits_y * per_y) / 256.0;
            const double us = c.fixed + c.step * work + c.longest * (double)std::max(per_x, per_y) + c.write_per_mb * (x.megabytes() + y.megabytes()) +
                              (of_x + of_y > 0 ? c.join + c.join_per_mb * (of_x * x.megabytes() + of_y * y.megabytes()) : 0.0);
            if (us >= least) continue;
            least = us;
            together = true;
            plan_x = {TILE, splits_x, (int32_t)per_x, us};
            plan_y = {TILE, splits_y, (int32_t)per_y, us};
        }
    return together;
}

// Those gradients that are planned, of one tile.
template <typename T> hipError_t launch(const mmm_maps *m, GradWork w, const GradPlan *x, const GradPlan *y, size_t bytes_x, hipStream_t s)
{
    const int tile = x != nullptr ? x->tile : y->tile;
    auto groups_of = [&](GradParams &p, const GradPlan &plan, int64_t r, int64_t l) -> int64_t {
        p.splits = plan.splits;
        p.steps_per_split = plan.steps_per_split;
        p.partials = m->partials;
        return ((r + tile - 1) / tile) * ((l + tile - 1) / tile) * plan.splits;
    };
    w.x.splits = w.y.splits = 1;
    const int64_t groups_x = x != nullptr ? (groups_of(w.x, *x, m->K, m->M) + 7) & ~7LL : 0, groups_y = y != nullptr ? (groups_of(w.y, *y, m->N, m->K) + 7) & ~7LL : 0;
    if (w.x.splits > 1) w.y.partials += (size_t)w.x.splits * bytes_x / sizeof(float);
    const int64_t groups = groups_x + groups_y + w.zeros.groups;
    if (groups > (1LL << 32) / 512 - 1) return hipErrorInvalidValue;   // threads of a launch
    w.groups_x = (uint32_t)groups_x;
    w.groups_y = (uint32_t)groups_y;
    w.y_first = x != nullptr && y != nullptr && y->steps_per_split > x->steps_per_split;
    void (*fn)(const GradWork) = tile == 256 ? mmm_grad_kernel<T, 2, 4, 8, 4> : tile == 128 ? mmm_grad_kernel<T, 2, 2, 4, 4> : mmm_grad_kernel<T, 2, 2, 2, 2>;
    hipLaunchKernelGGL(fn, dim3((uint32_t)groups), dim3(tile == 256 ? 512 : 256), 0, s, w);
    if (w.x.splits > 1 || w.y.splits > 1) {
        const int64_t r = std::max(w.x.splits > 1 ? m->K : 0, w.y.splits > 1 ? m->N : 0), l = std::max(w.x.splits > 1 ? m->M : 0, w.y.splits > 1 ? m->K : 0);
        const dim3 grid((uint32_t)((r + 1023) / 1024), (uint32_t)std::min<int64_t>(l, 65535), w.x.splits > 1 && w.y.splits > 1 ? 2 : 1);
        hipLaunchKernelGGL(mmm_grad_join_kernel<T>, grid, dim3(256), 0, s, w.x, w.y);
    }
    return hipGetLastError();
}

template <typename T> hipError_t launch_wanted(const mmm_maps *m, GradWork w, bool x, bool y, hipStream_t s)
{
    // row-compacted mode: as many k as the most recent count has found (a guess: the kernels go by the number the device has)
    const int64_t live = m->b_compact && m->stats_b_valid ? std::max<int64_t>(1, std::min<int64_t>(m->K, (int64_t)m->stats_rows_b)) : m->K;
    const auto quads = [](int64_t r) { return (size_t)((r + 3) & ~3LL); };
    const GradJob job_x{live, m->M, w.x.steps, quads(m->K) * (size_t)m->M * sizeof(float)}, job_y{m->N, live, w.y.steps, quads(m->N) * (size_t)m->K * sizeof(float)};
    const bool floats = sizeof(T) == 4;
    GradPlan plan_x = plan_one(job_x, floats, m->partial_bytes, w.x.lddc * (int64_t)sizeof(T)), plan_y = plan_one(job_y, floats, m->partial_bytes, w.x.lddc * (int64_t)sizeof(T));
    // (planned for both also where one is asked for: its sums are then the same)
    const bool together = plan_both(job_x, job_y, floats, m->partial_bytes, plan_x, plan_y);
    // Rows of dX written whole by the tiles, zeros and all: 16-bit types, where the tiles fill the machine and hold one k in sixteen at least.  Both gradients, us, against
    // results and zeros by themselves: 2048 x 16384 x 4096 bf16, a fiftieth of the rows 151 and 114, a tenth 177 and 214, nine tenths 549 and 638; 130 x 5000 x 328 half,
    // a fifth, 48 tiles, 15.4 and 12.4.  (Floats, whose products leave time for the zeros: a tenth 498 and 523, but 4096 x 2048 x 512 54 and 45.)
    w.x.whole_rows = m->b_compact && !floats && plan_x.splits == 1 && job_x.tiles(plan_x.tile) >= 256 && live * 16 >= m->K;
    if (w.x.whole_rows) w.zeros.dX = nullptr;
    w.zeros.groups = (uint32_t)std::min<int64_t>((w.zeros.dX != nullptr ? m->M : 0) + (w.zeros.dY != nullptr ? m->K : 0), 1024);
    if (together || !x || !y) return launch<T>(m, w, x ? &plan_x : nullptr, y ? &plan_y : nullptr, job_x.bytes, s);
    if (const hipError_t e = launch<T>(m, w, &plan_x, nullptr, job_x.bytes, s); e != hipSuccess) return e;
    w.zeros = {};   // (are written)
    return launch<T>(m, w, nullptr, &plan_y, job_x.bytes, s);
}

}   // namespace

hipError_t mmm_launch_grad(const mmm_maps *m, int32_t dtype, const void *Y, int64_t ldy, const void *dC, int64_t lddc, void *dX, int64_t lddx, float *dY,
                           int64_t lddy, int32_t accumulate, int32_t all_x, hipStream_t s)
{
    GradParams p{};
    p.Y = Y;
    p.ldy = ldy;
    p.dC = dC;
    p.lddc = lddc;
    p.a_img = m->a_img;
    p.a_bits = all_x ? nullptr : m->a_bits;
    p.b_bits = m->b_bits;
    p.kinfo = m->b_compact ? m->kinfo : nullptr;
    p.kmap = m->kmap;
    p.rows = m->rows_copy;
    p.M = m->M;
    p.K = m->K;
    p.N = m->N;
    p.WA = m->WA;
    p.WB = m->WB;
    p.KBA = (int32_t)m->KBA;
    p.bw_shift = m->bw == 8 ? 3 : m->bw == 16 ? 4 : 5;
    p.accumulate = accumulate;
    p.parts = m->a_form == MMM_FORM_PARTS;
    const int64_t esz = dtype == MMM_F32 ? 4 : 2;
    GradWork w{p, p, 0, 0, false, {}};
    w.x.out = dX;
    w.x.ldo = lddx;
    w.x.steps = (int32_t)((m->N * esz + ROWB - 1) / ROWB);
    w.y.out = dY;
    w.y.ldo = lddy;
    w.y.steps = (int32_t)(m->MBA * (dtype == MMM_F32 ? 2 : 1));
    // (of dX where its contraction is split: otherwise its tiles write them)
    if (m->b_compact)
        w.zeros = {static_cast<char *>(dX), accumulate ? nullptr : reinterpret_cast<char *>(dY), lddx * esz, m->M, lddy * 4, m->N * 4, m->K, m->rows_copy, 0};
    (void)hipGetLastError();
    const bool x = dX != nullptr, y = dY != nullptr;
    return dtype == MMM_F32 ? launch_wanted<float>(m, w, x, y, s) : dtype == MMM_BF16 ? launch_wanted<__bf16>(m, w, x, y, s) : launch_wanted<_Float16>(m, w, x, y, s);
}

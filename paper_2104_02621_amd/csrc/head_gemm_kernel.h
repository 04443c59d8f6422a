// Internal: the matrix products of a linear head over many classes (included by the files of its tiles), on the bf16 and fp16 matrix instructions:
//
//     out[m][n] = sum over k of a[m][k] * b[n][k]
//
// with the contracted index innermost in both operands.  fp32 operands lie in memory as three bf16 terms each (see
// bf16_split.h); the six products of terms that count are the same loop run six times, smallest products first.
//
// A workgroup of four waves owns a tile of out (256 x 256: 128 x 128 a wave).  A stage is 32 contracted values; LDS holds a
// ring of four stages, filled by copies that pass no registers.  Per stage a wave issues two steps of 16 matrix
// instructions (32x32x16); between them go, one at a time, the LDS reads of the next step's operands and the copies of
// the stage four ahead.  One barrier a stage, before its second step, whose operands are in registers by then.
//
// LDS stage: rows of 64 bytes, four 16-byte chunks, chunk c of row r in place c ^ (r / 4 % 4): the 16 lanes that read one
// chunk of 16 rows touch 16 different 16-byte columns of the banks.  Operands in blocks lie so in memory; of one that is
// rows, four neighbouring lanes of a copy bring a row's 64 bytes.  The n side is the matrix instruction's row operand, so that a lane ends up with runs of four
// neighbouring n of one m.
//
// Bound on large products: the matrix pipes, at the clock that the power limit leaves.  6144 x 131072 x 4096 in bf16 with the
// statistics as its end takes 4.9 ms (1340 TFLOP/s; a library's product of 8192 x 16384 x 4096 runs at 1310 on the same card), and
// 8192 x 65536 x 2048 with the gradients, whose 2 GB of 16-bit values nothing overlaps, 2.2 ms (1000 TFLOP/s).  One row against 50000 of
// 4096 values, on tiles of 64 x 128, takes 84 us, 4.9 TB/s of weights.
#pragma once
#include "head_gemm.h"

#include "bf16_split.h"
#include "conv_shape.h"
#include "igemm_common.h"
#include "lds_dma.h"
#include "row_vectors.h"

namespace capscaps {
namespace {

constexpr int OUT_OF_RANGE = (int)0x80000000u;

__device__ __forceinline__ unsigned half_pair(float lo, float hi)
{
    const float2v v = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, half2v));
}

// A row's part of 32 n values, for lanes of both halves: after it a lane holds eight neighbouring ones, those of
// lane half h beginning at 8 (2 pair + h).  v: packed pairs of 8g + 4h + 0..3 in v[2g], v[2g + 1].
__device__ __forceinline__ chunk_t neighbours(const unsigned* v, int pair)
{
    // (the upper half's register of run 2 pair goes to the lower half, the lower half's of run 2 pair + 1 to the upper)
    const auto a = __builtin_amdgcn_permlane32_swap(v[4 * pair], v[4 * pair + 2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(v[4 * pair + 1], v[4 * pair + 3], false, false);
    return {a[0], b[0], a[1], b[1]};
}

// Four lanes hold four n values each (two packed words), of neighbouring m; after it lane j of the four holds the
// four m values of n value j.
__device__ __forceinline__ void turn(unsigned& lo, unsigned& hi, int lane)
{
    auto moved = [](unsigned v, auto CTRL) {
        return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, decltype(CTRL)::value, 0xf, 0xf, true);
    };
    typedef std::integral_constant<int, 0xB1> One;  // quad_perm 1 0 3 2
    typedef std::integral_constant<int, 0x4E> Two;  // quad_perm 2 3 0 1
    const unsigned pick = lane & 1 ? 0x03020706u : 0x05040100u;
    const unsigned a = __builtin_amdgcn_perm(moved(lo, One()), lo, pick), b = __builtin_amdgcn_perm(moved(hi, One()), hi, pick);
    const bool late = lane & 2;
    const unsigned got = moved(late ? a : b, Two());
    lo = late ? got : a;
    hi = late ? b : got;
}

// NB: stages of the ring
template <typename Tag, int BM, int BN, int NWM, int NB, int TERMS, bool ROWS, int END>
__device__ __forceinline__ void head_gemm(const HeadGemm& G, int tiles_n, int block)
{
    constexpr int NWN = 4 / NWM, WM = BM / NWM, WN = BN / NWN, TM = WM / 32, TN = WN / 32;
    constexpr int A_BYTES = BM * 64, STAGE = (BM + BN) * 64;
    constexpr int CA = BM / 64, CB = BN / 64;  // copies of a wave and stage
    constexpr int NMMA = TM * TN, NFRAG = TM + TN;
    constexpr int KEEP = (NB - 2) * (CA + CB);
    static_assert(KEEP + CA < 64, "vmcnt is a 6-bit counter");
    static_assert(CA >= 1 && CB >= 1, "copies of every wave");
    extern __shared__ char smem[];

    // Tiles: an XCD (workgroups go to the eight in turn) takes a run of them, bands of eight rows of tiles, so that the 32
    // tiles its CUs work on at a time share operands in its L2.
    long long m_end = G.m_rows;
    if (G.m_count != nullptr) {
        const long long c = __builtin_amdgcn_readfirstlane(*G.m_count);
        m_end = c < m_end ? c : m_end;
    }
    // (of the rows that count: the others' workgroups end here, and leave no XCD without work)
    const int tiles_m = (int)((m_end + BM - 1) / BM), tiles = tiles_m * tiles_n, all = tiles * G.splits;
    if (block >= all) return;
    const int span = all & ~7;
    const int id = block < span ? (block & 7) * (span >> 3) + (block >> 3) : block;
    const int part = id / tiles, L = id - part * tiles;
    const int band = L / (8 * tiles_n), in_band = L - band * 8 * tiles_n;
    const int high = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
    const long long m0 = (long long)(band * 8 + in_band % high) * BM;
    const long long n0 = (long long)(in_band / high) * BN;
    // stages of this part
    long long k = G.k;
    if (G.k_count != nullptr) {
        const long long c = __builtin_amdgcn_readfirstlane(*G.k_count);
        k = c < k ? c : k;
    }
    const int all_stages = (int)((k + HEAD_K - 1) / HEAD_K);
    const int per = __builtin_amdgcn_readfirstlane((all_stages + G.splits - 1) / G.splits);
    const int first = __builtin_amdgcn_readfirstlane(part * per < all_stages ? part * per : all_stages);
    const int run = __builtin_amdgcn_readfirstlane(all_stages - first < per ? all_stages - first : per);  // of each product of terms
    constexpr int PRODUCTS = TERMS == 3 ? SPLIT_PRODUCTS : TERMS;
    const int stages = __builtin_amdgcn_readfirstlane(run * PRODUCTS);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % NWM, wn = wave / NWM;
    const int h = lane >> 5, lr = lane & 31;

    auto blocks_of = [](const void* base, long long stages, long long first_row, long long rows) {
        const long long bytes = ((rows + 15) / 16 - first_row / 16) * stages * 1024;
        return make_rsrc(static_cast<const char*>(base) + first_row / 16 * stages * 1024,
                         (unsigned)(bytes < 0x7fffffffll ? bytes : 0x7fffffffll));
    };
    const rsrc_t rs_a = blocks_of(G.a, G.stages_a, m0, m_end);
    rsrc_t rs_b;
    if constexpr (ROWS) {
        // (up to the last row's last value: rows may lie closer than they are long, or all in one place)
        const long long bytes = (G.n_rows - n0 - 1) * G.ldb + G.k * 2;
        rs_b = make_rsrc(static_cast<const char*>(G.b) + n0 * G.ldb, (unsigned)(bytes < 0x7fffffffll ? bytes : 0x7fffffffll));
    } else {
        rs_b = blocks_of(G.b, G.stages_b, n0, G.n_rows);
    }
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)smem;
    const unsigned lds_a = __builtin_amdgcn_readfirstlane((int)(lds0 + wave * CA * 1024));
    const unsigned lds_b = __builtin_amdgcn_readfirstlane((int)(lds0 + A_BYTES + wave * CB * 1024));
    // a copy is a block: 16 rows
    const int row_step_a = __builtin_amdgcn_readfirstlane((int)(G.stages_a * 1024));
    const int row_step_b = __builtin_amdgcn_readfirstlane((int)(ROWS ? 16 * G.ldb : G.stages_b * 1024));
    constexpr int step_b = ROWS ? 64 : 1024;  // bytes from stage to stage
    const unsigned a_voff = lane * 16;
    const unsigned b_voff = ROWS ? (lane >> 2) * (row_step_b >> 4) + ((lane & 3) ^ (lane >> 4)) * 16 : lane * 16;
    int a_row[CA], b_row[CB];
#pragma unroll
    for (int j = 0; j < CA; ++j) a_row[j] = __builtin_amdgcn_readfirstlane((wave * CA + j) * row_step_a);
#pragma unroll
    for (int j = 0; j < CB; ++j) b_row[j] = __builtin_amdgcn_readfirstlane((wave * CB + j) * row_step_b);

    // the stage whose copies go out next: byte offsets from a row's beginning (out of range past the last stage)
    int next = 0, product = 0, left = run;
    int a_off = stages > 0 ? first * 1024 : OUT_OF_RANGE, b_off = stages > 0 ? first * step_b : OUT_OF_RANGE;
    // terms of the products, two bits each, smallest products first
    constexpr int ta = TERMS == 3 ? SPLIT_TERM_A[0] | SPLIT_TERM_A[1] << 2 | SPLIT_TERM_A[2] << 4 | SPLIT_TERM_A[3] << 6 |
                                        SPLIT_TERM_A[4] << 8 | SPLIT_TERM_A[5] << 10
                                  : 1;
    constexpr int tb = TERMS == 3 ? SPLIT_TERM_B[0] | SPLIT_TERM_B[1] << 2 | SPLIT_TERM_B[2] << 4 | SPLIT_TERM_B[3] << 6 |
                                        SPLIT_TERM_B[4] << 8 | SPLIT_TERM_B[5] << 10
                                  : 0;
    if (TERMS > 1 && stages > 0) {
        a_off += (ta & 3) * G.plane_a * 1024;
        b_off += (tb & 3) * G.plane_b * 1024;
    }
    auto advance = [&]() {
        // (the empty statements hold the scalar arithmetic in the gap it is written in; where it drifts, the one wave of a SIMD
        // leaves the matrix pipe without work: 8192 x 2048 x 32768 in 1256 instead of 756 us on tiles of 256 x 256)
        if constexpr (TERMS == 1) asm volatile("" : "+s"(next), "+s"(a_off), "+s"(b_off));
        ++next;
        a_off += 1024;
        b_off += step_b;
        if constexpr (TERMS > 1) {
            const bool wrap = --left == 0;
            product += wrap ? 1 : 0;
            left = wrap ? run : left;
            const int at_a = (first + (ta >> 2 * product & 3) * G.plane_a) * 1024;
            const int at_b = (first + (tb >> 2 * product & 3) * G.plane_b) * 1024;
            a_off = wrap ? at_a : a_off;
            b_off = wrap ? at_b : b_off;
        }
        a_off = next < stages ? a_off : OUT_OF_RANGE;
        b_off = next < stages ? b_off : OUT_OF_RANGE;
        if constexpr (TERMS == 1) asm volatile("" : "+s"(next), "+s"(a_off), "+s"(b_off));
    };
    auto copy_a = [&](auto SLOT, auto J) {
        constexpr int slot = decltype(SLOT)::value, j = decltype(J)::value;
        copy_to_lds_16B<slot * STAGE + j * 1024>(rs_a, lds_a, a_voff, a_off, a_row[j]);
    };
    auto copy_b = [&](auto SLOT, auto J) {
        constexpr int slot = decltype(SLOT)::value, j = decltype(J)::value;
        copy_to_lds_16B<slot * STAGE + j * 1024>(rs_b, lds_b, b_voff, b_off, b_row[j]);
    };

    // operand reads: chunk 2t + h of row lr of a 32-row tile, in place (2t + h) ^ (lr / 4 % 4)
    const int place = h ^ ((lr >> 2) & 3);
    const char* const a_rd[2] = {smem + (wm * WM + lr) * 64 + place * 16, smem + (wm * WM + lr) * 64 + (place ^ 2) * 16};
    const char* const b_rd[2] = {smem + A_BYTES + (wn * WN + lr) * 64 + place * 16,
                                 smem + A_BYTES + (wn * WN + lr) * 64 + (place ^ 2) * 16};
    auto read_frag = [&](int slot, int t, int f) -> chunk_t {
        const char* p = f < TN ? b_rd[t] + slot * STAGE + f * 2048 : a_rd[t] + slot * STAGE + (f - TN) * 2048;
        return *reinterpret_cast<const chunk_t*>(p);
    };

    float16v acc[TN][TM];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;

    // stages 0 .. NB-2 whole, the m side of stage NB-1
    static_for<NB - 1>([&](auto S) {
        static_for<CA>([&](auto J) { copy_a(S, J); });
        static_for<CB>([&](auto J) { copy_b(S, J); });
        advance();
    });
    static_for<CA>([&](auto J) { copy_a(std::integral_constant<int, NB - 1>{}, J); });
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b) asm volatile("" : "+a"(acc[a][b]));
    {
        constexpr int keep0 = KEEP + CA;
        __builtin_amdgcn_s_waitcnt(0x0F70 | (keep0 & 15) | ((keep0 >> 4) << 14));
    }
    __syncthreads();
    chunk_t frag[2][NFRAG];
#pragma unroll
    for (int f = 0; f < NFRAG; ++f) frag[0][f] = read_frag(0, 0, f);

    auto mma = [&](const chunk_t& ka, const chunk_t& ib, float16v& c) {
        if constexpr (NMMA < 16) asm volatile("" : "+a"(c));
        Mma<Tag>::run(ka, ib, c);
        if constexpr (NMMA < 16) asm volatile("" : "+a"(c));
    };
    // reads before gap i of a step's gaps, one (two) in each of the first; copies, spread over all
    constexpr int per_gap = (NFRAG + NMMA - 1) / NMMA;
    constexpr auto reads_before = [](int i) { return i * per_gap < NFRAG ? i * per_gap : NFRAG; };
    constexpr auto copies_before = [](int i, int count) { return (i * count + NMMA / 2 - 1) / NMMA; };
    for (int st = 0; st < stages; st += NB) {
        static_for<NB>([&](auto SLOT) {
            constexpr int slot = decltype(SLOT)::value;
            constexpr int slot_next = (slot + 1) % NB;
            typedef std::integral_constant<int, (slot + NB - 1) % NB> SlotPrev;
            static_for<NMMA>([&](auto I) {
                constexpr int i = decltype(I)::value;
                mma(frag[0][i / TM], frag[0][TN + i % TM], acc[i / TM][i % TM]);
                static_for<NFRAG>([&](auto F) {
                    constexpr int f = decltype(F)::value;
                    if constexpr (f >= reads_before(i) && f < reads_before(i + 1)) frag[1][f] = read_frag(slot, 1, f);
                });
                static_for<CB>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    if constexpr (j >= copies_before(i, CB) && j < copies_before(i + 1, CB)) copy_b(SlotPrev{}, J);
                });
                if constexpr (i == NMMA - 1) advance();
                __builtin_amdgcn_sched_barrier(0);
            });
            // what this wave still needs of `slot` is in registers and its copies of the next stage have landed; after the
            // barrier that holds for all waves
            __builtin_amdgcn_s_waitcnt((0x0F70 | (KEEP & 15) | ((KEEP >> 4) << 14)) & 0xF0FF);
            __syncthreads();
            static_for<NMMA>([&](auto I) {
                constexpr int i = decltype(I)::value;
                mma(frag[1][i / TM], frag[1][TN + i % TM], acc[i / TM][i % TM]);
                static_for<NFRAG>([&](auto F) {
                    constexpr int f = decltype(F)::value;
                    if constexpr (f >= reads_before(i) && f < reads_before(i + 1))
                        frag[0][f] = read_frag(slot_next, 0, f);
                });
                static_for<CA>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    if constexpr (j >= copies_before(i, CA) && j < copies_before(i + 1, CA)) copy_a(SLOT, J);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    }
    // the copies of the surplus stages still write (zeros) into this workgroup's LDS
    __builtin_amdgcn_s_waitcnt(0x0F70);

    // lane (h, lr) of tile (a, b) holds in registers 4g .. 4g+3 the n values 8g + 4h + 0..3 of row lr
    const int n_left = (int)(G.n_rows - n0 < BN ? G.n_rows - n0 : BN) - wn * WN;  // columns of this wave's that exist
    if constexpr (END == HEAD_OUT) {
        const float scale = G.scale != nullptr ? *G.scale : 1.0f;
        const bool vectors = (G.ldo & 3) == 0;
        if (G.whole_vectors && n_left >= WN) {
            // All columns exist: 16 bytes a lane, two lanes side by side, at 32-bit offsets from the wave's first value; rows past
            // the last are dropped by the range check.  (Column by column with 64-bit addresses, below, a tile of 256 x 256 takes 25 us to
            // end.)
            // (The offsets within a row go into the instructions, not into a scalar register: after a 16-byte store with a scalar
            // offset the compiler lets the next instruction overwrite the stored registers, and some lanes then store the new value.)
            const int size = G.out_dtype == CAPSCAPS_FP32 ? 4 : 2;
            const long long first_row = m0 + wm * WM;
            const long long rows = m_end - first_row < WM ? m_end - first_row : WM;
            if (rows <= 0) return;
            const rsrc_t raw = make_rsrc(static_cast<char*>(G.out) + (first_row * G.ldo + part * G.out_split + n0 + wn * WN) * size,
                                         (unsigned)(((rows - 1) * G.ldo + WN) * size));
            const unsigned long long base = (unsigned long long)(unsigned)raw[0] | (unsigned long long)(unsigned)raw[1] << 32;
            const __amdgpu_buffer_rsrc_t rs =
                __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, raw[2], 0x00020000);
            static_for<TM>([&](auto B) {
                constexpr int b = decltype(B)::value;
                // (a row past the last may lie before the next one's end: its own mark)
                const int voff = b * 32 + lr < rows ? ((b * 32 + lr) * (int)G.ldo + (size == 4 ? 4 : 8) * h) * size : OUT_OF_RANGE;
                if (G.out_dtype == CAPSCAPS_FP32) {
                    float4v old[TN * 4];
                    if (G.accumulate)
                        static_for<TN * 4>([&](auto Q) {
                            constexpr int q = decltype(Q)::value;
                            old[q] = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(rs, voff + q * 32, 0, 0));
                        });
                    static_for<TN * 4>([&](auto Q) {
                        constexpr int q = decltype(Q)::value, a = q / 4, g = q % 4;
                        float4v r;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float z = acc[a][b][4 * g + j];
                            r[j] = (TERMS == 3 ? z * SPLIT_UNSCALE : z) * scale;
                        }
                        if (G.accumulate) r += old[q];
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(chunk_t, r), rs, voff + q * 32, 0, 0);
                    });
                } else {
                    static_for<TN>([&](auto A) {
                        constexpr int a = decltype(A)::value;
                        unsigned w[8];
#pragma unroll
                        for (int r = 0; r < 16; r += 2) {
                            float v[2];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const float z = acc[a][b][r + j];
                                v[j] = (TERMS == 3 ? z * SPLIT_UNSCALE : z) * scale;
                            }
                            w[r / 2] = G.out_dtype == CAPSCAPS_FP16 ? half_pair(v[0], v[1]) : round_pair(v[0], v[1]);
                        }
#pragma unroll
                        for (int pair = 0; pair < 2; ++pair)
                            __builtin_amdgcn_raw_buffer_store_b128(neighbours(w, pair), rs, voff + (a * 64 + pair * 32), 0, 0);
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            return;
        }
        const long long base = (m0 + wm * WM) * G.ldo + part * G.out_split + n0 + wn * WN;
        static_for<TM>([&](auto B) {
            constexpr int b = decltype(B)::value;
            if (m0 + wm * WM + b * 32 + lr < m_end)
                static_for<TN * 4>([&](auto Q) {
                    constexpr int a = decltype(Q)::value / 4, g = decltype(Q)::value % 4;
                    const int n = a * 32 + 8 * g + 4 * h;
                    const long long at = base + (b * 32 + lr) * G.ldo + n;
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)  // (one factor after the other: their product may be too small)
                        v[j] = (TERMS == 3 ? acc[a][b][4 * g + j] * SPLIT_UNSCALE : acc[a][b][4 * g + j]) * scale;
                    if (vectors && n + 4 <= n_left) {
                        if (G.out_dtype == CAPSCAPS_FP32) {
                            typedef float4v at4 __attribute__((aligned(4)));
                            at4* to = reinterpret_cast<at4*>(static_cast<float*>(G.out) + at);
                            float4v r = {v[0], v[1], v[2], v[3]};
                            if (G.accumulate) r += *to;
                            *to = r;
                        } else {
                            typedef unsigned u2 __attribute__((ext_vector_type(2)));
                            typedef u2 at2 __attribute__((aligned(2)));
                            const u2 r = G.out_dtype == CAPSCAPS_FP16 ? u2{half_pair(v[0], v[1]), half_pair(v[2], v[3])}
                                                                      : u2{round_pair(v[0], v[1]), round_pair(v[2], v[3])};
                            *reinterpret_cast<at2*>(static_cast<unsigned short*>(G.out) + at) = r;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (n + j < n_left) {
                                if (G.accumulate) v[j] += static_cast<const float*>(G.out)[at + j];
                                store_element(G.out, at + j, v[j], G.out_dtype);
                            }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
        });
        return;
    }
    // z + bias of the lane's values, in place
    if (TERMS == 3 || G.bias != nullptr)
        static_for<TN * 4>([&](auto Q) {
            constexpr int a = decltype(Q)::value / 4, g = decltype(Q)::value % 4;
            float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (G.bias != nullptr)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = a * 32 + 8 * g + 4 * h + j;
                    if (n < n_left) bias[j] = G.bias[n0 + wn * WN + n];
                }
            static_for<TM>([&](auto B) {
                constexpr int b = decltype(B)::value;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float z = acc[a][b][4 * g + j];
                    acc[a][b][4 * g + j] = (TERMS == 3 ? z * SPLIT_UNSCALE : z) + bias[j];
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    if (n_left < WN)  // (columns past the last class count nothing)
        static_for<TN * 16>([&](auto Q) {
            constexpr int a = decltype(Q)::value / 16, r = decltype(Q)::value % 16;
            const bool past = a * 32 + 8 * (r / 4) + 4 * h + r % 4 >= n_left;
#pragma unroll
            for (int b = 0; b < TM; ++b) acc[a][b][r] = past ? -__builtin_inff() : acc[a][b][r];
            __builtin_amdgcn_sched_barrier(0);
        });
    if constexpr (END == HEAD_STATS) {
        const long long first = (n0 + wn * WN) / WN * G.m_rows;
        const float minus = -__builtin_inff(), inv_log2 = G.inv_tau * 1.44269504f;
        static_for<TM>([&](auto B) {
            constexpr int b = decltype(B)::value;
            // (four chains: one wave on a SIMD waits for what it needs next.  v_max3_f32 by name: the compiler would make sure
            // of quiet NaN first, which v_exp_f32 does)
            float tops[4] = {minus, minus, minus, minus}, sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int a = 0; a < TN; ++a)
#pragma unroll
                for (int r = 0; r < 16; r += 2)
                    asm("v_max3_f32 %0, %1, %2, %0" : "+v"(tops[r / 2 & 3]) : "v"(acc[a][b][r]), "v"(acc[a][b][r + 1]));
            float top = __builtin_fmaxf(__builtin_fmaxf(tops[0], tops[1]), __builtin_fmaxf(tops[2], tops[3]));
            top = __builtin_fmaxf(top, __shfl_xor(top, 32));
            // (nothing but -infinity: every difference would be NaN)
            const float about = top == minus ? 0.0f : top;
            static_for<TN>([&](auto A) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sums[r & 3] += __builtin_amdgcn_exp2f((acc[decltype(A)::value][b][r] - about) * inv_log2);
                __builtin_amdgcn_sched_barrier(0);
            });
            float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            sum += __shfl_xor(sum, 32);
            const long long m = m0 + wm * WM + b * 32 + lr;
            if (h == 0 && m < m_end && n_left > 0) G.stats[first + m] = {top * G.inv_tau, sum};
        });
        return;
    }
    if constexpr (END == HEAD_GRADIENT) {
        const int terms = TERMS == 3 ? 3 : G.grad_terms;
        constexpr bool half = std::is_same<Tag, f16_tag>::value;
        float sums[TN * 16];
        static_for<TN * 16>([&](auto Q) { sums[decltype(Q)::value] = 0.0f; });
        // (columns up to a whole stage of the product that contracts classes are written, as zeros; so are rows up to one)
        const int n_out = ((n_left + wn * WN + HEAD_K - 1) / HEAD_K) * HEAD_K - wn * WN;
        const long long m_out = (m_end + HEAD_K - 1) / HEAD_K * HEAD_K;
        const long long sn = (long long)terms * G.planes_n, stt = (long long)terms * G.planes_t;
        static_for<TM>([&](auto B) {
            constexpr int b = decltype(B)::value;
            const long long m = m0 + wm * WM + b * 32 + lr;
            const bool row = m < m_end;
            const float lse = row ? G.lse[G.rows_of[m]] : 0.0f, coef = row ? G.coef[m] : 0.0f;
            const bool adds = row && __builtin_fabsf(coef) < __builtin_inff();  // (others: where the sums are added up)
            // row m at the wave's first class, without its chunk; stage of these 32 rows in gt
            unsigned short* const gn = G.gn + ((m >> 4) * sn + ((n0 + wn * WN) >> 5)) * 512 + (m & 15) * 32;
            const long long stage_t = (m0 + wm * WM + b * 32) >> 5;
            static_for<TN>([&](auto A) {
                constexpr int a = decltype(A)::value;
                float v[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float l = __builtin_fmaf(acc[a][b][r], G.inv_tau, -lse);
                    v[r] = coef * (TERMS == 3 ? expf(l) : __expf(l));
                    if (G.sums != nullptr) sums[a * 16 + r] += adds ? v[r] : 0.0f;
                    if constexpr (TERMS == 3) v[r] *= SPLIT_SCALE;
                }
#pragma unroll
                for (int p = 0; p < (TERMS == 3 ? 3 : 2); ++p) {
                    if (p >= terms) break;
                    unsigned w[8];
#pragma unroll
                    for (int r = 0; r < 16; r += 2) {
                        w[r / 2] = half ? half_pair(v[r], v[r + 1]) : round_pair(v[r], v[r + 1]);
                        if (!row) w[r / 2] = 0;  // (exp of a bias, with factor 0, may be NaN)
                        if constexpr (TERMS == 3) {
                            const bool lo = (w[r / 2] & 0x7f80u) == 0x7f80u, hi = (w[r / 2] & 0x7f800000u) == 0x7f800000u;
                            v[r] = lo ? 0.0f : v[r] - low_half(w[r / 2]);
                            v[r + 1] = hi ? 0.0f : v[r + 1] - high_half(w[r / 2]);
                        } else if (p == 0 && terms > 1) {
                            // (what is not finite: NaN in the second term too, as in the sums)
                            if constexpr (half) {
                                const half2v u = __builtin_bit_cast(half2v, w[r / 2]);
                                v[r] -= (float)u[0], v[r + 1] -= (float)u[1];
                            } else {
                                v[r] -= low_half(w[r / 2]), v[r + 1] -= high_half(w[r / 2]);
                            }
                        }
                    }
#pragma unroll
                    for (int pair = 0; pair < 2; ++pair) {
                        const chunk_t c = neighbours(w, pair);
                        const int place = (2 * pair + h) ^ ((lr >> 2) & 3);
                        if (row && a * 32 < n_out)
                            *reinterpret_cast<chunk_t*>(gn + ((long long)p * G.planes_n + a) * 512 + place * 8) = c;
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        typedef unsigned u2 __attribute__((ext_vector_type(2)));
                        u2 t = {w[2 * g], w[2 * g + 1]};
                        unsigned lo = t[0], hi = t[1];
                        turn(lo, hi, lane);
                        t = u2{lo, hi};
                        const int n = a * 32 + 8 * g + 4 * h + (lane & 3);
                        const int nr = n & 15, place = (lr >> 3) ^ (nr >> 2);
                        if (n < n_left && m - (lane & 3) < m_out)
                            *reinterpret_cast<u2*>(G.gt + (((n0 + wn * WN + n) >> 4) * stt + p * G.planes_t + stage_t) * 512 +
                                                   nr * 32 + place * 8 + (lr & 4)) = t;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        if (G.sums != nullptr && m0 + wm * WM < m_end) {
            float* const to = G.sums + ((m0 + wm * WM) / WM) * G.planes_n * HEAD_K + n0 + wn * WN;
            static_for<TN * 16>([&](auto Q) {
                constexpr int a = decltype(Q)::value / 16, r = decltype(Q)::value % 16;
                const float s = lanes_sum(sums[decltype(Q)::value], 32);
                const int n = a * 32 + 8 * (r / 4) + 4 * h + r % 4;
                if (lr == 0 && n < n_left) to[n] = s;
                __builtin_amdgcn_sched_barrier(0);
            });
        }
    }
}

template <typename Tag, int BM, int BN, int NWM, int NB, int TERMS, bool ROWS, int END>
__global__ __launch_bounds__(256, BM * BN == 65536 ? 1 : 2) void head_gemm_kernel(const HeadGemm G, int tiles_n)
{
    head_gemm<Tag, BM, BN, NWM, NB, TERMS, ROWS, END>(G, tiles_n, blockIdx.x);
}

// Two products that do not need each other in one launch: neither of few tiles leaves CUs without work, or its first copies
// waited for alone
struct HeadPair {
    HeadGemm g[2];
    int tiles_n[2], blocks;  // workgroups of the first
};
template <typename Tag, int BM, int BN, int NWM, int NB, int TERMS>
__global__ __launch_bounds__(256, 2) void head_gemm_pair_kernel(const HeadPair P)
{
    const int second = (int)blockIdx.x >= P.blocks ? 1 : 0;
    head_gemm<Tag, BM, BN, NWM, NB, TERMS, false, HEAD_OUT>(P.g[second], P.tiles_n[second],
                                                             (int)blockIdx.x - (second ? P.blocks : 0));
}

// Workgroups of a product, 0 where no launch holds them (the plan keeps within it)
template <int BM, int BN>
int workgroups_of(HeadGemm& g, int& tiles_n)
{
    const int size = g.out_dtype == CAPSCAPS_FP32 ? 4 : 2;
    g.whole_vectors = (reinterpret_cast<uintptr_t>(g.out) & 15) == 0 && g.ldo * size % 16 == 0 && g.out_split * size % 16 == 0 &&
                      g.ldo * size * BM < 0x7fffffffll;
    const long long tm = (g.m_rows + BM - 1) / BM, tn = (g.n_rows + BN - 1) / BN;
    if (tm * tn * g.splits > (1 << 23) || tm < 1 || tn < 1) return 0;
    tiles_n = (int)tn;
    return (int)(tm * tn * g.splits);
}

template <typename Tag, int BM, int BN, int NWM, int NB, int TERMS>
hipError_t launch_two(const HeadGemm& a, const HeadGemm& b, hipStream_t st)
{
    HeadPair p{{a, b}, {0, 0}, 0};
    p.blocks = workgroups_of<BM, BN>(p.g[0], p.tiles_n[0]);
    const int more = workgroups_of<BM, BN>(p.g[1], p.tiles_n[1]);
    if (p.blocks == 0 || more == 0) return hipErrorInvalidValue;
    const auto kernel = head_gemm_pair_kernel<Tag, BM, BN, NWM, NB, TERMS>;
    constexpr int lds = (BM + BN) * 64 * NB;
    static std::atomic<unsigned long long> done{0};
    const hipError_t err = set_dynamic_lds_once(reinterpret_cast<const void*>(kernel), lds, done);
    if (err != hipSuccess) return err;
    kernel<<<dim3((unsigned)p.blocks + (unsigned)more), dim3(256), lds, st>>>(p);
    return hipGetLastError();
}
template <int BM, int BN, int NWM, int NB>
hipError_t launch_pair(const HeadGemm& a, const HeadGemm& b, hipStream_t st)
{
    if (a.terms != b.terms || a.dtype != b.dtype || a.stages_b == 0 || b.stages_b == 0) return hipErrorInvalidValue;
    if (a.terms == 3) return launch_two<bf16_tag, BM, BN, NWM, NB, 3>(a, b, st);
    const bool bf16 = a.dtype == CAPSCAPS_BF16;
    if (a.terms == 2) return bf16 ? launch_two<bf16_tag, BM, BN, NWM, NB, 2>(a, b, st) : launch_two<f16_tag, BM, BN, NWM, NB, 2>(a, b, st);
    return bf16 ? launch_two<bf16_tag, BM, BN, NWM, NB, 1>(a, b, st) : launch_two<f16_tag, BM, BN, NWM, NB, 1>(a, b, st);
}

template <typename Tag, int BM, int BN, int NWM, int NB, int TERMS, bool ROWS, int END>
hipError_t launch(HeadGemm g, hipStream_t st)
{
    int tn = 0;
    const int blocks = workgroups_of<BM, BN>(g, tn);
    if (blocks == 0) return hipErrorInvalidValue;
    const auto kernel = head_gemm_kernel<Tag, BM, BN, NWM, NB, TERMS, ROWS, END>;
    constexpr int lds = (BM + BN) * 64 * NB;
    static std::atomic<unsigned long long> done{0};
    const hipError_t err = set_dynamic_lds_once(reinterpret_cast<const void*>(kernel), lds, done);
    if (err != hipSuccess) return err;
    kernel<<<dim3((unsigned)blocks), dim3(256), lds, st>>>(g, tn);
    return hipGetLastError();
}

template <int BM, int BN, int NWM, int NB, int END>
hipError_t launch_type(const HeadGemm& g, hipStream_t st)
{
    if (g.terms == 3) return launch<bf16_tag, BM, BN, NWM, NB, 3, false, END>(g, st);
    const bool bf16 = g.dtype == CAPSCAPS_BF16;
    if constexpr (END == HEAD_OUT) {
        if (g.terms == 2)
            return bf16 ? launch<bf16_tag, BM, BN, NWM, NB, 2, false, END>(g, st) : launch<f16_tag, BM, BN, NWM, NB, 2, false, END>(g, st);
    }
    if (g.terms != 1) return hipErrorInvalidValue;
    if (g.stages_b == 0)
        return bf16 ? launch<bf16_tag, BM, BN, NWM, NB, 1, true, END>(g, st) : launch<f16_tag, BM, BN, NWM, NB, 1, true, END>(g, st);
    return bf16 ? launch<bf16_tag, BM, BN, NWM, NB, 1, false, END>(g, st) : launch<f16_tag, BM, BN, NWM, NB, 1, false, END>(g, st);
}

template <int BM, int BN, int NWM, int NB>
hipError_t launch_end(const HeadGemm& g, HeadEnd end, hipStream_t st)
{
    if (end == HEAD_OUT) return launch_type<BM, BN, NWM, NB, HEAD_OUT>(g, st);
    if (end == HEAD_STATS) return launch_type<BM, BN, NWM, NB, HEAD_STATS>(g, st);
    return launch_type<BM, BN, NWM, NB, HEAD_GRADIENT>(g, st);
}

}  // namespace
}  // namespace capscaps

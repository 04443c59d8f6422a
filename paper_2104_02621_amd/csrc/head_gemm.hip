// The matrix products of a linear head over many classes, on the bf16 and fp16 matrix instructions:
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
// LDS stage: rows of 64 bytes, four 16-byte chunks, chunk c of row r in place c ^ (r / 4 % 4): four neighbouring lanes of a
// copy bring one row's 64 contiguous bytes, and the 16 lanes that read one chunk of 16 rows touch 16 different 16-byte
// columns of the banks.  The n side is the matrix instruction's row operand, so that a lane ends up with runs of four
// neighbouring n of one m.
#include "head_gemm.h"

#include "bf16_split.h"
#include "conv_shape.h"
#include "element.h"
#include "igemm_common.h"
#include "lds_dma.h"

namespace capscaps {
namespace {

constexpr int NB = 4;  // stages of the ring
constexpr int OUT_OF_RANGE = (int)0x80000000u;

template <typename Tag, int BM, int BN, int NWM, bool TERMS>
__global__ __launch_bounds__(256, BM * BN == 65536 ? 1 : 2) void head_gemm_kernel(const HeadGemm G, int tiles_m, int tiles_n)
{
    constexpr int NWN = 4 / NWM, WM = BM / NWM, WN = BN / NWN, TM = WM / 32, TN = WN / 32;
    constexpr int A_BYTES = BM * 64, STAGE = (BM + BN) * 64;
    constexpr int CA = BM / 64, CB = BN / 64;  // copies of a wave and stage
    constexpr int NMMA = TM * TN, NFRAG = TM + TN;
    constexpr int KEEP = (NB - 2) * (CA + CB);
    static_assert(KEEP + CA < 64, "vmcnt is a 6-bit counter");
    static_assert(NFRAG <= 2 * NMMA && CA >= 1 && CB >= 1, "side operations");
    extern __shared__ char smem[];

    // Tiles: an XCD (workgroups go to the eight in turn) takes a run of them, bands of eight rows of tiles, so that the 32
    // tiles its CUs work on at a time share operands in its L2.
    const int tiles = tiles_m * tiles_n;
    int part, L;
    {
        const int all = gridDim.x, span = all & ~7;
        const int id = (int)blockIdx.x < span ? ((int)blockIdx.x & 7) * (span >> 3) + ((int)blockIdx.x >> 3) : blockIdx.x;
        part = id / tiles;
        L = id - part * tiles;
    }
    const int band = L / (8 * tiles_n), in_band = L - band * 8 * tiles_n;
    const int high = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
    const long long m0 = (long long)(band * 8 + in_band % high) * BM;
    const long long n0 = (long long)(in_band / high) * BN;
    long long m_end = G.m_rows;
    if (G.m_count != nullptr) {
        const long long c = *G.m_count;
        m_end = c < m_end ? c : m_end;
    }
    if (m0 >= m_end) return;
    // stages of this part
    long long k = G.k;
    if (G.k_count != nullptr) {
        const long long c = *G.k_count;
        k = c < k ? c : k;
    }
    const int all_stages = (int)((k + HEAD_K - 1) / HEAD_K);
    const int per = (all_stages + G.splits - 1) / G.splits;
    const int first = part * per < all_stages ? part * per : all_stages;
    const int run = all_stages - first < per ? all_stages - first : per;  // of each product of terms
    const int stages = __builtin_amdgcn_readfirstlane(TERMS ? run * HEAD_PRODUCTS : run);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % NWM, wn = wave / NWM;
    const int h = lane >> 5, lr = lane & 31;

    auto rows_of = [](const void* base, long long ld, long long first_row, long long rows) {
        const long long bytes = (rows - first_row) * ld;
        return make_rsrc(static_cast<const char*>(base) + first_row * ld,
                         (unsigned)(bytes < 0x7fffffffll ? bytes : 0x7fffffffll));
    };
    const rsrc_t rs_a = rows_of(G.a, G.lda, m0, m_end), rs_b = rows_of(G.b, G.ldb, n0, G.n_rows);
    const int lda = __builtin_amdgcn_readfirstlane((int)G.lda), ldb = __builtin_amdgcn_readfirstlane((int)G.ldb);
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)smem;
    const unsigned lds_a = __builtin_amdgcn_readfirstlane((int)(lds0 + wave * CA * 1024));
    const unsigned lds_b = __builtin_amdgcn_readfirstlane((int)(lds0 + A_BYTES + wave * CB * 1024));
    // a copy is 16 rows; a lane's row of them and chunk
    const int copy_row = lane >> 2, copy_chunk = (lane & 3) ^ ((copy_row >> 2) & 3);
    const unsigned a_voff = copy_row * lda + copy_chunk * 16, b_voff = copy_row * ldb + copy_chunk * 16;
    int a_row[CA], b_row[CB];
#pragma unroll
    for (int j = 0; j < CA; ++j) a_row[j] = __builtin_amdgcn_readfirstlane((wave * CA + j) * 16 * lda);
#pragma unroll
    for (int j = 0; j < CB; ++j) b_row[j] = __builtin_amdgcn_readfirstlane((wave * CB + j) * 16 * ldb);

    // the stage whose copies go out next: byte offsets within a row (out of range past the last stage)
    int next = 0, product = 0, left = run;
    int a_off = stages > 0 ? first * 64 : OUT_OF_RANGE, b_off = a_off;
    if (TERMS && stages > 0) {
        a_off += SPLIT_TERM_A[0] * G.plane_a;
        b_off += SPLIT_TERM_B[0] * G.plane_b;
    }
    auto advance = [&]() {
        ++next;
        a_off += 64;
        b_off += 64;
        if constexpr (TERMS) {
            if (--left == 0) {
                left = run;
                ++product;
                // (terms of the products, two bits each)
                constexpr int ta = SPLIT_TERM_A[0] | SPLIT_TERM_A[1] << 2 | SPLIT_TERM_A[2] << 4 | SPLIT_TERM_A[3] << 6 |
                                   SPLIT_TERM_A[4] << 8 | SPLIT_TERM_A[5] << 10;
                constexpr int tb = SPLIT_TERM_B[0] | SPLIT_TERM_B[1] << 2 | SPLIT_TERM_B[2] << 4 | SPLIT_TERM_B[3] << 6 |
                                   SPLIT_TERM_B[4] << 8 | SPLIT_TERM_B[5] << 10;
                a_off = first * 64 + (ta >> 2 * product & 3) * G.plane_a;
                b_off = first * 64 + (tb >> 2 * product & 3) * G.plane_b;
            }
        }
        a_off = next < stages ? a_off : OUT_OF_RANGE;
        b_off = next < stages ? b_off : OUT_OF_RANGE;
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
    // reads before gap i of a step's NMMA gaps; copies, later, spread over them
    constexpr auto reads_before = [](int i) { return i * NFRAG / NMMA < NFRAG ? (NMMA >= NFRAG ? (i < NFRAG ? i : NFRAG) : i * NFRAG / NMMA) : NFRAG; };
    constexpr auto copies_before = [](int i, int count) {
        return NMMA >= 16 ? (i + 1) / 4 < count ? (i + 1) / 4 : count : i * count / NMMA;
    };
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
    const float scale = G.scale != nullptr ? *G.scale : 1.0f;
    const bool vectors = (G.ldo & 3) == 0;
    const long long n_end = G.n_rows;
#pragma unroll
    for (int b = 0; b < TM; ++b) {
        const long long m = m0 + wm * WM + b * 32 + lr;
        if (m >= m_end) continue;
        const long long row = m * G.ldo + part * G.out_split;
#pragma unroll
        for (int a = 0; a < TN; ++a)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const long long n = n0 + wn * WN + a * 32 + 8 * g + 4 * h;
                if (n >= n_end) continue;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (TERMS ? acc[a][b][4 * g + j] * SPLIT_UNSCALE : acc[a][b][4 * g + j]) * scale;  // (one factor after the other: their product may be too small)
                if (vectors && n + 4 <= n_end) {
                    if (G.out_dtype == CAPSCAPS_FP32) {
                        typedef float4v at __attribute__((aligned(4)));
                        at* to = reinterpret_cast<at*>(static_cast<float*>(G.out) + row + n);
                        float4v r = {v[0], v[1], v[2], v[3]};
                        if (G.accumulate) r += *to;
                        *to = r;
                    } else {
                        typedef unsigned u2 __attribute__((ext_vector_type(2)));
                        typedef u2 at __attribute__((aligned(2)));
                        const int kind = G.out_dtype == CAPSCAPS_FP16 ? 2 : 1;
                        const u2 r = {round_to_16(v[0], kind) | (unsigned)round_to_16(v[1], kind) << 16,
                                      round_to_16(v[2], kind) | (unsigned)round_to_16(v[3], kind) << 16};
                        *reinterpret_cast<at*>(static_cast<unsigned short*>(G.out) + row + n) = r;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (n + j < n_end) {
                            if (G.accumulate) v[j] += static_cast<const float*>(G.out)[row + n + j];
                            store_element(G.out, row + n + j, v[j], G.out_dtype);
                        }
                }
            }
    }
}

template <typename Tag, int BM, int BN, int NWM, bool TERMS>
hipError_t launch(const HeadGemm& g, hipStream_t st)
{
    const long long tm = (g.m_rows + BM - 1) / BM, tn = (g.n_rows + BN - 1) / BN;
    if (tm * tn * g.splits > (1 << 23) || tm < 1 || tn < 1) return hipErrorInvalidValue;
    const auto kernel = head_gemm_kernel<Tag, BM, BN, NWM, TERMS>;
    constexpr int lds = (BM + BN) * 64 * NB;
    static std::atomic<unsigned long long> done{0};
    const hipError_t err = set_dynamic_lds_once(reinterpret_cast<const void*>(kernel), lds, done);
    if (err != hipSuccess) return err;
    kernel<<<dim3((unsigned)(tm * tn * g.splits)), dim3(256), lds, st>>>(g, (int)tm, (int)tn);
    return hipGetLastError();
}

template <int BM, int BN, int NWM>
hipError_t launch_type(const HeadGemm& g, hipStream_t st)
{
    if (g.dtype == CAPSCAPS_FP32) return launch<bf16_tag, BM, BN, NWM, true>(g, st);
    if (g.dtype == CAPSCAPS_BF16) return launch<bf16_tag, BM, BN, NWM, false>(g, st);
    return launch<f16_tag, BM, BN, NWM, false>(g, st);
}

}  // namespace

hipError_t launch_head_gemm(const HeadGemm& g, int tile, hipStream_t st)
{
    if (tile == HEAD_TILE_256) return launch_type<256, 256, 2>(g, st);
    if (tile == HEAD_TILE_128) return launch_type<128, 128, 2>(g, st);
    return launch_type<64, 256, 1>(g, st);
}

}  // namespace capscaps

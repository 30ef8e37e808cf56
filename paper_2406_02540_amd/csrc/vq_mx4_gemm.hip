// GEMM on microscaled 4-bit operands, tiles that their wavefronts share.
//
// y[m,n] = sum over blocks of 2^(Ex + Ew) * (sum of 32 products of codes) + bias[n].  v_mfma_scale_f32_16x16x128_f8f6f4
// multiplies 16 channels x 16 tokens x 4 blocks; lane l holds block l/16 of row l%16, 16 bytes as they lie in memory, and that
// block's scale byte.  Channels are the rows of the product, so that a lane ends with four channels of a token, and the
// channels are dealt to the rows of the weight tile so that its sums of two neighbouring MFMA blocks are eight channels in a row; a
// store, after an exchange between lanes, is 16 bytes a lane, 8 tokens x 128 bytes.
//
// K in stages of 256: a row is one cache line of codes (128 bytes) and two dwords of scales.  The codes go from memory to LDS without
// registers, the scales through a register of the thread that spreads them there; the stage behind the one that is multiplied is on
// its way meanwhile, also from one tile of a workgroup to its next.
//
// Measured (captured, several hundred MB of inputs and outputs in turn, so that none is in the caches): 32768 x 1152 -> 4608 131 us (2.7
// PFLOP/s; its 324 MB alone are 63 us at the 5.2 TB/s of a copy), 32768 x 4608 -> 1152 133, 8192 x 1152 -> 1152 16.6, 8192 x 8192 -> 8192
// 277 (4.0 PFLOP/s).  At the last the matrix units were busy 42 % of the time at 2.07 GHz (counted before the stores' last form); where K is short a tile's outputs cost
// as much as its products.
#include "vq_internal.h"
#include "vq_mx4_product.h"

namespace vq {
namespace {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char* lds_bytes;

constexpr int kLineBytes = 128;
// Rows r of the weight tile and their channels: 32 channels are two MFMA blocks, of which lane group g has the rows 4g .. 4g+3.
__device__ __forceinline__ int row_channel(int r) {
    return (r & ~31) + ((r >> 2) & 3) * 8 + ((r >> 4) & 1) * 4 + (r & 3);
}
template <int TT_, int CC_, int WT_, int WC_>
struct Shape {
    static constexpr int TT = TT_, CC = CC_, WT = WT_, WC = WC_;         // a wavefront's MFMA blocks, and wavefronts
    static constexpr int kWaves = WT * WC, kTok = 16 * TT * WT, kCh = 16 * CC * WC;
    static constexpr int kXLoads = kTok / (8 * kWaves), kWLoads = kCh / (8 * kWaves);
    // two stages of codes, two of scales (of two stages of codes each), three tiles' bias
    static constexpr int kRows = kTok + kCh, kW = kTok * kLineBytes, kStage = kRows * kLineBytes;
    static constexpr int kScales = 2 * kStage, kScaleStage = 16 * kRows;
    static constexpr int kBias = kScales + 2 * kScaleStage, kBiasBytes = 2 * kCh;
    static constexpr int kLds = kBias + 3 * kBiasBytes;
    static constexpr int kStores = TT * CC / 2;
    static_assert(kTok % (8 * kWaves) == 0 && kCh % (8 * kWaves) == 0 && kRows <= 64 * kWaves, "whole loads, a row of scales a thread");
    static_assert(kBiasBytes / 4 % 64 == 0 && kBiasBytes / 256 <= kWaves && CC % 2 == 0, "whole loads of the bias");
};

// Where channel `to` of row m of a tile is, in bytes, where stores are range-checked (N below 2^21).  0 for rows that start anywhere:
// those are addressed in 64 bits, and with their N the product may not fit (an overflow is undefined even where nothing uses it).
template <bool ROWS16>
__host__ __device__ constexpr int checked_at(int m, int N, int to) {
    return ROWS16 ? 2 * (m * N + to) : 0;
}
static_assert(checked_at<true>(255, (1 << 21) - 1, 255) > 0 && checked_at<false>(255, 0x7FFFFFFF, 255) == 0, "nothing overflows");

struct TileArgsMx {
    Mx4GemmArgs g;
    int tiles_t, tiles_c, tiles, tiles_per_xcd, slots;
    bool whole_lines;        // rows of Y start on memory lines
};

// ROWS16: rows of Y are whole 16-byte pieces (N % 8 == 0, Y on 16 bytes): range-checked stores.  Otherwise 64-bit addresses, the same pieces
// unaligned, and a row's last channels one by one: 1001 x 1184 -> 2821 12.9 us, 14.6 with the bias straight from memory and 64 bytes of a row
// a store; 8192 x 1152 -> 4607 73 and 82 (4608 44, in tiles that this form has no registers for).
template <class TYPE, class S, bool ROWS16>
__global__ __launch_bounds__(64 * S::kWaves, 2) void mx4_gemm(TileArgsMx a) {
    __shared__ __align__(128) char lds[S::kLds];
    typedef typename TYPE::T T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, r16 = lane & 15;
    const int wt = wave % S::WT, wc = wave / S::WT;
    const int M = a.g.M, N = a.g.N, blocks = a.g.K / kMxBlock;
    const int row_bytes = a.g.K / 2, stride = mx_scale_stride(a.g.K);
    const int steps = (blocks + 3) / 4, stages = (steps + 1) / 2;
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds;

    // what this wavefront loads of a stage: 8 rows a turn, a lane 16 bytes
    int x_at[S::kXLoads], w_at[S::kWLoads];
    const int in8 = lane >> 3, slot = lane & 7;
#pragma unroll
    for (int i = 0; i < S::kXLoads; ++i) {
        const int r = 8 * (S::kXLoads * wave + i) + in8;
        x_at[i] = r * row_bytes + 16 * (slot ^ line_swizzle(r));
    }
#pragma unroll
    for (int i = 0; i < S::kWLoads; ++i) {
        const int r = 8 * (S::kWLoads * wave + i) + in8;
        w_at[i] = row_channel(r) * row_bytes + 16 * (slot ^ line_swizzle(r));
    }
    // and the scales of one row, tokens first
    const bool s_token = (int)threadIdx.x < S::kTok;
    const int s_row = s_token ? (int)threadIdx.x : row_channel((int)threadIdx.x - S::kTok);

    int row0 = 0, col0 = 0;            // the tile whose stages are asked for
    v4i rx, rw, rb;
    auto place = [&](int i) {
        const int tile = (int)(blockIdx.x % kXcds) * a.tiles_per_xcd + i;
        if (i >= a.tiles_per_xcd || tile >= a.tiles) return false;
        const int band = tile / (kBand * a.tiles_c), in_band = tile - band * kBand * a.tiles_c;
        const int band_rows = min(a.tiles_t - band * kBand, kBand);
        const int c = in_band / band_rows;
        row0 = (band * kBand + in_band - c * band_rows) * S::kTok;
        col0 = c * S::kCh;
        const int rows = min(M - row0, S::kTok), cols = min(N - col0, S::kCh);
        rx = make_rsrc(a.g.xq + (size_t)row0 * row_bytes, (unsigned)(rows * row_bytes));
        rw = make_rsrc(a.g.wq + (size_t)col0 * row_bytes, (unsigned)(cols * row_bytes));
        rb = make_rsrc((const char*)a.g.bias + 2 * (size_t)col0, a.g.bias ? 2u * (cols & ~1) : 0u);       // (whole dwords)
        return true;
    };
    // Scales go through registers, sixteen of a row at a time for two stages: a touch of their line costs the caches as much as 128
    // bytes of codes do.  Rows that do not exist, and blocks behind the row's end, whose codes are zeros, get zeros.
    v4i scales;
    auto ask_scales = [&](int stage) {
        const int from = s_token ? row0 + s_row : col0 + s_row, b0 = 8 * stage;
        const bool in = from < (s_token ? M : N) && threadIdx.x < S::kRows;
        const uint8_t* const p = (s_token ? a.g.x_scale : a.g.w_scale) + (size_t)from * stride + b0;
        scales = v4i{0, 0, 0, 0};
        if (in) {
            typedef v4i v4i_any __attribute__((aligned(4)));
            if (b0 + 16 <= stride) {
                scales = *(const v4i_any*)p;
            } else {
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    if (b0 + 4 * d < stride) scales[d] = *(const int*)(p + 4 * d);
            }
        }
    };
    auto keep_scales = [&](int stage, int to) {
        const int left = blocks - 8 * stage;
        v4i v;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int n = left - 4 * d;
            v[d] = n >= 4 ? scales[d] : n <= 0 ? 0 : scales[d] & ((1 << 8 * n) - 1);
        }
        // (a last stage of one step has the scale of block g where the other stages have that of 2g)
#pragma unroll
        for (int d = 0; d < 4; d += 2)
            if (2 * stage + d + 1 == steps) {
                v[d + 1] = (v[d] >> 16 & 0xFF) | (v[d] >> 8 & 0xFF0000);
                v[d] = (v[d] & 0xFF) | (v[d] << 8 & 0xFF0000);
            }
        if (S::kRows == 64 * S::kWaves || threadIdx.x < S::kRows) {
            const lds_bytes at = (lds_bytes)lds + S::kScales + to * S::kScaleStage + 8 * threadIdx.x;
            *(__attribute__((address_space(3))) v2i*)at = v2i{v[0], v[1]};
            *(__attribute__((address_space(3))) v2i*)(at + 8 * S::kRows) = v2i{v[2], v[3]};
        }
    };
    int buffer = 0, bias_to = 0;       // where the stage, and the tile's bias, go that are asked for next
    // Behind a row's end there are zeros.
    auto ask = [&](int stage) {
        const unsigned at = base + buffer * S::kStage;
        const int k0 = stage * kLineBytes;
        const bool tail = k0 + kLineBytes > row_bytes;
#pragma unroll
        for (int i = 0; i < S::kXLoads; ++i) {
            const int turn = S::kXLoads * wave + i;
            if (!tail) load_to_lds_16(rx, at + turn * 1024, x_at[i], k0);
            else load_to_lds_16(rx, at + turn * 1024, k0 + 16 * (slot ^ line_swizzle(8 * turn + in8)) < row_bytes ? x_at[i] + k0 : kNowhere, 0);
        }
#pragma unroll
        for (int i = 0; i < S::kWLoads; ++i) {
            const int turn = S::kWLoads * wave + i;
            if (!tail) load_to_lds_16(rw, at + S::kW + turn * 1024, w_at[i], k0);
            else load_to_lds_16(rw, at + S::kW + turn * 1024, k0 + 16 * (slot ^ line_swizzle(8 * turn + in8)) < row_bytes ? w_at[i] + k0 : kNowhere, 0);
        }
    };
    auto ask_bias = [&] {         // (every wavefront a turn: those beyond the bias write the same once more)
        const int turn = wave % (S::kBiasBytes / 256);
        load_to_lds_4(rb, base + S::kBias + bias_to * S::kBiasBytes + 256 * turn, 256 * turn + 4 * lane);
    };

    // Eight channels of a row that starts anywhere.
    auto put = [&](T* y, int m, int n, int rows, int cols, v4u v) {
        if (m >= rows) return;
        T* const to = y + (size_t)m * N + n;
        if (n + 8 <= cols) {
            typedef v4u v4u_any __attribute__((aligned(2)));
            *(v4u_any*)to = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (n + e < cols) ((unsigned short*)to)[e] = (unsigned short)(v[e >> 1] >> 16 * (e & 1));
        }
    };

    v4f acc[S::TT][S::CC];
    // the sums of the tile at (row, col), with its bias, to memory
    auto finish = [&](int row, int col, int bias_from) {
        const int rows = min(M - row, S::kTok), cols = min(N - col, S::kCh);
        T* const y = (T*)a.g.y + (size_t)row * N + col;
        const unsigned bytes = 2 * ((unsigned)(rows - 1) * (unsigned)N + (unsigned)cols);      // (meant for ROWS16 alone)
        const auto ry = __builtin_amdgcn_make_buffer_rsrc(y, 0, (int)bytes, (int)kRsrcFlags);
        const lds_bytes bias = (lds_bytes)lds + S::kBias + bias_from * S::kBiasBytes;
        // A lane has eight channels of its token in each of two neighbouring pairs of blocks, 64 bytes of a token's row a store.  Lanes
        // eight tokens apart exchange one of the two, and a store is 128 bytes of eight tokens: past the caches where these are whole
        // lines (32768 x 1152 -> 4608 131 us, 147 through them, 8192 x 1152 -> 1152 16.6 and 20.3; halves of lines past the caches are slower than either),
        // through them where rows start elsewhere and neighbouring stores share lines.
        const bool low = r16 < 8;
#pragma unroll
        for (int c = 0; c < S::CC; c += 4) {
            const int n = 16 * (S::CC * wc + c) + 8 * g;
            float b[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4i b8 = *(__attribute__((address_space(3))) v4i*)(bias + 2 * (n + 32 * h));
#pragma unroll
                for (int e = 0; e < 4; ++e) TYPE::unpack((unsigned)b8[e], b[h][2 * e], b[h][2 * e + 1]);
                if (!ROWS16 && (cols & 1) && a.g.bias) {       // the last of an odd number is in no whole dword
                    const int last = cols - 1 - (n + 32 * h);
                    if (last >= 0 && last < 8) {
                        const float its = (float)((const T*)a.g.bias)[col + cols - 1];
#pragma unroll
                        for (int e = 0; e < 8; e += 2) b[h][e] = e == last ? its : b[h][e];
                    }
                }
            }
            const int to = n + (low ? 0 : 32), m = 16 * S::TT * wt + (r16 & 7);
            const int at = to < cols ? checked_at<ROWS16>(m, N, to) : kNowhere;
#pragma unroll
            for (int t = 0; t < S::TT; ++t) {
                v4u piece[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v4f lo = acc[t][c + 2 * h], hi = acc[t][c + 2 * h + 1];
                    piece[h] = v4u{TYPE::pack(lo[0] + b[h][0], lo[1] + b[h][1]), TYPE::pack(lo[2] + b[h][2], lo[3] + b[h][3]),
                                   TYPE::pack(hi[0] + b[h][4], hi[1] + b[h][5]), TYPE::pack(hi[2] + b[h][6], hi[3] + b[h][7])};
                }
                v4u first, second;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned given = low ? piece[1][e] : piece[0][e];
                    const unsigned taken = (unsigned)__builtin_amdgcn_mov_dpp((int)given, 0x128, 0xF, 0xF, true);    // row_ror:8
                    first[e] = low ? piece[0][e] : taken;
                    second[e] = low ? taken : piece[1][e];
                }
                if (ROWS16) {
                    const int at_first = to < cols ? at + 32 * t * N : kNowhere, at_second = to < cols ? at + 32 * t * N + 16 * N : kNowhere;
                    if (a.whole_lines) {
                        __builtin_amdgcn_raw_buffer_store_b128(first, ry, at_first, 0, 2 /* nontemporal */);
                        __builtin_amdgcn_raw_buffer_store_b128(second, ry, at_second, 0, 2);
                    } else {
                        __builtin_amdgcn_raw_buffer_store_b128(first, ry, at_first, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b128(second, ry, at_second, 0, 0);
                    }
                } else {
                    put(y, m + 16 * t, to, rows, cols, first);
                    put(y, m + 16 * t + 8, to, rows, cols, second);
                }
            }
        }
    };
    // The stage in `from`, steps `step` and `step` + 1 of K, whose scales are in `s_from`.  Operands are read two groups of TT products
    // ahead of their use, the tokens' of the second step under the first one's products.
    auto multiply = [&](int from, int step, int s_from) {
        const lds_bytes at = (lds_bytes)lds + from * S::kStage + r16 * kLineBytes;
        const lds_bytes xp = at + 16 * S::TT * wt * kLineBytes, wp = at + S::kW + 16 * S::CC * wc * kLineBytes;
        const bool both = step + 1 < steps;       // (a last stage of one step: block g)
        const int chunk[2] = {16 * ((both ? 2 * g : g) ^ line_swizzle(r16)), 16 * ((2 * g + 1) ^ line_swizzle(r16))};
        const lds_bytes sp = (lds_bytes)lds + S::kScales + s_from * S::kScaleStage + 8 * S::kRows * ((step >> 1) & 1) + 8 * r16 + 2 * g;
        const lds_bytes xsp = sp + 128 * S::TT * wt, wsp = sp + 8 * S::kTok + 128 * S::CC * wc;
        typedef __attribute__((address_space(3))) v4i* lds_v4i;
        typedef __attribute__((address_space(3))) unsigned short* lds_u16;
        constexpr int kAhead = 2, kGroups = 2 * S::CC;
        v4i x[2][S::TT], w[kAhead + 1];
        int xs[S::TT], ws[S::CC];
        auto read_w = [&](int n) {      // group n of a step's products: channels n % CC of step n / CC
            w[n % (kAhead + 1)] = *(lds_v4i)(wp + 16 * kLineBytes * (n % S::CC) + chunk[n / S::CC]);
            if (n < S::CC) ws[n] = *(lds_u16)(wsp + 128 * n);
        };
#pragma unroll
        for (int t = 0; t < S::TT; ++t) {
            x[0][t] = *(lds_v4i)(xp + 16 * kLineBytes * t + chunk[0]);
            xs[t] = *(lds_u16)(xsp + 128 * t);
        }
#pragma unroll
        for (int n = 0; n < kAhead; ++n) read_w(n);
#pragma unroll
        for (int n = 0; n < S::CC; ++n) {
            read_w(n + kAhead);
            if (n < S::TT) x[1][n] = *(lds_v4i)(xp + 16 * kLineBytes * n + chunk[1]);
#pragma unroll
            for (int t = 0; t < S::TT; ++t) acc[t][n] = mx_mfma<0>(w[n % (kAhead + 1)], ws[n], x[0][t], xs[t], acc[t][n]);
            __builtin_amdgcn_sched_barrier(0);      // (the scheduler would put all reads of a step in front of its products)
        }
        if (!both) return;
#pragma unroll
        for (int n = S::CC; n < kGroups; ++n) {
            if (n + kAhead < kGroups) read_w(n + kAhead);
#pragma unroll
            for (int t = 0; t < S::TT; ++t)
                acc[t][n - S::CC] = mx_mfma<1>(w[n % (kAhead + 1)], ws[n - S::CC], x[1][t], xs[t], acc[t][n - S::CC]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    int i = (int)(blockIdx.x / kXcds);
    if (!place(i)) return;
    ask_scales(0);
    ask_bias();
    ask(0);
    buffer ^= 1;
    keep_scales(0, 0);
    int done_row = 0, done_col = 0, bias_from = 0, s_from = 0;
    bool done = false, stores = false, more = true;      // a tile's sums wait in the registers; its stores are the newest operations
    for (int from = 0; more;) {
        const int row = row0, col = col0;
        for (int s = 0; s < stages; ++s) {
            if (stores) wait_loads_before_and_barrier<S::kStores>();
            else wait_loads_and_barrier();
            stores = false;
            const bool last = s + 1 == stages;
            const int next = last ? 0 : s + 1;
            if (last) {
                i += a.slots;
                more = place(i);
                bias_to = bias_to == 2 ? 0 : bias_to + 1;
            }
            const bool new_scales = more && next % 2 == 0;
            if (new_scales) ask_scales(next);
            if (more && last) ask_bias();
            if (more) ask(next);
            if (s == 0) {
                if (done) {
                    finish(done_row, done_col, bias_from);
                    bias_from = bias_from == 2 ? 0 : bias_from + 1;
                    stores = ROWS16;
                }
#pragma unroll
                for (int t = 0; t < S::TT; ++t)
#pragma unroll
                    for (int c = 0; c < S::CC; ++c) acc[t][c] = v4f{0, 0, 0, 0};
            }
            multiply(from, 2 * s, s_from);
            buffer ^= 1;
            from ^= 1;
            if (new_scales) {
                s_from ^= 1;
                keep_scales(next, s_from);
            }
        }
        done = true;
        done_row = row, done_col = col;
    }
    finish(done_row, done_col, bias_from);
}

template <class S>
hipError_t launch(const Mx4GemmArgs& g, int dtype, int num_cus, hipStream_t stream) {
    TileArgsMx a{g, 0, 0, 0, 0, 0, g.N % 64 == 0 && (uintptr_t)g.y % 128 == 0};
    if (!mx4_gemm_takes(g.M, g.N)) return hipErrorInvalidValue;
    a.tiles_t = (g.M + S::kTok - 1) / S::kTok;
    a.tiles_c = (g.N + S::kCh - 1) / S::kCh;
    a.tiles = (int)((long)a.tiles_t * a.tiles_c);
    a.tiles_per_xcd = (a.tiles + kXcds - 1) / kXcds;
    const int resident = (int)(163840 / S::kLds) * (num_cus >= kXcds ? num_cus / kXcds : 1);
    a.slots = a.tiles_per_xcd < resident ? a.tiles_per_xcd : resident;
    const bool rows16 = g.N % 8 == 0 && g.N < 1 << 21;       // (a tile's rows within 2^31 bytes)
    const dim3 grid((unsigned)(a.slots * kXcds)), block(64 * S::kWaves);
    if (rows16) return enqueue(dtype == VQ_F16 ? mx4_gemm<F16, S, true> : mx4_gemm<BF16, S, true>, grid, block, stream, a);
    if constexpr (S::TT * S::CC <= 16)     // (a larger tile would spill registers where rows are written piece by piece)
        return enqueue(dtype == VQ_F16 ? mx4_gemm<F16, S, false> : mx4_gemm<BF16, S, false>, grid, block, stream, a);
    return hipErrorInvalidValue;
}

}  // namespace

// Rows and channels of a last tile fit an int, and so do the numbers of the smallest tiles, 64 x 128, and those that a workgroup asks for behind its last.
bool mx4_gemm_takes(int M, int N) {
    static_assert((0x7FFFFF00l + 127) / 128 * kBand <= 0x7FFFFFFFl, "tiles of a band");
    return M <= 0x7FFFFF00 && N <= 0x7FFFFF00 && (((long)M + 63) / 64) * (((long)N + 127) / 128) <= 0x7FFFF000l;
}

// The kernel for a product's sizes, by what each would take: rounds of its workgroups on the chip times a workgroup's time, fitted to
// measurements over M 1 .. 32768, N 1152 .. 8192, K 1152 .. 8192 (us; off by 10 to 15 %).  Where the wavefronts divide K, a
// workgroup counts as alone on its CU and takes 0.8 and 0.02 for each row of a line (256 of K), eight lines at a time; tiles of 256 x 256
// take 2.0 a stage and 3 for their outputs, of 128 x 128, two a CU, 1.1 and 2.7, of 64 x 128 0.9 and 1.7.
// (Tiles of 48 x 48 and 32 x 64 do fill a CU's LDS; two of 32 x 32 fit.  Counted as two with the same costs they take over up to 512 tiles:
// 32 x 4096 -> 8224 9.0 us as it is and 10.4 so, 128 x 4096 -> 4000 9.1 and 10.0, 16 x 4096 -> 12000 9.4 and 10.1, but 96 x 4096 -> 4096 9.7 and 8.8,
// 64 x 1152 -> 4608 5.1 and 4.4, 96 x 1152 -> 3456 5.1 and 4.6.)
Mx4Choice choose_mx4_gemm(int M, int N, int K, int num_cus) {
    const float lines = (float)((K + 255) / 256);
    const int turns = ((int)lines + 7) / 8;
    Mx4Choice best{0, 0, false};
    float least = 0;
    auto consider = [&](int t, int c, bool divide, int resident, float start, float each) {
        const long tiles = ((long)M + t - 1) / t * (((long)N + c - 1) / c), slots = (long)resident * num_cus;
        if (divide && tiles * 512 >= 1l << 32) return;       // (HIP takes less than 2^32 threads; the others are persistent)
        const float cost = start + (float)((tiles + slots - 1) / slots) * each;
        if (best.tile_t && cost >= least) return;
        best = {t, c, divide};
        least = cost;
    };
    // (rows that are no whole 16-byte pieces leave piece by piece, which the largest tile has no registers for)
    if (N % 8 == 0 && N < 1 << 21) consider(256, 256, false, 1, 1.5f, 2.0f * lines + 3.0f);
    consider(128, 128, false, 2, 1.5f, 1.1f * lines + 2.7f);
    consider(64, 128, false, 2, 1.5f, 0.9f * lines + 1.7f);
    consider(32, 32, true, 1, 1.0f, 0.8f + 0.02f * 64 * turns);
    consider(48, 48, true, 1, 1.0f, 0.8f + 0.02f * 96 * turns);
    consider(32, 64, true, 1, 1.0f, 0.8f + 0.02f * 96 * turns);
    return best;
}

// In one launch every workgroup quantizes the tokens once more: M rows, eight lines of K at a time, and again for every 16384 channels
// (workgroups that the chip holds at a time).  us in one launch / in two, captured: 1 x 1152 -> 3456 2.8 / 5.3, 1 x 4096 -> 4096 3.8 / 6.3,
// 8 x 4096 -> 4096 5.7 / 6.6, 16 x 1152 -> 1152 4.8 / 5.9, 1 x 4096 -> 32768 14.1 / 17.5; beyond the rule 16 x 4096 -> 4096 7.9 / 6.8,
// 16 x 4608 -> 1152 9.8 / 7.6.
bool small_mx4_layer(int M, int N, int K) {
    const long turns = (K + 2047) / 2048, rounds = ((long)N + 16383) / 16384;
    return M <= 16 && M * turns * rounds <= 16;
}

hipError_t launch_mx4_gemm(const Mx4GemmArgs& g, int dtype, int num_cus, hipStream_t stream) {
    const Mx4Choice c = choose_mx4_gemm(g.M, g.N, g.K, num_cus);
    if (c.divide_k) return launch_mx4_gemm_lines(c.tile_t, c.tile_c, g, dtype, stream);
    if (c.tile_t == 256) return launch<Shape<4, 8, 4, 2>>(g, dtype, num_cus, stream);
    if (c.tile_t == 128) return launch<Shape<4, 4, 2, 2>>(g, dtype, num_cus, stream);
    return launch<Shape<2, 4, 2, 2>>(g, dtype, num_cus, stream);
}

}  // namespace vq

extern "C" void vq_internal_mx4_choice(int M, int N, int K, int num_cus, int choice[3]) {
    const vq::Mx4Choice c = vq::choose_mx4_gemm(M, N, K, num_cus);
    choice[0] = c.tile_t;
    choice[1] = c.tile_c;
    choice[2] = c.divide_k;
}

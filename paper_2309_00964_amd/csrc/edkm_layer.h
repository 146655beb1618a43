// Internal declarations of the layer and optimizer operators: the products with
// 16-bit or palettized weights, the palette read-back and the AdamW step.
#pragma once
#include "edkm_internal.h"
#include "edkm_launch.h"

namespace edkm {

enum Activation : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3, ACT_COUNT = 4 };

// How an operand of a product lies in memory.  `row` is its output index (a token,
// an output feature), `depth` the index that is summed over.
enum Operand : int {
    OP_ROWS = 0,   // [row][depth], depth contiguous
    OP_DEPTH = 1,  // [depth][row], rows contiguous
    OP_PALETTE = 2 // [row][depth] as packed b-bit indices into a table
};

// out[r][c] = epilogue(sum_d a(r, d) b(c, d)); 16-bit operands of one format, fp32 sums.
struct ProductArgs {
    const uint16_t* a;
    const uint16_t* b;
    int64_t lda, ldb;       // elements between two rows of memory
    int32_t rows, cols, depth;
    // OP_PALETTE
    const uint8_t* idx;
    const float* lut;
    uint64_t idx_bytes;
    int bits;
    // epilogue: y = act(sum + bias[c]) + res[r][c]; z = sum + bias (nullable)
    const uint16_t* bias;
    const uint16_t* res;
    int64_t ldr;
    uint16_t* out;
    int64_t ldo;
    uint16_t* z;
    int act;
    int padded;             // OP_ROWS operands hold zeros up to the next multiple of eight depths
    // a split product: steps of 64 depths per part, and the parts' sums (null: not split)
    int split_steps;
    float* part;
    uint32_t first;         // the launch's first workgroup
};

// Whether a forward goes to k_few, which takes up to 64 tokens: always up to 16; past them,
// where every workgroup reads all tokens, only while those are no larger than given here.
// Measured (us, k_few against the tiles, bf16 and 3 bits): 32 x 4096 x 4096 12.7 (17.1) and
// 10.5 (17.6), 64 x 4096 x 4096 20.3 (15.9) and 18.0 (18.6), 48 x 11008 x 4096 25.6 (22.7) and
// 19.1 (26.6), 32 x 4096 x 11008 30.9 (25.5) and 22.9 (25.8), 33 x 4096 x 11008 33.2 (25.3)
// and 26.5 (29.0), 48 x 4096 x 11008 40.0 (25.6) and 34.1 (28.3).
inline bool few_tokens(int64_t rows, int64_t depth, bool palette) {
    return rows <= 16 || (rows <= 64 && rows * depth <= (palette ? 400 : 192) * 1000);
}

// Matrices to be copied to rows of whole 16-byte pieces in one launch.
struct AlignJob {
    const uint16_t* m;
    int64_t ld;
    int rows, cols;
    uint16_t* out;
};
struct AlignArgs {
    int count;
    AlignJob job[3];
};

constexpr int64_t DIRECT_LD_MOST = 1 << 22;    // of operands that go to LDS directly: a tile's offsets fit 32 bits
constexpr int SPLIT_TILE = 128;    // the only tile whose depths are ever split

// How a product is carried out.
struct ProductPlan {
    int tile;               // 256 or 128 outputs square
    int splits, split_steps;
    bool direct;            // operands can go to LDS by 16-byte pieces of memory
};
ProductPlan product_plan(const ProductArgs& p, int opa, int opb);
size_t product_part_bytes(int64_t rows, int64_t cols, int64_t depth);

// The gradient at the activation: dz = dy act'(z) (16 bits, only with an activation)
// and the bias gradient, summed over the rows of each chunk and then over the chunks.
struct DzArgs {
    const uint16_t* dy;
    int64_t lddy;
    const uint16_t* z;
    uint16_t* dz;
    int64_t lddz;           // a multiple of eight: dz's rows are followed by zeros up to it
    float* part;            // [chunks][cols]
    uint16_t* dbias;
    int32_t rows, cols;
    int act;
    int per;                // rows of a workgroup
    uint32_t first;         // the launch's first workgroup
};

constexpr int DZ_COLS = 512, DZ_ROWS_LEAST = 4, DZ_ROWS_MOST = 64;   // one workgroup's share of them
// Rows of a workgroup: as many as leave 1024 of them (four per CU).  With silu and the bias
// gradient 1001 x 1336 takes 7.4 us (11.8 by 64 rows each), 2048 x 4096 12.1 (16.7, and 14.6
// by 4 rows), 8192 x 11008 through the caches 111 (130 by 4).
inline int dz_rows(int64_t rows, int64_t cols) {
    int64_t r = DZ_ROWS_MOST;
    while (r > DZ_ROWS_LEAST && (rows + r - 1) / r * ((cols + DZ_COLS - 1) / DZ_COLS) < 1024) r /= 2;
    return (int)r;
}

enum ParamType : int { PT_FP16 = 0, PT_BF16 = 1, PT_FP32 = 2 };

struct AdamwTensor {
    void* p;
    float* master;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    uint64_t n;
};

constexpr int ADAMW_BLOCK = 256;       // elements of one 8-bit state's scale
// Elements of one workgroup: few where the tensors are small, so that all CUs take part,
// more where there are workgroups enough, so that fewer of them pay the start (8-bit states,
// us with the small and the large share: 8 tensors of 2^20 elements 24.0 and 30.7, one of
// 2^24 46.0 and 42.6, the seven of a decoder layer 433 and 383).
constexpr int ADAMW_CHUNK = 2048, ADAMW_CHUNK_MANY = 16384;
constexpr uint64_t ADAMW_MANY = 1ull << 24;

struct AdamwArgs {
    int count;
    uint32_t seed;
    int32_t* step;                     // steps done before this one
    const float* lr_dev;               // the rate on the device, or null: lr
    double lr, beta1, beta2, eps, decay;
    uint32_t chunk;                    // elements of one workgroup
    int aligned;                       // all arrays can be read and written eight elements at a time
    uint32_t wg_begin[MAXB];           // first workgroup of each tensor; 0xFFFFFFFF past them
    AdamwTensor t[MAXB];
};
static_assert(sizeof(AdamwArgs) <= 4096, "launch arguments fit the kernel-argument limit");

hipError_t launch_product(const ProductArgs& a, int fmt, int opa, int opb, float* part, hipStream_t s);
// Rows of whole 16-byte pieces of x, whole pieces of eight indices, four bytes of them at least.
hipError_t launch_tiled_palette(ProductArgs a, int fmt, float* part, hipStream_t s);
hipError_t launch_few(const ProductArgs& a, int fmt, int bits, hipStream_t s);
hipError_t launch_dz(const DzArgs& a, int fmt, hipStream_t s);
// past: by stores past the caches.
hipError_t launch_unpalettize(const uint8_t* idx, uint64_t idx_bytes, uint64_t n, int bits, int fmt, const float* lut,
                              uint16_t* out, bool past, hipStream_t s);
hipError_t launch_align_rows(const AlignArgs& a, hipStream_t s);
hipError_t launch_unpalettize_rows(const uint8_t* idx, uint64_t idx_bytes, int64_t rows, int64_t cols, int bits, int fmt,
                                   const float* lut, uint16_t* out, hipStream_t s);
hipError_t launch_adamw(const AdamwArgs& a, uint32_t grid, int param_type, int grad_type, int state_bits, hipStream_t s);
hipError_t launch_adamw_tick(int32_t* step, hipStream_t s);

}  // namespace edkm

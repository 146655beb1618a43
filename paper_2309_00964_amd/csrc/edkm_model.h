// Internal declarations of the operators at a model's ends and between its blocks: the
// embedding, the norms around a block and the cross entropy of a product.
#pragma once
#include "edkm_layer.h"

#include <algorithm>

namespace edkm {

enum IndexType : int { IDX_32 = 0, IDX_64 = 1 };

// ----------------------------------------------------------------------------
// embedding

struct EmbedArgs {
    uint32_t first;         // the launch's first workgroup
    const void* ids;
    const uint16_t* table;
    int64_t ldt;
    const uint8_t* idx;     // a palette's
    const float* lut;
    uint64_t idx_bytes;
    uint16_t* y;
    int64_t ldy;
    int64_t m;
    uint32_t v, d;
    uint32_t rows;          // tokens of a workgroup
    float scale;
};

// Tokens sorted by their row of the table, in order within a row (no token: row v, last).
struct SortArgs {
    uint32_t first;
    const void* ids;
    const uint32_t *key_in, *pos_in;    // the pass before's; null: the ids
    uint32_t *key, *pos;
    uint32_t* counts;       // [groups][digits]
    uint32_t m, v, per, groups, shift, digits;
};

struct EmbedGradArgs {
    uint32_t first;
    const uint32_t *key, *pos;
    const uint16_t* dy;
    int64_t lddy;
    uint16_t* dt;
    int64_t lddt;
    float* part;            // [chunks][2][up8(d)]
    uint32_t m, v, d, per, chunks;
    uint32_t chunk_groups;  // workgroups that sum; those after them write the rows of no token
    uint32_t zero_rows;     // ... so many rows each
    uint32_t lanes;         // log2 of the threads side by side that join
    float scale;
    int accumulate, past;
};

// Tokens that one launch ranks by comparing all with all (256 workgroups of 32, 67M
// comparisons: 10 us; 8000 tokens' gradient added to 32000 x 256 24.0 us, by digits 32.3), and that a
// digit's pass takes for a workgroup, at least.
constexpr int64_t RANK_MOST = 8192;
constexpr int RANK_TOKENS = 32, PLACE_LEAST = 1024, PLACE_GROUPS = 512, DIGIT_BITS = 10;
// Tokens of a chunk that one thread sums for its eight columns: from eight, so that there are
// threads enough, over sixteen from 16M values or 32768 tokens on to 64 at 256M, the more the fewer
// parts are joined (gradients added to a table, us by 8, 16, 32 and 64: 2000 tokens of 2000 x 512 14.3,
// 18.9, 24.9 and 39.9; 100000 of 40000 x 70 66, 71, 86 and 126; 8192 of 32000 x 4096 49.7, 46.7, 49.4 and
// 62.8; 131072 of 100000 x 1000 171, 147, 135 and 143; 65536 of 50000 x 4096 253, 204, 187 and 180).  And rows
// that one workgroup looks up to write those of no token: of 8192 values, 16 to 256 (gradients written, us
// by 8192, 32768 and 262144 values: 8192 tokens of 32000 x 256 25, 38 and 56, 20000 of 50000 x 1000 61, 60
// and 178; by 4096 that of 32000 x 256 takes 26, and 3000 of 300000 x 32 22 both ways).
constexpr int CHUNK_LEAST = 8, CHUNK_MANY = 16, CHUNK_MOST = 64, CHUNKS_FEW = 2048, ZERO_VALUES = 8192, ZERO_LEAST = 16, ZERO_MOST = 256;
constexpr int64_t CHUNK_ELEMENTS = 1 << 24;

struct SortPlan {
    int passes, width;      // digits' number and bits; 0 passes: ranked
    uint32_t per, groups;
};
inline SortPlan sort_plan(int64_t m, int64_t v) {
    SortPlan q{};
    if (m <= RANK_MOST) return q;
    int bits = 1;
    while (v >> bits) ++bits;           // keys are 0 .. v
    q.passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
    q.width = (bits + q.passes - 1) / q.passes;
    int64_t per = (m + PLACE_GROUPS - 1) / PLACE_GROUPS;
    if (per < PLACE_LEAST) per = PLACE_LEAST;
    q.per = (uint32_t)((per + 255) / 256 * 256);
    q.groups = (uint32_t)((m + q.per - 1) / q.per);
    return q;
}
inline uint32_t chunk_tokens(int64_t m, int64_t d) {
    const int64_t few = m * d > CHUNK_ELEMENTS || m / CHUNKS_FEW > CHUNK_MANY ? CHUNK_MANY : m / CHUNKS_FEW;
    const int64_t many = m * d / (CHUNK_ELEMENTS / 4), per = few > many ? few : many;
    return (uint32_t)(per < CHUNK_LEAST ? CHUNK_LEAST : per > CHUNK_MOST ? CHUNK_MOST : per);
}

hipError_t launch_embed(EmbedArgs a, int fmt, int index_type, int bits, hipStream_t s);
// key/pos: the sorted tokens' arrays; spare: two more of m, between passes
hipError_t launch_sort(const void* ids, int index_type, int64_t m, int64_t v, uint32_t* key, uint32_t* pos, uint32_t* spare,
                       uint32_t* counts, hipStream_t s);
hipError_t launch_embed_grad(EmbedGradArgs a, int fmt, hipStream_t s);

// ----------------------------------------------------------------------------
// norms

struct NormArgs {
    uint32_t first;
    const uint16_t *r, *u, *w, *post, *gate;
    int64_t ldr, ldu, ldg;
    int gate_rows;
    float scale, eps;
    uint16_t *h, *y;
    int64_t ldh, ldy;
    int64_t m;
    int n;
    // backward
    const uint16_t *dy, *dh;
    int64_t lddy, lddh;
    uint16_t *dr, *du, *dw, *dpost, *dgate;
    int64_t lddr, lddu;
    float* part;            // [groups][2][n]
    uint32_t groups;
};
uint32_t norm_groups(int64_t m, int64_t n);      // workgroups of a backward
hipError_t launch_norm(NormArgs a, int fmt, hipStream_t s);
hipError_t launch_norm_backward(NormArgs a, int fmt, hipStream_t s);

// ----------------------------------------------------------------------------
// cross entropy of a product

enum Reduction : int { RED_NONE = 0, RED_SUM = 1, RED_MEAN = 2, RED_COUNT = 3 };

// What the tokens with a target (in a backward: and a gradient other than 0) have, in order and without gaps.
struct LossRows {
    int32_t* count;         // [2]: how many there are
    float* alpha;           // [2] backward: what dz is a share of, as a product
    int32_t* row;           // [m] the token
    int32_t* word;          // [m] its target
    int32_t* slot;          // [m] backward: a token's place among them, -1 for none
    float* value;           // [m] forward: its target's logit, then its loss; backward: dz's factor
};

struct PickArgs {
    const void* targets;
    int64_t m, n;
    int reduction;
    LossRows r;
    float *loss, *lse;      // forward: zeros for tokens without a target
    const float* dloss;     // backward; may be null without tokens
    int backward;
};

// x's rows of those tokens, one after another with zeros up to ldo; nothing if all tokens
// have a target and x can be used as it is.  zero: rows of tokens without a target to clear.
struct GatherArgs {
    uint32_t first;
    LossRows r;
    const uint16_t* x;
    int64_t ldx;
    uint16_t* out;
    int64_t ldo;
    int64_t m;
    int k;
    int always;
    uint16_t* zero;
    int64_t ldz;
};

// How one of a loss's products is carried out.
struct LossPlan {
    int tile;               // outputs square: 256, 128 or SMALL
    int splits, split_steps;
    int groups;             // workgroups of a launch that splits the depths among them; 0: a workgroup to a tile
    bool direct;
};
constexpr int SMALL = 64, PART_STEPS = 8;
LossPlan loss_plan(int64_t rows, int64_t cols, int64_t depth, bool direct);
// Bytes of the parts' sums, whatever the operands' alignment.
size_t loss_part_bytes(int64_t rows, int64_t cols, int64_t depth);

struct LossArgs : ProductArgs {
    int splits;
    int groups, tile;       // workgroups of a launch that finds its splits by itself, and its tile; or 0
    LossRows rows_of;
    const uint16_t* all;    // x itself, where it can be used; else null
    int64_t ld_all;
    int32_t m, base;        // tokens in all; the first row of this launch
    int dynamic;            // what the count of tokens is here: 1 the rows, 2 the depths, 0 nothing (no list)
    const void* targets;    // without a list
    int index_type;
    // statistics: per 64 words and row the largest logit and the sum of exponentials
    float2* stats;
    int32_t stat_rows;
    int32_t col0;           // the first word of this launch
    const float* lse;
    // sums over several launches
    float* accum;
    int begins, ends, scatter;
};

struct LossEndArgs {
    LossRows r;
    const float2* stats;
    int32_t stat_rows, blocks, base, rows;
    int reduction;
    const void* targets;    // without a list of tokens
    int index_type;
    int64_t words;
    int whole;              // one workgroup has all rows, and sums them up
    float *loss, *lse;
};

hipError_t launch_pick(const PickArgs& a, int index_type, hipStream_t s);
hipError_t launch_gather(GatherArgs a, hipStream_t s);
// The two and the copy of w's rows (w.rows 0: none) in one, for 1 to ONE_LIST tokens (slot is not written).
hipError_t launch_pick_gather(const PickArgs& a, const GatherArgs& g, const AlignJob& w, int index_type, hipStream_t s);
hipError_t launch_loss_stats(const LossArgs& a, int fmt, const LossPlan& q, hipStream_t s);
hipError_t launch_loss_dz(const LossArgs& a, int fmt, const LossPlan& q, hipStream_t s);
hipError_t launch_loss_sum(const LossArgs& a, int fmt, int opa, const LossPlan& q, hipStream_t s);
hipError_t launch_few_loss(const LossArgs& a, int fmt, hipStream_t s);
hipError_t launch_loss_end(const LossEndArgs& a, hipStream_t s);
hipError_t launch_loss_reduce(const LossEndArgs& a, hipStream_t s);

// Words of a piece of the vocabulary whose dz is held at a time: as many as keep it within half
// the Infinity Cache, which the two products that read it then hit; 2048 at least.  The gradients of 8192 x
// 32000 x 4096 take 5280-5340 us by 64 MiB, 5140-5180 by 128 and 5230-5270 by 256, of which a quarter does not
// count 4560, 4130-4160 and 4160: 64 is too little, and above 128 there is no more to gain.
constexpr int64_t DZ_BYTES = 128 << 20, DZ_LEAST = 2048;
inline int64_t loss_piece(int64_t m, int64_t n) {
    int64_t p = DZ_BYTES / (2 * (m > 0 ? m : 1));
    if (p < DZ_LEAST) p = DZ_LEAST;
    if (p >= n) return n;
    const int64_t pieces = (n + p - 1) / p;
    return (((n + pieces - 1) / pieces) + 255) / 256 * 256;
}
// Tokens up to which a forward makes no list of those with a target: it would be a launch more
// (512 x 32000 x 4096 takes 119 us without, 124 with), and leaving out a quarter of the tokens pays
// where it saves the tiles a round over the CUs (1000 x 32000 x 4096 213 and 210, of 131072 x 2048 472 and
// 371).  At most 1024, which k_loss_reduce has threads for.
constexpr int64_t LIST_LEAST = 1024, ONE_LIST = 8192;
// Tokens up to which each workgroup takes sixteen words for all tokens: it is bound by the words'
// bytes, but up to sixteen tokens share a wave's loads of x, and its time grows with them (losses
// of 32000 x 4096, us by it and by the tiles: 1 token 50 and 58, 8 tokens 56 and 58, 16 tokens 68 and
// 58; of 131072 x 2048 108 and 124, 128 and 124, 140 and 126; their mean over 300 x 64 8 and 9 to 12).  The tiles
// need a copy of w where k is no multiple of eight, so there it is up to sixteen (1003 x 777 11.5 and 14 us,
// 9000 x 1500 22 and 29, 50001 x 1001 64 and 61).
constexpr int64_t LOSS_FEW = 16, LOSS_FEW_WHOLE = 8;
inline bool loss_few(int64_t m, int64_t k) { return m > 0 && m <= (k % 8 ? LOSS_FEW : LOSS_FEW_WHOLE); }
// Tokens of a forward's launch: as many as keep the statistics within 256 MiB, 256 at least.
inline int64_t loss_rows(int64_t m, int64_t n) {
    const int64_t blocks = (n + 63) / 64, r = (256 << 20) / (blocks * 8) / 256 * 256;
    return m < 256 || m < r ? m : r < 256 ? 256 : r;
}

}  // namespace edkm

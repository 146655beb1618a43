// Argument checks and workspace arithmetic that the layer and model operators share (host).
#pragma once
#include "../../include/edkm.h"
#include "edkm_layer.h"

#include <algorithm>

namespace edkm {

constexpr int64_t DIM_MAX = 0x7FFFFFFF - 1024;   // sizes are 32-bit in the kernels, tile ends included

constexpr int64_t MATRIX_MAX = (int64_t)1 << 40;     // elements of a matrix: its tiles are numbered in 32 bits

inline bool size_ok(int64_t v, int64_t least) { return v >= least && v <= DIM_MAX; }

inline bool product_ok(int64_t m, int64_t n, int64_t k, int format, int act) {
    return size_ok(m, 0) && size_ok(n, 1) && size_ok(k, 1) && std::max(m, k) <= MATRIX_MAX / n && m <= MATRIX_MAX / k && (format == EDKM_KEYS_FP16 || format == EDKM_KEYS_BF16) &&
           act >= 0 && act < ACT_COUNT;
}

// Leading dimension of a matrix with `rows` rows of `cols`: any for a single row, which
// then gets one that the kernels can work with.
inline bool ld_ok(int64_t& ld, int64_t rows, int64_t cols) {
    if (rows <= 1) ld = (cols + 7) & ~(int64_t)7;
    return ld >= cols && ld < (int64_t)1 << 40;
}

inline size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

inline int64_t up8(int64_t v) { return (v + 7) & ~(int64_t)7; }

// Rows whose length is no multiple of eight cannot be loaded by 16-byte pieces: a product
// first copies them to rows that can.
inline size_t aligned_bytes(int64_t rows, int64_t cols) { return cols % 8 ? up256((size_t)rows * up8(cols) * 2) : 0; }

// Has a matrix's rows copied to `to`, and points there.
inline void copy_rows(AlignArgs& a, const uint16_t*& p, int64_t& ld, int64_t rows, int64_t cols, char* to) {
    uint16_t* out = reinterpret_cast<uint16_t*>(to);
    a.job[a.count++] = {p, ld, (int)rows, (int)cols, out};
    p = out;
    ld = up8(cols);
}
// The same, if their length asks for it.
inline void align_rows(AlignArgs& a, const uint16_t*& p, int64_t& ld, int64_t rows, int64_t cols, char* to) {
    if (cols % 8 && rows > 0) copy_rows(a, p, ld, rows, cols, to);
}

inline edkm_status ws_ok(const void* ws, size_t have, size_t need) {
    if (need == 0) return EDKM_OK;
    return !ws || have < need || ((uintptr_t)ws & 255u) ? EDKM_ERR_WORKSPACE : EDKM_OK;
}

}  // namespace edkm

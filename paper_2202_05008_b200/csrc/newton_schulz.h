// What the Newton-Schulz kernels share with the host code: the list of matrices of a launch, the scales of the
// fp16 pairs, and the sizes of the buffers.  No device code.
#pragma once
#include <cmath>
#include <cstddef>
#include <cstdint>

namespace evo {
namespace ns {

// The tensor core cuts its sums off instead of rounding them, always towards zero: sums of squares come out short by kCut per MMA
// (A X of random matrices, one step: -6.1e-8 with one MMA a sum, -4.6e-7 with 8, -9.4e-7 with 16; 2048^2 was 1.6e-5 off after five
// steps with all products in one accumulator, a chain of fp32 torch products 3.6e-6).  So the small products have an accumulator of
// their own, the large ones' is taken out and added up in registers every kChunk of the contracted index, and what A's sums lack on
// average is given back: 2048^2 1.2e-6, 929 x 2,437 2.4e-6 (256 instead of 128: 2.2e-6 and 4.4e-6, 4 % faster).
constexpr uint32_t kChunk = 128;
constexpr float kCut = 5.7e-8f;

// What a matrix is made from, and what becomes of the result: a plain matrix of one of three types, or the gradient of a flat
// parameter vector (its momentum is updated on the way in, the centre on the way out).
enum Source : uint32_t { kF32 = 0, kBf16 = 1, kF16 = 2, kMuon = 3 };

constexpr uint32_t kMaxGroups = 32;      // groups of a launch; longer lists take several
constexpr uint32_t kMaxLarge = 16;       // ... of large matrices (each comes with its tensor maps)
constexpr uint32_t kTile = 128;          // rows and columns of a tile of the kernels for large matrices
constexpr uint32_t kPieceCols = 64;      // columns of a piece of the kernels that read the matrix (128 rows)

// `count` equal matrices.  The iteration works on the m x n matrix with m <= n: the matrix itself, or its transpose where it is
// taller than wide.
struct Group {
    uint64_t in, out;                    // element index of the first matrix in the source and the result
    uint64_t in_stride, out_stride;      // ... and from one matrix to the next
    uint64_t work;                       // large: byte offset of the first matrix' buffers in the workspace
    uint32_t in_ld, out_ld;              // row pitches
    uint32_t m, n, mp, np;               // m <= n, and what they are padded to (small: 16 and 16, np of a block's share; large: 128 and 64)
    uint32_t tall, count, first_matrix;
    uint32_t first_block;                // of this group among the blocks of the launch (small) or the pieces (large)
    uint32_t first_pair, first_tile;     // large: among the tiles on and under the diagonal, and among those of an m x n matrix
    float    gain;                       // Muon: lr x 0.2 sqrt(max(rows, cols))
};

struct Scalars {
    float a, b, c, eps;
    uint32_t steps;
    // x, A and B are carried times these powers of two, as large as fp16 lets them be
    float s_x, s_a, s_b;
    uint32_t growth;                     // a step makes no singular value more than 2^growth times as large
    // Muon
    float mu, rest, keep;                // rest = 1 - mu, keep = 1 - lr x decay
    uint32_t nesterov;
};

struct Args {
    const void* in;                      // matrices, or the gradient vector
    void* out;                           // matrices, or the new centre
    const float* m_in; float* m_out; const float* v_in; float* v_out; const float* c_in;      // Muon
    const double* skip;                  // Muon inside a tell: nothing is done where *skip is 0 (NULL: always)
    // Set in all launches of a Muon step but the first (one launch per product has none): the matrices have nothing in common, so a
    // launch need not wait for the one before it, and does so only at its end, which keeps the completions in order.  It starts when every block of
    // the one before has seen everything ahead of the step complete; what may be old in an SM's L1 by then is read from L2.
    // (28-128-128-8: 78 us without, 57 with)
    uint32_t late;
    char* work;
    double* partial;                     // large: sums of squares per piece
    uint32_t* sticky;                    // where a wait that ran out is noted (NULL: nowhere; what depends on it is NaN in any case)
    uint32_t wait_log2;
    uint32_t drop;                       // EVO_DEBUG_DROP_COMPLETION: block 0 leaves out the first commit that it waits for
    size_t partial_at, lift_at;          // byte offsets of the two in the workspace
    uint32_t* lift;                      // large: per matrix of the launch, see first_scale
    uint32_t groups, blocks, pairs, tiles, cluster;
    Scalars s;
    Group g[kMaxGroups];
};

// The largest power of two up to 2^15 that keeps `bound` (with room for what rounding adds) below fp16's largest number.
inline float scale_for(double bound)
{
    int e = 0;
    std::frexp(65504.0 / (1.03125 * bound), &e);
    return static_cast<float>(std::ldexp(1.0, (e - 1 < 15 ? e - 1 : 15)));
}

// Follows the largest singular value that `steps` of s -> a s + b s^3 + c s^5 can reach from [0, 1], and sets the scales from it.
// False where that grows beyond 64 (fp16 pairs would no longer carry the small singular values) or is no number.
inline bool set_scales(Scalars* s)
{
    const double a = s->a, b = s->b, c = s->c;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + c * x * x))); };
    double top = 1.0, most = 1.0;
    for (uint32_t k = 0; k < s->steps; ++k) {
        double next = f(top);
        double z[2] = { -1.0, -1.0 };                     // squares of the stationary points: 5 c z^2 + 3 b z + a = 0
        if (c != 0.0) {
            const double d = 9.0 * b * b - 20.0 * a * c;
            if (d >= 0.0) { z[0] = (-3.0 * b + std::sqrt(d)) / (10.0 * c); z[1] = (-3.0 * b - std::sqrt(d)) / (10.0 * c); }
        } else if (b != 0.0) {
            z[0] = -a / (3.0 * b);
        }
        for (double q : z)
            if (q > 0.0 && q < top * top && f(std::sqrt(q)) > next) next = f(std::sqrt(q));
        if (!(next <= 64.0)) return false;
        top = next;
        if (top > most) most = top;
    }
    const double r = most * most;                         // largest eigenvalue of A
    double poly = std::fabs(b * r + c * r * r), grow = std::fabs(a + b * r + c * r * r);
    if (std::fabs(a) > grow) grow = std::fabs(a);
    if (c != 0.0) {
        const double q = -b / (2.0 * c);
        if (q > 0.0 && q < r) {
            if (std::fabs(b * q + c * q * q) > poly) poly = std::fabs(b * q + c * q * q);
            if (std::fabs(a + b * q + c * q * q) > grow) grow = std::fabs(a + b * q + c * q * q);
        }
    }
    if (!(poly <= 1048576.0)) return false;
    s->growth = grow > 1.0 ? static_cast<uint32_t>(std::ceil(std::log2(grow * 1.0001))) : 0u;
    s->s_x = scale_for(most);
    s->s_a = scale_for(r);
    s->s_b = scale_for(poly > 1e-30 ? poly : 1e-30);
    return true;
}

// The kernel for matrices of one or two sixteens of rows: columns of a block (16 warps with four or two sixteens each), in clusters of
// 1, 2, 4 or 8 blocks.
constexpr uint32_t tiny_columns(uint32_t row_tiles) { return 1024u / row_tiles; }

// The kernel for small matrices: up to 128 rows, and 128 columns a block of a cluster of 1, 2, 4 or 8.
constexpr uint32_t kSmallRows = 128, kSmallCols = 128, kMostBlocks = 8;
constexpr size_t kSmallBytes = 200u * 1024u;
// Shared memory of a block: X as a pair of fp16 matrices, A or B as one, the other blocks' parts of A, and what a product reads beyond the last row
inline size_t small_bytes(uint32_t mp, uint32_t np, uint32_t blocks)
{
    const size_t eights = mp / 8u;
    return static_cast<size_t>(mp) * np * 4u + static_cast<size_t>(mp) * mp * 4u +
           (blocks > 1u ? (eights + blocks - 1u) / blocks * blocks * mp * 32u : 0u) + 2048u;
}
// Which kernel takes `count` m x n matrices, and how many blocks of a cluster each.
enum Kind : uint32_t { kTiny16 = 0, kTiny32 = 1, kSmall = 2, kLarge = 3 };
struct Choice { uint32_t kind, blocks; };
constexpr uint32_t kTogether = 148;      // blocks of the kernel for small matrices that run at the same time, one an SM
inline Choice cluster_for(uint32_t kind, uint32_t n)
{
    const uint32_t cols = kind == kSmall ? kSmallCols : tiny_columns(kind + 1u);
    for (uint32_t b = 1; b <= kMostBlocks; b *= 2u)
        if (n <= b * cols) return Choice{ kind, b };
    return Choice{ kLarge, 0u };
}
inline Choice choose(uint32_t m, uint32_t n, uint32_t count)
{
    if (m <= 16u) return cluster_for(kTiny16, n);
    if (m > kSmallRows) return Choice{ kLarge, 0u };
    if (m > 32u) return cluster_for(kSmall, n);
    // 17 to 32 rows in registers / in shared memory, us: 32 x 32 25 / 16.6, 28 x 128 21.6 / 22.1; 20 x 160 27.1 / 30.1, 32 x 256 32.2 / 32.9; 32 x 384 38.9 / 33.0,
    // 24 x 700 74 / 35, 12 of them 76 / 36, 24 of them 76 / 70.  Blocks of the second hold a quarter of the columns, so it falls behind where they
    // do not all run at once: 40 of 20 x 300 35.5 / 63.7, 300 of 24 x 600 349 / 682.  Beyond 1,024 columns the other side is a launch per product: 32 x 1,100 95 / 171.
    const Choice shared = cluster_for(kSmall, n);
    const bool registers = n > kSmallCols && (n <= 2u * kSmallCols || shared.kind == kLarge || static_cast<uint64_t>(shared.blocks) * count > kTogether);
    return registers ? cluster_for(kTiny32, n) : shared;
}

// Buffers of a large matrix in the workspace, each a matrix of high parts followed by one of low parts: X, the next X, A, B.
inline size_t x_bytes(uint32_t mp, uint32_t np) { return static_cast<size_t>(mp) * np * 4u; }
inline size_t a_bytes(uint32_t mp) { return static_cast<size_t>(mp) * mp * 4u; }
inline size_t large_bytes(uint32_t mp, uint32_t np) { return 2u * x_bytes(mp, np) + 2u * a_bytes(mp); }

}  // namespace ns
}  // namespace evo

// Which kernel multiplies the matrices of a launch of orthogonal.hip, and how much scratch they take.  Plain C++, so that the same lines run in the launcher and in a test
// on the host.
#pragma once
#include <math.h>
#include <stddef.h>

#include <algorithm>

namespace dr {

constexpr int NS_JOBS = 64;                  // most matrices of a launch
constexpr int NS_BLOCK = 1024;               // bytes of a block of 32 rows x 16 k of one piece of an operand
constexpr int SQUARES = 1024;                // most workgroups (and partial sums of squares) of a matrix
enum { GRAM = 0, POLY = 1, APPLY = 2, PRODUCTS = 3 };

// partial sums of squares of a matrix: workgroups of 256 threads, 16 elements each and more
constexpr int squares_of(int rows, int cols)
{
    return (int)std::min<size_t>(SQUARES, ((size_t)rows * cols + 4095) / 4096);
}

// Scales of the fp16 pieces of X and of A and Q, and whether those suffice: no element of X, A = X X^T or Q = a I + b A + c A A may pass 65504 by far.  Elements are at
// most the largest singular value, 1 at the start (|X|_F <= 1), which each step takes to at most the largest |a s + b s^3 + c s^5| of s up to it; that of Q is at most the
// largest |a + b t + c t^2| of t = s^2.  Beyond 3, 9 and 12 (a quarter left for roundings) the pieces are of bf16, three of them.
// growth, spare: a step multiplies a singular value by 2^(growth - spare) at most; growth is whole, spare below one of it, or what a polynomial below one takes away.
// Small values grow by |a|: where that is so much less that the steps together would take more than two bits from what X's scale leaves them, or where Q is so small
// itself that fp16's lower pieces end above its 2^-33, bf16 as well.
constexpr float NS_X_SCALE = 16384.f, NS_A_SCALE = 4096.f;
inline bool stays_small(int steps, double a, double b, double c, int* growth, float* spare = nullptr)
{
    double most = 1.0, fastest = 0.0;
    *growth = 0;
    for (int i = 0; i < steps; ++i) {
        const double end = most * most;
        double x = 0, q = fabs(a);
        auto look = [&](double t) {
            if (!(t >= 0 && t <= end)) return;
            q = std::max(q, fabs(a + b * t + c * t * t));
            x = std::max(x, sqrt(t) * fabs(a + b * t + c * t * t));
        };
        look(end);
        if (c != 0) {
            look(-b / (2 * c));                                      // where the derivative of Q's is zero
            const double d = 9 * b * b - 20 * a * c;                 // ... of X's: a + 3 b t + 5 c t^2 = 0
            const double far = -3 * b - copysign(sqrt(d), b);        // (a sum without cancellation: c may be nearly nothing beside b)
            if (d >= 0) { look(far / (10 * c)); if (far != 0) look(2 * a / far); }
        } else if (b != 0) look(-a / (3 * b));
        if (!(x <= 3 && q <= 12)) return false;
        fastest = std::max(fastest, q * 1.001);
        most = x * 1.001;                                            // (roundings)
    }
    if (!(fabs(a) >= 1.0 / 16 && steps * log2(fastest / fabs(a)) <= 2.0)) return false;
    while (fastest > (1 << *growth)) ++*growth;
    if (spare) *spare = (float)(*growth - log2(fastest));
    return true;
}

// A matrix whose norm is far below eps starts from an X as small, which fp16 does not hold: it is held multiplied by 2^shift, at step k by 2^(what is left), as much less as
// the steps before may have multiplied it by (in whole bits of all of them together: of each by itself, forty steps of a polynomial near one would take forty bits)
constexpr int held_at(int shift, int growth, float spare, int step)
{
    const int left = shift - growth * step + (int)(spare * (float)step);
    return left > 0 ? left : 0;
}

// matrices that fit the LDS of one workgroup: blocks of 32 of the short and of the long side
constexpr bool whole_fits(int mb, int nb) { return mb == 1 ? nb <= 28 : mb == 2 && nb <= 11; }

// a matrix whose products Q and Q X may be one launch has as many blocks of 32 rows at most
constexpr int NS_JOINED_ROWS = 8;

// blocks of 32 x 32 that a launch may have: its workgroups of 512 threads are counted in 32 bits
constexpr double NS_MOST_BLOCKS = 8388607;

// Kernels for a product, by the blocks of a tile's side; k-blocks that a wave of the first two has in flight, and their waves
enum { FINE, DIRECT, TILE4, TILE6, TILE8, KERNELS };
constexpr int SIDE[KERNELS] = {1, 2, 4, 6, 8}, AHEAD[] = {4, 1}, WAVES[] = {8, 8};

inline int tiles_of(int what, int mb, int nb, int T)
{
    const int tm = (mb + T - 1) / T, tn = (nb + T - 1) / T;
    return what == APPLY ? tm * tn : tm * (tm + 1) / 2;
}

// What one launch of a product has to do: tiles and tiles x k-blocks for each side of a tile, the longest contraction
struct Work {
    int tiles[KERNELS], longest;
    double blocks[KERNELS];
    void add(int what, int mb, int nb)
    {
        const int kblocks = 2 * (what == GRAM ? nb : mb);
        longest = std::max(longest, kblocks);
        for (int k = 0; k < KERNELS; ++k) {
            const int n = tiles_of(what, mb, nb, SIDE[k]);
            tiles[k] += n;
            blocks[k] += (double)n * kblocks;
        }
    }
};

// Microseconds that a launch takes, from 36 square and oblong shapes of 64 to 4096 rows with either number of pieces (of bf16 then, which multiply as fast): what a round of workgroups costs beside its products;
// a k-block on a compute unit by itself; what all of them multiply together, in blocks of 32 x 32 x 16 a microsecond; workgroups per compute unit.
struct Cost { float round, kblock, rate; int slots; };
constexpr Cost COSTS[2][KERNELS] = {
    {{3.f, 0.065f, 3900.f, 1}, {5.f, 0.2f, 5100.f, 1}, {7.f, 0.42f, 6600.f, 2}, {12.f, 0.8f, 7450.f, 1}, {18.f, 1.45f, 7150.f, 1}},           // three pieces
    {{2.6f, 0.045f, 5700.f, 1}, {4.f, 0.12f, 8500.f, 1}, {5.5f, 0.24f, 10200.f, 2}, {9.f, 0.45f, 12700.f, 1}, {12.5f, 0.8f, 13900.f, 1}},     // two
};
inline float cost_of(int P, int kernel, double tiles, double blocks, double longest, int cus)
{
    const Cost& c = COSTS[P == 3 ? 0 : 1][kernel];
    const double area = SIDE[kernel] * SIDE[kernel], slots = (double)c.slots * cus, each = blocks / tiles;
    const double full = floor(tiles / slots), rest = tiles - full * slots;
    auto time = [&](double n) { return n > 0 ? c.round + std::max(each * c.kblock, n * each * area / (c.rate * cus / 256.0)) : 0.0; };
    return (float)(1.0 + std::max(full * time(slots) + time(rest), (double)c.round + longest * c.kblock));
}

struct Choice { int kernel, splits; };
inline Choice choose(int P, int what, const Work& w, int cus)
{
    Choice best{FINE, 1};
    float least = 0.f;
    for (int k = 0; k < KERNELS; ++k) {
        const float t = cost_of(P, k, w.tiles[k], w.blocks[k], w.longest, cus);
        if (k == 0 || t < least) { least = t; best = Choice{k, 1}; }
    }
    if (what != GRAM) return best;
    // few tiles of long rows: up to a workgroup per compute unit, with as many k-blocks for each as its waves have in flight at least; the sums take a launch of 4 us
    for (int k = FINE; k <= DIRECT; ++k) {
        const int splits = std::min(cus / std::max(w.tiles[k], 1), w.longest / (WAVES[k] * AHEAD[k]));
        if (splits < 2) continue;
        const float t = 4.f + cost_of(P, k, (double)w.tiles[k] * splits, w.blocks[k], (double)w.longest / splits, cus);
        if (t < least) { least = t; best = Choice{k, splits}; }
    }
    return best;
}
inline size_t partial_bytes(const Choice& c, const Work& w) { return c.splits > 1 ? (size_t)w.tiles[c.kernel] * c.splits * SIDE[c.kernel] * SIDE[c.kernel] * 1024 * sizeof(float) : 0; }

// Operands of a matrix: X, X^T twice, A, Q
inline size_t operand_bytes(int mb, int nb, int P) { return ((size_t)3 * mb * nb + (size_t)2 * mb * mb) * 2 * P * NS_BLOCK; }

// The matrices that one sequence of launches works on: some of a list, its empty ones left out; made in the same way to size the workspace and to run
struct Group {
    Work work[PRODUCTS];
    int count, most_mb;
    bool whole;                              // all of them fit the LDS of a workgroup
    size_t squares, operands;                // bytes, of a piece
    size_t operands_bytes(int P) const { return operands * P; }
    size_t squares_bytes() const { return (squares + NS_JOBS * sizeof(int) + 1023) / 1024 * 1024; }     // ... and a shift for each matrix
    void start() { *this = Group{}; whole = true; }
    void add(int rows, int cols)
    {
        const int mb = (std::min(rows, cols) + 31) / 32, nb = (std::max(rows, cols) + 31) / 32;
        for (int w = 0; w < PRODUCTS; ++w) work[w].add(w, mb, nb);
        ++count;
        most_mb = std::max(most_mb, mb);
        whole = whole && whole_fits(mb, nb);
        squares += squares_of(rows, cols) * sizeof(double);
        operands += operand_bytes(mb, nb, 1);
    }
    // Q and Q X in one launch, a workgroup for each 32 x 32 of X: each makes its rows of Q for itself, which costs less than a launch as long as the workgroups come in one
    // round (two, where Q has 64 rows).  Five steps, two launches -> one, two pieces: 64 x 1728 88 -> 72 us, 64 x 8192 116 -> 102, 128 x 2048 88 -> 80, 192 x 576 77 -> 70,
    // 256 x 1024 86 -> 81; beyond that 128 x 6144 (768 workgroups) 115 -> 130, 256 x 1536 (384) 109 -> 117; three pieces: 192 x 576 95 -> 87, 256 x 1024 108 -> 108
    bool joined(int cus) const { return !whole && most_mb <= NS_JOINED_ROWS && work[APPLY].tiles[FINE] <= (most_mb <= 2 ? 2 : 1) * cus; }
    size_t bytes(int P, int cus) const
    {
        if (whole) return 256;               // (none is used)
        return squares_bytes() + operands_bytes(P) + partial_bytes(choose(P, GRAM, work[GRAM], cus), work[GRAM]);
    }
};

}  // namespace dr

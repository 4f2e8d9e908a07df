// Which kernel a matrix product takes, and whether k goes in shares (internal to the library; host only, no HIP).
//
// A call is estimated for each kernel and the least estimate taken.  The estimates are fits of what calls of 1 to 8192 rows with 128 to 11008
// channels and k from 300 to 11008 took on an MI355X, in ns, and meet those within a fifth mostly (not where more small tiles are than find
// place, four a CU, and a few are left for a second round, nor where rows begin off multiples of 16 bytes):
//   few rows       a CU takes in about 33 bytes a ns of rows of weights and activations (each as often as tiles need it), one workgroup
//                  after the other: 16 x 4096 x 11008 in bf16 22 us;
//   tiles          a step of 128 bytes of k takes at least `alone`, and `each` for every workgroup a CU has at a time (bf16, 8 bits): small tiles fill
//                  the chip with few rows, large ones read less from LDS and L2 for a product (8192 x 4096 x 4096 in bf16: 64 x 64 438 us, 128 x 128 277,
//                  256 x 256 219; 1024 x 4096 x 4096: 50, 53, 87);
//   shares of k    cost the join's launch and the partial sums' way to memory and back, where tiles alone leave CUs without work (64 x 4096 x 11008 in bf16
//                  42 us with the best kernel that has no shares, 27 with eight);
//   memory         gives 4.6 bytes a ps.
#ifndef ANSZP_LINEAR_PLAN_H
#define ANSZP_LINEAR_PLAN_H

#include <algorithm>
#include <cstdint>

enum LinearKernel : uint32_t { kLinearAny, kFew11, kFew21, kFew22, kFew24, kTile64, kTile128, kTile192, kTile256, kLinearKernels };

struct LinearPlan {
    LinearKernel kernel;
    uint32_t shares, share_steps;       // of k, in whole steps of 128 bytes; one share has them all
    uint64_t parts_stride, workspace;   // columns of a row of partial sums; bytes of all of them (one share: 0)
};

constexpr uint32_t kLinearStepBytes = 128u;

inline LinearPlan linear_plan(bool eight_bits, uint64_t rows, uint64_t cols, uint32_t k_bytes, uint64_t x_stride, uint64_t w_stride, uint32_t cus, bool may_share) {
    LinearPlan best = {kLinearAny, 1u, k_bytes / kLinearStepBytes, (cols + 7u) / 8u * 8u, 0u};
    // The others read whole pieces of 16 bytes, and tiles count rows' offsets in 32 bits.
    if (k_bytes < 16u) return best;
    double least = 1e300;
    const double memory = double(rows + cols) * k_bytes / 4600.0, launch = 1500.0;
    const auto groups = [](uint64_t n, uint32_t of) { return (n + of - 1u) / of; };
    const uint64_t most_groups = 1ull << 23;               // (a launch leaves out what is beyond 2^32 threads, and the largest of these workgroups have 512)
    struct Few { LinearKernel kernel; uint32_t tok, ch; };
    for (const Few& f : {Few{kFew11, 1u, 1u}, Few{kFew21, 2u, 1u}, Few{kFew22, 2u, 2u}, Few{kFew24, 2u, 4u}}) {
        if (rows > 4096u) break;
        if (groups(cols, 16u * f.ch) >= most_groups) continue;
        const uint64_t n = groups(groups(cols, 16u * f.ch) * groups(rows, 16u * f.tok), cus);
        const double t = launch + std::max(memory, double(n) * (f.tok + f.ch) * 16.0 * k_bytes / 33.0);
        if (t < least) {
            least = t;
            best.kernel = f.kernel;
        }
    }
    struct TileKind { LinearKernel kernel; uint32_t tok, ch; double alone[2], each[2]; uint32_t most_shares; };
    const TileKind tiles[] = {{kTile64, 64u, 64u, {550.0, 650.0}, {190.0, 250.0}, 16u},
                              {kTile128, 128u, 128u, {800.0, 1000.0}, {560.0, 720.0}, 16u},
                              {kTile192, 192u, 256u, {1350.0, 1780.0}, {1350.0, 1780.0}, 1u},
                              {kTile256, 256u, 256u, {1600.0, 2000.0}, {1600.0, 2000.0}, 1u}};
    const uint32_t steps = (k_bytes + kLinearStepBytes - 1u) / kLinearStepBytes, whole = k_bytes / kLinearStepBytes;
    if (std::max(x_stride, w_stride) <= 1u << 23)
        for (const TileKind& t : tiles) {
            if (groups(cols, t.ch) * groups(rows, t.tok) >= most_groups) continue;
            for (uint32_t s = 1u; s <= t.most_shares && (s == 1u || (may_share && steps >= 4u * s)); s *= 2u) {
                const uint32_t share_steps = s == 1u ? whole : (steps + s - 1u) / s, shares = s == 1u ? 1u : std::max(1u, (whole + share_steps - 1u) / share_steps);
                if (s > 1u && shares == 1u) continue;
                const double n = double(groups(groups(cols, t.ch) * groups(rows, t.tok) * shares, cus));
                double ns = launch + std::max(memory, (shares == 1u ? steps : share_steps) * std::max(t.alone[eight_bits], t.each[eight_bits] * n));
                if (shares > 1u) ns += 3500.0 + double(shares) * rows * best.parts_stride * 8.0 / 6000.0;
                if (ns < least) {
                    least = ns;
                    best.kernel = t.kernel;
                    best.shares = shares;
                    best.share_steps = share_steps;
                    best.workspace = shares > 1u ? uint64_t(shares) * rows * best.parts_stride * 4u : 0u;
                }
            }
        }
    return best;
}

#endif

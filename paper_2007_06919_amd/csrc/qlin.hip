// Linear layers on 8-bit codes: which kernel a launch takes, whether its k range is split, and
// the launches of a split one: partial sums, then the sum of those.

#include <algorithm>

#include "qlin_kernels.h"

namespace aqd {
namespace {

// A tile shape (outputs x tokens; with the gate twice as many rows of w), how many of its workgroups
// fit a CU, and its time in us per stage of 128 k while few CUs run and while all do, and per round
// of workgroups apart from the stages (first loads, stores), with the gate that many times as much.
// Fitted to launches of 1140 random sizes (1 to 11000 tokens, 128 to 16384 outputs and k, plain and
// gated, every shape with 1 to 8 parts, by least squares of the times' logarithms, each weighted by the
// square of the fastest's share of it, without those over twice the fastest). On 400 other sizes of that range, bf16, the
// plan's launch is 4.3% (rows at multiples of 4) and 3.2% (at any byte) slower than the fastest on average, 14% and 9% at the
// ninetieth percentile, 1.53 and 1.66 times at worst (gated 408 x 1034 x 14543 48.7 us, 31.9 with 256x128 in 6 parts;
// 1 x 11360 x 767 8.4, FEW16 5.1). On the sizes of the fit, without one of the shapes the
// fastest is 0.3% (128x128_TWO; 32% at worst, many tiles and a short k) to 1.8% slower on average; one shape
// for all, 2 to 10 times at the other end of the sizes.
struct Shape {
    int shape, out, gate_out, tokens, per_cu;
    double idle, busy, round, gate;
};
const Shape copied[] = {
    {QLIN_64x32, 64, 64, 32, 3, 0.130, 0.170, 1.56, 2.19},    {QLIN_64x64, 64, 0, 64, 2, 0.135, 0.205, 1.68, 0.0},
    {QLIN_128x64, 128, 64, 64, 2, 0.214, 0.355, 1.86, 1.40},  {QLIN_128x128, 128, 64, 128, 1, 0.272, 0.526, 2.57, 1.24},
    {QLIN_128x128_TWO, 128, 64, 128, 2, 0.380, 0.540, 3.40, 1.35}, {QLIN_256x128, 256, 128, 128, 1, 0.363, 0.889, 4.13, 1.07},
    {QLIN_256x256, 256, 128, 256, 1, 0.834, 1.616, 8.02, 1.01},
};
const Shape anywhere[] = {
    {QLIN_ANY, 64, 32, 64, 4, 0.812, 0.532, 2.24, 0.98},
    {QLIN_128x128_ANY, 128, 64, 128, 2, 0.597, 0.828, 4.30, 0.92},
    {QLIN_256x256_ANY, 256, 128, 256, 1, 1.039, 1.944, 8.98, 0.97},
};

constexpr int CUS = 256;
constexpr double LAUNCH = 2.5, MEMORY = 6.3e6;   // us; bytes per us

// how many b hold a
inline double up(double a, double b)
{
    const double q = a / b, whole = (double)(long long)q;
    return whole + (q > whole ? 1.0 : 0.0);
}

double part_bytes(const QlinArgs &a) { return 4.0 * a.rows * (4.0 * up(a.n, 4)) * (a.gate ? 2 : 1); }

double time_of(const QlinArgs &a, const Shape &s, int parts)
{
    const double groups = up(a.n, a.gate ? s.gate_out : s.out) * up(a.rows, s.tokens) * parts;
    const double stages = up(up(a.k, parts), 128), each = up(groups, CUS);
    const double stage = s.idle + (s.busy - s.idle) * std::min(1.0, groups / CUS);
    const double work = s.round * (a.gate ? s.gate : 1.0) * up(each, s.per_cu) + stages * each * stage;
    const double memory = ((double)a.rows * a.k + (double)a.wide * a.k + (double)a.rows * a.n * (a.type == AQD_F32 ? 4 : 2)) / MEMORY;
    // mostly under one another
    double t = std::max(work, memory) + 0.25 * std::min(work, memory);
    // the parts are written and read again, by a launch of its own
    if (parts > 1)
        t += 2.8 + 2.0 * parts * part_bytes(a) / 9.8e6;
    return LAUNCH + t;
}

// the copies into LDS take whole words
bool aligned_rows(const QlinArgs &a) { return (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.ld_x | (uintptr_t)a.ld_w) & 3) == 0; }

// The small launches' kernel, in the same way: us per round of 256 workgroups, a fixed part and one per
// 256 k (with the gate `gate` times as much), and the rate it reads weights at, bytes per us.
double time_of_few(const QlinArgs &a, int tokens, double fixed, double step, double gate, double rate)
{
    const double groups = up(a.n, 16) * up(a.rows, tokens), steps = up(a.k, 256) * (a.gate ? gate : 1.0);
    return LAUNCH + std::max((fixed + step * steps) * up(groups, CUS), (double)a.wide * a.k / rate);
}

}  // namespace

// The plan of a launch: the fastest shape and split by the times above. `room`: bytes for partial sums.
QlinPlan qlin_plan(const QlinArgs &a, size_t room)
{
    QlinPlan best = {QLIN_ANY, 1, 0};
    // offsets inside a tile have 32 bits, and the other kernels' loads 16 bytes
    if (std::max(a.ld_x, a.ld_w) >= 1 << 23 || a.k < 16)
        return best;
    double least = 1e30;
    const bool aligned = aligned_rows(a);
    const double one = part_bytes(a);
    auto consider = [&](const Shape &s) {
        if (a.gate && !s.gate_out)
            return;
        for (int parts : {1, 2, 3, 4, 5, 6, 8}) {
            if (parts > 1 && (one * parts > (double)room || a.k / parts < 512))
                break;
            const double t = time_of(a, s, parts);
            if (t < least) {
                least = t;
                best = {s.shape, parts, parts > 1 ? (size_t)(one * parts) : 0};
            }
        }
    };
    if (aligned)
        for (const Shape &s : copied)
            consider(s);
    else
        for (const Shape &s : anywhere)
            consider(s);
    // (its workgroups' second grid dimension ends at 65535)
    auto consider_few = [&](int shape, int tokens, double t) {
        if (t < least && up(a.rows, tokens) <= 65535) {
            least = t;
            best = {shape, 1, 0};
        }
    };
    if (aligned) {
        consider_few(QLIN_FEW16, 16, time_of_few(a, 16, 2.0, 0.09, 2.0, 4.1e6));
    } else {
        consider_few(QLIN_FEW16, 16, time_of_few(a, 16, 1.6, 0.26, 1.96, 2.6e6));
        consider_few(QLIN_FEW64, 64, time_of_few(a, 64, 1.8, 0.41, 1.82, 3.5e6));
    }
    return best;
}

namespace {

hipError_t launch_part(const QlinArgs &a, int shape, hipStream_t stream)
{
    const bool known = a.gate ? launch_shape<float, true, true>(a, shape, stream) : launch_shape<float, false, true>(a, shape, stream);
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

template <typename T>
void combine(const QlinArgs &a, hipStream_t stream)
{
    const long long items = (long long)a.rows * (a.n_pad / 4);   // few: their sums fit the workspace
    const dim3 grid((unsigned)((items + 255) / 256));
    if (a.gate)
        hipLaunchKernelGGL((qlin_combine_kernel<T, true>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((qlin_combine_kernel<T, false>), grid, dim3(256), 0, stream, a);
}

hipError_t launch_combine(const QlinArgs &a, hipStream_t stream)
{
    if (a.type == AQD_F32)
        combine<float>(a, stream);
    else if (a.type == AQD_F16)
        combine<_Float16>(a, stream);
    else
        combine<__bf16>(a, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_qlin(const QlinArgs &args, const QlinPlan &plan, hipStream_t stream)
{
    QlinArgs a = args;
    a.n_pad = (a.n + 3) & ~3;
    // Stores of whole lines pass the L2 by: 8192 x 8192 x 2048 148 -> 138 us (135 now), 2048 x 11264 x 4096 gated 191 -> 183 (180), and
    // a feed-forward block of 2048 rows that reads its hidden units at once 297 -> 290. Parts of lines, which the
    // L2 joins, do not (22300 x 720 x 256 19.4 us, and 23.1 past it), nor do small outputs.
    const int size = a.type == AQD_F32 ? 4 : 2;
    a.whole_lines = (((uintptr_t)a.y | (uintptr_t)a.ld_y * size) & 127) == 0 && (double)a.rows * a.n * size >= 4e6;
    // whole stages per part
    const int stages = a.k / 128 + (a.k % 128 != 0);
    a.kchunk = 128 * ((stages + plan.parts - 1) / plan.parts);
    a.ksplit = (a.k + a.kchunk - 1) / a.kchunk;
    if (a.ksplit > 1) {
        const hipError_t e = launch_part(a, plan.shape, stream);
        return e != hipSuccess ? e : launch_combine(a, stream);
    }
    a.kchunk = a.k;
    return a.type == AQD_F32   ? launch_qlin_f32(a, plan.shape, stream)
           : a.type == AQD_F16 ? launch_qlin_f16(a, plan.shape, stream)
                               : launch_qlin_bf16(a, plan.shape, stream);
}

}  // namespace aqd

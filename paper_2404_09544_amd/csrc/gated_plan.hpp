// Gated feed-forward blocks: which tiles a call's products take, how their sums are cut, and where everything lies in the workspace.
// Plain C++, by the sizes alone: nothing here asks the device.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace gnnav {

namespace {

constexpr int kFewRows = 8;   // rows, at most, of the kernels that multiply the weights as they lie

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

int64_t tiles(int64_t rows, int64_t cols, int64_t bn, int64_t bm) { return up(rows, bn) / bn * (up(cols, bm) / bm); }

// A tile: columns and rows of the output, workgroups that a unit holds at once, and what one takes, in us: a step `share` times the
// workgroups that share the unit and `alone` at least, all else `start`.  Fitted to 19 blocks of 20 to 100,000 rows in bf16 and 16
// in fp32, each in every tile; the launches' times are within some 15% of it, and the tile that it takes within 7% of the best
// in 9 of 10 cases.
// Measured: 8,192 x 1,024 outputs of 4,096 summed bf16 columns 126 us in tiles of 256 x 256, 104 of 128 x 256, 175 of 64 x 128,
// 256 of 64 x 64; 4,000 x 512 of 1,024 columns 42, 31, 19, 22.
struct Shape {
    int bm, bn, each;
    double share, alone, start;
};
constexpr int kUnits = 256;
enum { kLarge, kWide, kMedium, kSmall, kShapes };
const Shape kNone = {0, 0, 0, 0, 0, 0};
const Shape kOutBf16[kShapes] = {{256, 256, 1, 0.92, 0.92, 9.6}, {128, 256, 2, 0.63, 0.54, 7.6}, {64, 128, 4, 0.25, 0.26, 7.8}, {64, 64, 8, 0.16, 0.15, 8.8}};
const Shape kOutF32[kShapes] = {kNone, {128, 128, 2, 0.57, 0.63, 7.8}, {64, 128, 2, 0.37, 0.43, 6.7}, {64, 64, 4, 0.22, 0.31, 9.5}};
// the gradients, whose operands' rows are summed over: the same tiles
const Shape kGradsBf16[kShapes] = {{256, 256, 1, 0.83, 0.83, 8.8}, {128, 256, 2, 0.51, 0.52, 7.6}, {64, 128, 4, 0.21, 0.28, 5.5}, {64, 64, 8, 0.13, 0.19, 6.7}};
const Shape kGradsF32[kShapes] = {kNone, {128, 128, 2, 0.52, 0.64, 6.9}, {64, 128, 2, 0.34, 0.54, 4.8}, {64, 64, 4, 0.20, 0.36, 7.6}};
// h: columns of one projection
const Shape kGateBf16[kShapes] = {{128, 256, 1, 0.79, 0.79, 7.6}, kNone, {64, 128, 3, 0.22, 0.60, 7.2}, {32, 64, 6, 0.19, 0.49, 4.7}};
const Shape kGateF32[kShapes] = {kNone, {64, 128, 2, 0.51, 0.60, 11.9}, kNone, {32, 64, 4, 0.19, 0.26, 9.1}};
// da and db: a step of one product
const Shape kDgateBf16[kShapes] = {{128, 256, 1, 0.36, 0.36, 13.6}, kNone, {64, 128, 3, 0.12, 0.30, 10.0}, {64, 64, 4, 0.12, 0.20, 7.3}};
const Shape kDgateF32[kShapes] = {kNone, {128, 128, 2, 0.58, 0.23, 23.5}, kNone, {64, 64, 4, 0.23, 0.13, 10.3}};

// A product's part in a launch: tiles, steps of each, entries of the output.
struct Job {
    int64_t tiles, steps, entries;
    int32_t splits = 1;
};
// Time until a launch's last workgroup ends, its jobs' workgroups going to `slots` places in their order; in kTicks of a step, of
// which each takes `start` besides its steps.
constexpr int kTicks = 16;
int64_t makespan(const Job *jobs, int n, int64_t slots, int64_t start) {
    // times at which places become free, with how many do: few distinct ones
    int64_t at[64], count[64];
    int k = 1;
    at[0] = 0;
    count[0] = slots;
    int64_t last = 0;
    for (int j = 0; j < n; ++j) {
        int64_t left = jobs[j].tiles * jobs[j].splits;
        const int64_t each = (jobs[j].steps + jobs[j].splits - 1) / jobs[j].splits * kTicks + start;
        if (left > 16 * slots) return INT64_MAX;   // (long anyway)
        while (left > 0) {
            int first = 0;
            for (int i = 1; i < k; ++i)
                if (at[i] < at[first]) first = i;
            const int64_t take = std::min(left, count[first]), end = at[first] + each;
            left -= take;
            last = std::max(last, end);
            count[first] -= take;
            if (count[first] == 0) {
                at[first] = at[k - 1];
                count[first] = count[k - 1];
                --k;
            }
            int same = 0;
            while (same < k && at[same] != end) ++same;
            if (same < k) {
                count[same] += take;
            } else if (k < 64) {
                at[k] = end;
                count[k++] = take;
            } else {
                return INT64_MAX;
            }
        }
    }
    return last;
}
// us that a launch of these jobs takes, their parts' way to memory and back in a launch of its own among them (5 us and 4 TB/s).
double cost(const Job *jobs, int n, const Shape &shape) {
    const int64_t slots = (int64_t)kUnits * shape.each;
    int64_t groups = 0;
    double bytes = 0, t = 0;
    for (int j = 0; j < n; ++j) {
        groups += jobs[j].tiles * jobs[j].splits;
        if (jobs[j].splits > 1) bytes += jobs[j].entries * 8.0 * jobs[j].splits;
    }
    // a step, of so many workgroups
    auto step = [&](int64_t of) { return std::max(shape.alone, std::min<int64_t>(shape.each, (of + kUnits - 1) / kUnits) * shape.share); };
    const double full = step(groups);
    const int64_t m = n > 1 ? makespan(jobs, n, slots, (int64_t)(shape.start / full * kTicks)) : INT64_MAX;
    if (n == 1) {   // full rounds, and the last one
        const int64_t steps = (jobs[0].steps + jobs[0].splits - 1) / jobs[0].splits;
        t = groups / slots * (steps * full + shape.start) + (groups % slots ? steps * step(groups % slots) + shape.start : 0.0);
    } else if (m != INT64_MAX) {
        t = m * full / kTicks;
    } else {
        for (int j = 0; j < n; ++j) t += jobs[j].tiles * jobs[j].splits * ((jobs[j].steps + jobs[j].splits - 1) / jobs[j].splits * full + shape.start) / slots;
    }
    return t + (bytes > 0 ? 5.0 + bytes / 4e6 : 0.0);
}
// Splits of the jobs' sums that make it least.  Parts have 16 steps at least.
double split(Job *jobs, int n, const Shape &shape) {
    int64_t total = 0, longest = 0;
    for (int j = 0; j < n; ++j) {
        jobs[j].splits = 1;
        total += jobs[j].tiles * jobs[j].steps;
        longest = std::max(longest, jobs[j].tiles > 0 ? jobs[j].steps : 0);
    }
    double least = cost(jobs, n, shape);
    if (longest < 48) return least;
    Job best[3], now[3];
    for (int j = 0; j < n; ++j) best[j] = jobs[j];
    const int64_t even = std::max<int64_t>(1, total / ((int64_t)kUnits * shape.each));
    for (int r = 1; r <= 6; ++r)                   // parts of about this share of an even load
        for (int from = n - 1; from >= 0; --from) {   // the jobs from this one on
            const int64_t length = std::max<int64_t>(16, (even + r - 1) / r);
            for (int j = 0; j < n; ++j) {
                now[j] = jobs[j];
                if (j >= from && jobs[j].tiles > 0) {
                    const int64_t s = std::max<int64_t>(1, std::min<int64_t>({jobs[j].steps / 16, (jobs[j].steps + length - 1) / length, 64}));
                    const int64_t each = (jobs[j].steps + s - 1) / s;
                    now[j].splits = (int32_t)((jobs[j].steps + each - 1) / each);   // without empty ones
                }
            }
            const double c = cost(now, n, shape);
            if (c < least) {
                least = c;
                for (int j = 0; j < n; ++j) best[j] = now[j];
            }
        }
    for (int j = 0; j < n; ++j) jobs[j] = best[j];
    return least;
}
// The shape, of those that there are, whose launch takes least: `jobs_of` fills the jobs of a shape.
template <class F>
int choose(const Shape *shapes, Job *jobs, int n, bool may_split, F &&jobs_of) {
    int which = -1;
    double least = 0;
    Job best[3];
    for (int k = 0; k < kShapes; ++k) {
        if (shapes[k].bm == 0) continue;
        jobs_of(shapes[k], jobs);
        const double c = may_split ? split(jobs, n, shapes[k]) : cost(jobs, n, shapes[k]);
        if (which < 0 || c < least) {
            which = k;
            least = c;
            for (int j = 0; j < n; ++j) best[j] = jobs[j];
        }
    }
    for (int j = 0; j < n; ++j) jobs[j] = best[j];
    return which;
}

// Outputs of fewer entries take h, da and db in two bf16 parts: bf16's roundings average out over many entries and show in few.
// Those outputs are then off by their own rounding, 0.0016 by norm, and not by 0.0023; steps of 1,024 x 602 x 1,024 x 7 take
// 76 us (68 without), of 65,537 x 64 x 128 x 41, whose h of two parts costs more than elsewhere, 98 (86).
constexpr int64_t kFew = 8192;

// Where everything lies in the workspace, and how the products are cut.
struct Plan {
    int64_t m, d, f, o;
    int pl, bk;
    bool bf16, pack_x, pack_w, pack_wd, pack_dy;
    bool low_y, low_dx, low_dw, low_dd;
    int gate, down, dgate, grads;
    int32_t down_splits = 1, dx_splits = 1, dw_splits = 1, dd_splits = 1;
    size_t x = 0, wg = 0, wu = 0, wd = 0, dy = 0, h = 0, D = 0, part = 0, part2 = 0, part3 = 0, row_norms = 0, column_norms = 0, total = 0;
    int64_t fp() const { return up(f, 8); }
    size_t take(int64_t bytes) {
        const size_t here = total;
        total += (size_t)up(bytes, 256);
        return here;
    }
    size_t packed(int64_t rows, int64_t cols) { return take(rows * up(cols, 8) * 2 * pl); }
    static int64_t parts(int64_t rows, int64_t cols, const Shape &e, int32_t splits) {
        return splits > 1 ? splits * up(rows, e.bn) * up(cols, e.bm) * 4 : 0;
    }
    const Shape &out(int which) const { return (bf16 ? kOutBf16 : kOutF32)[which]; }   // (the gradients' have the same sizes)
    template <class Args>   // m, d, f, d_out, bf16, ld_wg and ld_wu of a call
    Plan(const Args &a, bool backward) : m(a.m), d(a.d), f(a.f), o(a.d_out), bf16(a.bf16) {
        pl = bf16 ? 1 : 3;
        bk = bf16 ? 32 : 16;
        low_y = bf16 && m * o < kFew;
        low_dx = bf16 && m * d < kFew;
        low_dw = bf16 && d * f < kFew;
        low_dd = bf16 && f * o < kFew;
        // (where the columns are summed over, the last chunk has to end in zeros)
        pack_x = !bf16 || d % 8;
        pack_wd = !bf16 || (backward && o % 8);
        pack_dy = !bf16 || o % 8;
        pack_w = !bf16 || (backward && (f % 8 || a.ld_wg != a.ld_wu));   // (a sum's matrices lie alike)
        if (pack_x) x = packed(m, d);
        if (pack_w || backward) {   // (whether their strides differ is not known to who asks for the size)
            wg = packed(d, f);
            wu = packed(d, f);
        }
        if (pack_wd) wd = packed(f, o);
        if (!backward) {
            h = take(std::max(fp() * m * 2 * (low_y ? 2 : pl), m <= kFewRows ? m * f * 4 : 0));
            Job j;
            gate = choose(bf16 ? kGateBf16 : kGateF32, &j, 1, false, [&](const Shape &e, Job *x) { *x = {tiles(m, f, e.bn, e.bm), (d + bk - 1) / bk, 0}; });
            down = choose(bf16 ? kOutBf16 : kOutF32, &j, 1, true,
                          [&](const Shape &e, Job *x) { *x = {tiles(m, o, e.bn, e.bm), (f + bk - 1) / bk * (low_y ? 2 : 1), m * o}; });
            down_splits = j.splits;
            part = take(parts(m, o, out(down), down_splits));
            if (!bf16) {   // (which activation it is, and whether a is kept, is not known to who asks for the size)
                row_norms = take(m * 4);
                column_norms = take(fp() * 4);
            }
        } else {
            if (pack_dy) dy = packed(m, o);
            D = take(2 * fp() * m * 2 * (low_dx || low_dw ? 2 : pl));
            if (low_dd) h = take(fp() * m * 4);
            Job j[3];
            dgate = choose(bf16 ? kDgateBf16 : kDgateF32, j, 1, false, [&](const Shape &e, Job *x) {
                *x = {tiles(m, f, e.bn, e.bm), (o + bk - 1) / bk + (bf16 ? (d + bk - 1) / bk * 2 : 0), 0};
            });
            const int64_t ks = (fp() + bk - 1) / bk * (low_dx ? 4 : 2), ms = (m + bk - 1) / bk;
            grads = choose(bf16 ? kGradsBf16 : kGradsF32, j, 3, true, [&](const Shape &e, Job *x) {
                x[0] = {tiles(m, d, e.bn, e.bm), ks, m * d};
                x[1] = {tiles(d, 2 * fp(), e.bn, e.bm), ms * (low_dw ? 2 : 1), 2 * d * fp()};
                x[2] = {tiles(f, o, e.bn, e.bm), ms * (low_dd ? 2 : 1), f * o};
            });
            const Shape &e = out(grads);
            dx_splits = j[0].splits;
            dw_splits = j[1].splits;
            dd_splits = j[2].splits;
            part = take(parts(m, d, e, dx_splits));
            part2 = take(parts(d, 2 * fp(), e, dw_splits));
            part3 = take(parts(f, o, e, dd_splits));
        }
    }
};

}  // namespace

}  // namespace gnnav

// The group norm's kernels, every thread of a full and of the last work-group's chunk with the kernels' own index arithmetic: the highest float
// of LDS that each touches, against what the launch asks for.  Reads lines "N HW C groups bytes vector backward", prints a line for
// each that is not covered and how many calls have a last chunk that uses more than a full one.
#include <cstdio>

#include "group_norm_plan.h"

using namespace anr::gnorm;

static size_t highest;
static void touch(size_t i) { highest = std::max(highest, i); }

// Columns and rows as a work-group divides its threads; tx of those left over has no column.
struct Threads {
    int columns, rows, wide;
    Threads(int channels, int V, int threads) : columns(channels / V), rows(threads / std::min(columns, threads)), wide(std::min(columns, threads)) {}
};

static void sums(const Shape& s, int channels, int V)
{
    const int table = (std::min(channels, 256 * V) + 3) / 4 * 4, tables = s.backward ? 4 * table : table;
    const Threads t(channels, V, 256);
    for (int tid = 0; tid < 256; ++tid) {
        const int ty = tid / t.wide, tx = ty < t.rows ? tid - ty * t.wide : t.columns;
        for (int base = 0; base < t.columns; base += 256) {
            const int here = std::min(channels - base * V, 256 * V), col = base + tx;
            for (int c = tid; c < here; c += 256) touch(s.backward ? 3 * (size_t)table + c : (size_t)c);
            if (col >= t.columns) continue;
            touch((size_t)tx * V + V - 1 + (s.backward ? 3 * table : 0));
            touch((size_t)tables + 2 * ((size_t)t.rows * channels + (size_t)((V - 1) * t.rows + ty) * t.columns + col) + 1);      // (64 bits)
        }
    }
}

static void apply(const Shape& s, int channels, int V, int cg)
{
    const int tables = s.backward ? 6 : 3, table = (std::min(channels, 256 * V) + 3) / 4 * 4;
    touch((size_t)tables * table - 1);
    touch((size_t)tables * table + (s.backward ? 2 : 3) * (channels / cg) - 1);
    if (s.backward) touch(2 * 255 + 1);              // the parameters' gradients: 64 bits a thread
}

static void resident(const Shape& s, int channels, int cg, int threads)
{
    const int table = (channels + 3) / 4 * 4, groups = channels / cg;
    const Threads t(channels, 4, threads);
    const size_t before = s.backward ? 6 * (size_t)table + (2 * groups + 3) / 4 * 4 : 2 * (size_t)table + 2 * ((groups + 3) / 4 * 4);
    for (int tid = 0; tid < threads; ++tid) {
        const int ty = tid / t.wide, tx = ty < t.rows ? tid - ty * t.wide : t.columns;
        const size_t at = (s.backward ? (size_t)(2 * ty + 1) : (size_t)ty) * channels + (size_t)tx * 4 + 3;
        if (tx < t.columns) touch(before + (s.backward ? at : 2 * at + 1));         // (forward: 64 bits)
        if (s.backward) touch(before + 2 * (size_t)t.rows * channels + 2 * tid + 1);
    }
}

int main()
{
    Shape s{};
    int vector, backward, more = 0, bad = 0;
    while (scanf("%d %d %d %d %d %d %d", &s.N, &s.HW, &s.C, &s.groups, &s.es, &vector, &backward) == 7) {
        if (vector && !vector_possible(s.C, s.groups, s.es)) continue;
        s.vector = vector;
        s.backward = backward;
        const Division d = divide(s);
        const int cg = s.C / s.groups, last = s.C - (d.chunks - 1) * d.chunk;
        size_t full[3] = {}, used[3] = {};
        for (int channels : {d.chunk, last}) {
            for (int kernel = 0; kernel < 3; ++kernel) {
                highest = 0;
                if (kernel < 2 && d.resident) continue;
                if (kernel == 2 && !d.resident) continue;
                if (kernel == 0) sums(s, channels, d.V);
                if (kernel == 1) apply(s, channels, d.V, cg);
                if (kernel == 2) resident(s, channels, cg, d.resident);
                if (channels == d.chunk) full[kernel] = std::max(full[kernel], highest);
                else more += highest > full[kernel];
                used[kernel] = std::max(used[kernel], highest);
            }
        }
        const size_t asked[3] = {d.sums_lds, d.apply_lds, d.resident_lds};
        for (int kernel = 0; kernel < 3; ++kernel)
            if (used[kernel] && 4 * (used[kernel] + 1) > asked[kernel]) {
                printf("N %d HW %d C %d groups %d bytes %d vector %d backward %d kernel %d: %zu of %zu\n", s.N, s.HW, s.C, s.groups, s.es, vector, backward, kernel,
                       4 * (used[kernel] + 1), asked[kernel]);
                ++bad;
            }
        if (std::max(d.sums_lds, d.resident_lds) > 160 * 1024) {
            printf("N %d HW %d C %d groups %d: more than a CU has\n", s.N, s.HW, s.C, s.groups);
            ++bad;
        }
    }
    printf("%d\n", more);
    return bad != 0;
}

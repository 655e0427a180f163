// layer_plan.h - how the layers' launches are cut: sizes in, blocks and shared memory out.  Plain C++ that needs no GPU, so that the rules can be
// checked for any size on the host; included by layers.cuh inside its unnamed namespace.
#pragma once

constexpr long long kBusy = 148 * 8;                   // blocks of 256 threads that fill the GPU; a constant, so that sums do not depend on the GPU
constexpr long long kMostBlocks = 0x7fffffff;

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ dropout
// Column vectors of a block and column blocks, for rows of `cols` elements in vectors of v.
void column_blocks(long long cols, int v, int &tx, int &blocks) {
    const long long vectors = ceil_div(cols, v);
    tx = 1;
    while (tx < 32 && tx < vectors) tx *= 2;
    blocks = (int)ceil_div(vectors, tx);
}

// Rows of cols elements to a walked row: as many as make whole vectors, and as fill a block's 32 of them.
long long rows_walked_as_one(long long cols, int v) {
    const long long least = v / std::gcd(cols, (long long)v);
    return least * std::max(1ll, ceil_div(32 * v, least * cols));
}
// Whether a call of this many rows has one such row.  Fewer are walked as they are: most of a longer row would not exist.
bool walked_as_one(long long rows, long long cols, int v) { return rows >= rows_walked_as_one(cols, v); }

constexpr int kSteps = 8, kSumSteps = 16;
// How the rows of a call are walked.
struct Walk {
    long long width, rows, chunk_rows, most_chunks;    // most_chunks: of this many rows or fewer
    int tx, col_blocks, chunks;
};
Walk walk_of(long long rows, long long cols, int n, int v, bool dense, bool sums) {
    Walk k;
    const long long fold = dense ? rows_walked_as_one(cols, v) : 1;
    k.width = fold * cols, k.rows = dense ? ceil_div(rows * cols + v - 1, k.width) : rows;
    column_blocks(k.width, v, k.tx, k.col_blocks);
    // Each thread kSteps rows, or fewer, but four, where that leaves the GPU idle.
    const long long step = 256 / k.tx, most = ceil_div(k.rows, 4 * step), want = ceil_div(kBusy, (long long)k.col_blocks * n);
    k.most_chunks = std::min(most, std::max(want, ceil_div(k.rows, (sums ? kSumSteps : kSteps) * step)));
    k.chunk_rows = ceil_div(k.rows, k.most_chunks);
    k.chunks = (int)ceil_div(k.rows, k.chunk_rows);
    return k;
}

// Floats a worker for the sums of up to max_rows rows, of which any call may have fewer; 0 where one chunk's sums are the result.
long long sums_of(long long max_rows, long long cols, int n, int v) {
    long long sums = 0;
    for (bool dense : {false, true}) {                 // walked either way
        if (dense && !walked_as_one(max_rows, cols, v)) continue;
        const Walk k = walk_of(max_rows, cols, n, v, dense, true);
        if (k.most_chunks > 1 || k.width != cols) sums = std::max(sums, k.most_chunks * k.width);
    }
    return sums;
}

// ------------------------------------------------------------------ group norm in one walk
struct Resident {
    int sv, log_tx, log_block, log_cluster, slots;     // sv: vectors of a slice; log_block: threads; slots: of a thread and array
    int fold, log_sub;                                 // neighbouring channels of a vector that share a group; lanes of a group's sums
    uint32_t group_magic;                              // 2^32 / channels of a group, rounded up; 0 for one
    int per;                                           // pixels of a block
    uint32_t slices, units;                            // of a sample, and of all
};

// Bytes of shared memory of the above.
inline size_t resident_shared(const Resident &r, int v, int size, bool two, bool bits) {
    const int width = (1 << r.log_tx) * v, rows = std::min(1 << (r.log_block - r.log_tx), 1 << (r.log_block - 5));
    const size_t sums = width / (two ? 1 : r.fold);
    return ((size_t)r.slots << r.log_block) * (v * size * (two ? 2 : 1) + (bits ? 1 : 0)) + (size_t)(6 + 2 * rows) * width * 4 + (4 << r.log_cluster) * sums * 4;
}

constexpr size_t kMostShared = size_t(220) << 10;      // of a block
struct NormSizes {
    int size;                                          // bytes of an element
    long long n, samples, pixels, channels, groups;
    bool drop;
};

// How a call is made in one walk, with v elements a vector; false: it does not fit, or vectors are too short for asynchronous copies.
// Clusters cost more than narrow slices: the fewest blocks that hold a slice of 64 bytes of a pixel at two blocks to an SM, then of 32, then at
// one to an SM (8 x 16 x 56 x 56 x 256 in bf16, forward: 64 bytes by 2 blocks 86 us, 128 by 4 96, 128 by 8 at four to an SM 100, 32 by one
// 106; gradient 133 by 4 and 156 of 128 bytes by 8).  Blocks of 256 threads, or of 128 where four fit an SM (28 x 28 x 256 forward 89 and
// 115 us).  Few units are spread over more blocks, at four pixels a thread and more.
bool plan_resident(const NormSizes &k, int v, bool two, Resident &r, size_t &shared) {
    const int size = k.size, per_group = (int)(k.channels / k.groups);
    if (v * size < 4) return false;
    const long long least = std::lcm(per_group, v) / v, all = k.channels / v, samples = k.n * k.samples;
    bool found = false;
    // 64 bytes, or more where a unit would be less than 16 KB and there are enough.
    long long widest = 64;
    while (widest < 4096 && widest * k.pixels < 16 << 10 && samples * ceil_div(k.channels * size, 2 * widest) >= kBusy / 2) widest *= 2;
    for (size_t most : {size_t(112) << 10, kMostShared}) {
        for (long long bytes : {widest, 32ll}) {
            r = Resident{};
            r.fold = std::gcd(per_group, v);
            const long long vectors = std::min(all, least * ceil_div(bytes, least * v * size)), slices = ceil_div(all, vectors);
            if (vectors > 128 || samples * slices > kMostBlocks / 8) continue;
            r.sv = (int)vectors, r.slices = (uint32_t)slices, r.units = (uint32_t)(samples * slices);
            while (1 << r.log_tx < r.sv) ++r.log_tx;
            auto cut = [&](Resident &r, int log_cluster) -> size_t {          // by so many blocks: bytes of shared memory of one
                r.log_cluster = log_cluster, r.per = (int)ceil_div(k.pixels, 1 << log_cluster);
                for (r.log_block = 7;; ++r.log_block) {
                    const long long slots = ceil_div(r.per, (1 << r.log_block) >> r.log_tx);
                    if (slots > 1 << 16) return ~size_t(0);              // (more than any block has)
                    r.slots = (int)slots;
                    const size_t bytes = resident_shared(r, v, size, two, two && k.drop);
                    if (r.log_block == 8 || bytes <= size_t(55) << 10) return bytes;
                }
            };
            int c = 0;
            for (shared = cut(r, c); shared > most && c < 3;) shared = cut(r, ++c);
            if (shared > most) continue;
            while (r.units << r.log_cluster < kBusy / 4 && c < 3 && r.per >= 4 * ((1 << r.log_block) >> r.log_tx)) {
                Resident more = r;
                const size_t bytes = cut(more, ++c);
                if (bytes > kMostShared) break;        // (the sums that more blocks exchange can outweigh the pixels that each has less)
                r = more, shared = bytes;
            }
            found = true;
            break;
        }
        if (found) break;
    }
    if (!found) return false;
    const int entries = two ? per_group : (per_group / r.fold) << r.log_cluster;
    while (r.log_sub < 5 && 1 << r.log_sub < entries) ++r.log_sub;
    r.group_magic = per_group == 1 ? 0 : (uint32_t)(((1ull << 32) + per_group - 1) / per_group);
    return true;
}

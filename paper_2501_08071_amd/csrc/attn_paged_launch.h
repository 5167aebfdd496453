// Internal: host-side launch interface of the operators on a paged key/value cache (not part of the ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

// A batch of sequences whose keys and values lie in pages.  Kernels take it by value.
struct PagedCache {
    void* k;                  // [n_pages][Hk][page size][D], pages page_stride elements apart
    void* v;
    const int* table;         // [B][table_stride], the first `width` of a row in use
    const int* cu_q;          // [B + 1]
    const int* kv_len;        // [B]
    long long page_stride;
    int n_pages, page_shift, Hk, table_stride, width, B, T;
};

// Bytes from the first key of a head in a page to key j of a sequence, of row_bytes each; mask: the page's keys - 1.  In 64 bits: a page of
// 2^24 keys of 256 bytes is 4 GiB.
__host__ __device__ inline uint64_t paged_key_offset(int j, int mask, int row_bytes) { return (uint64_t)(uint32_t)(j & mask) * (uint32_t)row_bytes; }

struct AppendLaunch {
    PagedCache c;
    const void *q, *k, *v;    // tokens q_stride, k_stride, v_stride elements apart
    long long q_stride, k_stride, v_stride;
    void* q_out;              // [T][Hq][D]
    const float *cos, *sin;   // [n_angles][rot / 2]
    int rot, interleaved, n_angles, pos_offset, Hq, D, dtype;
    void* stream;
};
hipError_t kv_append_launch(const AppendLaunch& a);

// n / d for 0 <= n < 2^31 as a product: with 2^(l-1) < d <= 2^l and m = floor(2^(31+l) / d) + 1, n m / 2^(31+l) exceeds n / d by less
// than n / 2^31 / d < 1 / d.  m has 32 bits: for d = 2^l it is 2^31 + 1, else d is 2^(l-1) + 1 or more, 2^(31+l) / d at most
// 2^32 - 2^32 / (2^(l-1) + 1), and with d < 2^31 that is below 2^32 - 3.  (A division by a number that is not known in advance takes 40 instructions; a small problem waits for several.)
struct Divisor {
    uint32_t m = 1, shift = 0;
    Divisor() = default;
    explicit Divisor(int d) {
        int l = 0;
        while ((1LL << l) < d) ++l;
        m = d == 1 ? 1u : (uint32_t)((1ULL << (31 + l)) / d + 1);   // d = 1: n * 1 / 1
        shift = d == 1 ? 0 : 31 + l;
    }
    __host__ __device__ int of(int n) const { return (int)(((uint64_t)(uint32_t)n * m) >> shift); }
};

struct PagedAttnLaunch {
    PagedCache c;
    const void* q;            // [T][Hq][D], tokens q_stride elements apart
    long long q_stride;
    void* o;                  // [T][Hq][D]
    float* lse;               // [T][Hq] or null
    const int* prefix_table;
    int prefix_len;
    int Hq, G, D, dtype, max_q, max_kv;
    Divisor by_G, by_Hk;
    float c_log2;             // |scale| * log2(e), kept off zero (a hidden logit of minus infinity times 0 would be NaN)
    uint32_t q_sign;          // 0x80008000 for a negative scale: flips the signs of q
    void* workspace;
    void* stream;
};

// How a problem is served: chosen from sizes that the host knows, the same for the launch and for the workspace's size.
struct PagedPlan {
    int rows;                 // of a workgroup: 16 or 32 (its wavefronts share out the keys), or 128 (they share out the rows)
    int workgroups, waves;    // of the pass over the sequences' own keys; wavefronts of each
    bool balanced;            // the keys shared out evenly over the workgroups, else one workgroup for each tile of rows and key head
    bool direct;              // not balanced, and every sequence has one tile of rows at most
    int prefix_rows, prefix_tiles, prefix_splits, prefix_waves;   // the pass over the shared prefix; 0 splits: none
    long long part_floats, prefix_floats, bytes;         // workspace: parts of split tiles, results of the prefix pass, all of it
};
constexpr int PAGED_WAVES = 2048;   // eight to a compute unit: what their LDS allows
constexpr int NARROW_PREFIX_WAVES = 8;   // of a workgroup of 16 or 32 rows in the pass over a shared prefix: few rows have few tiles

inline int paged_rows(long long rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 128; }
inline int paged_block_keys(int rows, int D) { return rows < 128 && D == 128 ? 32 : 64; }

inline PagedPlan paged_plan(int B, int T, int Hq, int Hk, int D, int max_q, int max_kv, int prefix_len) {
    PagedPlan p{};
    const int G = Hq / Hk;
    max_q = max_q < T ? max_q : T;   // (a hint may be any number; no sequence has more new tokens than there are)
    p.rows = paged_rows((long long)max_q * G);
    const int R = p.rows, KB = paged_block_keys(R, D);
    // tiles of rows: of every sequence at most, and of all its tokens together
    const long long each = (long long)B * (((long long)max_q * G + R - 1) / R), all = (long long)T * G / R + B;
    const long long segments = (each < all ? each : all) * Hk;
    // Whole tiles while they are short: sharing out costs a scan, sums through memory and a second launch, less so where there are more
    // tiles than compute units.  Decode steps, 32 / 8 heads, D = 128, bfloat16, us a call on the same inputs again and again, the four ways (this rule
    // and the next one) in one run:
    //                                            whole, 4 wavefronts   whole, 8   shared out, 4   shared out, 8   chosen
    //     1 sequence of 512 keys                         8.4              7.1         11.6            14.4        whole, 8
    //     1 of 1024                                     13.1              9.8         11.9            14.6        shared out, 4 (the second best)
    //     2 of 2048                                     22.8             16.0         12.7            15.1        shared out, 4
    //     4 of 4096                                     42.0             28.2         21.0            18.9        shared out, 8
    //     1 of 65537                                     612              377         50.5            48.4        shared out, 8
    //     16 of 1 to 2048                               22.9             16.1         17.5            17.6        shared out (the second best)
    //     64 of 1 to 1024                               14.7             15.3         22.3            26.8        whole, 4
    //     256 of 100 to 2048                             130              131          142             151        whole, 4
    //     64 of 200 to 8192                              140              136          110             112        shared out, 4
    // (Work is counted in 32 bits, of max_kv keys a tile at most: whatever may be past 2^31 blocks has tiles enough.  A division: the product with a
    // hint of 2^31 - 1 keys may pass 64 bits.)
    const long long often = segments / 256;
    p.balanced = max_kv > 16 * KB * (often < 1 ? 1 : often > 4 ? 4 : often) && each * Hk <= ((1LL << 31) - 1) / (max_kv / KB + 64);
    p.direct = !p.balanced && (long long)max_q * G <= R;
    // Eight wavefronts where a workgroup has a compute unit for itself: whole tiles take half the rounds, shared-out ones have half the parts,
    // if there is work for all, and two workgroups of four hide each other's ends where there are many tiles (figures: the table above).
    p.waves = R < 128 && segments <= 256 && (!p.balanced || segments * (max_kv / KB) >= 2048) ? 8 : 4;
    p.workgroups = p.balanced ? PAGED_WAVES / p.waves : p.direct ? B * Hk : (int)segments;
    p.part_floats = p.balanced ? 2LL * p.workgroups * R * (D + 2) + 8LL * p.workgroups : 0;
    if (prefix_len > 0) {
        p.prefix_rows = paged_rows((long long)T * G);
        const int PR = p.prefix_rows, PKB = paged_block_keys(PR, D);
        p.prefix_tiles = (int)(((long long)T * G + PR - 1) / PR);
        // As many pieces as fill the chip, of 8 blocks or more, and not so many that a row's sums take long to add up.  Of a short prefix
        // under many rows also smaller ones, the smaller the faster the own keys' pass adds them up: workgroups of 16 or 32 rows share
        // that out over their wavefronts (78 sequences behind 746 shared keys 16.8 us, 19.1 with 4 pieces at most).
        const long long groups = (long long)p.prefix_tiles * Hk, blocks = (prefix_len - 1) / PKB + 1, top = PR == 128 ? 32 : 64;
        const long long least = R < 128 ? 2 : 4, cap = R < 128 ? 16 : 4, fine = (blocks + least - 1) / least;
        long long most = (blocks + 7) / 8;
        if (PR == 128 && most < cap) most = fine < cap ? fine : cap;
        p.prefix_waves = PR < 128 ? NARROW_PREFIX_WAVES : 4;
        long long s = PAGED_WAVES / p.prefix_waves / groups;
        s = s > most ? most : s > top ? top : s;
        s = s < 1 ? 1 : s;
        p.prefix_splits = (int)s;
        p.prefix_floats = (s * T * Hq * (D + 2) + 3) / 4 * 4;   // what follows stays aligned to 16 bytes
    }
    p.bytes = 4 * (p.part_floats + p.prefix_floats);
    return p;
}
hipError_t paged_attn_launch(const PagedAttnLaunch& a);

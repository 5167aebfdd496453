// Attention over a paged key/value cache for gfx950.
//
// For token i of the n new ones of sequence b, query head h and its key head h / G (G = Hq / Hk):
//     z_j = scale q . k_j   over the shared prefix's keys and the first kv_len[b] - n + i + 1 keys of the sequence's own
//     o = sum_j exp(z_j) v_j / sum_j exp(z_j),   lse = ln sum_j exp(z_j)      (no key at all: o = 0, lse = -inf)
//
// The rows of a sequence that read the same keys -- its new tokens times the G query heads of a key head -- are one tile of
// 16 RT rows, so K and V are read once for all of them.  For a shared prefix the rows of the whole batch form such tiles, and a
// first pass over the prefix leaves its sums (maximum, sum of weights, weighted values) per row; the pass over the own keys
// adds them at the end.
//
// Few rows: the kernel is bound by the bytes of K and V, and has to keep many in flight.  Every wavefront therefore streams
// blocks of KB keys of its own from global memory straight into LDS buffers of its own, without a barrier in the loop (16 KiB for
// each of 8 wavefronts on a compute unit at D = 64 and 128, half of it at D = 32).  Everything is computed transposed, so that a lane
// only holds values of one query row per row tile:
//     S^T (keys x rows)  = K . Q^T     v_mfma_f32_16x16x32, A = K rows, B = Q^T
//     O^T (d x rows)    += V^T . P^T   A = V^T by transposing LDS reads, B = P^T, the weights as they lie in the accumulators:
// lane (c, row) (c = lane / 16) holds keys 4c .. 4c+3 of each 16-key tile; two tiles are the 8 contraction indices of its group
// of lanes, in the order  key(8c + e) = 16 (e / 4) + 4c + e % 4,  and V^T is fetched in that order.
// The wavefronts' sums are added in LDS at the end of a tile.
// Measured, 32 query and 8 key heads of 128, bfloat16: 64 sequences of 200 to 8192 keys 132 us (5.2 TB/s of keys and values; a copy moves
// 5.1 to 5.5), one of 65537 keys 55 to 57 us, one of 32 keys 4.8 us.
//
// The weights are rounded to the 16-bit type for the second product, their sum is not; references, sums and values stay in 32 bits, and so do
// the parts and the prefix's sums in the workspace.
#include <hip/hip_runtime.h>
#include <cstdint>

#include "attn_device.h"
#include "attn_paged_launch.h"
#include "gfx950_common.h"

namespace {

using namespace gfx950;

// Beginning and ending a tile, in blocks, where work is shared out; counted as 1, workgroups with many short tiles end last. Measured in us:
// narrow, 64 sequences of 200 to 8192 keys: 1: 140, 4: 132.5, 8: 131.7; wide, tokens up to 1024 in pieces of prompts beside decoding
// sequences: 1: 161, 4: 131, 8: 116, 12: 119, 16: 115; 16 sequences of up to 512 tokens behind up to 2000 keys: 6: 63.1, 8: 62.6, 12: 65.0,
// 16: 65.3; 48 of up to 128, 16 / 2 heads: 33.9, 32.5, 34.5, 33.0; 8 of up to 2000 behind up to 8000: 404, 401, 394, 410; equal tiles the same.
constexpr int PER_TILE_NARROW = 4, PER_TILE_WIDE = 8;
constexpr float NO_MAX = -3.0e38f;   // finite: the difference of two such maxima is 0, not NaN
constexpr float LN2 = 0.6931471805599453f;

// x of this lane and of lane l ^ 16 (or l ^ 32), in no order.  (The results are copied before their bits are taken as floats:
// __builtin_bit_cast of a vector's element reads element 0, whichever was named.)
__device__ __forceinline__ f32x2 pair16(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1];
    return f32x2{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ f32x2 pair32(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1];
    return f32x2{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
// over the four lanes l, l ^ 16, l ^ 32, l ^ 48 that hold a row
__device__ __forceinline__ float max_of_groups(float x) {
    f32x2 p = pair16(x);
    p = pair32(vmax(p[0], p[1]));
    return vmax(p[0], p[1]);
}
__device__ __forceinline__ float sum_of_groups(float x) {
    f32x2 p = pair16(x);
    p = pair32(p[0] + p[1]);
    return p[0] + p[1];
}
// x, but computed here: what is made from it is not kept in registers from one tile to the next
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}
// A kernel's first argument, to be read where it is used: a loop over pieces of work keeps no copy of it in scalar registers, which are
// too few and would be saved in vector registers, one lane each.
template <class T>
__device__ __forceinline__ const T& first_argument() {
    uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const T*)(const __attribute__((address_space(4))) T*)p;
}
// a value that is the same in every lane, for the scalar registers
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Of the 32 keys from key `first` on: which exist (bits of `there`) and come before `limit`.
__device__ __forceinline__ uint32_t seen_of(uint32_t there, int first, int limit) {
    const int left = limit - first;
    return left >= 32 ? there : left <= 0 ? 0u : there & ((1u << left) - 1u);
}

template <int D> struct Shape {
    static constexpr int KB = D == 128 ? 32 : 64;          // keys of a block
    static constexpr uint64_t ALL = KB == 64 ? ~0ull : (1ull << (KB & 63)) - 1;
    static constexpr int KT = KB / 16, KS = D / 32, DT = D / 16, ROW = 2 * D;
    static constexpr int BLOCK = KB * ROW;                 // bytes of a block of K or V
    static constexpr int NL = BLOCK / 1024;                // loads of a wavefront for one, 16 bytes a lane
    static constexpr int PITCH = D + 4;                    // floats of a row of sums in LDS
    static constexpr int BUF = 2 * BLOCK;                  // a wavefront's LDS: one block of K, one of V; its sums at the end
    static_assert(16 * PITCH * 4 <= BUF);
};

// A tile of rows and the keys it sees.
struct Tile {
    const int* table;     // pages of its keys
    int width;            // entries of it that may be read
    int row0, rows;       // first row within the sequence, rows in use (at most 16 RT)
    int tok0, hk;         // the sequence's first token; key head
    int first_limit;      // keys that row i of the sequence sees: first_limit + (i / G) * per_token
    int per_token;
    int keys;             // keys that its last row sees
};

// What a pass over a shared prefix left for every row: its sums, in `splits` pieces.
struct Prefix {
    const float *o, *ml;   // [splits][T * Hq][D]: weighted values; [splits][T * Hq][2]: maximum and sum of the weights
    int splits;
    long long rows;        // T * Hq
};
// where row r of a tile lies among the T * Hq rows of the result
__device__ __forceinline__ long long row_of(const PagedAttnLaunch& a, int tok0, int hk, int r) {
    const int i = a.by_G.of(r);
    return (long long)(tok0 + i) * a.Hq + hk * a.G + (r - i * a.G);
}

// 16 bytes per lane from global memory into LDS: lane l's land at lds_base + 16 l (lds_base uniform over the wavefront).  The
// compiler does not know of the transfer: the caller waits (wait_lds_dma) before it reads, and has read what it overwrites.
__device__ __forceinline__ void dma16(uint32_t lds_base, const void* p) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds_base), "v"(p) : "memory", "m0");
}
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Loads blocks of KB keys of the cache into LDS, rows of D with their 16-byte pieces swapped about against bank conflicts.  A wavefront
// loads N KiB of each, from the FIRST-th on.
//
// Page numbers come from the table 64 at a time: lane e holds page e % NP of the e / NP-th block from the first on (a wavefront's
// blocks are `stride` apart; NP pages a block, 1 where a page holds several blocks).  One load for many blocks: it waits for every
// load under way.  A load moves 4 to 16 whole rows; where those lie in one page, its address is a scalar and this lane's
// constant part of it.
template <int D, int KB, int N> struct Pager {
    static constexpr int ROW = 2 * D, ROWS = 1024 / ROW, KINDS = 16 / ROWS;   // rows of a load; loads whose pieces are swapped differently
    const PagedCache& c;
    const int lane, first;
    const int np_shift, ahead, stride;
    int index = 0;            // of the next block since the pages were fetched
    long long at = 0;         // byte offset of this lane's page
    uint64_t valid = 0;       // lanes that have a page
    uint32_t part[KINDS];     // this lane's part of an address

    __device__ Pager(const PagedCache& c, int lane, int first, int stride)
        : c(c), lane(lane), first(first), np_shift(c.page_shift < (KB == 32 ? 5 : 6) ? (KB == 32 ? 5 : 6) - c.page_shift : 0), ahead(64 >> np_shift), stride(stride) {
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int j = i * ROWS + 16 * lane / ROW, piece = 16 * lane % ROW / 16;
            part[i] = 16 * lane / ROW * ROW + ((piece ^ attn_device::swz<D>(j & 15)) << 4);
        }
    }
    __device__ __forceinline__ void fetch(const Tile& t, int kb) {
        const long long key = (long long)(kb + (lane >> np_shift) * stride) * KB + ((long long)(lane & ((1 << np_shift) - 1)) << c.page_shift);
        const int e = (int)(key >> c.page_shift);
        int p = -1;
        if (key < t.keys && e < t.width) p = t.table[e];
        const bool is = p >= 0 && p < c.n_pages;
        valid = __ballot(is);
        at = 2 * ((is ? p : 0) * c.page_stride);   // (a key that does not exist is read from where one could be)
        index = 0;
    }
    __device__ __forceinline__ void next(const Tile& t, int kb) {
        if (++index == ahead) fetch(t, kb);
    }
    // which keys of block kb exist
    __device__ __forceinline__ uint64_t there(const Tile& t, int kb) const {
        constexpr uint64_t ALL = KB == 64 ? ~0ull : (1ull << (KB & 63)) - 1;
        const int from = index << np_shift;
        const uint64_t pages = np_shift == 6 ? ~0ull : (1ull << (1 << np_shift)) - 1;
        if (((valid >> from) & pages) == pages && (long long)(kb + 1) * KB <= t.keys) return ALL;
        const int j = lane & (KB - 1);
        return __ballot(((valid >> (from + (np_shift ? j >> c.page_shift : 0))) & 1) && kb * KB + j < t.keys) & ALL;
    }
    __device__ __forceinline__ void load(uint32_t lds, const char* base, int kb) const {
        const int mask = (1 << c.page_shift) - 1, from = index << np_shift;
        if (mask >= ROWS - 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j = ROWS * (first + i), e = from + (np_shift ? j >> c.page_shift : 0);
                const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, e);
                const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)at >> 32), e);
                lds_dma16(lds + 1024 * i, base + ((uint64_t)hi << 32 | lo) + paged_key_offset(kb * KB + j, mask, ROW), part[i % KINDS]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j = ROWS * (first + i) + 16 * lane / ROW;
                const long long page = __shfl(at, from + (j >> c.page_shift), 64);
                dma16(lds + 1024 * i, base + page + paged_key_offset(kb * KB + j, mask, ROW) + (part[i % KINDS] & (ROW - 1)));
            }
        }
    }
    // what is not there becomes 0: a hidden value has weight 0, but 0 * NaN is not 0
    __device__ __forceinline__ void clear(uint32_t lds, uint64_t there) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = ROWS * (first + i) + 16 * lane / ROW;
            if (!((there >> j) & 1)) lds_write_b128(lds + 1024 * i + 16 * lane, u32x4{0u, 0u, 0u, 0u});
        }
        lds_reads_done();
    }
};

template <int DTY, int D, int RT, int NW> struct Worker {
    using S = Shape<D>;
    const PagedAttnLaunch& a;
    const int lane = here(threadIdx.x & 63), wave = here(threadIdx.x >> 6), c = lane >> 4, r16 = lane & 15;
    char* lds;            // this wavefront's buffer
    const uint32_t kbuf, vbuf;
    u32x4 q[RT][S::KS];
    f32x4 o[RT][S::DT];
    float m[RT], l[RT];
    int limit[RT];
    Pager<D, S::KB, S::NL> pager;

    __device__ Worker(const PagedAttnLaunch& a, char* all)
        : a(a), lds(all + wave * S::BUF), kbuf(uniform((int)(uintptr_t)(LDS_AS char*)all) + uniform(wave) * S::BUF), vbuf(kbuf + S::BLOCK), pager(a.c, lane, 0, NW) {}

    // the weights of a block: its logits against this lane's rows, the references moved up where need be
    __device__ __forceinline__ void weights(u32x4 (&p)[RT][S::KT / 2], int kb, uint64_t there, int first_limit) {
        f32x4 s[RT][S::KT];
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < S::KS; ++ks) {
                const u32x4 k = lds_read_b128(kbuf + (16 * kt + r16) * S::ROW + (((c + 4 * ks) ^ attn_device::swz<D>(r16)) << 4));
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][kt] = Elem<DTY>::mfma16(k, q[rt][ks], s[rt][kt]);
            }
        }
        const bool holes = there != S::ALL;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (holes || (kb + 1) * S::KB > first_limit) {
#pragma unroll
                for (int kp = 0; kp < S::KT / 2; ++kp) {
                    const uint32_t seen = seen_of((uint32_t)(there >> (32 * kp)), kb * S::KB + 32 * kp, limit[rt]) >> (4 * c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = s[rt][2 * kp + e / 4][e % 4];
                        s[rt][2 * kp + e / 4][e % 4] = (seen & (1u << (16 * (e / 4) + e % 4))) ? x : -__builtin_inff();
                    }
                }
            }
            float mx = s[rt][0][0];
#pragma unroll
            for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = vmax(mx, s[rt][kt][i]);
            mx = max_of_groups(mx) * a.c_log2;
            // the reference follows the maximum when that has grown by more than 2^8: weights stay far from overflow
            if (__ballot(mx > m[rt] + 8.f)) {
                const float n = vmax(m[rt], mx), f = __builtin_amdgcn_exp2f(m[rt] - n);
                m[rt] = n;
                l[rt] *= f;
#pragma unroll
                for (int d = 0; d < S::DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[rt][d][i] *= f;
            }
#pragma unroll
            for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[rt][kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][kt][i], a.c_log2, -m[rt]));
                    l[rt] += s[rt][kt][i];
                }
#pragma unroll
            for (int kp = 0; kp < S::KT / 2; ++kp)
                p[rt][kp] = u32x4{Elem<DTY>::pack2(s[rt][2 * kp][0], s[rt][2 * kp][1]), Elem<DTY>::pack2(s[rt][2 * kp][2], s[rt][2 * kp][3]),
                                  Elem<DTY>::pack2(s[rt][2 * kp + 1][0], s[rt][2 * kp + 1][1]), Elem<DTY>::pack2(s[rt][2 * kp + 1][2], s[rt][2 * kp + 1][3])};
        }
    }
    __device__ __forceinline__ void values(const u32x4 (&p)[RT][S::KT / 2], uint64_t there) {
        if (there != S::ALL) pager.clear(vbuf, there);
        const int j = 4 * c + (r16 >> 2), z = attn_device::swz<D>(j);
#pragma unroll
        for (int kp = 0; kp < S::KT / 2; ++kp)
#pragma unroll
            for (int d = 0; d < S::DT; ++d) {
                const uint32_t at = vbuf + (32 * kp + j) * S::ROW + (((2 * d + ((r16 >> 1) & 1)) ^ z) << 4) + 8 * (r16 & 1);
                const u32x2 lo = lds_read_tr16(at), hi = lds_read_tr16(at + 16 * S::ROW);
                const u32x4 vt = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][d] = Elem<DTY>::mfma16(vt, p[rt][kp], o[rt][d]);
            }
    }

    // the sums over the prefix, its pieces shared out over the wavefronts
    __device__ __forceinline__ void start_from(const Prefix& px, const Tile& t) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (16 * rt + r16 >= t.rows) continue;
            const long long row = row_of(a, t.tok0, t.hk, t.row0 + 16 * rt + r16);
#pragma unroll 2
            for (int s = wave; s < px.splits; s += NW) {
                const long long at = s * px.rows + row;
                const f32x2 ml = *(const f32x2*)(px.ml + 2 * at);
                f32x4 x[S::DT];
#pragma unroll
                for (int d = 0; d < S::DT; ++d) x[d] = *(const f32x4*)(px.o + at * D + 16 * d + 4 * c);
                const float n = __builtin_fmaxf(m[rt], ml[0]), f = __builtin_amdgcn_exp2f(m[rt] - n), g = __builtin_amdgcn_exp2f(ml[0] - n);
                m[rt] = n;
                l[rt] = l[rt] * f + (c == 0 ? g * ml[1] : 0.f);   // the four lanes of a row are added up at the end
#pragma unroll
                for (int d = 0; d < S::DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[rt][d][i] = o[rt][d][i] * f + x[d][i] * g;
            }
        }
    }

    // the blocks from, from + NW, ... below `to` of the tile's keys, on top of what px holds
    __device__ __forceinline__ void run(const Tile& t, int from, int to, const Prefix& px) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = 16 * rt + r16, row = t.row0 + r, i = a.by_G.of(row), g = row - i * a.G;
            limit[rt] = r < t.rows ? t.first_limit + i * t.per_token : 0;
            const char* src = (const char*)a.q + 2 * ((long long)(t.tok0 + i) * a.q_stride + (t.hk * a.G + g) * D);
#pragma unroll
            for (int ks = 0; ks < S::KS; ++ks) {
                q[rt][ks] = u32x4{0u, 0u, 0u, 0u};
                if (r < t.rows) q[rt][ks] = *(const u32x4*)(src + 64 * ks + 16 * c) ^ a.q_sign;
            }
            m[rt] = NO_MAX;
            l[rt] = 0.f;
#pragma unroll
            for (int d = 0; d < S::DT; ++d) o[rt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int first_limit = t.first_limit + a.by_G.of(t.row0) * t.per_token;
        const int end = (t.keys + S::KB - 1) / S::KB;
        to = to < end ? to : end;
        int kb = from + uniform(wave);
        const size_t head = ((size_t)t.hk << a.c.page_shift) * S::ROW;
        const char *kc = (const char*)a.c.k + head, *vc = (const char*)a.c.v + head;
        uint64_t now = 0;
        if (kb < to) {
            pager.fetch(t, kb);
            pager.load(kbuf, kc, kb);
            pager.load(vbuf, vc, kb);
            now = pager.there(t, kb);
        }
        if (px.splits > 0) start_from(px, t);
        if (kb >= to) return;
        // One block of K and one of V, each refilled as soon as it is used up: while the weights of a block are computed its V is on its
        // way, while V is used the next K.
        while (true) {
            const bool more = kb + NW < to;
            u32x4 p[RT][S::KT / 2];
            wait_lds_dma<S::NL>();
            weights(p, kb, now, first_limit);
            if (more) {
                pager.next(t, kb + NW);
                lds_reads_done();
                pager.load(kbuf, kc, kb + NW);
                wait_lds_dma<S::NL>();
            } else {
                wait_lds_dma<0>();
            }
            values(p, now);
            if (!more) break;
            lds_reads_done();
            kb += NW;
            pager.load(vbuf, vc, kb);
            now = pager.there(t, kb);
        }
        lds_reads_done();
    }
};

// four values of a row's result: divides, rounds, stores
template <int DTY, int D>
__device__ __forceinline__ void finish(const PagedAttnLaunch& a, long long row, int d, float m, float l, f32x4 o) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const u32x2 w = {Elem<DTY>::pack2(o[0] * inv, o[1] * inv), Elem<DTY>::pack2(o[2] * inv, o[3] * inv)};
    *(u32x2*)((uint16_t*)a.o + row * D + d) = w;
    if (a.lse && d == 0) a.lse[row] = LN2 * (m + __builtin_amdgcn_logf(l));
}

// Adds up the wavefronts' sums of row tile rt; out(row of the tile, d, m, l, four values).
template <int DTY, int D, int RT, int NW, class Out>
__device__ __forceinline__ void merge(Worker<DTY, D, RT, NW>& w, char* lds, float (*ml)[16][2], int rt, Out out) {
    using S = Shape<D>;
    const float l = sum_of_groups(w.l[rt]);
    if (w.c == 0) {
        ml[w.wave][w.r16][0] = w.m[rt];
        ml[w.wave][w.r16][1] = l;
    }
#pragma unroll
    for (int d = 0; d < S::DT; ++d) *(f32x4*)(w.lds + 4 * (w.r16 * S::PITCH + 16 * d + 4 * w.c)) = w.o[rt][d];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * D / 4; e += 64 * NW) {
        const int r = e / (D / 4), d = 4 * (e % (D / 4));
        float m = NO_MAX, l = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) m = vmax(m, ml[v][r][0]);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float f = __builtin_amdgcn_exp2f(ml[v][r][0] - m);
            l += f * ml[v][r][1];
            const f32x4 x = *(const f32x4*)(lds + v * S::BUF + 4 * (r * S::PITCH + d));
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += f * x[i];
        }
        out(16 * rt + r, d, m, l, o);
    }
    __syncthreads();
}

// One split tile, for the kernel that adds its parts up.
struct Split {
    int parts;            // 0: this workgroup's last tile was not split
    int row0, rows, tok0, hk, pad[3];
};

struct Schedule {
    int balanced, workgroups;
    float* parts;         // [2 * workgroups][16 RT * (D + 2)]: the part of a tile that began in an earlier workgroup; of one that goes on
    Split* splits;        // [workgroups]
};

// A sequence as the kernel takes it: whatever the tensors hold, no index leaves its buffer.
struct Seq {
    int tok0, n, rows, keys;
};
__device__ __forceinline__ Seq seq_of(const PagedAttnLaunch& a, int b) {
    Seq s;
    const int lo = a.c.cu_q[b], hi = a.c.cu_q[b + 1], keys = a.c.kv_len[b];
    const long long most = (long long)a.c.width << a.c.page_shift;
    s.tok0 = lo < 0 ? 0 : lo > a.c.T ? a.c.T : lo;
    s.n = (hi > a.c.T ? a.c.T : hi) - s.tok0;
    s.n = s.n < 0 ? 0 : s.n;
    s.rows = (s.n < a.max_q ? s.n : a.max_q) * a.G;
    s.keys = keys < 0 ? 0 : keys > most ? (int)most : keys;
    return s;
}

// Shares the tiles of R rows out over the workgroups, and calls body(tile, first, from, to, part) for each piece of this one's: blocks
// from .. to - 1 of KB keys; first: the piece that the prefix goes with; part: null where the piece is the whole tile, else where its sums go.
// DIRECT: a workgroup for each sequence and key head, whose rows are one tile.  Else, not balanced: a workgroup for each tile.  Balanced: the work of all tiles in a row (sequence, tile, key head), cut into equal
// pieces; tiles that are cut are added up by attn_paged_join_kernel.
__device__ __forceinline__ Seq uniform(Seq s) { return Seq{uniform(s.tok0), uniform(s.n), uniform(s.rows), uniform(s.keys)}; }
template <int R, int KB, int D, int NW, int PER_TILE, int LEAST, bool DIRECT, class Body>
__device__ __forceinline__ void share_out(const PagedAttnLaunch& a, const Schedule& sc, Body body) {
    constexpr int THREADS = 64 * NW;
    __shared__ int sums[NW], found[2];
    __shared__ Seq found_seq;
    const int Hk = a.c.Hk, B = a.c.B;

    auto tiles_of = [&](const Seq& s) { return (s.rows + R - 1) / R; };
    // a tile's share of the work: its blocks (those past max_kv keys go with the last piece), and what it costs to begin and to end
    // one.  (All of it together fits 32 bits: paged_plan.)
    auto work_of = [&](const Seq& s) { return sc.balanced ? ((s.keys < a.max_kv ? s.keys : a.max_kv) + KB - 1) / KB + PER_TILE : 1; };
    const int w = blockIdx.x;
    int total = 1, N = 1, u = 0, u_end = 1;
    int b, index, at = 0, size = 1, tiles = 1;      // (tile, key head) as one number; how far into its work, and all of that
    Seq s;
    // where the work of workgroup x begins: x * total / N, the whole part and the rest of total / N by themselves (x * rest < 2^18)
    int each = 1, over = 0;
    auto begin_of = [&](int x) {
        const int n = x * over;
        int q = (int)((float)n * __builtin_amdgcn_rcpf((float)N));
        q += n - q * N >= N ? 1 : n - q * N < 0 ? -1 : 0;
        return x * each + q;
    };
    if constexpr (DIRECT) {   // a tile to a workgroup, and a tile a sequence
        b = a.by_Hk.of(w);
        index = w - b * Hk;
        s = uniform(seq_of(a, b));
        if (s.rows == 0) return;
    } else {
        // every thread sums the work of a strip of sequences, a scan over the threads places the strips
        const int strip = (B + THREADS - 1) / THREADS, b0 = threadIdx.x * strip, b1 = b0 + strip < B ? b0 + strip : B;
        auto weight = [&](const Seq& s) { return tiles_of(s) * Hk * work_of(s); };
        int mine = 0;
        Seq first = {0, 0, 0, 0};
        for (int b = b0; b < b1; ++b) {
            const Seq s = seq_of(a, b);
            if (b == b0) first = s;
            mine += weight(s);
        }
        int upto = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int x = __shfl_up(upto, off, 64);
            if ((int)(threadIdx.x & 63) >= off) upto += x;
        }
        if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = upto;
        if (threadIdx.x == 0) found[0] = -1;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            if (v < (int)(threadIdx.x >> 6)) upto += sums[v];
            total += sums[v];
        }
        total = uniform(total);
        // workgroups with work; a piece is a block or more for each wavefront that takes blocks of its own
        const int most = (total + LEAST - 1) / LEAST;
        N = sc.balanced ? (most < sc.workgroups ? most : sc.workgroups) : total;
        if (w >= N) {
            if (sc.balanced && threadIdx.x == 0) sc.splits[w].parts = 0;
            return;
        }
        each = sc.balanced ? (int)((unsigned)total / (unsigned)N) : 1;
        over = sc.balanced ? total - each * N : 0;
        u = uniform(begin_of(w));
        u_end = uniform(begin_of(w + 1));
        if (upto - mine <= u && u < upto) {
            int rest = u - (upto - mine), b = b0;
            for (int x = weight(first); rest >= x && b + 1 < b1; x = weight(first)) {
                rest -= x;
                first = seq_of(a, ++b);
            }
            found[0] = b;
            found[1] = rest;
            found_seq = first;
        }
        __syncthreads();
        b = uniform(found[0]);
        s = uniform(found_seq);
        size = work_of(s), tiles = tiles_of(s);
        const int rest = uniform(found[1]);
        index = rest / size, at = rest - index * size;
        // (offsets that overlap can make sums past 32 bits: their results mean nothing, but no index leaves its range)
        if (b < 0 || rest < 0 || index >= tiles * Hk) {
            if (sc.balanced && threadIdx.x == 0) sc.splits[w].parts = 0;
            return;
        }
    }
    bool told = false;

    while (u < u_end) {
        // the key head runs fastest: workgroups that follow each other go to the 8 chiplets in turn, so that with 8 key heads
        // each chiplet's cache sees one; the last tiles, which see the most keys, come first
        const int order = a.by_Hk.of(index), hk = index - order * Hk, tile = tiles - 1 - order;
        Tile t;
        t.table = a.c.table + (size_t)b * a.c.table_stride;
        t.width = a.c.width;
        t.row0 = tile * R;
        t.rows = s.rows - t.row0 < R ? s.rows - t.row0 : R;
        t.tok0 = s.tok0;
        t.hk = hk;
        t.first_limit = s.keys - s.n + 1;
        t.per_token = 1;
        t.keys = t.first_limit + a.by_G.of(t.row0 + t.rows - 1);
        t.keys = t.keys < 0 ? 0 : t.keys;
        const int left = u_end - u, to = size - at <= left ? size : at + left;
        const bool split = !DIRECT && (at != 0 || to != size);
        // the blocks of this piece, at * (size - PER_TILE) / size and so on; there may be none
        auto block_of = [&](int x) { return x - (int)(((unsigned)x * PER_TILE + size - 1) / (unsigned)size); };
        body(t, DIRECT || at == 0, split ? block_of(at) : 0, !DIRECT && to < size ? block_of(to) : 0x7fffffff,
             split ? sc.parts + (2LL * w + (at == 0)) * R * (D + 2) : (float*)nullptr);
        if (split && at == 0) {
            if (threadIdx.x == 0) {
                // how many workgroups follow this one in the tile
                int parts = 2;
                const int end = u + size;
                while (w + parts < N && begin_of(w + parts) < end) {
                    const int more = (end - begin_of(w + parts)) / (each + 1);
                    parts += more > 0 ? more : 1;
                }
                parts = parts < N - w ? parts : N - w;
                sc.splits[w] = Split{parts, t.row0, t.rows, t.tok0, t.hk, {0, 0, 0}};
            }
            told = true;
        }
        if constexpr (DIRECT) return;
        u += to - at;
        at = 0;
        if (++index == tiles * Hk && u < u_end) {
            index = 0;
            do {
                if (++b >= B) break;
                s = uniform(seq_of(a, b));
            } while (s.rows == 0);
            if (b >= B) break;
            size = work_of(s);
            tiles = tiles_of(s);
        }
    }
    if (sc.balanced && !told && threadIdx.x == 0) sc.splits[w].parts = 0;
}

template <int DTY, int D, int RT, int NW, bool DIRECT>
__global__ __launch_bounds__(64 * NW, 2) void attn_paged_kernel(PagedAttnLaunch arg, Schedule sc, Prefix px) {
    using S = Shape<D>;
    constexpr int R = 16 * RT;
    __shared__ __align__(16) char lds[NW * S::BUF];
    __shared__ float ml[NW][16][2];
    share_out<R, S::KB, D, NW, PER_TILE_NARROW, NW, DIRECT>(arg, sc, [&](const Tile& t, bool first, int from, int to, float* part) {
        const PagedAttnLaunch& a = DIRECT ? arg : first_argument<PagedAttnLaunch>();
        Worker<DTY, D, RT, NW> worker(a, lds);
        worker.run(t, from, to, first ? px : Prefix{});
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            merge(worker, lds, ml, rt, [&](int r, int d, float m, float l, f32x4 o) {
                if (r >= t.rows) return;
                if (part) {
                    *(f32x4*)(part + r * D + d) = o;
                    if (d == 0) *(f32x2*)(part + R * D + 2 * r) = f32x2{m, l};
                } else {
                    finish<DTY, D>(a, row_of(a, t.tok0, t.hk, t.row0 + r), d, m, l, o);
                }
            });
    });
}

// Adds up the parts of the tile that workgroup blockIdx.x of the kernel above began and others went on with.
__device__ __forceinline__ const float* part_of(const Schedule& sc, int w, int p, int size) { return sc.parts + (2LL * (w + p) + (p == 0)) * size; }
// s, o += the sums of which m is the maximum: the loads of some parts come before the first is used
struct Sums {
    float m = NO_MAX, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float pm, float pl, const f32x4& po) {
        const float n = __builtin_fmaxf(m, pm), f = __builtin_amdgcn_exp2f(m - n), g = __builtin_amdgcn_exp2f(pm - n);
        m = n;
        l = l * f + pl * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = o[i] * f + po[i] * g;
    }
    // parts p0, p0 + step, ... below p1 of row r, four values from d on
    template <int R, int D, int AT_ONCE>
    __device__ __forceinline__ void add_parts(const Schedule& sc, int w, int p0, int p1, int step, int r, int d) {
        for (int p = p0; p < p1; p += AT_ONCE * step) {
            f32x2 ml[AT_ONCE];
            f32x4 x[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                ml[u] = f32x2{NO_MAX, 0.f};
                x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (p + u * step < p1) {
                    const float* part = part_of(sc, w, p + u * step, R * (D + 2));
                    ml[u] = *(const f32x2*)(part + R * D + 2 * r);
                    x[u] = *(const f32x4*)(part + r * D + d);
                }
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) add(ml[u][0], ml[u][1], x[u]);
        }
    }
};
constexpr int JOIN_THREADS = 256;
// Few parts: the lanes of a wavefront hold 64 / (D / 4) rows.
template <int DTY, int D, int R>
__global__ __launch_bounds__(JOIN_THREADS) void attn_paged_join_kernel(PagedAttnLaunch a, Schedule sc) {
    constexpr int Q = D / 4, ROWS = JOIN_THREADS / Q;
    const Split sp = sc.splits[blockIdx.x];
    if (sp.parts == 0) return;
    const int d = 4 * (threadIdx.x % Q);
    for (int r = blockIdx.y * ROWS + threadIdx.x / Q; r < sp.rows; r += ROWS * gridDim.y) {
        Sums s;
        s.add_parts<R, D, 4>(sc, blockIdx.x, 0, sp.parts, 1, r, d);
        finish<DTY, D>(a, row_of(a, sp.tok0, sp.hk, sp.row0 + r), d, s.m, s.l, s.o);
    }
}
// Many parts, few rows: a workgroup a row, its threads share out the parts.
template <int DTY, int D, int R>
__global__ __launch_bounds__(JOIN_THREADS) void attn_paged_join_many_kernel(PagedAttnLaunch a, Schedule sc) {
    constexpr int Q = D / 4, SHARES = JOIN_THREADS / Q;
    __shared__ __align__(16) f32x4 sums[SHARES][Q];
    __shared__ f32x2 ml[SHARES];
    const Split sp = sc.splits[blockIdx.x];
    if (sp.parts == 0) return;
    const int piece = threadIdx.x % Q, share = threadIdx.x / Q;
    for (int r = blockIdx.y; r < sp.rows; r += gridDim.y) {
        Sums s;
        s.add_parts<R, D, 8>(sc, blockIdx.x, share, sp.parts, SHARES, r, 4 * piece);
        sums[share][piece] = s.o;
        if (piece == 0) ml[share] = f32x2{s.m, s.l};
        __syncthreads();
        if (share == 0) {
#pragma unroll
            for (int v = 1; v < SHARES; ++v) s.add(ml[v][0], ml[v][1], sums[v][piece]);
            finish<DTY, D>(a, row_of(a, sp.tok0, sp.hk, sp.row0 + r), 4 * piece, s.m, s.l, s.o);
        }
        __syncthreads();
    }
}

// The pass over the shared prefix: tiles of the batch's rows, each key head, `splits` pieces of the keys.
template <int R, int KB>
__device__ __forceinline__ Tile prefix_tile(const PagedAttnLaunch& a, int splits, int& split, int& from, int& to) {
    // the key head fastest, as in share_out
    const int rest = a.by_Hk.of(blockIdx.x), hk = blockIdx.x - rest * a.c.Hk, tile = rest / splits;
    split = rest - tile * splits;
    Tile t;
    t.table = a.prefix_table;
    t.width = ((a.prefix_len - 1) >> a.c.page_shift) + 1;
    t.row0 = tile * R;
    const int rows = a.c.T * a.G;
    t.rows = rows - t.row0 < R ? rows - t.row0 : R;
    t.tok0 = 0;
    t.hk = hk;
    t.first_limit = t.keys = a.prefix_len;
    t.per_token = 0;
    const long long nb = (a.prefix_len - 1) / KB + 1;
    from = (int)(nb * split / splits);
    to = (int)(nb * (split + 1) / splits);
    return t;
}
// four values of a row's sums over the prefix, for finish()
template <int D>
__device__ __forceinline__ void leave(const PagedAttnLaunch& a, const Prefix& px, int split, long long row, int d, float m, float l, f32x4 o) {
    const long long at = split * px.rows + row;
    *(f32x4*)(const_cast<float*>(px.o) + at * D + d) = o;
    if (d == 0) *(f32x2*)(const_cast<float*>(px.ml) + 2 * at) = f32x2{m, l};
}

template <int DTY, int D, int RT>
__global__ __launch_bounds__(64 * NARROW_PREFIX_WAVES, 2) void attn_paged_prefix_kernel(PagedAttnLaunch a, Prefix px) {
    using S = Shape<D>;
    constexpr int NW = NARROW_PREFIX_WAVES;
    __shared__ __align__(16) char lds[NW * S::BUF];
    __shared__ float ml[NW][16][2];
    int split, from, to;
    const Tile t = prefix_tile<16 * RT, S::KB>(a, px.splits, split, from, to);
    Worker<DTY, D, RT, NW> worker(a, lds);
    worker.run(t, from, to, Prefix{});
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
        merge(worker, lds, ml, rt, [&](int r, int d, float m, float l, f32x4 o) {
            if (r < t.rows) leave<D>(a, px, split, row_of(a, 0, t.hk, t.row0 + r), d, m, l, o);
        });
}

// ---- Many rows: bound by the matrix and vector pipes.  A workgroup has 128 rows, 32 to a wavefront, and its four wavefronts share
// blocks of 64 keys, double-buffered in LDS.  As above everything is transposed, on v_mfma_f32_32x32x16: register r of key block jb
// holds  S[row = lane % 32][key = 32 jb + 8 (r / 4) + 4 h + r % 4]  (h = lane / 32), registers 8t .. 8t + 7 are the B operand of the second
// product as they are, and V^T is fetched in that order of keys.
// Measured, 32 query and 8 key heads of 128, bfloat16: 4096 tokens of one sequence 158 us (870 TFLOP/s), pieces of up to 1024 tokens beside
// decoding sequences 111 to 116 us (710 to 675), 256 rows a key head over 8192 shared keys 22 us (390: a workgroup a compute unit).
template <int D> struct Wide {
    static constexpr int NW = 4, R = 32 * NW, KB = 64, JB = KB / 32, KS = D / 16, DB = D / 32, ROW = 2 * D;
    static constexpr int BLOCK = KB * ROW, NL = BLOCK / 1024 / NW;   // bytes of a block of K or V; loads of a wavefront for its quarter
    static constexpr int LDS = 4 * BLOCK;
};

template <int DTY, int D> struct WideWorker {
    using S = Wide<D>;
    const PagedAttnLaunch& a;
    const int lane = here(threadIdx.x & 63), wave = here(threadIdx.x >> 6), h = lane >> 5, r32 = lane & 31;
    const uint32_t lds;
    u32x4 q[S::KS];
    f32x16 o[S::DB];
    float m, l;
    int limit;
    Pager<D, S::KB, S::NL> pager;
    // this lane's addresses in a block: its row of K, a piece for each step; its part of V's transposing reads
    const LDS_AS char *kp[S::KS], *vp[S::DB][2];

    __device__ WideWorker(const PagedAttnLaunch& a, char* all)
        : a(a), lds(uniform((int)(uintptr_t)(LDS_AS char*)all)), pager(a.c, lane, uniform(wave) * S::NL, 1) {
        const LDS_AS char* base = (const LDS_AS char*)all;
        const int i = lane & 15, row = 4 * h + (i >> 2), chunk = 2 * ((lane >> 4) & 1) + ((i >> 1) & 1);
#pragma unroll
        for (int ks = 0; ks < S::KS; ++ks) kp[ks] = base + r32 * S::ROW + (((2 * ks + h) ^ attn_device::swz<D>(r32 & 15)) << 4);
#pragma unroll
        for (int d = 0; d < S::DB; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                vp[d][u] = base + S::BLOCK + (row + 8 * u) * S::ROW + (((4 * d + chunk) ^ attn_device::swz<D>(row + 8 * u)) << 4) + 8 * (i & 1);
    }

    __device__ __forceinline__ void load(int buf, const char* kc, const char* vc, int kb) const {
        const uint32_t to = lds + buf * 2 * S::BLOCK + pager.first * 1024;
        pager.load(to, kc, kb);
        pager.load(to + S::BLOCK, vc, kb);
    }
    template <int BUF>
    __device__ __forceinline__ u32x4 key_piece(int jb, int ks) const { return *(const LDS_AS u32x4*)(kp[ks] + BUF * 2 * S::BLOCK + 32 * jb * S::ROW); }
    template <int BUF>
    __device__ __forceinline__ u32x4 value_piece(int step, int d) const {   // step: 16 keys
        s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(vp[d][0] + BUF * 2 * S::BLOCK + 16 * step * S::ROW));
        s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(vp[d][1] + BUF * 2 * S::BLOCK + 16 * step * S::ROW));
        const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
        return u32x4{a[0], a[1], b[0], b[1]};
    }
    template <int BUF>
    __device__ __forceinline__ void compute(int kb, uint64_t there, int first_limit) {
        f32x16 s[S::JB];
        // the reads of the next 32 keys run ahead of the products of these
        u32x4 k[2][S::KS];
#pragma unroll
        for (int ks = 0; ks < S::KS; ++ks) k[0][ks] = key_piece<BUF>(0, ks);
#pragma unroll
        for (int jb = 0; jb < S::JB; ++jb) {
            s[jb] = f32x16{};
            if (jb + 1 < S::JB)
#pragma unroll
                for (int ks = 0; ks < S::KS; ++ks) k[(jb + 1) & 1][ks] = key_piece<BUF>(jb + 1, ks);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int ks = 0; ks < S::KS; ++ks) s[jb] = Elem<DTY>::mfma(k[jb & 1][ks], q[ks], s[jb]);
        }
        if (there != ~0ull || (kb + 1) * S::KB > first_limit) {
#pragma unroll
            for (int jb = 0; jb < S::JB; ++jb) {
                const uint32_t seen = seen_of((uint32_t)(there >> (32 * jb)), kb * S::KB + 32 * jb, limit) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[jb][r] = (seen & (1u << (8 * (r / 4) + r % 4))) ? s[jb][r] : -__builtin_inff();
            }
        }
        u32x4 v[2][S::DB];
#pragma unroll
        for (int d = 0; d < S::DB; ++d) v[0][d] = value_piece<BUF>(0, d);
        float mx = s[0][0];
#pragma unroll
        for (int jb = 0; jb < S::JB; ++jb)
#pragma unroll
            for (int r = 0; r < 16; r += 2) mx = attn_device::vmax3(mx, s[jb][r], s[jb][r + 1]);
        const f32x2 both = pair32(mx);
        mx = vmax(both[0], both[1]) * a.c_log2;
        if (__ballot(mx > m + 8.f)) {
            const float n = vmax(m, mx), f = __builtin_amdgcn_exp2f(m - n);
            m = n;
            l *= f;
#pragma unroll
            for (int d = 0; d < S::DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= f;
        }
        // the wavefront that has weights to compute and products to feed goes before one that waits for its next block (4096 tokens,
        // 32 / 8 heads, D = 128: 157 us, 167 without)
        __builtin_amdgcn_s_setprio(1);
        constexpr int STEPS = 2 * S::JB;   // of 16 keys
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            float w8[8];
            u32x4 p;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w8[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t / 2][8 * (t % 2) + e], a.c_log2, -m));
                l += w8[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = Elem<DTY>::pack2(w8[2 * e], w8[2 * e + 1]);
            if (t + 1 < STEPS)
#pragma unroll
                for (int d = 0; d < S::DB; ++d) v[(t + 1) & 1][d] = value_piece<BUF>(t + 1, d);
#pragma unroll
            for (int d = 0; d < S::DB; ++d) o[d] = Elem<DTY>::mfma(v[t & 1][d], p, o[d]);
        }
        __builtin_amdgcn_s_setprio(0);
    }

    __device__ __forceinline__ void start_from(const Prefix& px, const Tile& t) {
        if (32 * wave + r32 >= t.rows) return;
        const long long row = row_of(a, t.tok0, t.hk, t.row0 + 32 * wave + r32);
#pragma unroll 1
        for (int s = 0; s < px.splits; ++s) {
            const long long at = s * px.rows + row;
            const f32x2 ml = *(const f32x2*)(px.ml + 2 * at);
            f32x4 x[S::DB][4];
#pragma unroll
            for (int d = 0; d < S::DB; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[d][e] = *(const f32x4*)(px.o + at * D + 32 * d + 8 * e + 4 * h);
            const float n = __builtin_fmaxf(m, ml[0]), f = __builtin_amdgcn_exp2f(m - n), g = __builtin_amdgcn_exp2f(ml[0] - n);
            m = n;
            l = l * f + (h == 0 ? g * ml[1] : 0.f);   // the two lanes of a row are added up at the end
#pragma unroll
            for (int d = 0; d < S::DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * f + x[d][r / 4][r % 4] * g;
        }
    }

    // the blocks from .. to - 1 of the tile's keys, on top of what px holds
    __device__ __forceinline__ void run(const Tile& t, int from, int to, const Prefix& px) {
        const int r = 32 * wave + r32, row = t.row0 + r, i = a.by_G.of(row), g = row - i * a.G;
        limit = r < t.rows ? t.first_limit + i * t.per_token : 0;
        const char* src = (const char*)a.q + 2 * ((long long)(t.tok0 + i) * a.q_stride + (t.hk * a.G + g) * D);
#pragma unroll
        for (int ks = 0; ks < S::KS; ++ks) {
            q[ks] = u32x4{0u, 0u, 0u, 0u};
            if (r < t.rows) q[ks] = *(const u32x4*)(src + 32 * ks + 16 * h) ^ a.q_sign;
        }
        m = NO_MAX;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < S::DB; ++d) o[d] = f32x16{};
        // what this wavefront's first row sees, and its last
        const int w32 = 32 * uniform(wave), rows = t.rows - w32 < 32 ? t.rows - w32 : 32;
        const int first_limit = t.first_limit + a.by_G.of(t.row0 + w32) * t.per_token;
        const int last_limit = rows > 0 ? t.first_limit + a.by_G.of(t.row0 + w32 + rows - 1) * t.per_token : 0;
        const int end = (t.keys + S::KB - 1) / S::KB;
        to = to < end ? to : end;
        int kb = from;
        const size_t head = ((size_t)t.hk << a.c.page_shift) * S::ROW;
        const char *kc = (const char*)a.c.k + head, *vc = (const char*)a.c.v + head;
        uint64_t there = 0;
        if (kb < to) {
            pager.fetch(t, kb);
            load(0, kc, vc, kb);
            there = pager.there(t, kb);
        }
        if (px.splits > 0) start_from(px, t);
        if (kb >= to) return;
        auto arrived = [&](int buf) {
            wait_lds_dma<0>();
            if (there != ~0ull) pager.clear(lds + (2 * buf + 1) * S::BLOCK + pager.first * 1024, there);
        };
        arrived(0);
        __syncthreads();
        // while one block is computed the next one is on its way to the other half of LDS
        auto step = [&]<int BUF>() {
            const uint64_t now = there;
            const bool more = kb + 1 < to;
            if (more) {
                pager.next(t, kb + 1);
                load(BUF ^ 1, kc, vc, kb + 1);
                there = pager.there(t, kb + 1);
            }
            if (kb * S::KB < last_limit) compute<BUF>(kb, now, first_limit);
            if (more) arrived(BUF ^ 1);
            __syncthreads();
            ++kb;
        };
        while (true) {
            step.template operator()<0>();
            if (kb >= to) break;
            step.template operator()<1>();
            if (kb >= to) break;
        }
    }

    // out(row of the tile, d, m, l, four values) for all that this wavefront holds, turned round in its quarter of LDS so that
    // neighbouring lanes have neighbouring elements of a row
    template <class Out>
    __device__ __forceinline__ void results(const Tile& t, Out out) {
        constexpr int Q = D / 4;   // pieces of four values in a row; they change places with the row against bank conflicts
        static_assert(32 * D * 4 * S::NW <= S::LDS);
        const f32x2 ls = pair32(l);
        const float sum = ls[0] + ls[1];
        const int lane = here(threadIdx.x & 63), h = lane >> 5, r32 = lane & 31;
        const uint32_t mine = lds + uniform(wave) * (32 * D * 4);
#pragma unroll
        for (int d = 0; d < S::DB; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(LDS_AS f32x4*)(uintptr_t)(mine + r32 * (4 * D) + (((8 * d + 2 * e + h) ^ (r32 & (Q - 1))) << 4)) =
                    f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
        const int rows = t.rows - 32 * uniform(wave);
        constexpr int AT_ONCE = 64 / Q < 8 ? 4 : 32 / (64 / Q);   // steps whose reads come before the first is used
#pragma unroll 1
        for (int r0 = 0; r0 < 32 && r0 < rows; r0 += AT_ONCE * (64 / Q)) {
            f32x4 x[AT_ONCE];
            float rm[AT_ONCE], rl[AT_ONCE];
            const int piece = lane % Q;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int r = r0 + u * (64 / Q) + lane / Q;
                rm[u] = __shfl(m, r, 64), rl[u] = __shfl(sum, r, 64);
                x[u] = *(const LDS_AS f32x4*)(uintptr_t)(mine + r * (4 * D) + ((piece ^ (r & (Q - 1))) << 4));
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int r = r0 + u * (64 / Q) + lane / Q;
                if (r < rows) out(32 * uniform(wave) + r, 4 * piece, rm[u], rl[u], x[u]);
            }
        }
        __syncthreads();
    }
};

template <int DTY, int D, bool DIRECT>
__global__ __launch_bounds__(64 * Wide<D>::NW, 2) void attn_paged_wide_kernel(PagedAttnLaunch arg, Schedule sc, Prefix px) {
    using S = Wide<D>;
    __shared__ __align__(16) char lds[S::LDS];
    share_out<S::R, S::KB, D, S::NW, PER_TILE_WIDE, 2, DIRECT>(arg, sc, [&](const Tile& t, bool first, int from, int to, float* part) {
        const PagedAttnLaunch& a = DIRECT ? arg : first_argument<PagedAttnLaunch>();
        WideWorker<DTY, D> worker(a, lds);
        worker.run(t, from, to, first ? px : Prefix{});
        worker.results(t, [&](int r, int d, float m, float l, f32x4 o) {
            if (part) {
                *(f32x4*)(part + r * D + d) = o;
                if (d == 0) *(f32x2*)(part + S::R * D + 2 * r) = f32x2{m, l};
            } else {
                finish<DTY, D>(a, row_of(a, t.tok0, t.hk, t.row0 + r), d, m, l, o);
            }
        });
    });
}

template <int DTY, int D>
__global__ __launch_bounds__(64 * Wide<D>::NW, 2) void attn_paged_wide_prefix_kernel(PagedAttnLaunch a, Prefix px) {
    using S = Wide<D>;
    __shared__ __align__(16) char lds[S::LDS];
    int split, from, to;
    const Tile t = prefix_tile<S::R, S::KB>(a, px.splits, split, from, to);
    WideWorker<DTY, D> worker(a, lds);
    worker.run(t, from, to, Prefix{});
    worker.results(t, [&](int r, int d, float m, float l, f32x4 o) { leave<D>(a, px, split, row_of(a, 0, t.hk, t.row0 + r), d, m, l, o); });
}

template <class... A>
hipError_t start(void (*kernel)(A...), dim3 grid, int threads, void* stream, A... arg) {
    void* args[] = {(void*)&arg...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), args, 0, (hipStream_t)stream);
}

template <int DTY, int D, bool DIRECT>
auto own_kernel(const PagedPlan& p) {
    const bool w8 = p.waves == 8;
    return p.rows == 16 ? (w8 ? &attn_paged_kernel<DTY, D, 1, 8, DIRECT> : &attn_paged_kernel<DTY, D, 1, 4, DIRECT>)
           : p.rows == 32 ? (w8 ? &attn_paged_kernel<DTY, D, 2, 8, DIRECT> : &attn_paged_kernel<DTY, D, 2, 4, DIRECT>)
                          : &attn_paged_wide_kernel<DTY, D, DIRECT>;
}

template <int DTY, int D>
hipError_t launch(const PagedAttnLaunch& a) {
    const PagedPlan p = paged_plan(a.c.B, a.c.T, a.Hq, a.c.Hk, D, a.max_q, a.max_kv, a.prefix_len);
    float* ws = (float*)a.workspace;
    const long long rows = (long long)a.c.T * a.Hq;
    Prefix px{ws, ws + p.prefix_splits * rows * D, p.prefix_splits, rows};
    if (p.prefix_splits > 0) {
        auto kernel = p.prefix_rows == 16 ? &attn_paged_prefix_kernel<DTY, D, 1>
                      : p.prefix_rows == 32 ? &attn_paged_prefix_kernel<DTY, D, 2> : &attn_paged_wide_prefix_kernel<DTY, D>;
        const hipError_t e = start(kernel, dim3(p.prefix_tiles * a.c.Hk * p.prefix_splits), 64 * p.prefix_waves, a.stream, a, px);
        if (e != hipSuccess) return e;
    }
    float* parts = ws + p.prefix_floats;
    Schedule sc{p.balanced, p.workgroups, parts, (Split*)(parts + 2LL * p.workgroups * p.rows * (D + 2))};
    auto kernel = p.direct ? own_kernel<DTY, D, true>(p) : own_kernel<DTY, D, false>(p);
    const hipError_t e = start(kernel, dim3(p.workgroups), 64 * p.waves, a.stream, a, sc, px);
    if (e != hipSuccess || !p.balanced) return e;
    const long long most = (long long)a.max_q * a.G;
    const int rows_used = most < 1 ? 1 : most < p.rows ? (int)most : p.rows;   // of a tile
    const bool many = p.rows < 128 && (long long)a.c.B * a.c.Hk * 8 <= p.workgroups;
    auto join = p.rows == 16 ? (many ? &attn_paged_join_many_kernel<DTY, D, 16> : &attn_paged_join_kernel<DTY, D, 16>)
                : p.rows == 32 ? (many ? &attn_paged_join_many_kernel<DTY, D, 32> : &attn_paged_join_kernel<DTY, D, 32>)
                               : &attn_paged_join_kernel<DTY, D, 128>;
    constexpr int AT_ONCE = JOIN_THREADS / (D / 4);   // rows of a workgroup
    return start(join, dim3(p.workgroups, many ? rows_used : (rows_used + AT_ONCE - 1) / AT_ONCE), JOIN_THREADS, a.stream, a, sc);
}

}  // namespace

hipError_t paged_attn_launch(const PagedAttnLaunch& a) {
    if (a.dtype == 0) return a.D == 32 ? launch<0, 32>(a) : a.D == 64 ? launch<0, 64>(a) : launch<0, 128>(a);
    return a.D == 32 ? launch<1, 32>(a) : a.D == 64 ? launch<1, 64>(a) : launch<1, 128>(a);
}

// Append to a paged key/value cache for gfx950: the new tokens' keys and values go to their pages, keys and queries rotated by
// their positions on the way.
//
// Token i of the n new ones of sequence b is key p = kv_len[b] - n + i of that sequence: page table[b][p >> page_shift], slot
// p mod page size.  With c, s the cosine and sine of its angles, a rotated pair (a, b) becomes (a c - b s, b c + a s), in 32 bits,
// rounded once.  Pairs are (j, j + rot / 2) or (2 j, 2 j + 1); the rest of a head and all of v pass unchanged.
//
// Bound by memory: a token's row is read once and written once.  A small step (a token for each of some sequences) is bound by
// the chain of dependent loads instead: which sequence -> the page -> the store.  Therefore
//   * a workgroup takes one token and finds its sequence with one round of loads: thread b looks at cu_q[b], cu_q[b + 1] and
//     kv_len[b], and names itself in LDS if the token lies between (a search would be log2(B) loads deep);
//   * the row's own loads do not depend on that and are under way meanwhile;
//   * a thread's unit of work is two chunks of 8 elements, the two halves of 8 rotated pairs; with 2, 4 or 8 units a head it is the
//     same unit in every head it visits, so a thread loads its angles once.
// Measured (us; 32 query and 8 key heads of 128): 64 tokens 3.2 in a replayed graph, 9947 tokens of 6 sequences 50 (4.9 TB/s; four tokens a
// workgroup 54, beside 51 with the kernel of then).  With 512 threads instead of 256, in turn: 3.0 and 3.2, 49.5 and 49.8; 8000 tokens with 64 query
// heads on the same inputs again and again 62.0 and 62.9.
// Every workgroup looks at all sequences: 1024 sequences of a token each 6.9 us (3.6 TB/s), 4096 28 (512 threads 26), 16384 226 (191; 1.8 TB/s): from
// some thousands of sequences in a step on, the search is what it waits for.
#include <hip/hip_runtime.h>
#include <cstdint>

#include "attn_paged_launch.h"
#include "gfx950_common.h"

namespace {

using gfx950::u32x4;

template <int DT>
__device__ __forceinline__ void widen8(const u32x4& p, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = gfx950::Elem<DT>::widen((uint16_t)(p[i] & 0xFFFFu));
        f[2 * i + 1] = gfx950::Elem<DT>::widen((uint16_t)(p[i] >> 16));
    }
}
template <int DT>
__device__ __forceinline__ u32x4 narrow8(const float (&f)[8]) {
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = gfx950::Elem<DT>::pack2(f[2 * i], f[2 * i + 1]);
    return p;
}

constexpr int MOST = 256;   // threads of a workgroup

// What a thread does to the two chunks of its unit.
template <int DT>
__device__ __forceinline__ void rotate(u32x4& x, u32x4& y, const float (&cs)[8], const float (&sn)[8], int interleaved) {
    float p[8], q[8];
    widen8<DT>(x, p);
    widen8<DT>(y, q);
    auto turn = [](float& a, float& b, float c, float s) {
        const float m = a * c - b * s, n = b * c + a * s;
        a = m;
        b = n;
    };
    if (!interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) turn(p[j], q[j], cs[j], sn[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            turn(p[2 * j], p[2 * j + 1], cs[j], sn[j]);
            turn(q[2 * j], q[2 * j + 1], cs[4 + j], sn[4 + j]);
        }
    }
    x = narrow8<DT>(p);
    y = narrow8<DT>(q);
}

template <int DT, int D>
__global__ __launch_bounds__(MOST) void kv_append_kernel(AppendLaunch a) {
    constexpr int U = D / 16;                        // units of a head
    constexpr int AHEAD = 2;                         // visits whose loads are issued before the token's page is known
    const int HEADS = blockDim.x / U;                // heads the workgroup visits at once
    __shared__ int seq, pos;
    const PagedCache& c = a.c;
    const int t = blockIdx.x;
    const int u = threadIdx.x % U, h0 = threadIdx.x / U, heads = a.Hq + 2 * c.Hk;
    const bool turned = u < a.rot / 16;              // else both chunks pass as they are
    const int e0 = turned && !a.interleaved ? 8 * u : 16 * u, e1 = turned && !a.interleaved ? e0 + a.rot / 2 : e0 + 8;

    auto load = [&](int h, u32x4& x, u32x4& y) {
        const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + c.Hk;
        const uint16_t* src = is_q ? (const uint16_t*)a.q + t * a.q_stride + h * D
                                   : is_k ? (const uint16_t*)a.k + t * a.k_stride + (h - a.Hq) * D
                                          : (const uint16_t*)a.v + t * a.v_stride + (h - a.Hq - c.Hk) * D;
        x = *(const u32x4*)(src + (is_q || is_k ? e0 : 16 * u));
        y = *(const u32x4*)(src + (is_q || is_k ? e1 : 16 * u + 8));
    };
    u32x4 x[AHEAD], y[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (h0 + i * HEADS < heads) load(h0 + i * HEADS, x[i], y[i]);

    if (threadIdx.x == 0) seq = -1;
    __syncthreads();
    for (int b = threadIdx.x; b < c.B; b += blockDim.x) {
        const int lo = c.cu_q[b], hi = c.cu_q[b + 1], n = c.kv_len[b];
        if (lo <= t && t < hi) {
            seq = b;
            pos = n - (hi - t);
        }
    }
    __syncthreads();
    // where the token's key goes in head 0, if its page exists
    const int b = seq, p = b < 0 ? -1 : pos, page_at = p >> c.page_shift;
    long long at = -1;
    if (p >= 0 && page_at < c.width) {
        const int page = c.table[(size_t)b * c.table_stride + page_at];
        if (page >= 0 && page < c.n_pages) at = page * c.page_stride + (long long)(p & ((1 << c.page_shift) - 1)) * D;
    }
    float cs[8], sn[8];
    if (turned) {
        int row = p + a.pos_offset;
        row = row < 0 ? 0 : row >= a.n_angles ? a.n_angles - 1 : row;
        const float *pc = a.cos + (size_t)row * (a.rot / 2) + 8 * u, *ps = a.sin + (size_t)row * (a.rot / 2) + 8 * u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cs[j] = pc[j];
            sn[j] = ps[j];
        }
    }
    const size_t head_stride = (size_t)D << c.page_shift;
    auto finish = [&](int h, u32x4 x, u32x4 y) {
        const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + c.Hk;
        const bool rot = is_q || is_k;
        if (turned && rot) rotate<DT>(x, y, cs, sn, a.interleaved);
        uint16_t* dst = is_q ? (uint16_t*)a.q_out + ((size_t)t * a.Hq + h) * D
                             : is_k ? (uint16_t*)c.k + at + (h - a.Hq) * head_stride : (uint16_t*)c.v + at + (h - a.Hq - c.Hk) * head_stride;
        if (is_q || at >= 0) {
            *(u32x4*)(dst + (rot ? e0 : 16 * u)) = x;
            *(u32x4*)(dst + (rot ? e1 : 16 * u + 8)) = y;
        }
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (h0 + k * HEADS < heads) finish(h0 + k * HEADS, x[k], y[k]);
#pragma unroll 2
    for (int h = h0 + AHEAD * HEADS; h < heads; h += HEADS) {
        u32x4 x, y;
        load(h, x, y);
        finish(h, x, y);
    }
}

template <int DT, int D>
hipError_t launch(const AppendLaunch& a) {
    AppendLaunch arg = a;
    void* args[] = {&arg};
    // threads for a token's units in as few visits as can be, none idle for long
    const long long units = ((long long)a.Hq + 2 * a.c.Hk) * (D / 16), visits = (units + MOST - 1) / MOST;
    const unsigned threads = (unsigned)(((units + visits - 1) / visits + 63) / 64 * 64);
    return hipLaunchKernel(reinterpret_cast<const void*>(&kv_append_kernel<DT, D>), dim3(a.c.T), dim3(threads), args, 0, (hipStream_t)a.stream);
}

}  // namespace

hipError_t kv_append_launch(const AppendLaunch& a) {
    if (a.dtype == 0) return a.D == 32 ? launch<0, 32>(a) : a.D == 64 ? launch<0, 64>(a) : launch<0, 128>(a);
    return a.D == 32 ? launch<1, 32>(a) : a.D == 64 ? launch<1, 64>(a) : launch<1, 128>(a);
}

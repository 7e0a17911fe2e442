// kv_slots.cu -- the slots and positions of the tokens that a batch of sequences
// adds, from lengths and page tables on the device, with new pages out of a free
// list (parason_kv_slots).
//
//   tokens   p_r = sum over r' < r of added_r'          (rows p_r .. p_r + added_r - 1)
//   pages    need_r = ceil((held_r + added_r) / 16) - ceil(held_r / 16), and their sums
//   slot     of token i of sequence r: x = held_r + i, 16 page(r, x / 16) + x % 16
//
// A few KB in, 8 bytes a token out: launch and one chain of dependent loads
// (lengths, two scans, page, stores) are its time.  So it is one launch, whose CTAs
// make both scans for themselves in shared memory and share the rows (4.5 us with 256
// requests or 64 branches; its 32 registers, bounded for 1024 threads, spill 28 bytes).  Where the
// lengths or the count of taken pages advance in place, the CTAs are one cluster, and its
// barrier stands between the last read of them and the first write.
#include <cooperative_groups.h>

#include <algorithm>
#include <iterator>

#include "device_common.cuh"
#include "internal.h"

namespace parason {
namespace {

constexpr int kMaxSeqs = 16384;          // 12 bytes each in shared memory
constexpr int kClusterCtas = 8;          // the portable size
constexpr int kMaxCtas = 128;            // without a cluster: each reads all lengths
constexpr int kMaxThreads = 1024, kFewThreads = 256;
constexpr int kFewSeqs = 1024;           // up to this many: kFewThreads a CTA
constexpr int kTokensPerThread = 4;      // neighbours, stored in 16 bytes
constexpr int32_t kMaxPage = INT32_MAX / kPageSize;

struct SlotArgs {
    const int32_t *held, *added, *first, *free_pages, *free_used;
    int32_t *table, *slots, *positions, *token_ptr, *held_out, *used_out;
    int64_t table_stride;
    int32_t num_seqs, table_pages, num_free, num_rows;
    bool aligned;                        // slots and positions to 16 bytes
    bool in_place;                       // held_out or used_out are inputs too
};

// Inclusive sums over the CTA's threads of a and b; `part` holds two values a warp.
__device__ __forceinline__ void scan_pair(int64_t &a, int64_t &b, int64_t (&part)[2][32], int warps) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) a += x, b += y;
    }
    if (lane == 31) part[0][warp] = a, part[1][warp] = b;
    __syncthreads();
    int64_t x = lane < warps && lane < warp ? part[0][lane] : 0, y = lane < warps && lane < warp ? part[1][lane] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        x += __shfl_xor_sync(0xffffffffu, x, o);
        y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    a += x;
    b += y;
    __syncthreads();
}

__device__ __forceinline__ int pages_of(int64_t tokens) { return static_cast<int>((tokens + kPageSize - 1) / kPageSize); }

// Every CTA scans all sequences; the grid's threads then share the rows, a thread
// kTokensPerThread neighbours a step (mostly of one page: it is looked up when it changes),
// and CTA 0 writes what there is per sequence.
__global__ void __launch_bounds__(kMaxThreads) kv_slots_kernel(const SlotArgs a) {
    extern __shared__ int32_t mem[];
    __shared__ int64_t part[2][32];
    int32_t *row0 = mem;                              // [num_seqs + 1] first row of a sequence
    int32_t *page0 = mem + a.num_seqs + 1;            // [num_seqs + 1] its first new page in the list
    int32_t *held = page0 + a.num_seqs + 1;           // [num_seqs]
    const int R = a.num_seqs, warps = blockDim.x / 32;
    const int per = (R + blockDim.x - 1) / blockDim.x, r0 = min(R, static_cast<int>(threadIdx.x) * per), r1 = min(R, r0 + per);
    dev::grid_wait();
    const int used = a.free_used ? max(0, *a.free_used) : 0;

    auto added_of = [&](int r, int h) { return min(max(a.added ? a.added[r] : 1, 0), INT32_MAX - h); };
    auto need_of = [&](int h, int64_t n) {
        return a.free_pages ? max(0, min(pages_of(h + n), a.table_pages) - pages_of(h)) : 0;
    };
    int64_t tokens = 0, pages = 0;
    for (int r = r0; r < r1; ++r) {
        const int h = max(a.held[r], 0), n = added_of(r, h);
        held[r] = h;
        tokens += n;
        pages += need_of(h, n);
    }
    int64_t t = tokens, p = pages;
    scan_pair(t, p, part, warps);
    // (more tokens than rows: those past them are not added, and need no pages)
    if (__syncthreads_or(t > a.num_rows)) {
        int64_t at = t - tokens;
        pages = 0;
        for (int r = r0; r < r1; ++r) {
            const int64_t n = added_of(r, held[r]);
            pages += need_of(held[r], min(n, max(static_cast<int64_t>(0), a.num_rows - at)));
            at += n;
        }
        int64_t none = 0;
        p = pages;
        scan_pair(p, none, part, warps);
    }
    {
        int64_t at = t - tokens, page = p - pages;
        for (int r = r0; r < r1; ++r) {
            const int64_t n = added_of(r, held[r]);
            row0[r] = static_cast<int32_t>(min(at, static_cast<int64_t>(a.num_rows)));
            page0[r] = static_cast<int32_t>(min(page, static_cast<int64_t>(INT32_MAX)));
            page += need_of(held[r], min(n, max(static_cast<int64_t>(0), a.num_rows - at)));
            at += n;
        }
        if (threadIdx.x == blockDim.x - 1) {
            row0[R] = static_cast<int32_t>(min(t, static_cast<int64_t>(a.num_rows)));
            page0[R] = static_cast<int32_t>(min(p, static_cast<int64_t>(INT32_MAX)));
        }
    }
    if (a.in_place)
        cooperative_groups::this_cluster().sync();    // lengths are read, scans written
    else
        __syncthreads();

    const int left = max(0, a.num_free - used);       // of the list
    const int ctas = gridDim.x, cta = blockIdx.x;
    if (cta == 0) {
        for (int r = threadIdx.x; r <= R; r += blockDim.x) {
            if (a.token_ptr) a.token_ptr[r] = row0[r];
            if (r == R || !a.held_out) continue;
            // tokens as far as the pages go
            const int h = held[r], n = row0[r + 1] - row0[r];
            const int64_t had = pages_of(h);
            int64_t room = a.table_pages;
            if (a.free_pages) room = min(room, had + min(page0[r + 1] - page0[r], max(0, left - page0[r])));
            a.held_out[r] = h + static_cast<int>(min(static_cast<int64_t>(n), max(static_cast<int64_t>(0), room * kPageSize - h)));
        }
        if (threadIdx.x == 0 && a.used_out) a.used_out[0] = used + min(page0[R], left);
    }
    const int total = row0[R];
    const int64_t step = static_cast<int64_t>(ctas) * blockDim.x * kTokensPerThread;
    for (int64_t q0 = (static_cast<int64_t>(cta) * blockDim.x + threadIdx.x) * kTokensPerThread; q0 < a.num_rows; q0 += step) {
        int r = 0;                                    // the last sequence that starts at q0 or before
        if (q0 < total) {
            int lo = 0, hi = R;                       // row0[lo] <= q0 < row0[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (row0[mid] <= q0)
                    lo = mid;
                else
                    hi = mid;
            }
            r = lo;
        }
        int32_t slot[kTokensPerThread], pos[kTokensPerThread];
        int64_t known = -1;                           // (sequence, page) that `page` is of
        int page = -1;
#pragma unroll
        for (int i = 0; i < kTokensPerThread; ++i) {
            const int64_t q = q0 + i;
            slot[i] = -1;
            pos[i] = 0;
            if (q >= total) continue;
            while (row0[r + 1] <= q) ++r;             // (row0[R] = total > q)
            const int h = held[r], x = h + static_cast<int>(q - row0[r]), j = x / kPageSize;
            pos[i] = x + (a.first ? __ldg(a.first + r) : 0);
            const int64_t id = static_cast<int64_t>(r) << 32 | j;
            if (id != known) {
                known = id;
                page = -1;
                const int fresh = j - pages_of(h);
                if (j >= a.table_pages) {
                } else if (!a.free_pages || fresh < 0) {
                    page = a.table[r * a.table_stride + j];
                } else if (page0[r] + static_cast<int64_t>(fresh) < left) {
                    page = __ldg(a.free_pages + (used + page0[r] + fresh));
                    if (x % kPageSize == 0) a.table[r * a.table_stride + j] = page;
                }
            }
            if (page >= 0 && page <= kMaxPage) slot[i] = page * kPageSize + x % kPageSize;
        }
        if (a.aligned && q0 + kTokensPerThread <= a.num_rows) {
            *reinterpret_cast<int4 *>(a.slots + q0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
            if (a.positions) *reinterpret_cast<int4 *>(a.positions + q0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
#pragma unroll
            for (int i = 0; i < kTokensPerThread; ++i) {
                if (q0 + i >= a.num_rows) break;
                a.slots[q0 + i] = slot[i];
                if (a.positions) a.positions[q0 + i] = pos[i];
            }
        }
    }
}

// Whether outputs lie over what is read, or over one another: CTAs read while others write.
// held_out may be held, and used_out free_used (their writes wait for every read).
bool overlaps(const parason_slot_map &m) {
    struct Array {
        const int32_t *at;
        int64_t n;
    };
    const int64_t seqs = m.num_seqs;
    const Array in[] = {{m.held, seqs}, {m.added, seqs}, {m.first, seqs}, {m.free_pages, m.num_free}, {m.free_used, 1}};
    const Array out[] = {{m.held_out, seqs}, {m.used_out, 1}, {m.slots, m.num_rows}, {m.positions, m.num_rows},
                         {m.token_ptr, seqs + 1}};
    auto meet = [](const Array &a, const Array &b) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
        return a.at && b.at && a.n > 0 && b.n > 0 && (x <= y ? (y - x) / 4 < static_cast<uintptr_t>(a.n)
                                                              : (x - y) / 4 < static_cast<uintptr_t>(b.n));
    };
    // an array and the table's rows, which may lie apart: its first element's row, or the next one
    auto meets_table = [&](const Array &a) {
        if (!a.at || a.n <= 0 || seqs == 0 || m.table_pages == 0) return false;
        const intptr_t off = static_cast<intptr_t>(reinterpret_cast<uintptr_t>(a.at) - reinterpret_cast<uintptr_t>(m.page_table));
        const int64_t from = off >> 2, to = from + a.n;       // (both 4-byte aligned)
        if (seqs == 1 || from < 0) return to > 0 && from < m.table_pages;
        const int64_t r = from / m.table_stride, at = from % m.table_stride;
        return r < seqs && (at < m.table_pages || (r + 1 < seqs && at + a.n > m.table_stride));
    };
    for (const Array &o : out) {
        for (const Array &i : in)
            if (meet(o, i) && !(o.at == i.at && ((&o == &out[0] && &i == &in[0]) || (&o == &out[1] && &i == &in[4]))))
                return true;
        for (const Array *p = &o + 1; p != std::end(out); ++p)
            if (meet(o, *p)) return true;
        if (meets_table(o)) return true;
    }
    // (the table is written where there is a free list)
    if (m.free_pages)
        for (const Array &i : in)
            if (meets_table(i)) return true;
    return false;
}

bool misaligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace
}  // namespace parason

using namespace parason;

extern "C" parason_status parason_kv_slots(const parason_slot_map *m, parason_stream_t stream) {
    if (!m || m->num_seqs < 0 || m->num_rows < 0 || m->table_pages < 0 || m->num_free < 0) return PARASON_EINVAL;
    if (m->num_seqs > kMaxSeqs) return PARASON_EUNSUPPORTED;
    if (m->num_rows == INT32_MAX) return PARASON_EUNSUPPORTED;
    for (const void *p : {static_cast<const void *>(m->held), static_cast<const void *>(m->added),
                          static_cast<const void *>(m->first), static_cast<const void *>(m->page_table),
                          static_cast<const void *>(m->free_pages), static_cast<const void *>(m->free_used),
                          static_cast<const void *>(m->slots), static_cast<const void *>(m->positions),
                          static_cast<const void *>(m->token_ptr), static_cast<const void *>(m->held_out),
                          static_cast<const void *>(m->used_out)})
        if (misaligned4(p)) return PARASON_EINVAL;
    if (m->num_seqs > 0 && (!m->held || (m->table_pages > 0 && !m->page_table))) return PARASON_EINVAL;
    if (m->num_seqs > 1 && m->table_stride < m->table_pages) return PARASON_EINVAL;
    if (m->num_rows > 0 && !m->slots) return PARASON_EINVAL;
    if (!m->free_pages && (m->free_used || m->used_out || m->num_free > 0)) return PARASON_EINVAL;
    if (overlaps(*m)) return PARASON_EINVAL;
    SlotArgs a{};
    a.held = m->held;
    a.added = m->added;
    a.first = m->first;
    a.free_pages = m->free_pages;
    a.free_used = m->free_used;
    a.table = m->page_table;
    a.slots = m->slots;
    a.positions = m->positions;
    a.token_ptr = m->token_ptr;
    a.held_out = m->held_out;
    a.used_out = m->used_out;
    a.table_stride = m->table_stride;
    a.num_seqs = m->num_seqs;
    a.table_pages = m->table_pages;
    a.num_free = m->num_free;
    a.num_rows = m->num_rows;
    a.aligned = (reinterpret_cast<uintptr_t>(m->slots) | reinterpret_cast<uintptr_t>(m->positions)) % 16 == 0;
    a.in_place = (m->held_out && m->held_out == m->held) || (m->used_out && m->used_out == m->free_used);
    const int64_t groups = (static_cast<int64_t>(a.num_rows) + kTokensPerThread - 1) / kTokensPerThread;
    const int most = a.in_place || a.num_seqs > kFewSeqs ? kMaxThreads : kFewThreads;
    const int threads =
        static_cast<int>(std::min<int64_t>(most, std::max<int64_t>(32, (std::max<int64_t>(a.num_seqs, groups) + 31) / 32 * 32)));
    const int64_t ctas64 = std::max<int64_t>(1, (groups + threads - 1) / threads);
    int ctas = static_cast<int>(std::min<int64_t>(ctas64, kMaxCtas));
    if (a.in_place) {
        ctas = 1;
        while (ctas < kClusterCtas && ctas < ctas64) ctas *= 2;
    }
    const size_t smem = (3 * static_cast<size_t>(a.num_seqs) + 2) * sizeof(int32_t);
    if (smem > 47 * 1024 &&
        cudaFuncSetAttribute(kv_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>((3 * kMaxSeqs + 2) * sizeof(int32_t))) != cudaSuccess)
        return PARASON_ECUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(ctas));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = reinterpret_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.in_place ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kv_slots_kernel, a) == cudaSuccess ? PARASON_OK : PARASON_ECUDA;
}

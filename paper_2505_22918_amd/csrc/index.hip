// Block-index builder (gfx950): the static mask M of Sec.3 as a block CSR, and a mask's transpose.
//
// Three launches on the caller's stream (an EXPLICIT input may stack several
// masks, one per head or per (batch, head); mask m owns row_ptr[m][0 .. n_blk]):
//   1. row_count   one workgroup per (mask, query block) writes its kept-block
//                  count into row_ptr[m][qb + 1] (closed form for the window
//                  patterns, a count of the 0/1 row for EXPLICIT);
//   2. row_scan    one workgroup turns all counts into absolute offsets in place;
//   3. row_fill    one workgroup per (mask, query block) ranks the candidate key
//                  blocks and writes the kept ones in ascending order.
//
// Ranking is exact integer arithmetic: a block's centroid is the sum of its
// token coordinates scaled by lcm / count (lcm over the candidate blocks' token
// counts), so squared distances compare exactly, and the key
// (distance^2, |kb - qb|, kb) is a total order.  Each candidate's rank is the
// number of candidates with a smaller key; a block is kept when its rank is
// below the keep count.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "train.h"

namespace rt {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 4096;
constexpr int kMaxRows = 32768;  // (mask, query block) rows one scan handles

__device__ int row_count_of(const IndexArgs& a, int qb) {
    if (a.kind == 1) return a.keep < a.n_blk ? a.keep : a.n_blk;
    if (a.kind == 2) {
        if (qb < a.n_tblk) return a.n_tblk;
        const int nv = a.n_blk - a.n_tblk;
        return a.n_tblk + (a.keep < nv ? a.keep : nv);
    }
    return -1;  // explicit: counted by the caller
}

__global__ __launch_bounds__(kThreads) void row_count(IndexArgs a) {
    const int m = blockIdx.x / a.n_blk;
    const int qb = blockIdx.x - m * a.n_blk;
    int32_t* const rp = a.row_ptr + (size_t)m * (a.n_blk + 1);
    __shared__ int total;
    if (a.kind != 0) {
        if (threadIdx.x == 0) rp[qb + 1] = row_count_of(a, qb);
        return;
    }
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    int n = 0;
    const uint8_t* row = a.mask + ((size_t)m * a.n_blk + qb) * a.n_blk;
    for (int kb = threadIdx.x; kb < a.n_blk; kb += kThreads) n += row[kb] != 0;
    atomicAdd(&total, n);
    __syncthreads();
    if (threadIdx.x == 0) rp[qb + 1] = total;
}

// Exclusive scan of the n_masks * n_blk row counts, in row order, into absolute
// offsets: row_ptr[m][qb] = entries of all earlier rows, row_ptr[m][n_blk] =
// row_ptr[m + 1][0] (the total after the last mask).
__global__ __launch_bounds__(kThreads) void row_scan(IndexArgs a) {
    __shared__ int cnt[kMaxRows];
    __shared__ int part[kThreads + 1];
    const int nb = a.n_blk;
    const int n = a.n_masks * nb;
    const int tid = threadIdx.x;
    for (int i = tid; i < n; i += kThreads) {
        const int m = i / nb, qb = i - m * nb;
        cnt[i] = a.row_ptr[(size_t)m * (nb + 1) + qb + 1];
    }
    __syncthreads();
    // each thread owns a contiguous segment; segment sums are scanned serially
    const int seg = (n + kThreads - 1) / kThreads;
    const int s0 = tid * seg < n ? tid * seg : n;
    const int s1 = s0 + seg < n ? s0 + seg : n;
    int local = 0;
    for (int i = s0; i < s1; ++i) local += cnt[i];
    part[tid + 1] = local;
    __syncthreads();
    if (tid == 0) {
        part[0] = 0;
        for (int i = 1; i <= kThreads; ++i) part[i] += part[i - 1];
    }
    __syncthreads();
    int run = part[tid];
    for (int i = s0; i < s1; ++i) {
        const int c = cnt[i];
        cnt[i] = run;
        run += c;
    }
    __syncthreads();
    const int total = part[kThreads];
    for (int i = tid; i < n; i += kThreads) {
        const int m = i / nb, qb = i - m * nb;
        a.row_ptr[(size_t)m * (nb + 1) + qb] = cnt[i];
    }
    for (int m = tid; m < a.n_masks; m += kThreads)
        a.row_ptr[(size_t)m * (nb + 1) + nb] = m + 1 < a.n_masks ? cnt[(m + 1) * nb] : total;
}

// scaled centroid coordinates of block b (video: b holds video tokens only)
__device__ void centroid(const IndexArgs& a, int b, int64_t c[3]) {
    const int t0 = b * a.block;
    const int t1 = (t0 + a.block < a.T) ? t0 + a.block : a.T;
    int64_t s0 = 0, s1 = 0, s2 = 0;
    if (a.kind == 1) {
        for (int t = t0; t < t1; ++t) {
            s0 += t / a.grid_w;
            s1 += t % a.grid_w;
        }
    } else {
        const int hw = a.grid_h * a.grid_w;
        for (int t = t0; t < t1; ++t) {
            const int v = t - a.n_text;
            s0 += v / hw;
            s1 += (v / a.grid_w) % a.grid_h;
            s2 += v % a.grid_w;
        }
    }
    const int64_t f = a.lcm / (t1 - t0);
    c[0] = s0 * f;
    c[1] = s1 * f;
    c[2] = s2 * f;
}

__global__ __launch_bounds__(kThreads) void row_fill(IndexArgs a) {
    __shared__ int64_t dist[kMaxBlocks];
    __shared__ uint8_t kept[kMaxBlocks];
    __shared__ int part[kThreads + 1];

    const int nb = a.n_blk;
    const int m = blockIdx.x / nb;
    const int qb = blockIdx.x - m * nb;
    const int tid = threadIdx.x;

    // candidate range and how many of them to keep
    int lo = 0, k = 0;
    bool ranked = false;
    if (a.kind == 1) {
        ranked = true;
        k = a.keep < nb ? a.keep : nb;
    } else if (a.kind == 2 && qb >= a.n_tblk) {
        ranked = true;
        lo = a.n_tblk;
        k = a.keep < nb - lo ? a.keep : nb - lo;
    }

    if (ranked) {
        int64_t cq[3];
        centroid(a, qb, cq);
        for (int kb = lo + tid; kb < nb; kb += kThreads) {
            int64_t ck[3];
            centroid(a, kb, ck);
            const int64_t d0 = ck[0] - cq[0], d1 = ck[1] - cq[1], d2 = ck[2] - cq[2];
            dist[kb] = d0 * d0 + d1 * d1 + d2 * d2;
        }
        __syncthreads();
        for (int kb = lo + tid; kb < nb; kb += kThreads) {
            const int64_t dk = dist[kb];
            const int ak = kb > qb ? kb - qb : qb - kb;
            int rank = 0;
            for (int j = lo; j < nb; ++j) {
                const int64_t dj = dist[j];
                const int aj = j > qb ? j - qb : qb - j;
                rank += (dj < dk) || (dj == dk && (aj < ak || (aj == ak && j < kb)));
            }
            kept[kb] = rank < k;
        }
        // text key blocks of a video row are always kept
        for (int kb = tid; kb < lo; kb += kThreads) kept[kb] = 1;
    } else if (a.kind == 2) {
        // text query block: text key blocks only
        for (int kb = tid; kb < nb; kb += kThreads) kept[kb] = kb < a.n_tblk;
    } else {
        const uint8_t* row = a.mask + ((size_t)m * nb + qb) * nb;
        for (int kb = tid; kb < nb; kb += kThreads) kept[kb] = row[kb] != 0;
    }
    __syncthreads();

    // ordered write: each thread owns a contiguous segment of key blocks
    const int seg = (nb + kThreads - 1) / kThreads;
    const int s0 = tid * seg;
    const int s1 = (s0 + seg < nb) ? s0 + seg : nb;
    int n = 0;
    for (int kb = s0; kb < s1; ++kb) n += kept[kb];
    part[tid + 1] = n;
    __syncthreads();
    if (tid == 0) {
        part[0] = 0;
        for (int i = 1; i <= kThreads; ++i) part[i] += part[i - 1];
    }
    __syncthreads();
    int pos = a.row_ptr[(size_t)m * (nb + 1) + qb] + part[tid];
    for (int kb = s0; kb < s1; ++kb) {
        if (kept[kb]) {
            if (pos >= 0 && pos < a.capacity) a.col_idx[pos] = kb;
            ++pos;
        }
    }
}

// ---- transpose of a block mask -------------------------------------------------------------
//
// Row kb of the transposed mask lists the query blocks whose rows hold kb, ascending, and a plan says how the
// gradients' call splits long rows (train.h).
//
// Up to kSmall blocks: one workgroup to a mask sets a bit for each entry in LDS, and a thread to a key block counts its
// row of bits and writes it out in order.  Masks keep their places by what row_ptr says they hold.  More blocks: one
// wave to a (mask, kb) looks at 64 rows at a time, each lane with a binary search of its row (rows are ascending),
// once to count and once, after a scan of the counts, to write; ballots keep the order.
//
// Latency: 12 masks of 83 blocks 16 us in three launches, 9 in one (its kernel alone 6.6).  In one launch 32 blocks take
// 5 us, 256 15, 640 33.  The searches are of every row for every key block, so their time grows with the square of the
// blocks: 641 29 us (30 masks of them 267), 1024 44, 2048 107, 4096 340 to 730, 16384 4.7 ms, 131072 (the longest head)
// 240 ms.

constexpr int kSmall = 640;  // its bits take 51 KB

// item j's entry of a list of n pieces, {row, first, entries, part or -1}
__device__ __forceinline__ int4 plan_item(int row, int at, int count, int seg, int j, int n, int part) {
    const int first = j * seg, left = count - first;
    return int4{row, at < 0 ? -1 : at + first, left < seg ? left : seg, n > 1 ? part + j : -1};
}
__device__ __forceinline__ int pieces_of(int count, int seg) { return count <= seg ? 1 : (count + seg - 1) / seg; }

__global__ __launch_bounds__(1024) void transpose_small(TransposeArgs a) {
    extern __shared__ uint32_t bits[];
    // entries of the masks before this one, their room for further parts, entries of all masks
    __shared__ unsigned long long before[3];
    __shared__ int waves[16][4];
    const int m = blockIdx.x, n = a.n_blk, words = (n + 31) >> 5, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < n * words; i += 1024) bits[i] = 0u;
    if (tid < 3) before[tid] = 0;
    __syncthreads();
    auto entries = [&](int k) {  // of mask k, by its row offsets (as far as the array goes)
        const int32_t* p = a.row_ptr + (size_t)k * (n + 1);
        const int b = p[0] < 0 ? 0 : p[0], e = p[n] > a.nnz ? a.nnz : p[n];
        return e < b ? 0 : e - b;
    };
    for (int k = tid; k < a.n_masks; k += 1024) {
        const int c = entries(k);
        atomicAdd(&before[2], (unsigned long long)c);
        if (k >= m) continue;
        atomicAdd(&before[0], (unsigned long long)c);
        if (n > a.seg) atomicAdd(&before[1], (unsigned long long)(c / a.seg));
    }
    const int32_t* rp = a.row_ptr + (size_t)m * (n + 1);
    for (int q = tid >> 4; q < n; q += 64) {  // 16 lanes a row
        int b = rp[q], e = rp[q + 1];
        b = b < 0 ? 0 : (b > a.nnz ? a.nnz : b);
        e = e < b ? b : (e > a.nnz ? a.nnz : e);
        for (int j = b + (tid & 15); j < e; j += 16) {
            const int c = a.col_idx[j];
            if (c >= 0 && c < n) atomicOr(&bits[c * words + (q >> 5)], 1u << (q & 31));
        }
    }
    __syncthreads();
    int count = 0;
    if (tid < n)
        for (int i = 0; i < words; ++i) count += __popc(bits[tid * words + i]);
    const int pieces = tid < n ? pieces_of(count, a.seg) : 1;
    // running sums of entries, further parts, parts of split lists, split lists
    int own[4] = {count, pieces - 1, pieces > 1 ? pieces : 0, pieces > 1}, sum[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        int s = own[k];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(s, d);
            if (lane >= d) s += x;
        }
        if (lane == 63) waves[wave][k] = s;
        sum[k] = s - own[k];
    }
    __syncthreads();
    int all = 0;
    for (int w = 0; w < 16; ++w) {
        all += waves[w][0];
        if (w < wave)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += waves[w][k];
    }
    // Where all entries fit, so does their room for further parts.
    const int mine = entries(m);
    const bool fits = all <= mine && before[2] <= (unsigned long long)a.t_nnz;
    const int base = fits ? (int)before[0] : -1;
    const int skip = before[1] < (unsigned long long)a.max_more ? (int)before[1] : a.max_more;
    int4* item = reinterpret_cast<int4*>(a.plan);
    int4* more = item + (size_t)a.n_masks * n + skip;
    // this mask's room for further parts and split lists; the last mask's is all that is left
    int left = n > a.seg && m < a.n_masks - 1 ? mine / a.seg : a.max_more - skip;
    left = left < a.max_more - skip ? left : a.max_more - skip;
    int n_more = 0, n_split = 0;
    for (int w = 0; w < 16; ++w) {
        n_more += waves[w][1];
        n_split += waves[w][3];
    }
    for (int i = tid; i < left; i += 1024) {
        if (!fits || i >= n_more) more[i] = int4{-1, 0, 0, 0};
        if (!fits || i >= n_split) more[a.max_more + i] = int4{-1, 0, 0, 0};
    }
    int32_t* t_rp = a.t_row_ptr + (size_t)m * (n + 1);
    if (tid == 0) t_rp[0] = base;
    if (tid < n) {
        const int at = fits ? base + sum[0] : -1, row = m * n + tid;
        t_rp[tid + 1] = fits ? at + count : -1;
        for (int j = 0; j < (fits ? pieces : 1); ++j) {
            const int4 x = plan_item(row, at, count, a.seg, j, pieces, 2 * skip + sum[2]);
            if (j == 0)
                item[row] = x;
            else
                more[sum[1] + j - 1] = x;
        }
        if (fits && pieces > 1) more[a.max_more + sum[3]] = int4{row, 2 * skip + sum[2], pieces, 0};
        int to = at;
        for (int i = 0; fits && i < words; ++i)
            for (uint32_t w = bits[tid * words + i]; w; w &= w - 1) a.t_col_idx[to++] = 32 * i + __ffs(w) - 1;
    }
}

// whether row qb of mask m holds key block kb
__device__ __forceinline__ bool row_holds(const TransposeArgs& a, int m, int qb, int kb) {
    if (qb >= a.n_blk) return false;
    const int32_t* p = a.row_ptr + (size_t)m * (a.n_blk + 1) + qb;
    int b = p[0], e = p[1];
    b = b < 0 ? 0 : (b > a.nnz ? a.nnz : b);
    e = e < b ? b : (e > a.nnz ? a.nnz : e);
    const int end = e;
    while (b < e) {
        const int mid = b + ((e - b) >> 1);
        if (a.col_idx[mid] < kb)
            b = mid + 1;
        else
            e = mid;
    }
    return b < end && a.col_idx[b] == kb;
}

template <bool FILL>
__global__ __launch_bounds__(64) void transpose_rows(TransposeArgs a) {
    const int m = blockIdx.x / a.n_blk, kb = blockIdx.x - m * a.n_blk, lane = threadIdx.x;
    int32_t* row = a.t_row_ptr + (size_t)m * (a.n_blk + 1) + kb;
    int at = FILL ? row[0] : 0;
    if (FILL && at < 0) return;
    for (int q0 = 0; q0 < a.n_blk; q0 += 64) {
        const bool holds = row_holds(a, m, q0 + lane, kb);
        const uint64_t all = __builtin_amdgcn_ballot_w64(holds);
        if (FILL && holds) {
            const int i = at + __popcll(all & ((1ull << lane) - 1));
            if (i < a.t_nnz) a.t_col_idx[i] = q0 + lane;
        }
        at += __popcll(all);
    }
    if (!FILL && lane == 0) row[1] = at;
}

// One workgroup: counts in row_ptr[m][kb + 1] become absolute offsets (-1 if the entries do not fit), and the plan is
// written.
__global__ __launch_bounds__(1024) void transpose_scan(TransposeArgs a) {
    __shared__ int64_t part[4][1024];  // entries, further parts, parts of split lists, split lists
    const int64_t rows = (int64_t)a.n_masks * a.n_blk, each = (rows + 1023) / 1024;
    const int64_t i0 = threadIdx.x * each, i1 = i0 + each < rows ? i0 + each : rows;
    int64_t sum[4] = {0, 0, 0, 0}, own[4];
    for (int64_t i = i0; i < i1; ++i) {
        const int c = a.t_row_ptr[i + i / a.n_blk + 1], n = pieces_of(c, a.seg);
        sum[0] += c;
        sum[1] += n - 1;
        sum[2] += n > 1 ? n : 0;
        sum[3] += n > 1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        own[k] = sum[k];
        part[k][threadIdx.x] = sum[k];
    }
    __syncthreads();
    for (int d = 1; d < 1024; d *= 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] = (int)threadIdx.x >= d ? part[k][threadIdx.x - d] : 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) part[k][threadIdx.x] += sum[k];
        __syncthreads();
    }
    const bool fits = part[0][1023] <= a.t_nnz;
    int64_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = part[k][threadIdx.x] - own[k];
    int4* item = reinterpret_cast<int4*>(a.plan);
    int4* more = item + rows;
    for (int64_t i = threadIdx.x; i < a.max_more; i += 1024) {
        if (!fits || i >= part[1][1023]) more[i] = int4{-1, 0, 0, 0};
        if (!fits || i >= part[3][1023]) more[a.max_more + i] = int4{-1, 0, 0, 0};
    }
    for (int64_t i = i0; i < i1; ++i) {
        const int64_t m = i / a.n_blk;
        const int c = a.t_row_ptr[i + m + 1], n = pieces_of(c, a.seg), to = fits ? (int)at[0] : -1;
        if (i == m * a.n_blk) a.t_row_ptr[i + m] = to;
        a.t_row_ptr[i + m + 1] = fits ? to + c : -1;
        for (int j = 0; j < (fits ? n : 1); ++j) {
            const int4 x = plan_item((int)i, to, c, a.seg, j, n, (int)at[2]);
            if (j == 0)
                item[i] = x;
            else
                more[at[1]++] = x;
        }
        if (fits && n > 1) {
            more[a.max_more + at[3]++] = int4{(int)i, (int)at[2], n, 0};
            at[2] += n;
        }
        at[0] += c;
    }
}

}  // namespace

hipError_t launch_index_transpose(const TransposeArgs& a, hipStream_t stream) {
    if (a.n_blk <= kSmall) {
        const size_t lds = (size_t)a.n_blk * ((a.n_blk + 31) / 32) * 4;
        hipLaunchKernelGGL(transpose_small, dim3(a.n_masks), dim3(1024), lds, stream, a);
        return hipGetLastError();
    }
    const dim3 rows((uint32_t)a.n_masks * (uint32_t)a.n_blk);
    hipLaunchKernelGGL(transpose_rows<false>, rows, dim3(64), 0, stream, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(transpose_scan, dim3(1), dim3(1024), 0, stream, a);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(transpose_rows<true>, rows, dim3(64), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_index_build(const IndexArgs& a, hipStream_t stream) {
    const int rows = a.n_masks * a.n_blk;
    hipLaunchKernelGGL(row_count, dim3(rows), dim3(kThreads), 0, stream, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(row_scan, dim3(1), dim3(kThreads), 0, stream, a);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(row_fill, dim3(rows), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace rt

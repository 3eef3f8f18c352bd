// The kernels of include/qknorm_pages.h.
#include "qknorm_pages.cuh"

namespace qknorm {

// Exclusive prefix sum over the CTA of a count per thread, and the total.  scratch: 33 ints.
__device__ __forceinline__ int plan_scan(int v, int* scratch, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  __syncthreads();  // the last call's readers are done
  if (lane == 31) scratch[warp] = upto;
  __syncthreads();
  if (warp == 0) {
    int w = scratch[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += x;
    }
    scratch[lane] = w;
  }
  __syncthreads();
  total = scratch[31];
  return upto - v + (warp > 0 ? scratch[warp - 1] : 0);
}

// refs of pages p0 .. p0 + kPlanAhead - 1, 1 where nothing is there.
__device__ __forceinline__ void plan_refs(const PageParams& P, long long p0, long long end, int (&r)[kPlanAhead]) {
  if (p0 + kPlanAhead <= end && (reinterpret_cast<uintptr_t>(P.refs + p0) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < kPlanAhead; i += 4) {
      const int4 v = *reinterpret_cast<const int4*>(P.refs + p0 + i);
      r[i] = v.x, r[i + 1] = v.y, r[i + 2] = v.z, r[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPlanAhead; ++i) r[i] = p0 + i < end ? P.refs[p0 + i] : 1;
  }
}

// One CTA.  For every fork: src, dst (pages to copy, -1: none) and len (-1: left out).
__global__ void __launch_bounds__(kPlanThreads) pages_fork_plan_kernel(const __grid_constant__ PageParams P) {
  __shared__ int scratch[33];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x;
  auto in = [&](int row) { return row >= 0 && row < P.rows; };
  for (int i = tid; i < P.n; i += kPlanThreads)
    if (in(P.children[i])) P.claim[P.children[i]] = 0x7fffffff;
  __syncthreads();
  for (int i = tid; i < P.n; i += kPlanThreads)
    if (in(P.children[i])) atomicMin(P.claim + P.children[i], i);
  __syncthreads();
  // which forks can be made, and which of them need a page
  int wanted = 0;
  for (int i0 = 0; i0 < P.n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int len = -1, part = 0, src = -1;
    if (i < P.n) {
      const int parent = P.parents[i], child = P.children[i];
      if (in(parent) && in(child) && parent != child && P.lens[child] == 0 && __ldcg(P.claim + child) == i) {
        len = P.lens[parent];
        const int full = len / P.page_size;
        part = len % P.page_size != 0;
        if (len < 0 || full + part > P.cols) len = -1, part = 0;
        if (part) src = P.table[parent * P.ld + full];
      }
    }
    int total;
    const int rank = wanted + plan_scan(part, scratch, total);
    wanted += total;
    if (i < P.n) {
      P.len[i] = len;
      P.src[i] = src;
      P.dst[i] = part ? rank : -1;
    }
  }
  // the first `wanted` free pages
  int found = 0;
  for (long long p0 = 0; p0 < P.num_pages && found < wanted; p0 += kPlanThreads * kPlanAhead) {
    int r[kPlanAhead], mine = 0, total;
    const long long p = p0 + tid * kPlanAhead;
    plan_refs(P, p, P.num_pages, r);
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) mine += r[k] <= 0;
    int at = found + plan_scan(mine, scratch, total);
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k)
      if (r[k] <= 0) {
        if (at < wanted) P.free_page[at] = (int)(p + k);
        ++at;
      }
    found += total;
  }
  if (found > wanted) found = wanted;
  __syncthreads();
  for (int i = tid; i < P.n; i += kPlanThreads) {
    const int rank = P.dst[i];
    if (rank >= found) {  // no page left
      P.len[i] = -1;
      P.dst[i] = -1;
    } else if (rank >= 0) {
      const int page = __ldcg(P.free_page + rank);
      P.dst[i] = page;
      P.refs[page] = 1;
    }
    if (P.ok != nullptr) P.ok[i] = P.len[i] >= 0;
  }
}

__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_read(const int* mine, unsigned rank) {  // the same variable of another CTA
  uint32_t at = (uint32_t)__cvta_generic_to_shared(mine);
  int v;
  asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %1, %2;\n\tld.shared::cluster.s32 %0, [r];\n\t}" : "=r"(v) : "r"(at), "r"(rank) : "memory");
  return v;
}

// One cluster.  Lists of pages that move (src) and where to (dst), map from the one to the other, their number, and `live`.
__global__ void __cluster_dims__(kPlanCluster, 1, 1) __launch_bounds__(kPlanThreads) pages_compact_plan_kernel(const __grid_constant__ PageParams P) {
  __shared__ int scratch[33];
  __shared__ int held, holes, movers;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, rank = (int)cluster_rank();
  constexpr int kStep = kPlanThreads * kPlanAhead;
  const long long per = ((P.num_pages + kPlanCluster - 1) / kPlanCluster + kPlanAhead - 1) / kPlanAhead * kPlanAhead;
  const long long begin = per * rank < P.num_pages ? per * rank : P.num_pages, end = begin + per < P.num_pages ? begin + per : P.num_pages;
  const bool once = per <= kStep;  // a thread's pages are looked at once and stay in its registers
  int r[kPlanAhead], total;
  // held pages
  int mine = 0;
  for (long long p0 = begin + tid * kPlanAhead; p0 < end; p0 += kStep) {
    plan_refs(P, p0, end, r);
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) mine += p0 + k < end && r[k] > 0;
  }
  plan_scan(mine, scratch, total);
  if (tid == 0) held = total;
  __syncthreads();
  cluster_sync();
  int live = 0;
  for (int c = 0; c < kPlanCluster; ++c) live += cluster_read(&held, c);
  // free pages before `live`, and held ones from there on, of a thread's kPlanAhead pages: in the lower and the upper half of a word
  auto both = [&](long long p0) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) {
      if (p0 + k >= end) continue;
      n += r[k] <= 0 && p0 + k < live ? 1 : r[k] > 0 && p0 + k >= live ? 1 << 16 : 0;
    }
    return n;
  };
  auto list = [&](long long p0, int ia, int ib) {
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) {
      const long long p = p0 + k;
      if (p >= end) continue;
      if (r[k] <= 0 && p < live) P.dst[ia++] = (int)p;
      if (p >= live) {
        P.map[p] = (int)p;  // a free page that a row names all the same
        if (r[k] > 0) P.src[ib++] = (int)p;
      }
    }
  };
  int before = 0, n_holes = 0, n_movers = 0;
  const long long mine0 = begin + tid * kPlanAhead;
  for (long long at = begin; at < end; at += kStep) {
    const long long p0 = at + tid * kPlanAhead;
    if (!once && p0 < end) plan_refs(P, p0, end, r);
    before = plan_scan(both(p0), scratch, total);
    n_holes += total & 0xffff;
    n_movers += total >> 16;
  }
  if (tid == 0) {
    holes = n_holes;
    movers = n_movers;
  }
  __syncthreads();
  cluster_sync();
  int hole = 0, mover = 0, moves = 0;
  for (int c = 0; c < kPlanCluster; ++c) {
    const int a = cluster_read(&holes, c), b = cluster_read(&movers, c);
    if (c < rank) hole += a, mover += b;
    moves += b;
  }
  if (once) {
    list(mine0, hole + (before & 0xffff), mover + (before >> 16));
  } else {
    for (long long at = begin; at < end; at += kStep) {
      const long long p0 = at + tid * kPlanAhead;
      if (p0 < end) plan_refs(P, p0, end, r);
      before = plan_scan(both(p0), scratch, total);
      list(p0, hole + (before & 0xffff), mover + (before >> 16));
      hole += total & 0xffff;
      mover += total >> 16;
    }
  }
  __threadfence();
  cluster_sync();  // the lists are complete, and nobody reads another's shared memory any more
  for (int k = rank * kPlanThreads + tid; k < moves; k += kPlanCluster * kPlanThreads) P.map[__ldcg(P.src + k)] = __ldcg(P.dst + k);
  if (rank == 0 && tid == 0) {
    *P.count = moves;
    *P.live = live;
  }
}

// Rows give up their pages: a CTA per row.
__global__ void __launch_bounds__(kPageThreads) pages_free_kernel(const __grid_constant__ PageParams P) {
  __shared__ int tokens;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int i = blockIdx.x; i < P.n; i += gridDim.x) {
    const int row = P.children[i];
    if (row < 0 || row >= P.rows) continue;
    __syncthreads();
    if (threadIdx.x == 0) tokens = atomicExch(P.lens + row, 0);  // a row named twice has nothing left the second time
    __syncthreads();
    const long long len = tokens;
    long long held = len <= 0 ? 0 : (len + P.page_size - 1) / P.page_size;
    if (held > P.cols) held = P.cols;
    for (int j = threadIdx.x; j < held; j += kPageThreads) {
      const int e = P.table[row * P.ld + j];
      if (e >= 0 && e < P.num_pages) atomicSub(P.refs + e, 1);
    }
  }
}

// One run of bytes, by the CTA; n <= kPageChunk.
template <class V>
__device__ __forceinline__ void copy_run(char* dst, const char* src, int n) {
  const V* s = reinterpret_cast<const V*>(src);
  V* d = reinterpret_cast<V*>(dst);
  const int m = n / (int)sizeof(V);
  constexpr int kAhead = 4;
  for (int i0 = threadIdx.x; i0 < m; i0 += kAhead * kPageThreads) {
    V v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + k * kPageThreads < m) v[k] = __ldcs(s + i0 + k * kPageThreads);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + k * kPageThreads < m) __stcs(d + i0 + k * kPageThreads, v[k]);
  }
}

// blockIdx.y: a pool, or behind the last one the books.
__global__ void __launch_bounds__(kPageThreads) pages_move_kernel(const __grid_constant__ MoveParams M) {
  const PageParams& P = M.P;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int pairs = P.n_device != nullptr ? *P.n_device : P.n;
  if ((int)blockIdx.y < M.pools) {
    const PagePool& pool = M.pool[blockIdx.y];
    const long long chunks = (pool.bytes + kPageChunk - 1) / kPageChunk, per = pool.pieces * chunks;
    for (long long it = blockIdx.x; it < per * pairs; it += gridDim.x) {
      const int i = (int)(it / per);
      const long long rest = it - i * per, piece = rest / chunks, at = (rest - piece * chunks) * kPageChunk;
      const int a = P.from[i], b = P.to[i];
      if (a < 0 || b < 0 || a >= P.num_pages || b >= P.num_pages || a == b) continue;
      const long long off = piece / pool.count1 * pool.stride0 + piece % pool.count1 * pool.stride1 + at;
      const char* src = pool.base + a * pool.page + off;
      char* dst = pool.base + b * pool.page + off;
      const int n = pool.bytes - at < kPageChunk ? (int)(pool.bytes - at) : kPageChunk;
      if (pool.unit == 16) copy_run<uint4>(dst, src, n);
      else if (pool.unit == 4) copy_run<unsigned>(dst, src, n);
      else copy_run<unsigned char>(dst, src, n);
    }
    return;
  }
  if (P.books == 1) {  // forks: a CTA per child
    for (int i = blockIdx.x; i < P.n; i += gridDim.x) {
      const int len = P.len[i];
      if (len < 0) continue;
      const int parent = P.parents[i], child = P.children[i], full = len / P.page_size, fresh = P.to[i];
      for (int j = threadIdx.x; j < P.cols; j += kPageThreads) {
        int e = -1;
        if (j < full) {
          e = P.table[parent * P.ld + j];
          if (e >= 0 && e < P.num_pages) atomicAdd(P.refs + e, 1);
        } else if (j == full && fresh >= 0) {
          e = fresh;
        }
        P.table[child * P.ld + j] = e;
      }
      if (threadIdx.x == 0) P.lens[child] = len;
    }
  } else {  // compact: entries follow their pages, refs move
    for (int row = blockIdx.x; row < P.rows; row += gridDim.x) {
      const long long len = P.lens[row];
      long long held = len <= 0 ? 0 : (len + P.page_size - 1) / P.page_size;
      if (held > P.cols) held = P.cols;
      for (int j = threadIdx.x; j < held; j += kPageThreads) {
        const int e = P.table[row * P.ld + j];
        if (e >= *P.live && e < P.num_pages) P.table[row * P.ld + j] = P.map[e];
      }
    }
    for (int k = blockIdx.x * kPageThreads + threadIdx.x; k < pairs; k += gridDim.x * kPageThreads) {
      const int a = P.from[k], b = P.to[k];
      P.refs[b] = P.refs[a];
      P.refs[a] = 0;
    }
  }
}

PageKernel pages_kernel_for(int which) {
  switch (which) {
    case kPagesForkPlan: return pages_fork_plan_kernel;
    case kPagesCompactPlan: return pages_compact_plan_kernel;
    default: return pages_free_kernel;
  }
}
MoveKernel pages_move_kernel_for() { return pages_move_kernel; }

}  // namespace qknorm

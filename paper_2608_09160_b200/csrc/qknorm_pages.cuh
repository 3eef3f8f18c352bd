// Pages of a paged cache: copying, forking, freeing, compacting (include/qknorm_pages.h).
//
// The bookkeeping is a few thousand integers and bound by latency: which page is free, and which moves where, are prefix sums over
// refs, done by one CTA (fork: it stops as soon as it has found the pages it needs) or by one cluster of eight that exchanges its counts
// through distributed shared memory (compact: it has to see all of refs).  The k-th fork takes the k-th free page whichever thread finds it,
// so that nothing depends on the order of atomics; those that remain only add to refs.
// A second launch moves the data, bound by HBM (each byte read once, written once), and brings the tables up to date beside it.
// Measured: 96 rows dropped and forked anew over 32 layers, 403 MB moved: 66 us, 92 % of the copy rate with three launches; 983 of 4096 pages of
// eight layers packed, 515 MB: 102 us with two copies of the tables before it, of which the plan is about 7; eight forks of one layer 8.2 us.
#pragma once
#include <stdint.h>

namespace qknorm {

constexpr int kPagePools = 48;  // pools of a launch: what its parameters hold
constexpr int kPageThreads = 256, kPlanThreads = 1024, kPlanCluster = 8;
constexpr int kPageChunk = 16384;  // bytes that a CTA copies at a time: four vectors of 16 bytes a thread
constexpr int kPlanAhead = 8;      // refs that a thread looks at together

struct PagePool {
  char* base;
  long long page, stride0, stride1, bytes;
  long long pieces;  // count[0] * count[1]
  int count1;
  int unit;          // 16, 4 or 1: what divides everything
};

struct PageParams {  // the books
  long long num_pages;
  int* refs;
  int* table;
  int cols;
  long long ld;
  int* lens;
  int rows, page_size;
  const int *from, *to;  // pairs of pages
  const int *parents, *children;  // fork; free: the rows are children
  int n;                 // of pairs, forks or rows
  const int* n_device;   // compact: how many pairs there are
  int* ok;               // fork
  int* live;             // compact
  int *claim, *free_page, *src, *dst, *len, *map, *count;  // workspace
  int books;             // the launch that moves pages keeps the tables, too: 1 fork, 2 compact
};
struct MoveParams {
  PageParams P;
  int pools;
  PagePool pool[kPagePools];
};

typedef void (*PageKernel)(const PageParams);
typedef void (*MoveKernel)(const MoveParams);
enum { kPagesForkPlan, kPagesCompactPlan, kPagesFree };
PageKernel pages_kernel_for(int which);  // in qknorm_pages_inst.cu
MoveKernel pages_move_kernel_for();

}  // namespace qknorm

// The paged key/value cache: its handle, and the two calls that write into it.
//
// A page holds page_size positions of every key/value head, [Hkv, page_size, Dh]; position p of item b is slot p % page_size of
// page table[b][p / page_size].  Both calls are pure data movement, 16 bytes a lane, bound by the loads that wait for each
// other (lengths and path, then the page's number, then the stores; the rows are asked for beside the page's number) where the
// rows are few (16 items' paths, 24 heads of 64: 2.4 us), and by memory where they are many.  A position whose table entry
// names no page of the pool is not written: what a read may clamp, a write may not.
#include <new>

#include "lpp_internal.h"

extern "C" int32_t lpp_paged_create(int32_t dtype, int32_t Hkv, int32_t Dh, int32_t page_size, int32_t n_pages,
                                    lpp_paged** out) {
  if (!out) return LPP_EINVAL;
  *out = nullptr;
  if (Hkv < 1 || Dh < 1 || page_size < 1 || n_pages < 1) return LPP_EINVAL;
  if (dtype != LPP_F32 && dtype != LPP_BF16) return LPP_EUNSUPPORTED;
  if (Dh != 64 && Dh != 128) return LPP_EUNSUPPORTED;
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return LPP_EUNSUPPORTED;
  if (Hkv > 4096) return LPP_EUNSUPPORTED;                   // (a page stays below 2^31 bytes)
  lpp_paged* c = new (std::nothrow) lpp_paged();
  if (!c) return LPP_EHIP;
  c->dtype = dtype; c->Hkv = Hkv; c->Dh = Dh; c->page_size = page_size; c->n_pages = n_pages;
  while ((1 << c->page_shift) < page_size) ++c->page_shift;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) {
    (void)hipGetLastError();
    *out = c;                                                // host-only handle
    return LPP_OK;
  }
  auto fail = [&]() {
    (void)hipGetLastError();
    lpp_paged_destroy(c);
    return (int32_t)LPP_EHIP;
  };
  int v = 0;
  if (hipGetDevice(&c->device) != hipSuccess) return fail();
  if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, c->device) != hipSuccess) return fail();
  if (v > 0) c->n_cu = v;
  if (hipMalloc((void**)&c->d_counters, sizeof(int32_t) * LPP_COUNTER_SLOTS) != hipSuccess) return fail();
  if (hipMemset(c->d_counters, 0, sizeof(int32_t) * LPP_COUNTER_SLOTS) != hipSuccess) return fail();
  if (hipStreamSynchronize(nullptr) != hipSuccess) return fail();            // (whatever stream uses them first)
  *out = c;
  return LPP_OK;
}

extern "C" int32_t lpp_paged_destroy(lpp_paged* c) {
  if (!c) return LPP_OK;
  if (c->d_counters) (void)hipFree(c->d_counters);
  delete c;
  return LPP_OK;
}

namespace {

struct PagedWriteArgs {
  const unsigned char* k_new;
  const unsigned char* v_new;
  unsigned char* k_pages;
  unsigned char* v_pages;
  const int32_t* table;
  const int32_t* seq_len;
  const int32_t* path;              // commit
  const int32_t* accept_len;        // commit
  const int32_t* row_len;           // append, or null
  int32_t* new_len;
  int32_t Hkv, M, depth, table_stride, capacity, page_shift, n_pages;
  int32_t chunk_shift;              // log2 of the 16-byte chunks of a row
  int32_t tiles;                    // append: blocks of a (item, head)
};

__device__ __forceinline__ int64_t page_row(const PagedWriteArgs& a, int page, int h, int pos) {
  const int slot = pos & ((1 << a.page_shift) - 1);
  return ((((int64_t)page * a.Hkv + h) << a.page_shift) + slot) << a.chunk_shift;      // in chunks
}

// A block is one kept row of one item, all heads: row 0 is the root, row i the i-th of the accepted path.
__global__ __launch_bounds__(256) void paged_commit_kernel(PagedWriteArgs a) {
  const int b = (int)(blockIdx.x / (unsigned)(a.depth + 1)), i = (int)(blockIdx.x - (unsigned)b * (a.depth + 1));
  const int accepted = a.accept_len[b], len = a.seq_len[b];
  const int node = a.path[(int64_t)b * a.depth + max(i - 1, 0)];
  const int n = min(max(accepted, 0), a.depth), base = min(max(len, 0), a.capacity);
  if (i == 0 && threadIdx.x == 0 && a.new_len) a.new_len[b] = min(base + 1 + n, a.capacity);
  const int pos = base + i;
  if (i > n || pos >= a.capacity) return;
  const int page = a.table[(int64_t)b * a.table_stride + (pos >> a.page_shift)];
  if ((unsigned)page >= (unsigned)a.n_pages) return;
  const int row = i > 0 ? min(max(node, 0), a.M - 1) : 0;
  const int chunks = 1 << a.chunk_shift;
  const uint4* kn = reinterpret_cast<const uint4*>(a.k_new);
  const uint4* vn = reinterpret_cast<const uint4*>(a.v_new);
  for (int t = threadIdx.x; t < a.Hkv * chunks; t += 256) {
    const int h = t >> a.chunk_shift, c = t & (chunks - 1);
    const int64_t src = ((((int64_t)b * a.Hkv + h) * a.M + row) << a.chunk_shift) + c;
    const int64_t dst = page_row(a, page, h, pos) + c;
    const uint4 k = kn[src], v = vn[src];
    reinterpret_cast<uint4*>(a.k_pages)[dst] = k;
    reinterpret_cast<uint4*>(a.v_pages)[dst] = v;
  }
}

// A block is 256 chunks (16 rows of 256 bytes) of one (item, head), one of K and of V a lane.  (Four of each a lane, 640 blocks
// in all: 22.6 us for 4 chunks of up to 2048 rows, 8 heads of 128; so 8.7, which is 4.8 TB/s: as fast as a copy.)
__global__ __launch_bounds__(256) void paged_append_kernel(PagedWriteArgs a) {
  const int bh = (int)(blockIdx.x / (unsigned)a.tiles), tile = (int)(blockIdx.x - (unsigned)bh * a.tiles);
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int base = min(max(a.seq_len[b], 0), a.capacity);
  const int n = a.row_len ? min(max(a.row_len[b], 0), a.M) : a.M;
  if (h == 0 && tile == 0 && threadIdx.x == 0 && a.new_len) a.new_len[b] = (int)min((int64_t)base + n, (int64_t)a.capacity);
  const int row = tile * (256 >> a.chunk_shift) + (int)(threadIdx.x >> a.chunk_shift), c = threadIdx.x & ((1 << a.chunk_shift) - 1);
  if (row >= min(n, a.capacity - base)) return;
  const int page = a.table[(int64_t)b * a.table_stride + ((base + row) >> a.page_shift)];
  const int64_t src = (((int64_t)bh * a.M + row) << a.chunk_shift) + c;
  const uint4 k = reinterpret_cast<const uint4*>(a.k_new)[src], v = reinterpret_cast<const uint4*>(a.v_new)[src];
  if ((unsigned)page >= (unsigned)a.n_pages) return;
  const int64_t dst = page_row(a, page, h, base + row) + c;
  reinterpret_cast<uint4*>(a.k_pages)[dst] = k;
  reinterpret_cast<uint4*>(a.v_pages)[dst] = v;
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int32_t paged_write(const lpp_paged* cache, const void* k_new, const void* v_new, const int32_t* page_table,
                    int32_t table_stride, const int32_t* seq_len, int32_t B, int32_t M, void* k_pages, void* v_pages,
                    int32_t* new_len, PagedWriteArgs* a) {
  if (!cache || !k_new || !v_new || !page_table || !seq_len || !k_pages || !v_pages) return LPP_EINVAL;
  if (B < 1 || M < 1 || table_stride < 1) return LPP_EINVAL;
  if (new_len == seq_len) return LPP_EINVAL;                // every block reads seq_len
  if (misaligned(k_new) || misaligned(v_new) || misaligned(k_pages) || misaligned(v_pages)) return LPP_EINVAL;
  const int64_t capacity = (int64_t)table_stride << cache->page_shift;
  if (capacity + M > 0x7FFFFFFF) return LPP_EUNSUPPORTED;
  a->k_new = (const unsigned char*)k_new; a->v_new = (const unsigned char*)v_new;
  a->k_pages = (unsigned char*)k_pages; a->v_pages = (unsigned char*)v_pages;
  a->table = page_table; a->seq_len = seq_len; a->new_len = new_len;
  a->path = nullptr; a->accept_len = nullptr; a->row_len = nullptr;
  a->Hkv = cache->Hkv; a->M = M; a->depth = 1; a->tiles = 1;
  a->table_stride = table_stride; a->capacity = (int32_t)capacity; a->page_shift = cache->page_shift; a->n_pages = cache->n_pages;
  const int chunks = cache->Dh * (cache->dtype == LPP_F32 ? 4 : 2) / 16;      // 8, 16 or 32
  a->chunk_shift = chunks == 8 ? 3 : chunks == 16 ? 4 : 5;
  return LPP_OK;
}

}  // namespace

extern "C" int32_t lpp_paged_commit_kv(const lpp_paged* cache, const lpp_tree* tree, const void* k_tree, const void* v_tree,
                                       const int32_t* path, const int32_t* accept_len, const int32_t* page_table,
                                       int32_t table_stride, const int32_t* seq_len, int32_t B, void* k_pages, void* v_pages,
                                       int32_t* new_len, void* stream) {
  if (!tree || !path || !accept_len) return LPP_EINVAL;
  if (new_len == accept_len || (new_len && (new_len == path || new_len == page_table))) return LPP_EINVAL;
  PagedWriteArgs a;
  const int32_t st = paged_write(cache, k_tree, v_tree, page_table, table_stride, seq_len, B, tree->M, k_pages, v_pages, new_len, &a);
  if (st != LPP_OK) return st;
  // (a tree of the root alone has no path entries, [B, 0]: what the kernel reads ahead is then something else of B words)
  a.path = tree->depth > 0 ? path : seq_len; a.accept_len = accept_len;
  a.depth = tree->depth > 0 ? tree->depth : 1;
  const int64_t blocks = (int64_t)B * (a.depth + 1);
  if (!lpp_launch_fits(blocks, 256)) return LPP_EUNSUPPORTED;
  if (!cache->d_counters || !tree->d_anc) return LPP_EHIP;   // host-only handle: no device
  if (!lpp_is_current(cache->device)) return LPP_EINVAL;
  hipLaunchKernelGGL(paged_commit_kernel, dim3((unsigned)blocks), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}

extern "C" int32_t lpp_paged_append_kv(const lpp_paged* cache, const void* k_new, const void* v_new, const int32_t* row_len,
                                       const int32_t* page_table, int32_t table_stride, const int32_t* seq_len, int32_t B,
                                       int32_t M, void* k_pages, void* v_pages, int32_t* new_len, void* stream) {
  if (new_len && (new_len == row_len || new_len == page_table)) return LPP_EINVAL;
  PagedWriteArgs a;
  const int32_t st = paged_write(cache, k_new, v_new, page_table, table_stride, seq_len, B, M, k_pages, v_pages, new_len, &a);
  if (st != LPP_OK) return st;
  a.row_len = row_len;
  a.tiles = (int32_t)((((int64_t)M << a.chunk_shift) + 255) >> 8);
  const int64_t blocks = (int64_t)B * cache->Hkv * a.tiles;
  if (!lpp_launch_fits(blocks, 256)) return LPP_EUNSUPPORTED;
  if (!cache->d_counters) return LPP_EHIP;
  if (!lpp_is_current(cache->device)) return LPP_EINVAL;
  hipLaunchKernelGGL(paged_append_kernel, dim3((unsigned)blocks), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
  LPP_HIP_TRY(hipGetLastError());
  return LPP_OK;
}

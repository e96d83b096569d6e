// Runs the library's token_at on the host for every thread of a launch, those past the last item included.  The arrays
// that it may read end where an inaccessible page begins, so a read past either of them ends the program.
#include <sys/mman.h>
#include <unistd.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "gl_cache4.cuh"

// n values whose last one is the last of its page
static int32_t* guarded(int64_t n) {
  const int64_t page = sysconf(_SC_PAGESIZE), bytes = (n * 4 + page - 1) / page * page;
  char* p = static_cast<char*>(mmap(nullptr, bytes + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
  if (p == MAP_FAILED || mprotect(p + bytes, page, PROT_NONE)) exit(3);
  return reinterpret_cast<int32_t*>(p + bytes - n * 4);
}

int main(int argc, char** argv) {
  if (argc != 8) return 2;
  const int batch = atoi(argv[1]), T = atoi(argv[2]), heads = atoi(argv[3]), D = atoi(argv[4]), page = atoi(argv[5]),
            width = atoi(argv[6]), per_block = atoi(argv[7]);
  int32_t* lengths = guarded(batch);
  int32_t* table = guarded(static_cast<int64_t>(batch) * width);
  const int pages = batch * width + 1;
  for (int b = 0; b < batch; ++b) lengths[b] = b % 3 == 0 ? width * page : b % 3 == 1 ? T / 2 : width * page + 7;
  for (int i = 0; i < batch * width; ++i) table[i] = (i * 7 + 3) % (pages + 2) - 1;
  TokensParams p;
  memset(&p, 0, sizeof(p));
  uint8_t* const data = reinterpret_cast<uint8_t*>(uintptr_t{1} << 20);
  p.c.data = data;
  p.c.table = table;
  p.c.lengths = lengths;
  p.c.pages = pages;
  p.c.head_stride = static_cast<int64_t>(page / kGroup) * group_bytes(D);
  p.c.page_stride = p.c.head_stride * heads;
  p.c.kv_heads = heads;
  p.c.page_tokens = page;
  p.c.batch = batch;
  p.c.width = width;
  p.c.capacity = width * page;
  p.c.div_page.set(page);
  p.T = T;
  p.D = D;
  p.pitch = static_cast<int64_t>(heads) * D;
  p.items = static_cast<uint32_t>(batch) * T * heads * (D / 8);
  p.div_row.set(D / 8);
  p.div_heads.set(heads);
  p.div_T.set(T);
  const uint32_t threads = (p.items + per_block - 1) / per_block * per_block;
  for (uint32_t item = 0; item < threads; ++item) {
    const TokenAt at = token_at(p, item);
    if (item >= p.items) {
      if (at.group) { printf("item %u of %u has a place\n", item, p.items); return 1; }
      continue;
    }
    const int w = item % (D / 8), h = item / (D / 8) % heads, i = item / (D / 8) / heads % T, b = item / (D / 8) / heads / T;
    const int pos = (lengths[b] > width * page ? width * page : lengths[b]) - T + i;
    uint8_t* group = nullptr;
    if (pos >= 0) {
      const int pg = table[static_cast<int64_t>(b) * width + pos / page];
      if (pg >= 0 && pg < pages)
        group = data + pg * p.c.page_stride + h * p.c.head_stride + static_cast<int64_t>(pos % page / kGroup) * group_bytes(D);
    }
    if (at.group != group || at.w != w || (group && at.tok != pos % page % kGroup) ||
        at.dense != (static_cast<int64_t>(b) * T + i) * p.pitch + h * D + w * 8) {
      printf("item %u: wrong place\n", item);
      return 1;
    }
  }
  printf("ok %u\n", p.items);
  return 0;
}

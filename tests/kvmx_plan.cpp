// Runs, on the host alone, the microscaled attention's planning: launches are recorded here
// instead of reaching a GPU, and the split schedule's index arithmetic is followed in 64
// bits.  Each argument is a call, "hd bits H T shared cached,q cached,q ...", and gives a
// line of its launches, and the status:
//   <workgroups> <threads each> <kernel> <figures of its schedule>; ... status <status>
#include "k_attn_mx.hip"

#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <utility>
#include <vector>

using namespace ardit;

static const AttnStream& stream_of_item(const AttnArgs& a, int64_t item) {
  int si = 0;
  for (int i = 1; i < a.n_streams; ++i)
    if (item >= a.s[i].item_begin) si = i;
  return a.s[si];
}

static void split_figures(const AttnArgs& a) {
  // per item: how many of its tiles are taken, and the furthest one; the largest number formed
  // on the way, and the slots of partial results
  std::map<int64_t, std::pair<int64_t, int64_t>> got;
  std::map<int64_t, int> slots;
  int64_t most = 0;
  bool inside = true;
  const int64_t items = a.total_items - a.item0;
  auto take = [&](const AttnStream& s, int64_t item, int64_t tb, int64_t te, int64_t slot) {
    inside = inside && item >= 0 && item < static_cast<int64_t>(s.n_qtiles) * a.H && tb >= 0 && tb < te && te <= s.n_tiles;
    auto& g = got[s.item_begin + item];
    g.first += te - tb;
    g.second = std::max(g.second, te);
    if (slot >= 0) ++slots[slot];
  };
  for (int64_t gi = a.item0; gi < a.total_items; ++gi) {
    const AttnStream& s = stream_of_item(a, gi);
    if (s.main_tiles > 0) take(s, gi - s.item_begin, 0, s.main_tiles, s.main_tiles == s.n_tiles ? -1 : gi - a.item0);
  }
  for (int64_t r = 0; r < a.split_blocks - items; ++r) {
    int64_t pos = r * a.split_tiles;
    const int64_t end = std::min<int64_t>(pos + a.split_tiles, a.total_tiles);
    most = std::max(most, pos + a.split_tiles);
    while (pos < end) {
      int si = 0;
      for (int i = 1; i < a.n_streams; ++i)
        if (pos >= a.s[i].tail_begin) si = i;
      const AttnStream& s = a.s[si];
      const int64_t tl = s.n_tiles - s.main_tiles, rel = pos - s.tail_begin;
      const int64_t item = std::max(0, a.item0 - s.item_begin) + rel / tl;
      const int64_t tb = s.main_tiles + rel % tl, te = std::min<int64_t>(s.n_tiles, tb + (end - pos));
      pos += te - tb;
      take(s, item, tb, te, items + s.item_begin + item - a.item0 + r);
    }
  }
  bool all = inside && static_cast<int64_t>(got.size()) == items;
  for (const auto& g : got) {
    const AttnStream& s = stream_of_item(a, g.first);
    all = all && g.second.first == s.n_tiles && g.second.second == s.n_tiles;
  }
  for (const auto& s : slots) all = all && s.second == 1 && s.first < 2 * kAttnSplitBlocks;
  printf("most %lld covered %d", static_cast<long long>(most), all ? 1 : 0);
}

template <int HD, int BITS>
static bool figures(const void* f, void** args) {
  if (f == reinterpret_cast<const void*>(&attn_mx_join_kernel<HD>)) {
    const MxSmallArgs& a = *static_cast<const MxSmallArgs*>(args[0]);
    int64_t rows = 0;   // that have something to join
    for (int i = a.shared; i < a.n_spans; ++i)
      if (a.s[i].part_begin >= 0) rows += a.s[i].q_len;
    printf("join %lld %d", static_cast<long long>(rows), a.groups);
  } else if (f == reinterpret_cast<const void*>(&attn_mx_small_kernel<HD, BITS>)) {
    const MxSmallArgs& a = *static_cast<const MxSmallArgs*>(args[0]);
    int pieces = 0;
    bool sound = true;
    for (int i = 0; i < a.n_spans; ++i) {
      const MxSpan& s = a.s[i];
      pieces = std::max(pieces, s.pieces);
      sound = sound && s.pieces >= 1 && s.per_piece >= 1 && static_cast<int64_t>(s.pieces) * s.per_piece >= s.tile1 - s.tile0 &&
              static_cast<int64_t>(s.pieces - 1) * s.per_piece < s.tile1 - s.tile0;
    }
    printf("few %d sound %d", pieces, sound ? 1 : 0);
  } else if (f == reinterpret_cast<const void*>(&attn_mx_split_kernel<HD, BITS>)) {
    printf("split ");
    split_figures(static_cast<const MxLargeArgs*>(args[0])->a);
  } else if (f == reinterpret_cast<const void*>(&attn_mx_kernel<HD, BITS, false>) ||
             f == reinterpret_cast<const void*>(&attn_mx_kernel<HD, BITS, true>)) {
    printf("items %d", static_cast<const MxLargeArgs*>(args[0])->a.total_items);
  } else {
    return false;
  }
  return true;
}

// A launch, taken over from the runtime.
static dim3 g_grid, g_block;
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = g_grid;
  *block = g_block;
  *lds = 0;
  *stream = nullptr;
  return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }
extern "C" hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  printf("%u %u ", grid.x, block.x);
  if (!figures<128, 8>(f, args) && !figures<128, 4>(f, args) && !figures<64, 8>(f, args) && !figures<64, 4>(f, args)) printf("merge");
  printf("; ");
  return hipSuccess;
}

int main(int argc, char** argv) {
  for (int i = 1; i < argc; ++i) {
    MxPages p;
    memset(&p, 0, sizeof(p));
    RowStreams rs;
    memset(&rs, 0, sizeof(rs));
    int shared = 0, at = 0;
    if (sscanf(argv[i], "%d %d %d %d %d%n", &p.hd, &p.bits, &p.H, &p.T, &shared, &at) != 5) return 2;
    p.nt = (p.T + 63) / 64;
    p.fT = make_fastdiv(p.T);
    p.fnt = make_fastdiv(p.nt);
    int rows = 0, cached, q, n;
    for (const char* s = argv[i] + at; rs.n < kMaxStreams && sscanf(s, " %d,%d%n", &cached, &q, &n) == 2; s += n) {
      rs.s[rs.n].row_begin = rows;
      rs.s[rs.n].len = q;
      rs.s[rs.n].cache_len = cached;
      rows += q;
      ++rs.n;
    }
    p.max_frames = 1 << 30;
    p.n_pages = 1;
    const int status = launch_attention_mx(nullptr, p, nullptr, nullptr, rs, shared, reinterpret_cast<float*>(uintptr_t(1) << 40));
    printf("status %d\n", status);
    fflush(stdout);
  }
  return 0;
}

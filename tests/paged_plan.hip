// The index arithmetic of ppd_paged_attention on the host, for tests: built without device code and called through ctypes.
#include "../paper_2307_05908_amd/csrc/ppd_paged_attn.h"

extern "C" int t_first_seen(int pos, int window) { return ppd::first_seen(pos, window); }

extern "C" void t_span(int pos0, int n, int tile, int tile_rows, int group, int part, int parts, int room, int window, int* lo, int* hi) {
  const ppd::Span s = ppd::span_of(pos0, n, tile, tile_rows, group, part, parts, room, window);
  *lo = s.lo; *hi = s.hi;
}

extern "C" int t_have_places(int first, int parts, int items) { return ppd::have_places(first, parts, items); }

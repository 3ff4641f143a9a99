// The index arithmetic of ppd_paged_attention on the host, for tests: built without device code and called through ctypes.
#include "../paper_2307_05908_amd/csrc/ppd_paged_attn.h"

extern "C" int t_first_seen(int pos, int window) { return ppd::first_seen(pos, window); }

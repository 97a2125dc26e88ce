// Prints the layout that the library chooses for each call of attention over the 8-bit cache on
// its input: "dtype batch hkv group d cap T window sinks prefix" per line. Built and run by
// tests/test_cache8_rule.py on the CPU.
#include <stdio.h>

#include "spla_layout.h"

int main() {
  int dt, batch, hkv, group, d, cap, T, window, sinks, prefix;
  while (scanf("%d %d %d %d %d %d %d %d %d %d", &dt, &batch, &hkv, &group, &d, &cap, &T, &window,
               &sinks, &prefix) == 10) {
    spla_config c{};
    c.batch = batch;
    c.n_kv_heads = hkv;
    c.n_q_heads = hkv * group;
    c.head_dim = d;
    c.block_size = 32;
    c.max_seq_len = cap;
    c.dtype = dt;
    const spla::Dims m = spla::make_dims(c);
    spla_attend8_opts o{};
    const int32_t some = 0;
    o.window = window;
    o.sinks = sinks;
    o.attend.prefix_len = prefix ? &some : nullptr;
    const spla::AttendWs w = spla::attend8_ws_layout(m, T, spla::attend8_keys(m, T, o));
    printf("%d %d %d %d %d %d\n", w.rows, w.n_tiles, w.n_split, w.shares, w.join > 0,
           w.total <= spla::attend8_ws_bytes(m, T));
  }
  return 0;
}

// Gathers over the stand-in for the HIP runtime of host_steps.cpp, whose scenarios' names end at main.
#define main host_steps_main
#include "host_steps.cpp"
#undef main

// A gather out of a pool in 8 bits is laid out for the compute units that it runs on, as a page write is: those of its phase's share, a staged
// one among them.
static void shares_of_gathers() {
  const spd_pool_desc desc = {SPD_KV_GQA_FP8, 16, 8, 128, 128, 64};
  uint64_t bytes;
  spd_pool* p;
  CHECK(spd_pool_bytes(&desc, &bytes) == SPD_OK);
  CHECK(spd_pool_create(ctx, aligned_alloc(4096, bytes), bytes, &desc, &p) == SPD_OK);
  CHECK(spd_kv_reserve(p, 1, 40, nullptr) == SPD_OK);
  CHECK(spd_kv_gather(ctx, p, SPD_PHASE_DECODE, 1, 40, tensor, tensor) == SPD_OK && seen_cus == std::vector<int>{256});
  CHECK(spd_set_partition(ctx, 192, 64) == SPD_OK);
  for (const int phase : {SPD_PHASE_PREFILL, SPD_PHASE_DECODE}) CHECK(spd_kv_gather(ctx, p, phase, 1, 40, tensor, tensor) == SPD_OK);
  CHECK(seen_cus == (std::vector<int>{256, 192, 64}));
  CHECK(spd_pool_destroy(p) == SPD_OK);
}

int main() {
  setup();
  shares_of_gathers();
  puts("ok");
}

// GQA pools in 8 bits over host_steps.cpp's stand-in for the HIP runtime.  host_gqa_fp8 NAME runs one scenario.
#define main host_steps_main
#include "host_steps.cpp"
#undef main

static spd_pool* pool_of(int64_t pages, int32_t dim) {
  const spd_pool_desc desc = {SPD_KV_GQA_FP8, 16, 8, dim, dim, pages};
  uint64_t bytes;
  spd_pool* p;
  CHECK(spd_pool_bytes(&desc, &bytes) == SPD_OK);
  CHECK(spd_pool_create(ctx, aligned_alloc(4096, (bytes + 4095) / 4096 * 4096), bytes, &desc, &p) == SPD_OK);
  return p;
}

// A gather is laid out for the compute units that it runs on, as a page write is: those of its phase's share, a staged one among them.
static void shares_of_gathers() {
  spd_pool* p = pool_of(64, 128);
  CHECK(spd_kv_reserve(p, 1, 40, nullptr) == SPD_OK);
  CHECK(spd_kv_gather(ctx, p, SPD_PHASE_DECODE, 1, 40, tensor, tensor) == SPD_OK && seen_cus == std::vector<int>{256});
  CHECK(spd_set_partition(ctx, 192, 64) == SPD_OK);
  for (const int phase : {SPD_PHASE_PREFILL, SPD_PHASE_DECODE}) CHECK(spd_kv_gather(ctx, p, phase, 1, 40, tensor, tensor) == SPD_OK);
  CHECK(seen_cus == (std::vector<int>{256, 192, 64}));
}

// Launches of a decode step with append: records copied and tokens appended ahead of the attention only where a compute unit has more workgroups
// than run on it at once (three), and HBM does not hide what they do first.
static void launches_of_appends() {
  for (const int dim : {64, 128}) {
    spd_pool* p = pool_of(40000, dim);
    auto step = [&](int n, int32_t len, bool rotate) -> int {
      std::vector<uint64_t> ids((size_t)n);
      std::vector<int32_t> lens((size_t)n, len);
      for (int i = 0; i < n; ++i) ids[(size_t)i] = (uint64_t)i + 1;
      spd_rope_config r = rope(10000.0);
      r.rotary_dim = dim;
      const spd_decode_batch b = {n, ids.data(), lens.data(), tensor, tensor, tensor, tensor, 32, 0.1f, rotate ? &r : nullptr};
      CHECK(spd_decode_step(ctx, p, &b) == SPD_OK && spd_phase_sync(ctx, SPD_PHASE_DECODE) == SPD_OK);
      const int before = n_launches;
      CHECK(spd_decode_step(ctx, p, &b) == SPD_OK && spd_phase_sync(ctx, SPD_PHASE_DECODE) == SPD_OK);
      for (const uint64_t id : ids) CHECK(spd_kv_free(p, id, nullptr) == SPD_OK);
      return n_launches - before;
    };
    for (const bool rotate : {false, true}) {
      CHECK(step(96, 45, rotate) == 1);              // three workgroups per compute unit
      CHECK(step(128, 45, rotate) == 1);
      CHECK(step(200, 45, rotate) == 3);
      CHECK(step(200, 150, rotate) == 3);
    }
    CHECK(step(200, 300, false) == 2 && step(200, 300, true) == 3);      // records alone, or all of it
    CHECK(step(200, 600, true) == 2);
  }
}

int main(int argc, char** argv) {
  CHECK(argc == 2);
  const std::string name = argv[1];
  setup();
  if (name == "shares_of_gathers") shares_of_gathers();
  else if (name == "launches_of_appends") launches_of_appends();
  else CHECK(!"a scenario of that name");
  puts("ok");
}

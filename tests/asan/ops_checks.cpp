// Host-side checks, under AddressSanitizer, of the calls for queries and keys
// (jn_qk_norm_rope*) and for token heads (jn_tenant_tokens_*): argument checks,
// workspace sizes, plans and launch shapes over random sizes, as host_checks.cpp
// does it for the others.  Test infrastructure only.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "joynexus.h"

extern "C" long long jn_fake_launches;

namespace {

int g_checks = 0;

#define CHECK(cond)                                                                   \
  do {                                                                                \
    ++g_checks;                                                                       \
    if (!(cond)) {                                                                    \
      std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
      std::exit(2);                                                                   \
    }                                                                                 \
  } while (0)

struct Rng {
  uint64_t s;
  explicit Rng(uint64_t seed) : s(seed * 6364136223846793005ull + 1442695040888963407ull) {}
  uint32_t next() {
    s = s * 6364136223846793005ull + 1442695040888963407ull;
    return (uint32_t)(s >> 33);
  }
  int range(int lo, int hi) { return lo + (int)(next() % (uint32_t)(hi - lo + 1)); }
};

// Device addresses that nothing on the host reads: 256-byte aligned.
void* at(uintptr_t k) { return (void*)(uintptr_t)(0x100000000ull + k * 0x1000000000ull); }

void check_qk(jn_ctx* c) {
  Rng r(1);
  int32_t pos[4] = {};
  for (int t = 0; t < 400; ++t) {
    jn_qk_args a{};
    a.rows = t % 7 == 0 ? 0 : r.range(1, t % 5 == 0 ? 2000000 : 3000);
    a.n_heads = r.range(0, 20);
    a.n_kv_heads = r.range(a.n_heads == 0, 8);
    a.head_dim = 16 * r.range(1, 16);
    const int64_t width = (int64_t)(a.n_heads + a.n_kv_heads) * a.head_dim;
    a.ld_in = width + 8 * r.range(0, 9);
    a.ld_out = width + 8 * r.range(0, 9);
    a.ld_grad = width + 8 * r.range(0, 9);
    const bool norm = t % 3 != 0, rope = !norm || t % 2 == 0;
    a.gq = norm ? at(1) : nullptr;
    a.gk = norm ? at(2) : nullptr;
    a.eps = norm ? 1e-6f : 0.f;
    a.rope_theta = rope ? 1e4f : 0.f;
    a.pos = rope ? pos : nullptr;
    a.rope_axes = r.range(0, 4);
    a.rope_interleaved = t & 1;
    const int half = a.head_dim / 2;
    if (a.rope_axes > 1) {
      const int rest = half / (a.rope_axes + 1);
      a.rope_sections[0] = half - rest * (a.rope_axes - 1);
      for (int k = 1; k < a.rope_axes; ++k) a.rope_sections[k] = rest;
    }
    CHECK(jn_qk_norm_rope(c, &a, at(3), at(4)) == JN_OK);
    if (a.rows > 0) {
      CHECK(jn_qk_norm_rope(c, &a, nullptr, at(4)) == JN_EINVAL);
      CHECK(jn_qk_norm_rope(c, &a, at(3), (char*)at(4) + 2) == JN_EUNSUPPORTED);
      if (a.ld_in != a.ld_out) CHECK(jn_qk_norm_rope(c, &a, at(3), at(3)) == JN_EINVAL);
    }
    size_t ws = 1;
    CHECK(jn_qk_norm_rope_workspace_size(&a, &ws) == JN_OK);
    CHECK(ws % (2 * a.head_dim * 4) == 0 && (norm || ws == 0));
    float* dg[2] = {norm ? (float*)at(5) : nullptr, norm ? (float*)at(6) : nullptr};
    CHECK(jn_qk_norm_rope_bwd(c, &a, norm ? at(3) : nullptr, at(4), at(7), dg[0], dg[1], ws ? at(8) : nullptr, ws) == JN_OK);
    if (ws > 0) CHECK(jn_qk_norm_rope_bwd(c, &a, at(3), at(4), at(7), dg[0], dg[1], at(8), ws - 1) == JN_ENOSPACE);
    if (norm) CHECK(jn_qk_norm_rope_bwd(c, &a, at(3), at(4), at(7), nullptr, dg[1], at(8), ws) == JN_EINVAL);
    auto refused = [&](jn_status want, auto change) {
      jn_qk_args b = a;
      change(b);
      CHECK(jn_qk_norm_rope(c, &b, at(3), at(4)) == want);
      CHECK(jn_qk_norm_rope_bwd(c, &b, at(3), at(4), at(7), (float*)at(5), (float*)at(6), at(8), 1u << 30) == want);
    };
    refused(JN_EINVAL, [](jn_qk_args& b) { b.rows = -1; });
    refused(JN_ESHAPE, [](jn_qk_args& b) { b.rows = (1 << 26) - 3; });  // 2^32 threads in one launch
    refused(JN_EINVAL, [](jn_qk_args& b) { b.n_heads = b.n_kv_heads = 0; });
    refused(JN_EUNSUPPORTED, [](jn_qk_args& b) { b.head_dim += 8; });
    refused(JN_EUNSUPPORTED, [](jn_qk_args& b) { b.head_dim = 272; });
    refused(JN_EINVAL, [&](jn_qk_args& b) { b.ld_out = width - 8; });
    refused(JN_EUNSUPPORTED, [](jn_qk_args& b) { b.ld_out += 4; });
    refused(JN_EINVAL, [](jn_qk_args& b) { b.rope_axes = 5; });
    refused(JN_EINVAL, [](jn_qk_args& b) { b.rope_theta = -1.f; });
    if (a.rope_axes > 1) refused(JN_EINVAL, [](jn_qk_args& b) { b.rope_sections[0] += 1; });
    if (rope && a.rows > 0) refused(JN_EINVAL, [](jn_qk_args& b) { b.pos = nullptr; });
  }
  jn_qk_args a{};
  size_t ws;
  CHECK(jn_qk_norm_rope(c, nullptr, at(1), at(2)) == JN_EINVAL);
  CHECK(jn_qk_norm_rope(nullptr, &a, at(1), at(2)) == JN_EINVAL);
  CHECK(jn_qk_norm_rope_workspace_size(nullptr, &ws) == JN_EINVAL);
}

struct Group {
  std::vector<jn_token_head> h;
  std::vector<jn_token_io> io;
  std::vector<jn_token_pick> pick;
};

Group make(Rng& r, int G, int most_n, int most_v, bool f32) {
  Group g;
  for (int k = 0; k < G; ++k) {
    jn_token_head h{};
    h.vocab = r.range(1, most_v);
    h.W = at(10);
    jn_token_io io{};
    io.n = r.range(0, 9) == 0 ? 0 : r.range(1, most_n);
    io.dw_f32 = f32;
    io.rows = (const int32_t*)at(11);
    io.targets = (const int32_t*)at(12);
    io.logp = (float*)at(13);
    io.loss = (float*)at(14);
    io.dW = at(15);
    io.dh = r.range(0, 1) ? at(16) : nullptr;
    g.h.push_back(h);
    g.io.push_back(io);
    g.pick.push_back(jn_token_pick{io.n, 0, io.rows, (int32_t*)at(17), io.logp});
  }
  return g;
}

void run(jn_ctx* c, Group& g, int d) {
  const int G = (int)g.h.size();
  size_t ws = 0, dws = 0;
  CHECK(jn_tokens_workspace_size(d, g.h.data(), g.io.data(), G, &ws) == JN_OK);
  CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), 100, d, g.h.data(), g.io.data(), G, at(2), ws) == JN_OK);
  if (ws > 0) CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), 100, d, g.h.data(), g.io.data(), G, at(2), ws - 1) == JN_ENOSPACE);
  CHECK(jn_tokens_decode_workspace_size(d, g.h.data(), g.pick.data(), G, &dws) == JN_OK);
  CHECK(jn_tenant_tokens_decode(c, at(1), 100, d, g.h.data(), g.pick.data(), G, at(2), dws) == JN_OK);
  if (dws > 0) CHECK(jn_tenant_tokens_decode(c, at(1), 100, d, g.h.data(), g.pick.data(), G, at(2), dws - 1) == JN_ENOSPACE);
}

void check_tokens(jn_ctx* c) {
  Rng r(2);
  const int widths[] = {64, 128, 192, 768, 1024, 2048, 2176, 4096, 8192};
  for (int t = 0; t < 300; ++t) {
    const int d = widths[r.range(0, 8)];
    Group g = make(r, r.range(1, t % 10 == 0 ? 70 : 9), t % 3 == 0 ? 64 : 5000, t % 4 == 0 ? 300000 : 4000, t & 1);
    run(c, g, d);
  }
  // the limits: the longest lists, the largest vocabulary, many pieces, many tenants
  for (int k = 0; k < 5; ++k) {
    Group g = make(r, k == 3 ? 3000 : 1, 8, 100, false);
    if (k == 0) g.io[0].n = 1 << 20;
    if (k == 1) {
      g.h[0].vocab = 1 << 24;
      g.io[0].n = 16;
      g.io[0].dh = at(16);
    }
    if (k == 2) {
      g.h[0].vocab = 1 << 24;
      g.io[0].n = 5000;
      g.io[0].dh = at(16);
    }
    if (k == 4) {
      g.h[0].vocab = 300000;
      g.io[0].n = 1 << 20;
    }
    g.pick[0].n = g.io[0].n;
    run(c, g, k == 1 ? 8192 : 64);
  }
  Group g = make(r, 3, 500, 3000, false);
  for (auto& io : g.io) io.n = 70, io.dh = at(16);
  size_t ws = 0;
  CHECK(jn_tokens_workspace_size(256, g.h.data(), g.io.data(), 3, &ws) == JN_OK);
  auto refused = [&](jn_status want, int d, auto change) {
    Group b = g;
    change(b);
    CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), 100, d, b.h.data(), b.io.data(), 3, at(2), (size_t)1 << 40) == want);
    size_t n;
    CHECK(jn_tokens_workspace_size(d, b.h.data(), b.io.data(), 3, &n) == want);
  };
  const long long before = jn_fake_launches;
  refused(JN_EUNSUPPORTED, 96, [](Group&) {});
  refused(JN_EUNSUPPORTED, 0, [](Group&) {});
  refused(JN_EUNSUPPORTED, 8256, [](Group&) {});
  refused(JN_ESHAPE, 256, [](Group& b) { b.h[1].vocab = 0; });
  refused(JN_ESHAPE, 256, [](Group& b) { b.h[2].vocab = (1 << 24) + 1; });
  refused(JN_ESHAPE, 256, [](Group& b) { b.io[1].n = -1; });
  refused(JN_ESHAPE, 256, [](Group& b) { b.io[1].n = (1 << 20) + 1; });
  refused(JN_ESHAPE, 8192, [](Group& b) { b.io[1].n = 1 << 18; });
  refused(JN_EINVAL, 256, [](Group& b) { b.io[1].dw_f32 = 1; });
  refused(JN_EINVAL, 256, [](Group& b) { b.io[0].dw_f32 = 2; });
  refused(JN_EINVAL, 256, [](Group& b) { b.h[0].W = nullptr; });
  refused(JN_EUNSUPPORTED, 256, [](Group& b) { b.h[0].W = (const char*)b.h[0].W + 8; });
  refused(JN_EINVAL, 256, [](Group& b) { b.io[0].targets = nullptr; });
  refused(JN_EUNSUPPORTED, 256, [](Group& b) { b.io[0].dh = (char*)b.io[0].dh + 4; });
  CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), -1, 256, g.h.data(), g.io.data(), 3, at(2), ws) == JN_EINVAL);
  CHECK(jn_tenant_tokens_fwd_bwd(c, nullptr, 100, 256, g.h.data(), g.io.data(), 3, at(2), ws) == JN_EINVAL);
  CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), 100, 256, g.h.data(), g.io.data(), 3, (char*)at(2) + 16, ws) == JN_EUNSUPPORTED);
  CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), 100, 256, g.h.data(), g.io.data(), 0, at(2), ws) == JN_EINVAL);
  CHECK(jn_tenant_tokens_fwd_bwd(c, at(1), 100, 256, nullptr, g.io.data(), 3, at(2), ws) == JN_EINVAL);
  CHECK(jn_tenant_tokens_decode(nullptr, at(1), 100, 256, g.h.data(), g.pick.data(), 3, at(2), ws) == JN_EINVAL);
  CHECK(jn_fake_launches == before);  // nothing enqueued
}

}  // namespace

int main() {
  jn_ctx* c = nullptr;
  CHECK(jn_ctx_create(&c, nullptr) == JN_OK);
  check_qk(c);
  check_tokens(c);
  jn_ctx_destroy(c);
  std::printf("ops checks ok: %d checks, %lld launches\n", g_checks, jn_fake_launches);
  return 0;
}

// Host-side checks, under AddressSanitizer, of the calls over a paged cache (jn_kv_*,
// jn_backbone_extend) and of jn_tenant_tokens_verify: argument checks, workspace sizes
// and launch shapes over random sizes, as host_checks.cpp does it for the others. Test
// infrastructure only.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
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

struct Case {
  jn_kv_cache k{};
  jn_kv_batch b{};
  jn_kv_attn a{};
  jn_qk_args qk{};
};

Case make(Rng& r, int t) {
  Case c;
  const int hds[] = {32, 64, 128, 256};
  c.k.n_layers = r.range(1, 30);
  c.k.n_pages = r.range(1, 100000);
  c.k.page_size = 16 << r.range(0, 4);
  c.k.n_kv_heads = r.range(1, 16);
  c.k.head_dim = hds[r.range(0, 3)];
  const int64_t page = (int64_t)c.k.n_kv_heads * c.k.page_size * c.k.head_dim;
  if (t & 1) {
    c.k.ld_page = page + 8 * r.range(0, 5);
    c.k.ld_layer = c.k.ld_page * c.k.n_pages + 8 * r.range(0, 5);
  } else {
    c.k.ld_layer = page + 8 * r.range(0, 5);
    c.k.ld_page = c.k.ld_layer * c.k.n_layers;
  }
  c.k.k = at(1);
  c.k.v = at(2);
  const bool tree = t % 3 == 0;
  c.b.n_seqs = t % 11 == 0 ? 0 : r.range(1, t % 5 == 0 ? 65535 : 300);
  c.b.max_pages = r.range(1, (1 << 30) / c.k.page_size / (t % 4 == 0 ? 1 : 1000));
  c.b.rows = t % 13 == 0 ? 0 : r.range(1, t % 7 == 0 ? 2000000 : 5000);
  c.b.max_new = tree ? r.range(1, 256) : r.range(1, t % 9 == 0 ? 2000 : 40);
  c.b.whole = !tree && t % 2;
  c.b.pages = (const int32_t*)at(3);
  c.b.past = (const int32_t*)at(4);
  c.b.cu_rows = (const int32_t*)at(5);
  c.b.parents = tree ? (const int32_t*)at(6) : nullptr;
  const int group = r.range(1, 16);
  c.a.n_heads = c.k.n_kv_heads * group;
  c.a.scale = t % 2 ? 0.f : 0.3f;
  c.a.ld_q = (int64_t)c.a.n_heads * c.k.head_dim + 8 * r.range(0, 3);
  c.a.ld_out = (int64_t)c.a.n_heads * c.k.head_dim + 8 * r.range(0, 3);
  c.qk.rows = c.b.rows;
  c.qk.n_heads = r.range(0, 20);
  c.qk.n_kv_heads = c.k.n_kv_heads;
  c.qk.head_dim = c.k.head_dim;
  c.qk.ld_in = ((int64_t)c.qk.n_heads + 2 * c.qk.n_kv_heads) * c.k.head_dim + 8 * r.range(0, 3);
  c.qk.ld_out = (int64_t)c.qk.n_heads * c.k.head_dim + 8 * r.range(0, 3);
  if (t % 2) c.qk.gq = at(7), c.qk.gk = at(8), c.qk.eps = 1e-6f;
  if (t % 3) c.qk.rope_theta = 1e4f;
  return c;
}

void check_cache(jn_ctx* c) {
  Rng r(3);
  for (int t = 0; t < 600; ++t) {
    Case x = make(r, t);
    const bool none = x.b.rows == 0 || x.b.n_seqs == 0;
    void* const q = x.qk.n_heads > 0 ? at(10) : nullptr;
    long long before = jn_fake_launches;
    CHECK(jn_kv_append(c, &x.k, x.k.n_layers - 1, &x.b, &x.qk, at(9), q) == JN_OK);
    CHECK(jn_fake_launches - before == (none ? 0 : 1));
    size_t ws = 7;
    const jn_status st = jn_kv_attention_workspace_size(&x.k, &x.b, &x.a, &ws);
    before = jn_fake_launches;
    if (st == JN_OK) {
      CHECK((ws == 0) == none && ws < (size_t)160 << 20);
      CHECK(jn_kv_attention(c, &x.k, 0, &x.b, &x.a, at(10), at(11), ws ? at(12) : nullptr, ws) == JN_OK);
      CHECK(jn_fake_launches - before == (none ? 0 : 2));
      if (!none) {
        CHECK(jn_kv_attention(c, &x.k, 0, &x.b, &x.a, at(10), at(11), at(12), ws - 1) == JN_ENOSPACE);
        CHECK(jn_kv_attention(c, &x.k, 0, &x.b, &x.a, at(10), at(11), (char*)at(12) + 64, ws) == JN_EUNSUPPORTED);
        CHECK(jn_kv_attention(c, &x.k, 0, &x.b, &x.a, at(10), at(10), at(12), ws) == JN_EINVAL);
        CHECK(jn_kv_attention(c, &x.k, 0, &x.b, &x.a, (char*)at(10) + 8, at(11), at(12), ws) == JN_EUNSUPPORTED);
      }
    } else {
      CHECK(st == JN_ESHAPE);
      CHECK(jn_kv_attention(c, &x.k, 0, &x.b, &x.a, at(10), at(11), at(12), (size_t)1 << 40) == JN_ESHAPE);
    }
    const int32_t* const path = (const int32_t*)at(13);
    const int32_t* const count = (const int32_t*)at(14);
    before = jn_fake_launches;
    const jn_status sk = jn_kv_keep(c, &x.k, &x.b, path, r.range(1, 300), count, t % 3 ? (int32_t*)at(15) : nullptr);
    CHECK(sk == JN_OK || (sk == JN_ESHAPE && x.b.n_seqs > 1000));
    CHECK(jn_fake_launches - before == (sk == JN_OK && x.b.n_seqs > 0 ? 1 : 0));
    before = jn_fake_launches;
    if (sk == JN_OK && x.b.n_seqs > 0) {
      CHECK(jn_kv_keep(c, &x.k, &x.b, path, 4, count, (int32_t*)x.b.past) == JN_OK);
      CHECK(jn_fake_launches - before == 2);
    }
    before = jn_fake_launches;
    auto refused = [&](jn_status want, auto change) {
      Case y = x;
      change(y);
      CHECK(jn_kv_append(c, &y.k, 0, &y.b, &y.qk, at(9), q) == want);
      CHECK(jn_kv_keep(c, &y.k, &y.b, path, 4, count, nullptr) == want);
      size_t n;
      CHECK(jn_kv_attention_workspace_size(&y.k, &y.b, &y.a, &n) == want);
    };
    refused(JN_EUNSUPPORTED, [](Case& y) { y.k.page_size = 48; });
    refused(JN_EUNSUPPORTED, [](Case& y) { y.k.page_size = 8; });
    refused(JN_EUNSUPPORTED, [](Case& y) { y.k.head_dim = 24; });
    refused(JN_EINVAL, [](Case& y) { y.k.n_layers = 0; });
    refused(JN_EINVAL, [](Case& y) { y.k.ld_page -= y.k.n_layers == 1 || y.k.ld_layer > y.k.ld_page ? 1 << 24 : 8; });
    refused(JN_EINVAL, [](Case& y) { y.k.v = y.k.k; });
    refused(JN_EUNSUPPORTED, [](Case& y) { y.k.v = (char*)y.k.v + 2; });
    refused(JN_EINVAL, [](Case& y) { y.b.n_seqs = -1; });
    refused(JN_ESHAPE, [](Case& y) { y.b.n_seqs = 65536; });
    refused(JN_EINVAL, [](Case& y) { y.b.max_pages = 0; });
    refused(JN_ESHAPE, [](Case& y) { y.b.max_pages = (1 << 30) / y.k.page_size + 1; });
    refused(JN_EINVAL, [](Case& y) { y.b.max_new = 0; });
    refused(JN_EINVAL, [](Case& y) { y.b.whole = 3; });
    if (x.b.n_seqs > 0) refused(JN_EINVAL, [](Case& y) { y.b.cu_rows = nullptr; });
    refused(JN_EINVAL, [](Case& y) { y.b.parents = (const int32_t*)at(6), y.b.whole = 1; });
    refused(JN_EUNSUPPORTED, [](Case& y) { y.b.parents = (const int32_t*)at(6), y.b.whole = 0, y.b.max_new = 257; });
    auto row = [&](jn_status want, auto change) {
      Case y = x;
      change(y);
      CHECK(jn_kv_append(c, &y.k, 0, &y.b, &y.qk, at(9), at(10)) == want);
    };
    row(JN_EINVAL, [](Case& y) { y.qk.rows += 1; });
    row(JN_EINVAL, [](Case& y) { y.qk.n_kv_heads += 1; });
    row(JN_EINVAL, [](Case& y) { y.qk.ld_in = 8; });
    row(JN_EUNSUPPORTED, [](Case& y) { y.qk.ld_in += 4; });
    row(JN_EINVAL, [](Case& y) { y.qk.gq = y.qk.gq ? nullptr : at(7); });
    row(JN_EINVAL, [](Case& y) { y.qk.rope_theta = -1.f; });
    row(JN_EINVAL, [](Case& y) { y.qk.rope_theta = INFINITY; });
    row(JN_EINVAL, [](Case& y) { y.qk.rope_axes = 5; });
    CHECK(jn_kv_append(c, &x.k, x.k.n_layers, &x.b, &x.qk, at(9), q) == JN_ESHAPE);
    CHECK(jn_kv_append(c, &x.k, -1, &x.b, &x.qk, at(9), q) == JN_ESHAPE);
    if (!none) CHECK(jn_kv_append(c, &x.k, 0, &x.b, &x.qk, nullptr, q) == JN_EINVAL);
    CHECK(jn_kv_keep(c, &x.k, &x.b, path, 0, count, nullptr) == JN_EINVAL);
    CHECK(jn_kv_keep(c, &x.k, &x.b, path, (1 << 26) + 1, count, nullptr) == JN_ESHAPE);
    CHECK(jn_kv_keep(c, &x.k, &x.b, (const int32_t*)((char*)at(13) + 2), 4, count, nullptr) == JN_EINVAL);
    if (x.b.n_seqs > 0) CHECK(jn_kv_keep(c, &x.k, &x.b, nullptr, 4, count, nullptr) == JN_EINVAL);
    CHECK(jn_fake_launches == before);  // nothing enqueued
  }
  Case x = make(r, 1);
  CHECK(jn_kv_append(nullptr, &x.k, 0, &x.b, &x.qk, at(9), at(10)) == JN_EINVAL);
  CHECK(jn_kv_append(c, nullptr, 0, &x.b, &x.qk, at(9), at(10)) == JN_EINVAL);
  CHECK(jn_kv_append(c, &x.k, 0, nullptr, &x.qk, at(9), at(10)) == JN_EINVAL);
  CHECK(jn_kv_append(c, &x.k, 0, &x.b, nullptr, at(9), at(10)) == JN_EINVAL);
  CHECK(jn_kv_attention_workspace_size(&x.k, &x.b, &x.a, nullptr) == JN_EINVAL);
}

void check_extend(jn_ctx* c) {
  Rng r(5);
  for (int t = 0; t < 60; ++t) {
    const int d = 128 * r.range(1, 8), heads = d / (t % 2 ? 64 : 128) , layers = r.range(1, 4);
    std::vector<jn_layer> L(layers);
    for (auto& l : L) {
      l = jn_layer{at(1), at(2), at(3), t % 3 ? at(4) : nullptr, at(5), at(6), at(7), nullptr, nullptr};
      if (t % 2) l.gq = at(8), l.gk = at(9);
    }
    jn_backbone bb{};
    bb.n_layers = layers;
    bb.d = d;
    bb.n_heads = heads;
    bb.ffn = 128 * r.range(1, 10);
    bb.eps = 1e-6f;
    bb.layers = L.data();
    bb.gf = at(10);
    bb.causal = t % 4 != 0;
    bb.rope_theta = t % 5 ? 1e4f : 0.f;
    Case x = make(r, t % 4 != 0 && t % 3 == 0 ? 3 * t : 3 * t + 2);
    x.k.n_layers = layers;
    x.k.n_kv_heads = heads;
    x.k.head_dim = d / heads;
    x.k.ld_page = (int64_t)heads * x.k.page_size * x.k.head_dim;
    x.k.ld_layer = x.k.ld_page * x.k.n_pages;
    x.b.n_seqs = r.range(1, 50);
    x.b.rows = t % 7 ? r.range(1, 3000) : 0;
    if (!bb.causal) x.b.parents = nullptr;
    x.b.whole = !bb.causal;
    size_t ws = 0;
    CHECK(jn_backbone_extend_workspace_size(&bb, &x.k, &x.b, &ws) == JN_OK);
    const long long before = jn_fake_launches;
    CHECK(jn_backbone_extend(c, &bb, &x.k, &x.b, at(11), at(12), at(13), ws) == JN_OK);
    CHECK((jn_fake_launches > before) == (x.b.rows > 0));
    const long long after = jn_fake_launches;
    if (x.b.rows > 0) {
      CHECK(jn_backbone_extend(c, &bb, &x.k, &x.b, at(11), at(12), at(13), ws - 1) == JN_ENOSPACE);
      CHECK(jn_backbone_extend(c, &bb, &x.k, &x.b, nullptr, at(12), at(13), ws) == JN_EINVAL);
      CHECK(jn_backbone_extend(c, &bb, &x.k, &x.b, at(11), at(12), (char*)at(13) + 16, ws) == JN_EUNSUPPORTED);
    }
    x.k.n_layers += 1;
    CHECK(jn_backbone_extend(c, &bb, &x.k, &x.b, at(11), at(12), at(13), ws) != JN_OK);
    x.k.n_layers -= 1;
    bb.causal = !bb.causal;
    CHECK(jn_backbone_extend(c, &bb, &x.k, &x.b, at(11), at(12), at(13), ws) == JN_EINVAL);
    CHECK(jn_fake_launches == after);
  }
}

void check_verify(jn_ctx* c) {
  Rng r(9);
  for (int t = 0; t < 300; ++t) {
    const int G = r.range(1, t % 6 == 0 ? 70 : 4);
    std::vector<jn_token_verify> v(G);
    for (auto& x : v) {
      x = jn_token_verify{};
      x.n_trees = r.range(0, t % 5 == 0 ? 900 : 20);
      x.n = r.range(0, 30) * x.n_trees;
      x.vocab = r.range(1, t % 4 == 0 ? 1 << 20 : 3000);
      x.max_path = r.range(1, 300);
      x.ld_p = x.vocab + r.range(0, 3);
      x.ld_q = x.vocab + r.range(0, 3);
      x.cu_nodes = (const int32_t*)at(1);
      x.parents = r.range(0, 1) ? (const int32_t*)at(2) : nullptr;
      x.tokens = (const int32_t*)at(3);
      if (r.range(0, 3)) {
        x.p = (const float*)at(4);
        x.q = r.range(0, 1) ? (const float*)at(5) : nullptr;
        x.u = (const float*)at(6);
        x.r = (const float*)at(7);
      } else {
        x.greedy = (const int32_t*)at(8);
      }
      x.path = (int32_t*)at(9);
      x.n_path = (int32_t*)at(10);
      x.next = (int32_t*)at(11);
    }
    size_t ws = 0;
    CHECK(jn_tokens_verify_workspace_size(v.data(), G, &ws) == JN_OK);
    CHECK(jn_tenant_tokens_verify(c, v.data(), G, ws ? at(12) : nullptr, ws) == JN_OK);
    const long long before = jn_fake_launches;
    if (ws > 0) {
      CHECK(jn_tenant_tokens_verify(c, v.data(), G, at(12), ws - 1) == JN_ENOSPACE);
      CHECK(jn_tenant_tokens_verify(c, v.data(), G, (char*)at(12) + 4, ws) == JN_EUNSUPPORTED);
    }
    auto refused = [&](jn_status want, auto change) {
      std::vector<jn_token_verify> w = v;
      w[0].n_trees = 3;
      w[0].n = 9;
      change(w[0]);
      CHECK(jn_tenant_tokens_verify(c, w.data(), G, at(12), (size_t)1 << 40) == want);
    };
    refused(JN_EINVAL, [](jn_token_verify& x) { x.n = -1; });
    refused(JN_EINVAL, [](jn_token_verify& x) { x.max_path = 0; });
    refused(JN_ESHAPE, [](jn_token_verify& x) { x.vocab = 0; });
    refused(JN_ESHAPE, [](jn_token_verify& x) { x.n_trees = 70000; });
    refused(JN_ESHAPE, [](jn_token_verify& x) { x.n = 1 << 30, x.vocab = 1 << 20, x.ld_p = x.ld_q = 1 << 20; });
    refused(JN_EINVAL, [](jn_token_verify& x) { x.tokens = nullptr; });
    refused(JN_EINVAL, [](jn_token_verify& x) { x.p = x.p ? nullptr : (const float*)at(4); });
    refused(JN_EINVAL, [](jn_token_verify& x) { x.path = (int32_t*)((char*)at(9) + 1); });
    CHECK(jn_tenant_tokens_verify(c, v.data(), 0, at(12), ws) == JN_EINVAL);
    CHECK(jn_tenant_tokens_verify(c, nullptr, G, at(12), ws) == JN_EINVAL);
    CHECK(jn_tenant_tokens_verify(nullptr, v.data(), G, at(12), ws) == JN_EINVAL);
    CHECK(jn_fake_launches == before);
  }
}

}  // namespace

int main() {
  jn_ctx* c = nullptr;
  CHECK(jn_ctx_create(&c, nullptr) == JN_OK);
  check_cache(c);
  check_extend(c);
  check_verify(c);
  jn_ctx_destroy(c);
  std::printf("kv checks ok: %d checks, %lld launches\n", g_checks, jn_fake_launches);
  return 0;
}

"""CPU checks of the C structs of the calls over a cache, their workspaces and refusals, and the binding's own checks."""
import ctypes as C
import os
import subprocess

import pytest
import torch  # before the library: both then share one HIP runtime

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, I32 = torch.bfloat16, torch.int32


def test_struct_layout_matches_c(tmp_path, lib):
    from paper_2607_16074_amd import _abi
    structs = {n: getattr(_abi, n) for n in ("jn_kv_cache", "jn_kv_batch", "jn_kv_attn", "jn_token_verify")}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "joynexus.h"', "int main(void){"]
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, cls in structs.items():
        assert int(got[name]) == C.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, f"{name}.{f}"


def parts(lib, layers=1, pages=4, kv=2, page=16, hd=64, seqs=2, per=2, rows=5, new=3, tree=False):
    k, v = (torch.zeros(layers, pages, kv, page, hd, dtype=BF16) for _ in range(2))
    i = lambda *n: torch.zeros(n, dtype=I32)  # noqa: E731
    return (lib.KVCache(k, v), lib.KVBatch(i(seqs, per), i(seqs), i(seqs + 1), rows, new, i(rows) if tree else None))


def refused(lib, status, change, heads=4, **kw):
    cache, b = parts(lib, **kw)
    change(cache.struct, b.struct)
    with pytest.raises(lib.JNError) as e:
        lib.jn_kv_attention_workspace_size(cache, b, heads)
    assert str(e.value).startswith(status), e.value


def test_refusals_before_anything_runs(lib):
    n = lib.jn_kv_attention_workspace_size(*parts(lib), 4)
    assert 0 <= n < 1 << 26
    set_ = lambda **f: lambda c, b: [setattr(c if hasattr(c, k) else b, k, x) for k, x in f.items()]  # noqa: E731
    refused(lib, "JN_EUNSUPPORTED", set_(page_size=24))
    refused(lib, "JN_EUNSUPPORTED", set_(page_size=512))
    refused(lib, "JN_EUNSUPPORTED", set_(head_dim=40))
    refused(lib, "JN_EUNSUPPORTED", set_(head_dim=48))  # of attention only
    refused(lib, "JN_EINVAL", set_(n_pages=0))
    refused(lib, "JN_EINVAL", set_(ld_page=8))
    refused(lib, "JN_EUNSUPPORTED", set_(ld_page=2 * 16 * 64 + 4))
    refused(lib, "JN_EINVAL", set_(ld_page=1 << 62))
    refused(lib, "JN_EINVAL", set_(ld_layer=2 * 16 * 64), layers=2)
    refused(lib, "JN_EINVAL", set_(k=None))
    refused(lib, "JN_EUNSUPPORTED", lambda c, b: setattr(c, "k", c.k + 8))
    refused(lib, "JN_EINVAL", lambda c, b: setattr(c, "k", c.v))
    refused(lib, "JN_EINVAL", set_(rows=-1))
    refused(lib, "JN_EINVAL", set_(max_new=0))
    refused(lib, "JN_EINVAL", set_(whole=2))
    refused(lib, "JN_ESHAPE", set_(n_seqs=65536))
    refused(lib, "JN_ESHAPE", set_(rows=(1 << 26) - 3))
    refused(lib, "JN_ESHAPE", set_(max_pages=(1 << 26) + 1))
    refused(lib, "JN_EINVAL", set_(past=None))
    refused(lib, "JN_EINVAL", lambda c, b: setattr(b, "cu_rows", b.cu_rows + 2))
    refused(lib, "JN_EINVAL", set_(whole=1), tree=True)
    refused(lib, "JN_EUNSUPPORTED", set_(max_new=257), tree=True)
    refused(lib, "JN_EINVAL", set_(), heads=3)
    refused(lib, "JN_EINVAL", set_(), heads=0)
    refused(lib, "JN_ESHAPE", set_(max_new=1 << 22, rows=1 << 22, n_seqs=60000), heads=64)


def test_sizes_beyond_a_batch_are_taken(lib):
    """What a batch may hold at most: 256 sequences in buffers for 75,529 rows, each allowed all of them."""
    cache, b = parts(lib, kv=4, seqs=256, rows=75529, new=75529)
    assert 0 < lib.jn_kv_attention_workspace_size(cache, b, 16) < 1 << 28
    refused(lib, "JN_ESHAPE", lambda c, x: setattr(x, "max_new", x.rows), heads=4096, kv=2, rows=(1 << 15) + 1)


def test_the_cache_and_batch_binding_checks_types(lib):
    k = torch.zeros(1, 4, 2, 16, 64, dtype=BF16)
    for bad in ((k.float(), k.float()), (k, k[:, :3]), (k[0], k[0]), (k[..., ::2], k[..., ::2]), (k, k.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(TypeError):
            lib.KVCache(*bad)
    i = lambda *n: torch.zeros(n, dtype=I32)  # noqa: E731
    for bad in ((i(2), i(2), i(3)), (i(2, 2), i(3), i(3)), (i(2, 2), i(2), i(2)), (i(2, 2).long(), i(2), i(3))):
        with pytest.raises(TypeError):
            lib.KVBatch(*bad, 4, 2)
    with pytest.raises(TypeError):
        lib.KVBatch(i(2, 2), i(2), i(3), 4, 2, i(3))


def tree(lib, n=4, trees=2, width=9, **kw):
    i = lambda *s: torch.zeros(s, dtype=I32)  # noqa: E731
    a = dict(p=torch.zeros(n, width), u=torch.zeros(n), r=torch.zeros(trees))
    a.update(kw)
    return lib.TokenVerify(i(trees + 1), i(n), i(trees, 3), i(trees), i(trees), **a)


def test_refusals_of_a_verification(lib):
    lib.jn_tokens_verify_workspace_size([tree(lib), tree(lib, q=torch.zeros(4, 9))])
    lib.jn_tokens_verify_workspace_size([tree(lib, p=None, u=None, r=None, greedy=torch.zeros(4, dtype=I32), vocab=9)])

    def bad(status, io, **f):
        for k, x in f.items():
            setattr(io.struct, k, x)
        with pytest.raises(lib.JNError) as e:
            lib.jn_tokens_verify_workspace_size([tree(lib), io])
        assert str(e.value).startswith(status), e.value

    bad("JN_EINVAL", tree(lib), u=None)
    bad("JN_EINVAL", tree(lib), r=None)
    bad("JN_EINVAL", tree(lib), p=None)
    bad("JN_EINVAL", tree(lib), ld_p=8)
    bad("JN_EINVAL", tree(lib, q=torch.zeros(4, 9)), ld_q=8)
    bad("JN_EINVAL", tree(lib), max_path=0)
    bad("JN_EINVAL", tree(lib), n_trees=-1)
    bad("JN_EINVAL", tree(lib), next=None)
    bad("JN_ESHAPE", tree(lib), vocab=(1 << 24) + 1, ld_p=1 << 25)
    bad("JN_ESHAPE", tree(lib), n=1 << 30, vocab=1 << 12, ld_p=1 << 12)
    bad("JN_EINVAL", tree(lib, greedy=torch.zeros(4, dtype=I32)))
    with pytest.raises(lib.JNError):
        lib.jn_tokens_verify_workspace_size([])
    for kw in (dict(p=torch.zeros(3, 9)), dict(p=torch.zeros(4, 9).double()), dict(u=torch.zeros(3)), dict(q=torch.zeros(4, 8)),
               dict(p=None), dict(vocab=10), dict(p=torch.zeros(1, 9).expand(4, 9)), dict(parents=torch.zeros(3, dtype=I32))):
        with pytest.raises(TypeError):
            tree(lib, **kw)

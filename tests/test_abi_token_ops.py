"""CPU checks of the C structs of the calls for queries and keys and for token heads, and of the binding's own checks."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch  # before the library: both then share one HIP runtime

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layout_matches_c(tmp_path, lib):
    from paper_2607_16074_amd import _abi
    structs = {n: getattr(_abi, n) for n in ("jn_qk_args", "jn_token_head", "jn_token_io", "jn_token_pick", "jn_layer",
                                             "jn_backbone")}
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


def test_sizes_of_workspaces(lib):
    """Sizes come from the host alone; a larger piece budget than JN_TOKEN_PIECE_BYTES is never asked for by much."""
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    small, big = lib.TokenHead(bf(100, 64)), lib.TokenHead(bf(120001, 64))
    io = lib.TokenIO(i32(9), i32(9), torch.zeros(9), torch.zeros(1), bf(100, 64))
    assert 0 < lib.jn_tokens_workspace_size([small], [io]) < 1 << 20
    many = lib.TokenIO(i32(20000), i32(20000), torch.zeros(20000), torch.zeros(1), bf(120001, 64))
    n = lib.jn_tokens_workspace_size([big], [many])
    # one piece (up to a whole round of tiles more: 65,536 columns here would be; 256 it is below a round), 8 bytes a
    # part of 128 columns, and the rows
    assert n < (1 << 30) * 1.05 + 8 * 20000 * (120001 / 64 + 8) + 20000 * 64 * 8 + (1 << 20)
    # tenants of few rows keep whole logits only up to a piece: 40 of them, 64 rows of 120,001 each
    few = [lib.TokenIO(i32(64), i32(64), torch.zeros(64), torch.zeros(1), big.W, bf(64, 64)) for _ in range(40)]
    assert lib.jn_tokens_workspace_size([big] * 20, few[:20]) < (1 << 30) * 1.05
    assert lib.jn_tokens_workspace_size([big] * 40, few) < (1 << 30) * 1.35
    pick = lib.TokenPick(i32(3), i32(3), torch.zeros(3))
    assert lib.jn_tokens_decode_workspace_size([small], [pick]) < 1 << 16
    with pytest.raises(lib.JNError):
        lib.jn_tokens_workspace_size([lib.TokenHead(bf(100, 96))], [lib.TokenIO(i32(1), i32(1), torch.zeros(1), torch.zeros(1), bf(100, 96))])
    qk = lib.QKNormRope(4, 2, 64, 1e-6, bf(64), bf(64), 1e4)
    assert lib.jn_qk_norm_rope_workspace_size(qk, 0) == 0 and lib.jn_qk_norm_rope_workspace_size(qk, 10 ** 6) == 1024 * 2 * 64 * 4
    assert lib.jn_qk_norm_rope_workspace_size(lib.QKNormRope(4, 2, 64, theta=1e4), 1000) == 0


def test_the_binding_checks_types(lib):
    bf = torch.zeros(8, 64, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    for bad in (torch.zeros(8, 64), bf[:, ::2], bf[0]):
        with pytest.raises(TypeError):
            lib.TokenHead(bad)
    f = torch.zeros(3)
    with pytest.raises(TypeError):
        lib.TokenIO(i, i.long(), f, f[:1], bf)
    with pytest.raises(TypeError):
        lib.TokenIO(i, i, f[:2], f[:1], bf)
    with pytest.raises(TypeError):
        lib.TokenIO(i, i, f, f[:1], bf, dh=torch.zeros(3, 63, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        lib.TokenPick(i, f, f)
    with pytest.raises(TypeError):
        lib._token_arrays([lib.TokenHead(bf)], [lib.TokenIO(i, i, f, f[:1], bf[:4])], lib.TokenIO)
    with pytest.raises(ValueError):
        lib.QKNormRope(1, 1, 64, sections=[8] * 5)
    qk = lib.QKNormRope(1, 0, 64, theta=1e4)
    with pytest.raises(TypeError):
        qk.at(8, torch.zeros(8, dtype=torch.int64), bf, bf)
    with pytest.raises(TypeError):
        qk.at(8, torch.zeros(7, dtype=torch.int32), bf, bf)
    with pytest.raises(TypeError):
        qk.at(8, torch.zeros(8, dtype=torch.int32), bf[:, :32], bf)
    a = qk.at(8, torch.zeros(8, dtype=torch.int32), bf, torch.zeros(8, 80, dtype=torch.bfloat16)[:, :64])
    assert (a.ld_in, a.ld_out, a.rows) == (64, 80, 8)


def test_rows_of_targets_and_positions(lib):
    from paper_2607_16074_amd import step
    lens, ten = [[3, 5], [4]], [1, 0]
    reqs = [lib.Request(t, 4096, np.array(n, np.int32), 6) for t, n in zip(ten, lens)]
    maps = lib.jn_pack_maps_host(reqs, [lib.Tenant(7, 64)] * 2, 64, 4)
    assert maps["cu_seqlens"].tolist() == [0, 4, 12, 16]
    got = step.target_rows(maps, 1, np.array([0, 1, 1, 2, 0, -1]), np.array([2, 0, 4, 0, 3, 0]))
    assert got.tolist() == [2, 4, 8, -1, -1, -1] and got.dtype == np.int32
    assert step.target_rows(maps, 0, np.array([0]), np.array([3])).tolist() == [15]
    pos = [np.arange(2 * 6 * 2).reshape(2, 6, 2), 100 + np.arange(12).reshape(1, 6, 2)]
    p = step.packed_positions(reqs, maps, pos)
    assert p.shape == (maps["T"], 2) and p[2].tolist() == [4, 5] and p[3].tolist() == [0, 0] and p[4].tolist() == [12, 13]
    assert p[12].tolist() == [100, 101]

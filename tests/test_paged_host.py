"""The calls of the paged cache on the host: struct layouts, defaults, workspace sizes, rotary frequencies and every
refusal.  Nothing here reaches a launch."""
import ctypes
import json
import math
import os
import subprocess

import pytest
import torch

from paper_2607_16213_amd import selkv as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EDTYPE, EUNSUPPORTED, EALIGN, EWORKSPACE, EHIP = 1, 2, 3, 4, 5, 6
FAKE, NULL = 0x10000, None
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers are only passed where no GPU exists")


def cache(page=64, n_pages=100, columns=8, **kw):
    c = S.PagedStruct()
    S.lib.selkv_paged_init(c)
    c.page, c.n_pages, c.columns = page, n_pages, columns
    c.K = c.V = c.table = c.bias = FAKE
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(data=FAKE, sb=1024, sn=1024, sh=128):
    return S.RowsStruct(data, sb, sn, sh)


def rope(**kw):
    r = S.RopeStruct()
    S.lib.selkv_rope_init(r)
    r.rot_dim, r.freq = 64, FAKE
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def append(p, c, k=rows(), v=rows(), bias=NULL, rp=NULL, positions=NULL, q=NULL, q_out=NULL, n=8, cache_len=64,
           lens=NULL, counts=NULL):
    return S.lib.selkv_paged_append(p, c, k, v, bias, rp, positions, q, q_out, n, cache_len, lens, counts, None)


def attn(p, c, q=FAKE, parent=NULL, n=8, cache_len=64, lens=NULL, counts=NULL, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return S.lib.selkv_tree_attn(p, c, q, parent, n, cache_len, lens, counts, out, ws, ws_bytes, None)


def keep(p, c, path=FAKE, n_path=FAKE, n=8, cache_len=64, lens=NULL):
    return S.lib.selkv_paged_keep(p, c, path, n_path, n, cache_len, lens, None)


def verify(batch=2, n=8, vocab=1000, dtype=0, tokens=FAKE, parent=NULL, target=FAKE, draft=NULL, u=FAKE, counts=NULL,
           path=FAKE, n_path=FAKE, nxt=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return S.lib.selkv_tree_verify(batch, n, vocab, dtype, tokens, parent, target, draft, u, counts, path, n_path, nxt,
                                   ws, ws_bytes, None)


@pytest.mark.parametrize("name,struct", [("selkv_paged", S.PagedStruct), ("selkv_rows", S.RowsStruct),
                                         ("selkv_rope", S.RopeStruct)])
def test_struct_layouts(tmp_path, name, struct):
    fields = [f for f, _ in struct._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "selkv.h"', "int main(void){",
           f'printf("{{\\"size\\": %zu", sizeof({name}));']
    src += [f'printf(", \\"{f}\\": %zu", offsetof({name}, {f}));' for f in fields]
    (tmp_path / "l.c").write_text("\n".join(src + ['printf("}\\n"); return 0; }']))
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", f"-I{ROOT}/include", "-I/opt/rocm/include", str(tmp_path / "l.c"),
                    "-o", str(tmp_path / "l")], check=True)
    layout = json.loads(subprocess.run([str(tmp_path / "l")], capture_output=True, text=True).stdout)
    assert layout["size"] == ctypes.sizeof(struct)
    assert all(layout[f] == getattr(struct, f).offset for f in fields)


def test_defaults():
    c, r = S.PagedStruct(), S.RopeStruct()
    S.lib.selkv_paged_init(c)
    S.lib.selkv_rope_init(r)
    assert (c.struct_size, c.page, c.n_pages, c.columns, c.K) == (ctypes.sizeof(c), 64, 0, 0, None)
    assert (r.struct_size, r.layout, r.rot_dim, r.scale, r.freq) == (ctypes.sizeof(r), 0, 0, 1.0, None)
    S.lib.selkv_paged_init(None)
    S.lib.selkv_rope_init(None)


@no_gpu
@pytest.mark.parametrize("call", [append, attn, keep])
def test_refusals_of_every_cache_call(call):
    p = S.params()
    assert call(p, cache()) == EHIP                            # valid: it gets as far as the launch
    assert call(p, cache(bias=None)) == EHIP
    assert call(None, cache()) == EINVAL and call(p, None) == EINVAL
    assert call(S.params(struct_size=4), cache()) == EINVAL
    assert call(p, cache(struct_size=4)) == EINVAL
    assert call(S.params(kv_dtype=7), cache()) == EDTYPE
    assert call(S.params(batch=0), cache()) == EINVAL
    assert call(S.params(n_heads_kv=0), cache()) == EINVAL
    assert call(S.params(head_dim=96), cache()) == EUNSUPPORTED
    assert call(S.params(batch=8192), cache()) == EUNSUPPORTED      # 65536 KV heads
    for page in (0, 8, 48, 512, -64):
        assert call(p, cache(page=page)) == EUNSUPPORTED
    assert call(p, cache(columns=0)) == EINVAL and call(p, cache(n_pages=0)) == EINVAL
    assert call(p, cache(columns=(1 << 22) + 1)) == EUNSUPPORTED and call(p, cache(n_pages=(1 << 22) + 1)) == EUNSUPPORTED
    assert call(p, cache(columns=1 << 22)) == EHIP and call(p, cache(n_pages=1 << 22)) == EHIP
    for f in ("K", "V", "table"):
        assert call(p, cache(**{f: None})) == EINVAL
    for f in ("K", "V", "bias"):
        assert call(p, cache(**{f: FAKE + 8})) == EALIGN
    assert call(p, cache(table=FAKE + 2)) == EALIGN and call(p, cache(table=FAKE + 4)) == EHIP
    assert call(p, cache(), n=0) == EINVAL and call(p, cache(), n=-1) == EINVAL
    assert call(p, cache(), cache_len=-1) == EINVAL and call(p, cache(), cache_len=513) == EINVAL
    assert call(p, cache(), cache_len=504) == EHIP and call(p, cache(), cache_len=505) == EINVAL    # no room
    assert call(p, cache(), cache_len=512, lens=FAKE) == EHIP        # the lengths are on the device
    assert call(p, cache(), lens=FAKE + 2) == EALIGN
    assert call(p, cache(), n=513, lens=FAKE) != EHIP


@no_gpu
def test_refusals_of_append():
    p, c = S.params(), cache()
    for bad in (rows(data=None), rows(sb=-8), rows(sn=-8), rows(sh=-8), NULL):
        assert append(p, c, k=bad) == EINVAL and append(p, c, v=bad) == EINVAL
    for bad in (rows(data=FAKE + 8), rows(sb=4), rows(sn=4), rows(sh=4)):
        assert append(p, c, k=bad) == EALIGN and append(p, c, v=bad) == EALIGN
    assert append(S.params(kv_dtype="fp32"), c, k=rows(sn=4)) == EHIP
    assert append(p, c, k=rows(sn=0)) == EHIP
    assert append(p, c, bias=FAKE) == EHIP and append(p, cache(bias=None), bias=FAKE) == EINVAL
    assert append(p, c, bias=FAKE + 2) == EALIGN and append(p, c, positions=FAKE + 2) == EALIGN
    assert append(p, c, counts=FAKE + 1) == EALIGN and append(p, c, n=512, cache_len=0) == EHIP
    assert append(p, c, cache_len=512, counts=FAKE) == EHIP
    assert append(p, c, rp=rope()) == EHIP
    for bad, why in ((dict(struct_size=8), EINVAL), (dict(layout=2), EINVAL), (dict(rot_dim=0), EINVAL),
                     (dict(rot_dim=144), EINVAL), (dict(rot_dim=24), EUNSUPPORTED), (dict(scale=float("nan")), EINVAL),
                     (dict(scale=float("inf")), EINVAL), (dict(freq=None), EINVAL), (dict(freq=FAKE + 4), EALIGN)):
        assert append(p, c, rp=rope(**bad)) == why, bad
    assert append(p, c, rp=rope(rot_dim=128)) == EHIP and append(S.params(head_dim=64), c, rp=rope(rot_dim=80)) == EINVAL
    assert append(p, c, rp=rope(), q=rows(), q_out=FAKE) == EHIP
    assert append(p, c, q=rows(), q_out=FAKE) == EINVAL              # nothing to turn them by
    assert append(p, c, rp=rope(), q=rows()) == EINVAL and append(p, c, rp=rope(), q=rows(), q_out=FAKE + 8) == EALIGN
    assert append(p, c, rp=rope(), q=rows(sh=4), q_out=FAKE) == EALIGN
    assert append(S.params(group=0), c, rp=rope(), q=rows(), q_out=FAKE) == EINVAL
    assert append(S.params(group=65), c, rp=rope(), q=rows(), q_out=FAKE) == EUNSUPPORTED
    assert append(S.params(group=65), c) == EHIP                     # without queries the group is not used


@no_gpu
def test_refusals_of_the_tree_calls():
    p, c = S.params(), cache()
    big = cache(columns=4096)
    assert attn(S.params(group=0), c) == EINVAL and attn(S.params(group=65), c) == EUNSUPPORTED
    assert attn(S.params(group=64), c, n=64) == EHIP
    for scale in (-1.0, float("nan"), float("inf")):
        assert attn(S.params(scale=scale), c) == EINVAL
    assert attn(p, c, n=65) == EUNSUPPORTED and keep(p, c, n=65) == EUNSUPPORTED
    assert attn(p, c, q=NULL) == EINVAL and attn(p, c, out=NULL) == EINVAL
    assert attn(p, c, q=FAKE + 8) == EALIGN and attn(p, c, out=FAKE + 8) == EALIGN and attn(p, c, parent=FAKE + 2) == EALIGN
    assert attn(p, c, counts=FAKE + 2) == EALIGN and attn(p, c, cache_len=512, counts=FAKE) == EHIP
    assert attn(p, big, cache_len=100000, ws=NULL) == EWORKSPACE
    assert attn(p, big, cache_len=100000, ws_bytes=64) == EWORKSPACE
    assert attn(p, big, cache_len=100000, ws=FAKE + 16) == EALIGN
    assert keep(p, c, path=NULL) == EINVAL and keep(p, c, n_path=NULL) == EINVAL
    assert keep(p, c, path=FAKE + 2) == EALIGN and keep(p, c, n_path=FAKE + 2) == EALIGN
    n = ctypes.c_size_t()
    f = S.lib.selkv_tree_workspace_size
    assert f(p, c, 8, None) == EINVAL and f(p, None, 8, ctypes.byref(n)) == EINVAL and f(None, c, 8, ctypes.byref(n)) == EINVAL
    assert f(p, c, 65, ctypes.byref(n)) == EUNSUPPORTED and f(p, c, 0, ctypes.byref(n)) == EINVAL
    assert f(p, cache(K=None, V=None, table=None, n_pages=0), 8, ctypes.byref(n)) == 0


@no_gpu
def test_refusals_of_verify():
    assert verify() == EHIP and verify(parent=FAKE, draft=FAKE, counts=FAKE, dtype=1) == EHIP
    assert verify(dtype=2) == EDTYPE
    for bad in (dict(batch=0), dict(n=0), dict(vocab=0), dict(tokens=NULL), dict(target=NULL), dict(u=NULL),
                dict(path=NULL), dict(n_path=NULL), dict(nxt=NULL)):
        assert verify(**bad) == EINVAL, bad
    for bad in (dict(batch=65536), dict(n=65), dict(vocab=(1 << 21) + 1)):
        assert verify(**bad) == EUNSUPPORTED, bad
    for bad in ("tokens", "parent", "u", "counts", "path", "n_path", "nxt"):
        assert verify(**{bad: FAKE + 2}) == EALIGN, bad
    assert verify(target=FAKE + 8) == EALIGN and verify(draft=FAKE + 8) == EALIGN
    assert verify(batch=65535, n=64, vocab=1 << 21) == EHIP
    n = ctypes.c_size_t()
    f = S.lib.selkv_tree_verify_workspace_size
    assert f(1, 1, 1, None) == EINVAL and f(0, 1, 1, ctypes.byref(n)) == EINVAL and f(1, 65, 1, ctypes.byref(n)) == EUNSUPPORTED


@no_gpu
def test_the_workspaces_pass_at_every_length_and_count():
    """The calls then fail at the launch, there being no GPU, never with EWORKSPACE."""
    need = ctypes.c_size_t()
    for (B, H, G, d, page, columns, n, dtype) in [(1, 8, 4, 128, 64, 600, 64, "bf16"), (1, 2, 2, 64, 16, 50, 7, "fp32"),
                                                  (3, 5, 3, 128, 32, 300, 26, "fp32"), (1, 1, 64, 64, 256, 40, 64, "bf16"),
                                                  (128, 8, 8, 128, 64, 1600, 33, "bf16"), (1, 1, 1, 128, 256, 1 << 20, 64, "bf16")]:
        p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype)
        c = cache(page=page, columns=columns)
        assert S.lib.selkv_tree_workspace_size(p, c, n, ctypes.byref(need)) == 0
        cap = page * columns
        for length in [x for x in (0, 1, 100, 129, 1000, 5000, cap // 3, cap // 2, cap - n) if x <= cap - n]:
            for k in range(1, n + 1):
                for lens in (NULL, FAKE):
                    assert attn(p, c, n=k, cache_len=length, lens=lens, ws_bytes=need.value) == EHIP, (B, H, length, k)
        assert attn(p, c, n=n, cache_len=cap, lens=FAKE, ws_bytes=need.value) == EHIP
    for (B, n, vocab) in [(1, 1, 1), (3, 64, 151936), (32, 8, 1 << 21), (65535, 2, 4)]:
        assert S.lib.selkv_tree_verify_workspace_size(B, n, vocab, ctypes.byref(need)) == 0
        for k in {1, n // 2 + 1, n}:
            assert verify(batch=B, n=k, vocab=vocab, ws_bytes=need.value) == EHIP


def test_refusals_of_the_binding():
    p = S.params(batch=1, n_heads_kv=2, group=2, head_dim=64, kv_dtype="fp32")
    z = torch.zeros
    with pytest.raises(ValueError, match="page"):
        S.PagedCache(p, 4, 4, "cpu", page=48)
    with pytest.raises(ValueError, match="device tensor"):      # host memory
        S.PagedCache(p, 4, 4, "cpu")
    with pytest.raises(ValueError, match="four"):
        S.PagedCache.over(p, z(2, 64, 64), z(1), z(1, 1))
    with pytest.raises(ValueError, match="there must be some"):
        S.PagedCache.over(p, z(4, 2, 48, 64), z(4, 2, 48, 64), z(1, 4))
    with pytest.raises(ValueError, match="there must be some"):
        S.PagedCache.over(p, z(4, 2, 64, 64), z(4, 2, 64, 64), z(1, 0))
    with pytest.raises(ValueError, match="one dimension"):
        S.Rope(z(2, 2))
    with pytest.raises(ValueError, match="device tensor"):
        S.Rope(z(16, dtype=torch.float64))
    with pytest.raises(ValueError, match="four"):
        S.paged_append(p, None, z(2, 2), z(2, 2), 0)
    with pytest.raises(ValueError, match="four"):
        S.tree_attn(p, None, z(2, 2), None, 0, None, None)
    with pytest.raises(ValueError, match="two"):
        S.paged_keep(p, None, z(2), z(2), 0)
    with pytest.raises(ValueError, match="three"):
        S.tree_verify(None, None, z(2, 2), None, None, None, None, None, None)
    with pytest.raises(ValueError, match="dtype"):
        S.tree_verify(None, None, z(2, 2, 2, dtype=torch.float64), None, None, None, None, None, None)


def test_rope_frequencies():
    f, s = S.rope_frequencies(128, 10000.0, "cpu")
    assert s == 1.0 and f.dtype == torch.float64 and f.shape == (64,)
    assert f[0] == 1.0 and math.isclose(f[63], 10000.0 ** (-126 / 128), rel_tol=1e-14)
    g, s = S.rope_frequencies(128, 10000.0, "cpu", "linear", 4.0)
    assert s == 1.0 and torch.equal(g, f / 4)
    g, s = S.rope_frequencies(128, 10000.0, "cpu", "ntk", 4.0)
    assert s == 1.0 and g[0] == 1.0 and math.isclose(g[63], f[63] / 4, rel_tol=1e-12) and bool((g <= f).all())
    g, s = S.rope_frequencies(128, 10000.0, "cpu", "yarn", 4.0, original_len=4096)
    turns = f * 4096 / (2 * math.pi)
    assert math.isclose(s, 0.1 * math.log(4.0) + 1.0)
    assert torch.equal(g[turns > 36], f[turns > 36]) and torch.equal(g[turns < 0.85], f[turns < 0.85] / 4)
    assert bool(((g <= f) & (g >= f / 4)).all()) and bool((g[1:] < g[:-1]).all())
    assert torch.equal(S.rope_frequencies(2, 10000.0, "cpu", "ntk", 4.0)[0], torch.ones(1, dtype=torch.float64))
    for bad in (dict(rot_dim=3), dict(theta=1.0), dict(factor=0.5), dict(scaling="yarn"), dict(scaling="cubic")):
        with pytest.raises(ValueError):
            S.rope_frequencies(**{**dict(rot_dim=64, theta=1e4, device="cpu"), **bad})

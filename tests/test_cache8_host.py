"""The 8-bit cache's calls on the host: struct layout, defaults, workspace sizes and every refusal.  Nothing here
reaches a launch."""
import ctypes
import json
import os
import subprocess

import pytest
import torch

from paper_2607_16213_amd import selkv as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EDTYPE, EUNSUPPORTED, EALIGN, EWORKSPACE, EHIP = 1, 2, 3, 4, 5, 6
FAKE, NULL = 0x10000, None
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers are only passed where no GPU exists")


def cache(code=0, block=64, capacity=256, **kw):
    c = S.Cache8Struct()
    S.lib.selkv_cache8_init(c)
    c.code, c.block, c.capacity = code, block, capacity
    for f in ("K", "V", "k_scale", "v_scale", "k_tail", "v_tail"):
        setattr(c, f, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def write(p, c, K=FAKE, V=FAKE, n_new=16, cache_len=0, lens=NULL, counts=NULL):
    return S.lib.selkv_cache8_write(p, c, K, V, n_new, cache_len, lens, counts, None)


def read(p, c, K=FAKE, V=FAKE, first=0, count=16, cache_len=64, lens=NULL):
    return S.lib.selkv_cache8_read(p, c, K, V, first, count, cache_len, lens, None)


def attn(p, c, q=FAKE, bias=NULL, cache_len=64, lens=NULL, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return S.lib.selkv_decode8_attn(p, c, q, bias, cache_len, lens, out, ws, ws_bytes, None)


def append(p, c, q=FAKE, k=FAKE, v=FAKE, bias=NULL, cache_len=64, lens=NULL, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return S.lib.selkv_decode8_append(p, c, q, k, v, bias, cache_len, lens, out, ws, ws_bytes, None)


def test_struct_layout_and_defaults(tmp_path):
    fields = [f for f, _ in S.Cache8Struct._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "selkv.h"', "int main(void){",
           'printf("{\\"size\\": %zu", sizeof(selkv_cache8));']
    src += [f'printf(", \\"{f}\\": %zu", offsetof(selkv_cache8, {f}));' for f in fields]
    (tmp_path / "l.c").write_text("\n".join(src + ['printf("}\\n"); return 0; }']))
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", f"-I{ROOT}/include", "-I/opt/rocm/include", str(tmp_path / "l.c"),
                    "-o", str(tmp_path / "l")], check=True)
    layout = json.loads(subprocess.run([str(tmp_path / "l")], capture_output=True, text=True).stdout)
    assert layout["size"] == ctypes.sizeof(S.Cache8Struct)
    assert all(layout[f] == getattr(S.Cache8Struct, f).offset for f in fields)
    c = S.Cache8Struct()
    S.lib.selkv_cache8_init(c)
    assert (c.struct_size, c.code, c.block, c.capacity, c.K) == (ctypes.sizeof(c), 0, 64, 0, None)


def test_workspace_covers_every_shorter_cache():
    need = ctypes.c_size_t()
    for (B, H, G, d, block) in [(1, 8, 4, 128, 64), (1, 2, 2, 64, 16), (4, 32, 1, 128, 128), (64, 8, 8, 128, 32)]:
        p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d)
        last = 0
        for cap in range(block, 20 * 1024, 7 * block):
            assert S.lib.selkv_decode8_workspace_size(p, cache(block=block, capacity=cap), ctypes.byref(need)) == 0
            assert need.value >= last
            last = need.value


@no_gpu
def test_the_capacity_workspace_passes_at_every_length():
    """The calls then fail at the launch, there being no GPU, never with EWORKSPACE."""
    need = ctypes.c_size_t()
    for (B, H, G, block, cap) in [(1, 8, 4, 64, 64 * 67), (1, 2, 2, 16, 1600), (2, 32, 1, 128, 128 * 40)]:
        p = S.params(batch=B, n_heads_kv=H, group=G)
        c = cache(block=block, capacity=cap)
        S.lib.selkv_decode8_workspace_size(p, c, ctypes.byref(need))
        for n in range(0, cap, 37):
            for lens in (NULL, FAKE):
                assert attn(p, c, cache_len=n, lens=lens, ws_bytes=need.value) == EHIP
                assert append(p, c, cache_len=n, lens=lens, ws_bytes=need.value) == EHIP
    for heads in (1, 2, 7, 60, 100, 255, 256, 400, 768, 769, 2304, 2305, 65535):
        p = S.params(batch=heads, n_heads_kv=1, group=2)
        c = cache(capacity=1 << 28)
        assert S.lib.selkv_decode8_workspace_size(p, c, ctypes.byref(need)) == 0
        for n in (0, 769, 1000, 2048, 5000, 12801, 25600, 102400, 1 << 20, (1 << 28) - 1):
            for lens in (NULL, FAKE):
                assert attn(p, c, cache_len=n, lens=lens, ws_bytes=need.value) == EHIP, (heads, n)


@no_gpu
@pytest.mark.parametrize("call", [write, read, attn, append])
def test_refusals_of_every_call(call):
    p = S.params()
    assert call(p, cache()) == EHIP                            # valid: it gets as far as the launch
    assert call(S.params(struct_size=4), cache()) == EINVAL
    assert call(p, cache(struct_size=4)) == EINVAL
    assert call(S.params(kv_dtype=7), cache()) == EDTYPE
    assert call(p, cache(code=2)) == EDTYPE
    assert call(S.params(batch=0), cache()) == EINVAL
    assert call(S.params(n_heads_kv=0), cache()) == EINVAL
    assert call(S.params(head_dim=96), cache()) == EUNSUPPORTED
    assert call(S.params(batch=8192), cache()) == EUNSUPPORTED      # 65536 KV heads
    for block in (0, 8, 48, 256, -64):
        assert call(p, cache(block=block, capacity=768)) == EUNSUPPORTED
    assert call(p, cache(capacity=0)) == EINVAL
    assert call(p, cache(capacity=100)) == EINVAL
    assert call(p, cache(capacity=(1 << 28) + 64)) == EUNSUPPORTED
    assert call(p, cache(capacity=1 << 28)) == EHIP
    for f in ("K", "V", "k_scale", "v_scale", "k_tail", "v_tail"):
        assert call(p, cache(**{f: None})) == EINVAL
        assert call(p, cache(**{f: FAKE + 2})) == EALIGN
        assert call(p, cache(**{f: FAKE + 8})) == (EHIP if "scale" in f else EALIGN)
    for n in (-1, 257):
        assert call(p, cache(), cache_len=n) == EINVAL
    assert call(p, cache(), lens=FAKE + 2) == EALIGN


@no_gpu
def test_refusals_of_write_and_read():
    p, c = S.params(), cache()
    assert write(p, c, K=NULL) == EINVAL and write(p, c, V=NULL) == EINVAL
    assert write(p, c, K=FAKE + 8) == EALIGN and write(p, c, V=FAKE + 8) == EALIGN and write(p, c, counts=FAKE + 1) == EALIGN
    assert write(p, c, n_new=0) == EINVAL and write(p, c, n_new=-1) == EINVAL and write(p, c, n_new=257) == EINVAL
    assert write(p, c, n_new=16, cache_len=241) == EINVAL      # no room
    assert write(p, c, n_new=16, cache_len=240) == EHIP
    assert write(p, c, n_new=16, cache_len=256, lens=FAKE) == EHIP    # the lengths are on the device
    assert read(p, c, K=NULL) == EINVAL and read(p, c, V=NULL) == EINVAL
    assert read(p, c, K=FAKE + 8) == EALIGN and read(p, c, V=FAKE + 8) == EALIGN
    assert read(p, c, first=-1) == EINVAL and read(p, c, count=0) == EINVAL and read(p, c, first=250, count=7) == EINVAL
    assert read(p, c, first=250, count=6) == EHIP


@no_gpu
def test_refusals_of_the_decode_calls():
    p, c = S.params(), cache()
    big = cache(capacity=1 << 16)
    for call in (attn, append):
        assert call(S.params(group=0), c) == EINVAL and call(S.params(group=9), c) == EUNSUPPORTED
        for scale in (-1.0, float("nan"), float("inf")):
            assert call(S.params(scale=scale), c) == EINVAL
        assert call(p, c, q=NULL) == EINVAL and call(p, c, out=NULL) == EINVAL
        assert call(p, c, q=FAKE + 8) == EALIGN and call(p, c, out=FAKE + 8) == EALIGN and call(p, c, bias=FAKE + 2) == EALIGN
        assert call(p, big, cache_len=60000, ws=NULL) == EWORKSPACE
        assert call(p, big, cache_len=60000, ws_bytes=64) == EWORKSPACE
        assert call(p, big, cache_len=60000, ws=FAKE + 16) == EALIGN
    assert append(p, c, k=NULL) == EINVAL and append(p, c, v=NULL) == EINVAL
    assert append(p, c, k=FAKE + 8) == EALIGN and append(p, c, v=FAKE + 8) == EALIGN
    assert append(p, c, cache_len=256) == EINVAL and attn(p, c, cache_len=256) == EHIP    # full
    assert append(p, c, cache_len=255) == EHIP and attn(p, c, cache_len=0) == EHIP
    n = ctypes.c_size_t()
    f = S.lib.selkv_decode8_workspace_size
    assert f(p, c, None) == EINVAL and f(p, None, ctypes.byref(n)) == EINVAL and f(None, c, ctypes.byref(n)) == EINVAL
    assert f(S.params(group=9), c, ctypes.byref(n)) == EUNSUPPORTED and f(p, cache(block=5), ctypes.byref(n)) == EUNSUPPORTED


def test_refusals_of_the_binding():
    p = S.params(batch=1, n_heads_kv=2, group=2, head_dim=64, kv_dtype="fp32")
    with pytest.raises(ValueError):
        S.Cache8(p, 100, "cpu", block=48)
    with pytest.raises(KeyError):
        S.Cache8(p, 100, "cpu", code="fp4")
    with pytest.raises(ValueError, match="device tensor"):      # host memory
        S.Cache8(p, 100, "cpu")
    z = torch.zeros
    with pytest.raises(ValueError, match="dtype"):
        S.Cache8.over(p, z(1, 2, 64, 64), z(1), z(1), z(1), z(1), z(1))
    with pytest.raises(ValueError, match="four"):
        S.Cache8.over(p, z(2, 64, 64, dtype=torch.int8), z(1), z(1), z(1), z(1), z(1))
    with pytest.raises(ValueError, match="whole blocks"):
        S.Cache8.over(p, z(1, 2, 100, 64, dtype=torch.int8), z(1), z(1), z(1), z(1, 2, 64, 64), z(1))

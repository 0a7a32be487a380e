"""CPU tests of latent caches: sizes, refusals (nothing is launched), and the rules that divide their launches."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import oracle.latent as ol
import paper_2403_11805_amd as kvs
from paper_2403_11805_amd import binding

GOOD = kvs.LatentShape(2, 4, 512, 64, 128, 64, 256, 16, 64)
P = 1 << 20          # an address that is aligned and never read
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def pages(**other):
    f = dict(pool=P, pool_bytes=1 << 20, off=P, bits=P, len=P, n_seqs=3, stride=16)
    f.update(other)
    return binding.kv_pages_t(**f)


def refused(code, name, *args):
    with pytest.raises(kvs.KvError) as e:
        binding._check(getattr(binding.lib(), name)(*args))
    assert e.value.code == code, str(e.value)


def moved_args(shape=GOOD, pg=None, layer=0, c=P, c_stride=512, r=P, r_stride=64, n_rows=3, start=None):
    s, pg = shape.c(), pg or pages()
    return ctypes.byref(s), ctypes.byref(pg), layer, c, c_stride, r, r_stride, n_rows, start, None


def attend_args(shape=GOOD, pg=None, layer=0, q=P, stride=4 * 192, n_rows=3, start=None, max_rows=1, w=P, ws=P, ws_bytes=1 << 40, out=P):
    s, pg = shape.c(), pg or pages()
    return ctypes.byref(s), ctypes.byref(pg), layer, q, stride, n_rows, start, max_rows, w, ws, ws_bytes, out, None


def prompt_args(shape=GOOD, pg=None, layer=0, q=P, stride=4 * 192, n_rows=3, start=None, n_tokens=300, w=P, ws=P, ws_bytes=1 << 40, out=P):
    s, pg = shape.c(), pg or pages()
    return ctypes.byref(s), ctypes.byref(pg), layer, q, stride, n_rows, start, n_tokens, w, ws, ws_bytes, out, None


CALLS = [("kv_latent_append_tokens", moved_args), ("kv_latent_read_tokens", moved_args), ("kv_latent_attend_tokens", attend_args),
         ("kv_latent_attend_prompts", prompt_args)]
BAD_SHAPES = [dict(latent_dim=128), dict(latent_dim=384), dict(rope_dim=16), dict(rope_dim=128), dict(key_dim=96), dict(value_dim=256),
              dict(n_heads=0), dict(n_heads=1025), dict(group=32), dict(group=96), dict(latent_dim=256, group=512), dict(format=1), dict(format=4),
              dict(chunk_tokens=8), dict(chunk_tokens=24, n_tokens=240), dict(chunk_tokens=1040, n_tokens=1040), dict(n_tokens=250),
              dict(n_tokens=(1 << 24) + 16), dict(n_layers=0), dict(n_layers=65537)]


@pytest.mark.parametrize("name,args", CALLS)
def test_shapes_and_tables_are_checked(name, args):
    for bad in BAD_SHAPES:
        refused(binding.KV_ESHAPE, name, *args(shape=GOOD._replace(**bad)))
    for other in (dict(pool=None), dict(off=None), dict(bits=None), dict(len=None), dict(pool=P + 8), dict(off=P + 4), dict(len=P + 2),
                  dict(n_seqs=0), dict(n_seqs=65536), dict(stride=15)):
        refused(binding.KV_EINVAL, name, *args(pg=pages(**other)))
    for layer in (-1, 2):
        refused(binding.KV_EINVAL, name, *args(layer=layer))
    for i in (0, 1):
        call = list(args())
        call[i] = None
        refused(binding.KV_EINVAL, name, *call)
    refused(binding.KV_EINVAL, name, *args(n_rows=-1, start=P))
    refused(binding.KV_EINVAL, name, *args(n_rows=2))                       # without row_start: one row a sequence
    refused(binding.KV_EINVAL, name, *args(start=P + 2))


@pytest.mark.parametrize("name", ["kv_latent_append_tokens", "kv_latent_read_tokens"])
def test_refusals_of_moved_rows(name):
    for other in (dict(c=None), dict(r=None), dict(c=P + 8), dict(r=P + 8), dict(c_stride=504), dict(c_stride=516), dict(r_stride=56),
                  dict(r_stride=68)):
        refused(binding.KV_EINVAL, name, *moved_args(**other))
    assert getattr(binding.lib(), name)(*moved_args(n_rows=0, start=P, c=None, r=None)) == 0
    # a launch has less than 2^32 threads: 16777215 workgroups of 256, of 16 rows (append) or 8 (read)
    refused(binding.KV_ESHAPE, name, *moved_args(n_rows=1 << 28 if "append" in name else 1 << 27, start=P))


@pytest.mark.parametrize("name,args", CALLS[2:])
def test_refusals_of_attention(name, args):
    for other in (dict(q=None), dict(w=None), dict(out=None), dict(ws=None), dict(q=P + 8), dict(w=P + 8), dict(out=P + 8), dict(ws=P + 128),
                  dict(stride=4 * 192 - 8), dict(stride=4 * 192 + 4)):
        refused(binding.KV_EINVAL, name, *args(**other))
    assert getattr(binding.lib(), name)(*args(n_rows=0, start=P, q=None, w=None, out=None, ws=None)) == 0
    if args is attend_args:
        for max_rows in (0, 17, -1):
            refused(binding.KV_EINVAL, name, *args(max_rows=max_rows))
        need = [kvs.kv_latent_attend_workspace_bytes(GOOD, 3, m) for m in (1, 5, 16)]
        assert need == sorted(need)
        for m, n in zip((1, 5, 16), need):
            refused(binding.KV_ENOMEM, name, *args(max_rows=m, ws_bytes=n - 1))
    else:
        for n_tokens in (0, -1):
            refused(binding.KV_EINVAL, name, *args(n_tokens=n_tokens))
        refused(binding.KV_ESHAPE, name, *args(n_tokens=(1 << 26) + 1))
        refused(binding.KV_ENOMEM, name, *args(ws_bytes=kvs.kv_latent_prompts_workspace_bytes(GOOD, 3, 300) - 1))
        refused(binding.KV_ESHAPE, name, *args(shape=GOOD._replace(n_heads=1024), stride=1024 * 192, n_rows=1 << 22, start=P))


def test_sizes_that_no_call_can_have():
    wide = GOOD._replace(n_heads=1024, n_tokens=1 << 24)
    for ask in (lambda: kvs.kv_latent_attend_workspace_bytes(wide, 65535), lambda: kvs.kv_latent_attend_workspace_bytes(GOOD, 0),
                lambda: kvs.kv_latent_attend_workspace_bytes(GOOD, 3, 17), lambda: kvs.kv_latent_prompts_workspace_bytes(GOOD, 3, 0),
                lambda: kvs.kv_latent_prompts_workspace_bytes(wide, 3, 1 << 26), lambda: kvs.kv_latent_record_bytes(GOOD, 3),
                lambda: kvs.kv_latent_record_bytes(GOOD, 1), lambda: kvs.kv_latent_record_bytes(GOOD._replace(rope_dim=8), 16)):
        with pytest.raises(kvs.KvError):
            ask()


@pytest.mark.parametrize("fmt", [0, 3])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
def test_record_bytes(bits, fmt):
    for shape in (GOOD, GOOD._replace(n_layers=61, chunk_tokens=1024, n_tokens=1024), GOOD._replace(latent_dim=256, rope_dim=32, group=256)):
        s = shape._replace(format=fmt)
        assert kvs.kv_latent_record_bytes(s, bits) == ol.record_bytes(ol.Shape(*s), bits)


def test_the_prompts_workspace_holds_what_is_made_in_it():
    """Keys and values of all heads, latents and position parts of n_tokens tokens."""
    for n_seqs, n_tokens in ((1, 1), (3, 2), (1, 4096), (65535, 70000)):
        assert kvs.kv_latent_prompts_workspace_bytes(GOOD, n_seqs, n_tokens) >= n_tokens * 2 * (4 * 192 + 512 + 64)


def test_the_binding_refuses_tensors_that_do_not_fit():
    t = lambda *size, dtype=torch.float16: torch.zeros(size, dtype=dtype)
    with pytest.raises(ValueError):
        kvs.LatentPages(GOOD, t(64, dtype=torch.uint8), t(3, 16, dtype=torch.int64), t(3, 15, dtype=torch.uint8), t(3, dtype=torch.int32))
    with pytest.raises((ValueError, TypeError)):
        kvs.LatentPages(GOOD, t(64, dtype=torch.uint8), t(3, 16, dtype=torch.int64), t(3, 16, dtype=torch.uint8), t(3, dtype=torch.int32))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    at = tmp_path_factory.mktemp("latent_rules")
    source = at / "driver.cpp"
    source.write_text('#include "kv_launch_rules.hpp"\nextern "C" int latent_run(int u, int p, int g) { return kvs::latent_run(u, p, g); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2403_11805_amd", "csrc"),
                    str(source), "-o", str(at / "rules.so")], check=True)
    return ctypes.CDLL(str(at / "rules.so"))


def test_runs_of_the_line_of_work(rules):
    """Every place is in some workgroup's run, and a run has room for a pair's first tile."""
    cost = 4
    for pairs in (1, 2, 3, 16, 24, 100, 4096, 65535):
        for tiles in (0, 1, 2, 7, 32, 1024):
            for groups in (1, 5, 256):
                run = rules.latent_run(pairs * tiles, pairs, groups)
                assert run >= 1 and run * groups >= pairs * (tiles + cost)

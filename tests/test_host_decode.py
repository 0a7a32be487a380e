"""CPU tests of decoding on packed records: workspace sizes, refusals (nothing is launched), the rules that divide launches, and
the oracle against closed forms and against itself."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import oracle
import oracle.decode as od
import paper_2403_11805_amd as kvs
from paper_2403_11805_amd import binding

from paged import Paged, rows

GOOD = kvs.Shape(2, 2, 4, 128, 256, 16, 64)
P = 1 << 20          # an address that is aligned and never read


def pages(**other):
    f = dict(pool=P, pool_bytes=1 << 20, off=P, bits=P, len=P, n_seqs=3, stride=16)
    f.update(other)
    return binding.kv_pages_t(**f)


def refused(code, name, *args):
    with pytest.raises(kvs.KvError) as e:
        binding._check(getattr(binding.lib(), name)(*args))
    assert e.value.code == code, str(e.value)


def append_args(shape=GOOD, pg=None, layer=0, k=P, v=P, stride=256, n_rows=3, start=None, seen=None, mass=None, pos=None):
    s, pg = shape.c(), pg or pages()
    return ctypes.byref(s), ctypes.byref(pg), layer, k, v, stride, n_rows, start, seen, mass, pos, None


def attend_args(shape=GOOD, pg=None, layer=0, q=P, stride=512, n_rows=3, start=None, max_rows=1, mass_in=None, mass=None, ws=P,
                ws_bytes=1 << 40, out=P):
    s, pg = shape.c(), pg or pages()
    return ctypes.byref(s), ctypes.byref(pg), layer, q, stride, n_rows, start, max_rows, mass_in, mass, ws, ws_bytes, out, None


def evict_args(shape=GOOD, pg=None, begin=0, end=2, mass_in=P, pos_in=P, seen=None, keep=100, sink=4, recent=20, ws=P, ws_bytes=1 << 40,
               mass=P, pos=P):
    s, pg = shape.c(), pg or pages()
    return ctypes.byref(s), ctypes.byref(pg), begin, end, mass_in, pos_in, seen, keep, sink, recent, ws, ws_bytes, mass, pos, None


CALLS = [("kv_append_tokens", append_args), ("kv_attend_tokens", attend_args), ("kv_evict_tokens", evict_args)]


@pytest.mark.parametrize("name,args", CALLS)
def test_shapes_and_tables_are_checked(name, args):
    for bad in (GOOD._replace(format=1, chunk_tokens=16), GOOD._replace(head_dim=512, group=512), GOOD._replace(chunk_tokens=8),
                GOOD._replace(n_tokens=250), GOOD._replace(group=96), GOOD._replace(n_q_heads=3)):
        refused(binding.KV_ESHAPE, name, *args(shape=bad))
    for other in (dict(pool=None), dict(off=None), dict(bits=None), dict(len=None), dict(pool=P + 8), dict(off=P + 4), dict(len=P + 2),
                  dict(n_seqs=0), dict(n_seqs=65536), dict(stride=15)):
        refused(binding.KV_EINVAL, name, *args(pg=pages(**other)))
    call = list(args())
    call[1] = None
    refused(binding.KV_EINVAL, name, *call)
    call = list(args())
    call[0] = None
    refused(binding.KV_EINVAL, name, *call)


def test_append_refusals():
    for other in (dict(layer=2), dict(layer=-1), dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(stride=248), dict(stride=260),
                  dict(n_rows=-1, start=P), dict(n_rows=2), dict(start=P + 2), dict(seen=P + 1), dict(mass=P + 2), dict(pos=P + 3)):
        refused(binding.KV_EINVAL, "kv_append_tokens", *append_args(**other))
    assert binding.lib().kv_append_tokens(*append_args(n_rows=0, start=P, k=None, v=None)) == 0


def test_attend_refusals():
    for other in (dict(layer=2), dict(q=None), dict(out=None), dict(ws=None), dict(q=P + 8), dict(out=P + 8), dict(ws=P + 128), dict(stride=504),
                  dict(stride=516), dict(n_rows=-1, start=P), dict(n_rows=4), dict(max_rows=0), dict(max_rows=17), dict(mass_in=P),
                  dict(mass=P + 2), dict(mass=P, mass_in=P + 1)):
        refused(binding.KV_EINVAL, "kv_attend_tokens", *attend_args(**other))
    refused(binding.KV_ESHAPE, "kv_attend_tokens", *attend_args(shape=GOOD._replace(n_kv_heads=1, n_q_heads=65), stride=65 * 128, max_rows=16))
    for max_rows, mass in ((1, None), (5, P)):
        need = kvs.kv_attend_workspace_bytes(GOOD, 3, max_rows, mass is not None)
        refused(binding.KV_ENOMEM, "kv_attend_tokens", *attend_args(max_rows=max_rows, mass=mass, ws_bytes=need - 1))
    assert binding.lib().kv_attend_tokens(*attend_args(n_rows=0, start=P, q=None, out=None, ws=None)) == 0


def test_evict_refusals():
    for other in (dict(begin=-1), dict(begin=2, end=1), dict(end=3), dict(keep=0), dict(sink=-1), dict(recent=-1), dict(sink=50, recent=51),
                  dict(recent=2 ** 31 - 1), dict(mass_in=None), dict(pos_in=None), dict(mass=None), dict(pos=None), dict(ws=None),
                  dict(ws=P + 64), dict(mass=P + 1), dict(pos_in=P + 2), dict(seen=P + 2)):
        refused(binding.KV_EINVAL, "kv_evict_tokens", *evict_args(**other))
    need = kvs.kv_evict_workspace_bytes(GOOD, 3, 2, 100)
    refused(binding.KV_ENOMEM, "kv_evict_tokens", *evict_args(ws_bytes=need - 1))
    assert binding.lib().kv_evict_tokens(*evict_args(begin=1, end=1, mass=None, ws=None)) == 0


def test_grids_that_no_launch_can_have_are_refused():
    """A launch has less than 2^32 threads: 16777215 workgroups of 256, 4194303 of 1024."""
    tiny = GOOD._replace(n_tokens=16, n_kv_heads=1, n_q_heads=1, head_dim=64)
    most = pages(n_seqs=65535)
    refused(binding.KV_ESHAPE, "kv_append_tokens", *append_args(shape=tiny, n_rows=1 << 28, start=P))
    wide = tiny._replace(n_kv_heads=32, n_q_heads=256)
    refused(binding.KV_ESHAPE, "kv_attend_tokens", *attend_args(shape=wide, pg=most, stride=256 * 64, n_rows=65535))
    with pytest.raises(kvs.KvError):
        kvs.kv_attend_workspace_bytes(wide, 65535)
    deep = tiny._replace(n_layers=65, n_kv_heads=1)
    refused(binding.KV_ESHAPE, "kv_evict_tokens", *evict_args(shape=deep, pg=most, end=65, keep=4, sink=0, recent=0))


def test_workspace_sizes():
    assert kvs.kv_attend_workspace_bytes(GOOD, 1, 1) > 0
    # the logits of every row, for the weights
    assert kvs.kv_attend_workspace_bytes(GOOD, 3, 4, True) - kvs.kv_attend_workspace_bytes(GOOD, 3, 4) == 3 * 2 * (2 * 4) * 256 * 4
    for bad in ((GOOD, 0, 1), (GOOD, 65536, 1), (GOOD, 1, 0), (GOOD, 1, 17), (GOOD._replace(chunk_tokens=8), 1, 1)):
        with pytest.raises(kvs.KvError):
            kvs.kv_attend_workspace_bytes(*bad)
    for bad in ((GOOD, 0, 1, 1), (GOOD, 1, 0, 1), (GOOD, 1, 3, 1), (GOOD, 1, 1, 0)):
        with pytest.raises(kvs.KvError):
            kvs.kv_evict_workspace_bytes(*bad)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_launch_rules(tmp_path):
    root, lib = os.path.dirname(os.path.dirname(os.path.abspath(__file__))), str(tmp_path / "librules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I",
                    os.path.join(root, "paper_2403_11805_amd", "csrc"), os.path.join(root, "tests", "decode_rules_driver.cpp"), "-o", lib],
                   check=True)
    rules = ctypes.CDLL(lib)
    for name in ("attend_groups", "evict_blocks", "append_pieces"):
        getattr(rules, name).restype = ctypes.c_int64
    rules.attend_groups.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
    rules.evict_blocks.argtypes = [ctypes.c_int64] * 3
    rules.append_pieces.argtypes = [ctypes.c_int64, ctypes.c_int]
    for d, step, most in ((64, 4, 512), (128, 4, 512), (256, 2, 512)):
        assert rules.attend_groups(1, 1, d) == 1 and rules.attend_groups(3, 32 * step, d) == 3 and rules.attend_groups(3, 32 * step + 1, d) == 6
        assert rules.attend_groups(1 << 20, 1 << 15, d) == most
    # never none, never more than the list has work for
    assert rules.evict_blocks(1, 0, 64) == 1 and rules.evict_blocks(1, 65, 64) == 2 and rules.evict_blocks(1, 1 << 20, 64) == 2048
    assert rules.evict_blocks(1 << 16, 1 << 20, 64) == 4
    assert rules.append_pieces(1, 256) == 1 and rules.append_pieces(1 << 20, 256) == 4


def test_binding_checks_tensors():
    """On CPU tensors: sizes are looked at before anything is taken to be on a device."""
    pool, off = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros((3, 16), dtype=torch.int64)
    bits, length = torch.zeros((3, 16), dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    for args in ((off[0], bits, length), (off, bits[:, :8], length), (off, bits, length[:2])):
        with pytest.raises(ValueError):
            kvs.Pages(GOOD, pool, *args)
    with pytest.raises(TypeError):
        kvs.Pages(GOOD, pool, off, bits, length)


def test_oracle_row_is_the_compressed_row():
    """Appending token by token gives the bytes of compressing the chunk (groups never span two tokens)."""
    for fmt in (0, 3):
        for w in (16, 8, 4, 2):
            s = oracle.Shape(1, 2, 2, 128, 32, 32, 64, fmt)
            rng = np.random.RandomState(w)
            kv = rng.standard_normal((1, 2, 2, 32, 128)).astype(np.float16)
            off = np.array([0, oracle.record_bytes(s, w)], dtype=np.uint64)
            want = oracle.compress_chunks(s, kv, np.array([w], dtype=np.uint8), off)
            pool = np.zeros(int(off[1]), dtype=np.uint8)
            k, v = (np.ascontiguousarray(kv[0, i].transpose(1, 0, 2)) for i in range(2))
            od.append(s, pool, np.zeros((1, 1), dtype=np.int64), np.array([[w]], dtype=np.uint8), np.array([32], dtype=np.int32), 0, k, v,
                      np.array([0, 32], dtype=np.int32))
            assert np.array_equal(pool, want)
            # and a row's values are what a Load gives back, before their last rounding
            out = np.zeros_like(kv)
            oracle.swapin_chunks(s, want, np.zeros(1, dtype=np.uint64), np.zeros(1, dtype=np.int32), np.array([w], dtype=np.uint8), out)
            slab = od.Slab(s, pool, 0, w, 0, 1, 1)
            assert np.array_equal(np.stack([slab.dequantised(s, r) for r in range(32)]).view(np.uint16), out[0, 1, 1].view(np.uint16))
            np.testing.assert_allclose(slab.values(s), out[0, 1, 1].astype(np.float64), rtol=2.0 ** -11, atol=2.0 ** -11 * 8)


def test_oracle_attention_closed_forms():
    p = Paged((1, 1, 2, 64, 64, 16, 64), [50, 3], (16, 4), 1)
    q = np.zeros((2, 2, 64), dtype=np.float16)                 # equal logits: the mean of V, weights 1 / n
    out, _, _, mass = od.attend(p.os, p.pool, *p.table(), 0, q)
    for s, n in enumerate((50, 3)):
        v = np.concatenate([od.Slab(p.os, p.pool, p.off[s, i], p.bits[s, i], 0, 1, 0).values(p.os) for i in range(4)])[:n]
        np.testing.assert_allclose(out[s, 0], v.mean(0), rtol=1e-12, atol=1e-14)
        np.testing.assert_allclose(mass[s, 0, :n], 2 / n)
        assert not mass[s, 0, n:].any()
    start, _ = rows([2, 0])                                    # the first of two new rows does not see the second
    out, _, _, mass = od.attend(p.os, p.pool, *p.table(), 0, q, start)
    np.testing.assert_allclose(mass[0, 0, 49], 2 / 50)
    np.testing.assert_allclose(mass[0, 0, 48], 2 / 50 + 2 / 49)


def test_oracle_eviction_small():
    p = Paged((1, 1, 1, 64, 16, 16, 64), [8], (16,), 1)
    mass, pos = np.array([5, 0, 3, 0, 1, 4, 3, 0, 9, 9, 9, 9, 9, 9, 9, 9], dtype=np.float32).reshape(1, 1, 1, 16), p.book(1)[1]
    before = p.pool.copy().view(np.float16).reshape(2, 16, 64)
    m, q = od.evict(p.os, p.pool, *p.table(), (0, 1), mass, pos, 4, 0, 1)      # kept: 7 (newest), 0, 5, 2 (ties with 6)
    assert q[0, 0, 0, :4].tolist() == [0, 5, 2, 7] and m[0, 0, 0, :4].tolist() == [5, 4, 3, 0]
    after = p.pool.view(np.float16).reshape(2, 16, 64)
    assert np.array_equal(after[:, :4], before[:, [0, 5, 2, 7]]) and np.array_equal(after[:, 4:8], before[:, 4:8])

"""What the host side of the 8-bit cache, its attention and the block tables promises: a launch that fails is reported, block
tables are as wide as their rows lie apart, and a workspace that serves a call serves every smaller one.  No GPU is used."""
import ctypes as C
import json
import os
import random
import subprocess
import sys

import pytest
import torch

from paper_2512_07993_amd import binding as B

from test_quant_refusals import _pages, _quant, _queries, _rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(B._LIB_PATH):
        from paper_2512_07993_amd.build import build_library
        build_library()
    yield


# ---- launches that fail -------------------------------------------------------------------------------------
# Stands in front of the runtime in a child process: no kernel is launched, the launch named by fail_at fails, and the last error is kept
# until it is asked for, as the runtime keeps it.
RUNTIME = r"""
#include <cstddef>
namespace { int count, at = -1, last; struct { unsigned g[3], b[3]; size_t lds; void *st; } conf; }
struct Dim { unsigned x, y, z; };
extern "C" {
void fail_at(int n) { count = 0, at = n, last = 0; }
int launches() { return count; }
int __hipPushCallConfiguration(Dim g, Dim b, size_t lds, void *st) {
  conf = {{g.x, g.y, g.z}, {b.x, b.y, b.z}, lds, st};
  return 0;
}
int __hipPopCallConfiguration(Dim *g, Dim *b, size_t *lds, void **st) {
  *g = {conf.g[0], conf.g[1], conf.g[2]}, *b = {conf.b[0], conf.b[1], conf.b[2]}, *lds = conf.lds, *st = conf.st;
  return 0;
}
int hipLaunchKernel(const void *, Dim, Dim, void **, size_t, void *) { return count++ == at ? last = 1 : 0; }
int hipGetLastError() { const int e = last; last = 0; return e; }
}
"""

ATTEND = {
    "one token": dict(max_len=60),
    "one token, cut caches": dict(max_len=64000),
    "fp32": dict(dtype=B.F32),
    "32 rows": dict(max_q=8, total_q=24),
    "many rows, cut alike": dict(max_q=200, total_q=600, max_len=1500),
    "many rows, dealt out": dict(max_q=900, total_q=2700, max_len=64000),
}


def _calls():
    lib = B.lib()
    qc = _quant(table_stride=4000)
    for name, kw in ATTEND.items():
        need = C.c_size_t(0)
        q = _queries(**kw)
        assert lib.skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(q), C.byref(need)) == B.OK
        yield name, lambda: lib.skipkv_quant_attend(C.byref(qc), 0, C.byref(q), 0xB000, None, 0x10000, need.value, None)
    for name, call in (("store", lib.skipkv_quant_store), ("load", lib.skipkv_quant_load)):
        yield name, lambda: call(C.byref(qc), C.byref(_rows()), 0, None, None, None, None)
    for name, slots, new in (("pages", 0x7000, 3), ("pages without slots", None, 0)):
        yield name, lambda: lib.skipkv_pages_update(C.byref(_pages()), 0x5000, 1, 0x6000, new, slots, None, 0x10000, 1 << 20, None)


def _child(runtime):
    rt = C.CDLL(runtime)
    seen = {}
    for name, call in _calls():
        rt.fail_at(-1)
        ok = call()
        n = rt.launches()
        failed = []
        for i in range(n):
            rt.fail_at(i)
            failed.append([call(), rt.launches()])
        seen[name] = [ok, n, failed]
    print(json.dumps(seen))


@pytest.fixture(scope="module")
def outcomes(tmp_path_factory):
    d = tmp_path_factory.mktemp("runtime")
    src, so = str(d / "runtime.cpp"), str(d / "runtime.so")
    with open(src, "w") as f:
        f.write(RUNTIME)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", so, src], check=True)
    first = [so] + [x for x in os.environ.get("LD_PRELOAD", "").split(":") if x]
    env = dict(os.environ, LD_PRELOAD=":".join(first), PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests")]))
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


@pytest.mark.parametrize("what", list(ATTEND) + ["store", "load", "pages", "pages without slots"])
def test_whichever_launch_fails_the_call_says_so(outcomes, what):
    ok, n, failed = outcomes[what]
    assert ok == B.OK and n >= 1
    for rc, _ in failed:
        assert rc == B.EHIP


@pytest.mark.parametrize("what", list(ATTEND))
def test_nothing_is_joined_when_the_first_kernel_was_not_launched(outcomes, what):
    _, n, failed = outcomes[what]
    assert n == (1 if what in ("one token", "32 rows") else 2) and failed[0] == [B.EHIP, 1]


# ---- block tables of the binding: table_stride is a row's pitch and its width --------------------------------

def _both(table):
    """The structures of the two kinds of callers over one block table [B, entries]."""
    z = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype)
    batch = table.shape[0]
    pool = lambda: z(1, 20, 16, 2, 128, dtype=torch.uint8)
    return [lambda: B.Pages(table, z(batch), z(20), z(1), 16).c(),
            lambda: B.QuantCache(pool(), pool(), z(1, 2, 20, dtype=torch.uint8), z(1, 2, 20, dtype=torch.uint8), table).c()]


BIG = torch.arange(32, dtype=torch.int32).view(4, 8)


@pytest.mark.parametrize("table", [BIG[:, :6], BIG[:, 3:], BIG[:, 3:6], BIG[::2], BIG[:, :1], BIG[1:2].expand(3, 8), BIG[:, ::2], BIG.t(),
                                   BIG.view(2, 16)[:, :8], BIG.long()],
                         ids=["left", "right", "middle", "every other row", "one column", "one row for all", "every other column", "transposed",
                              "half", "64-bit"])
def test_tables_whose_rows_lie_further_apart_than_they_are_wide_are_refused(table):
    """The library would take the entries behind a row for the row's own, and in the last one read and write beyond the storage."""
    for call in _both(table):
        with pytest.raises(AssertionError):
            call()


@pytest.mark.parametrize("table", [BIG, BIG[1:3], BIG[2:3], BIG[3:4, 2:7], torch.arange(9, dtype=torch.int32).view(9, 1).t(),
                                   BIG.view(-1)[5:].as_strided((1, 12), (3, 1)), torch.zeros(5, 1, dtype=torch.int32), BIG[1:2].expand(1, 8),
                                   torch.zeros(3, 0, dtype=torch.int32), BIG[:, 2:2]],
                         ids=["all", "some rows", "one row", "a piece of one row", "column of 9 as a row", "row of any pitch", "one column", "one row, expanded",
                              "nothing", "nothing of a table"])
def test_tables_are_as_wide_as_their_shape_says(table):
    for call in _both(table):
        c = call()
        assert c.batch == table.shape[0] and c.table_stride == table.shape[1]
        assert (c.block_table or 0) == table.data_ptr()


# ---- pools: codes are e4m3 -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.int8, torch.bool, torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int16, torch.bfloat16])
def test_pools_of_another_form_are_refused(dtype):
    z = lambda *shape, dt=torch.uint8: torch.zeros(shape, dtype=dt)
    exp, table = z(1, 2, 20), z(3, 8, dt=torch.int32)
    pool = (1, 20, 16, 2, 128)
    for k, v in ((dtype, dtype), (torch.uint8, dtype), (dtype, torch.float8_e4m3fn)):
        with pytest.raises(AssertionError):
            B.QuantCache(z(*pool, dt=k), z(*pool, dt=v), exp, exp, table).c()
    for good in (torch.uint8, torch.float8_e4m3fn):
        assert B.QuantCache(z(*pool, dt=good), z(*pool, dt=good), exp, exp, table).c().n_blocks == 20


# ---- workspaces and status words ----------------------------------------------------------------------------

def _entry_points():
    """The calls of the binding that take a workspace or a status word, on host tensors: (name, call(ws, dev_status))."""
    z = lambda *shape, dt=torch.int32: torch.zeros(shape, dtype=dt)
    u8, bf = torch.uint8, torch.bfloat16
    qc = B.QuantCache(z(1, 20, 16, 2, 128, dt=u8), z(1, 20, 16, 2, 128, dt=u8), z(1, 2, 20, dt=u8), z(1, 2, 20, dt=u8), z(3, 8))
    off = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    rows = B.Cache(z(1, 2, 3, 128, dt=bf), z(1, 2, 3, 128, dt=bf), 2, off, None, None, 3, 0)
    qs = B.Queries(z(3, 4, 128, dt=bf), z(3, 4, 128, dt=bf), off, max_q=1, max_len=128, scale=0.1)
    pages = B.Pages(qc.block_table, z(3), z(20), z(1), 16)
    return {"attend": lambda ws, st: B.skipkv_quant_attend(qc, 0, qs, z(2, 3), ws, st),
            "pages": lambda ws, st: B.skipkv_pages_update(pages, z(1, 3), off, 3, None, ws, st),
            "store": lambda ws, st: B.skipkv_quant_store(qc, rows, 0, None, None, st),
            "load": lambda ws, st: B.skipkv_quant_load(qc, rows, 0, None, None, st)}


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="tensors in host memory are refused where there is a GPU")
@pytest.mark.parametrize("name", ["attend", "pages"])
def test_a_workspace_with_gaps_is_refused(name):
    """Its size counts its elements, not the span that they lie in."""
    call = _entry_points()[name]
    for ws in (torch.zeros(1 << 20, dtype=torch.uint8)[::4], torch.zeros((64, 4096), dtype=torch.uint8)[:, :2048], torch.zeros(1, dtype=torch.uint8).expand(1 << 22)):
        with pytest.raises(AssertionError, match="workspace"):
            call(ws, None)


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="tensors in host memory are refused where there is a GPU")
@pytest.mark.parametrize("name", ["attend", "pages", "store", "load"])
def test_a_status_word_of_another_type_is_refused(name):
    call, ws = _entry_points()[name], torch.zeros(1 << 20, dtype=torch.uint8)
    for status in (torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.int16), torch.zeros(1)):
        with pytest.raises(AssertionError, match="status"):
            call(ws, status)


# ---- sizes of workspaces -------------------------------------------------------------------------------------

def _need(batch, max_q, total_q, max_len, hk=8, group=4, dtype=B.BF16, slots=64000):
    qc = _quant(batch=batch, n_kv_heads=hk, stride_tok=hk * 128, stride_block=16 * hk * 128, table_stride=slots // 16)
    q = _queries(dtype=dtype, n_q_heads=hk * group, q_stride_tok=hk * group * 128, out_stride_tok=hk * group * 128, max_q=max_q, total_q=total_q,
                 max_len=max_len)
    out = C.c_size_t(0)
    assert B.lib().skipkv_quant_attend_workspace_bytes(C.byref(qc), C.byref(q), C.byref(out)) == B.OK
    return out.value


def test_one_token_over_shorter_caches_needs_no_more():
    top = _need(1, 1, 1, 32768)
    assert all(_need(1, 1, 1, n) <= top for n in range(64, 32768, 64))


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
def test_fewer_tokens_and_fewer_sequences_need_no_more(dtype):
    need = [_need(16, m, 16 * m, 8192, dtype=dtype) for m in range(1, 300)]
    assert need == sorted(need)
    need = [_need(b, 1, b, 16384, dtype=dtype) for b in range(1, 300)]
    assert need == sorted(need)


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("hk,group", [(8, 4), (1, 1), (2, 7), (3, 5), (4, 8), (16, 2)])
def test_a_workspace_serves_every_smaller_call(hk, group, dtype):
    """One that shrinks in its sequences, its tokens, its longest query or cache, or in the room of a table row."""
    rng = random.Random(hk * 100 + group)
    log = lambda lo, hi: min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))
    for _ in range(1500):
        big = [log(1, 600), log(1, 1500), 0, log(1, 64000), 16 * log(1, 4000)]
        big[2] = rng.choice([big[0] * big[1], log(1, big[0] * big[1])])
        small = [log(1, x) if rng.random() < 0.6 else x for x in big[:4]] + [16 * log(1, big[4] // 16)]
        a, b = ([_need(*x[:4], hk=hk, group=group, dtype=dtype, slots=x[4])] for x in (big, small))
        assert b <= a, (big, small)


def test_short_caches_need_none():
    assert _need(64, 1, 64, 64) == 0


if __name__ == "__main__":
    _child(sys.argv[1])

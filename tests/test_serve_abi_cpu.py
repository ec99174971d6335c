"""The serving operators' C ABI on the CPU: struct layouts, workspace sizes,
and the refusal of invalid arguments before any device call."""
import os
import shutil
import subprocess

import pytest

import paper_2601_18999_amd as K
from paper_2601_18999_amd import serve as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

TABLES = ["struct_size", "rows", "width", "page_size", "ring_size", "num_tokens", "table_stride", "d_held", "d_delta",
          "d_base", "d_table", "d_ring", "d_state", "d_held_out", "d_state_out", "d_row_start", "d_slots",
          "d_positions"]
CACHE = ["struct_size", "dtype", "num_pages", "page_size", "kv_heads", "dim", "d_k", "d_v", "k_page", "k_slot",
         "k_head", "v_page", "v_slot", "v_head", "d_k_scale", "d_v_scale"]
STORE = ["struct_size", "dtype", "num_tokens", "pad", "d_k", "d_v", "k_token", "k_head", "v_token", "v_head", "d_slots",
         "d_status"]
ATTENTION = ["struct_size", "dtype", "num_tokens", "num_requests", "num_groups", "heads", "width", "prefix_width",
             "scale", "pad", "d_q", "d_out", "d_lse", "q_token", "q_head", "out_token", "out_head", "d_row_start",
             "d_length", "d_table", "d_group_start", "d_prefix_table", "d_prefix_length", "table_stride",
             "prefix_stride", "d_status"]
P = 4096  # stands for a device pointer: nothing dereferences it before a refusal

GOOD_TABLES = dict(rows=4, width=8, page_size=16, ring_size=100, num_tokens=10, table_stride=8, d_held=P, d_delta=2 * P,
                   d_base=P, d_table=P, d_ring=P, d_state=P, d_held_out=P, d_state_out=P, d_row_start=3 * P, d_slots=P,
                   d_positions=P)
GOOD_CACHE = dict(dtype=0, num_pages=100, page_size=16, kv_heads=2, dim=128, d_k=P, d_v=P, k_page=4096, k_slot=256,
                  k_head=128, v_page=4096, v_slot=256, v_head=128, d_k_scale=0, d_v_scale=0)
GOOD_STORE = dict(dtype=0, num_tokens=5, pad=0, d_k=P, d_v=P, k_token=256, k_head=128, v_token=256, v_head=128,
                  d_slots=P, d_status=0)
GOOD_ATTENTION = dict(dtype=0, num_tokens=5, num_requests=3, num_groups=1, heads=8, width=4, prefix_width=4, scale=0.1,
                      pad=0, d_q=P, d_out=P, d_lse=0, q_token=1024, q_head=128, out_token=1024, out_head=128,
                      d_row_start=P, d_length=P, d_table=P, d_group_start=P, d_prefix_table=P, d_prefix_length=P,
                      table_stride=4, prefix_stride=4, d_status=0)


def _pack(record, fields, good, change):
    d = dict(good, struct_size=record.size)
    d.update(change)
    return bytearray(record.pack(*[d[f] for f in fields]))


def tables(**kw):
    return _pack(S.TABLES_RECORD, TABLES, GOOD_TABLES, kw)


def cache(**kw):
    return _pack(S.CACHE_RECORD, CACHE, GOOD_CACHE, kw)


def store(**kw):
    return _pack(S.STORE_RECORD, STORE, GOOD_STORE, kw)


def attention(**kw):
    return _pack(S.ATTENTION_RECORD, ATTENTION, GOOD_ATTENTION, kw)


def test_records_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    kinds = (("kvr_tables", TABLES, S.TABLES_RECORD), ("kvr_cache", CACHE, S.CACHE_RECORD),
             ("kvr_store", STORE, S.STORE_RECORD), ("kvr_attention", ATTENTION, S.ATTENTION_RECORD))
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "kvr.h"', "int main(void) {"]
    for name, fields, _ in kinds:
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        lines += [f'  printf("%zu %zu\\n", offsetof({name}, {f}), sizeof((({name}*)0)->{f}));' for f in fields]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = iter(subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n"))
    for name, fields, record in kinds:
        assert int(next(out)) == record.size, name
        # each field packed alone shows where it lies: a value of all ones bits
        codes = [c for c in record.format.lstrip("<") ]
        expanded, count = [], ""
        for c in codes:
            if c.isdigit():
                count += c
            else:
                expanded += [c] * int(count or 1)
                count = ""
        assert len(expanded) == len(fields)
        at = 0
        for f, c in zip(fields, expanded):
            size = {"I": 4, "i": 4, "f": 4, "q": 8, "Q": 8}[c]
            assert [int(x) for x in next(out).split()] == [at, size], (name, f)
            at += size


def test_workspace_sizes():
    a = K.kvr_block_tables_workspace(tables())
    assert a > 0 and K.kvr_block_tables_workspace(tables(rows=4000)) > a + 8 * 3900
    b = K.kvr_attention_workspace(cache(), attention())
    assert b > 0 and K.kvr_attention_workspace(cache(), attention(num_tokens=50000)) > b


BAD_TABLES = [dict(struct_size=8), dict(rows=0), dict(rows=(1 << 20) + 1), dict(width=0), dict(width=1 << 30),
              dict(page_size=0), dict(page_size=24), dict(page_size=2048), dict(ring_size=0),
              dict(ring_size=1 << 28), dict(num_tokens=-1), dict(table_stride=7)]
BAD_POINTERS = [dict(d_held=0), dict(d_delta=0), dict(d_table=0), dict(d_ring=0), dict(d_state=0), dict(d_held_out=0),
                dict(d_state_out=0), dict(d_row_start=0), dict(d_slots=0), dict(d_positions=0),
                dict(d_held_out=2 * P), dict(d_row_start=P)]


def _names(cases):
    return ["-".join(f"{k}={v}" for k, v in c.items()) for c in cases]


def _refused(call, status=K.KVR_EINVAL):
    with pytest.raises(K.KvrError) as ei:
        call()
    assert ei.value.status == status and K.kvr_last_error()


@pytest.mark.parametrize("bad", BAD_TABLES, ids=_names(BAD_TABLES))
def test_tables_refused(bad):
    _refused(lambda: K.kvr_block_tables_workspace(tables(**bad)))
    _refused(lambda: K.kvr_block_tables(tables(**bad), P, 1 << 20))


@pytest.mark.parametrize("bad", BAD_POINTERS, ids=_names(BAD_POINTERS))
def test_tables_pointers_refused(bad):
    _refused(lambda: K.kvr_block_tables(tables(**bad), P, 1 << 20))


def test_small_or_missing_workspaces_refused():
    _refused(lambda: K.kvr_block_tables(tables(), 0, 1 << 20))
    _refused(lambda: K.kvr_block_tables(tables(), P + 4, 1 << 20))
    _refused(lambda: K.kvr_block_tables(tables(), P, 16), K.KVR_ENOMEM)
    _refused(lambda: K.kvr_shared_attention(cache(), attention(), 0, 1 << 30))
    _refused(lambda: K.kvr_shared_attention(cache(), attention(), P + 16, 1 << 30))
    _refused(lambda: K.kvr_shared_attention(cache(), attention(), P, 16), K.KVR_ENOMEM)


BAD_CACHES = [dict(struct_size=8), dict(dtype=3), dict(dtype=-1), dict(num_pages=0), dict(num_pages=1 << 28),
              dict(page_size=3), dict(page_size=0), dict(kv_heads=0), dict(kv_heads=1025), dict(dim=96),
              dict(d_k_scale=P), dict(d_v_scale=P), dict(dtype=1)]
BAD_CACHE_BUFFERS = [dict(d_k=0), dict(d_v=0), dict(d_k=P + 8), dict(k_page=4100), dict(v_slot=260),
                     dict(v_head=129), dict(dtype=2, k_head=136)]


@pytest.mark.parametrize("bad", BAD_CACHES + BAD_CACHE_BUFFERS, ids=_names(BAD_CACHES + BAD_CACHE_BUFFERS))
def test_caches_refused(bad):
    _refused(lambda: K.kvr_cache_store(cache(**bad), store()))
    _refused(lambda: K.kvr_shared_attention(cache(**bad), attention(), P, 1 << 30))


BAD_STORES = [dict(struct_size=8), dict(dtype=2), dict(dtype=-1), dict(num_tokens=-1), dict(num_tokens=1 << 27),
              dict(d_k=0), dict(d_v=0), dict(d_slots=0), dict(d_v=P + 2), dict(k_token=260), dict(v_head=132)]


@pytest.mark.parametrize("bad", BAD_STORES, ids=_names(BAD_STORES))
def test_stores_refused(bad):
    _refused(lambda: K.kvr_cache_store(cache(), store(**bad)))


BAD_ATTENTIONS = [dict(struct_size=8), dict(dtype=2), dict(dtype=1), dict(num_tokens=-1), dict(num_requests=0),
                  dict(num_requests=(1 << 20) + 1), dict(num_groups=-1), dict(heads=0), dict(heads=7),
                  dict(num_tokens=1 << 29), dict(width=-1), dict(prefix_width=-1), dict(d_row_start=0),
                  dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(d_q=0),
                  dict(d_out=0), dict(d_length=0), dict(d_table=0), dict(d_group_start=0), dict(d_prefix_length=0),
                  dict(d_prefix_table=0), dict(table_stride=3), dict(prefix_stride=3), dict(d_q=P + 8),
                  dict(q_head=132), dict(d_out=P + 4), dict(out_token=1022)]


@pytest.mark.parametrize("bad", BAD_ATTENTIONS, ids=_names(BAD_ATTENTIONS))
def test_attentions_refused(bad):
    _refused(lambda: K.kvr_shared_attention(cache(), attention(**bad), P, 1 << 30))


def test_nothing_to_do_is_no_error_and_no_launch():
    K.kvr_cache_store(cache(), store(num_tokens=0))
    K.kvr_shared_attention(cache(), attention(num_tokens=0), P, 1 << 30)


def test_null_structs_refused():
    lib = K.load_library()
    assert lib.kvr_block_tables(None, P, 1 << 20, None) == K.KVR_EINVAL
    assert lib.kvr_cache_store(None, None, None) == K.KVR_EINVAL
    assert lib.kvr_shared_attention(None, None, P, 1 << 20, None) == K.KVR_EINVAL
    assert lib.kvr_attention_workspace(None, None, None) == K.KVR_EINVAL


def test_tensors_on_the_cpu_refused():
    import torch
    x = torch.zeros(4, dtype=torch.int32)
    _refused(lambda: K.block_tables(x, x, x[:, None], x, torch.zeros(3, dtype=torch.int64), 16, 4))
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    c = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    _refused(lambda: K.cache_store(k, k, c, c, x))
    _refused(lambda: K.shared_attention(k, c, c, None, x[:, None], x))


def test_status_bits_raise():
    K.check_status("block_tables", 0)
    for bits, word in ((1, "lengths"), (128, "ring"), (256, "row"), (512, "page number")):
        with pytest.raises(K.KvrError, match=word):
            K.check_status("block_tables", bits)

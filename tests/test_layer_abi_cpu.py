"""The C ABI of norms, 8-bit products and linear attention on the CPU: struct
layouts, workspace sizes, and the refusal of invalid arguments before any
device call."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2601_18999_amd as K
from paper_2601_18999_amd import layer as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # stands for a device pointer: nothing dereferences it before a refusal

NORM = ["struct_size", "dtype", "residual_dtype", "out_dtype", "num_tokens", "dim", "activation", "eps",
        "residual_scale", "pad", "d_x", "d_after", "d_gate", "d_residual", "d_before", "d_residual_out", "d_out",
        "d_out_scale", "x_token", "gate_token", "residual_token", "residual_out_token", "out_token"]
PRODUCT = ["struct_size", "dtype", "out_dtype", "num_tokens", "dim", "channels", "d_x", "d_w", "d_out", "d_x_scale",
           "d_w_scale", "d_bias", "x_token", "w_channel", "out_token"]
LINEAR = ["struct_size", "dtype", "num_tokens", "num_requests", "heads", "kv_heads", "dim", "num_slots", "scale", "pad",
          "d_q", "d_k", "d_v", "d_out", "d_state", "q_token", "q_head", "k_token", "k_head", "v_token", "v_head",
          "out_token", "out_head", "state_slot", "state_head", "d_log_decay", "d_row_start", "d_read", "d_write",
          "d_status"]

GOOD_NORM = dict(dtype=0, residual_dtype=0, out_dtype=0, num_tokens=5, dim=100, activation=0, eps=1e-6,
                 residual_scale=1.0, pad=0, d_x=P, d_after=P, d_gate=P, d_residual=P, d_before=P, d_residual_out=P,
                 d_out=P, d_out_scale=0, x_token=100, gate_token=0, residual_token=100, residual_out_token=100,
                 out_token=100)
GOOD_PRODUCT = dict(dtype=3, out_dtype=0, num_tokens=5, dim=64, channels=70, d_x=P, d_w=P, d_out=P, d_x_scale=P,
                    d_w_scale=P, d_bias=0, x_token=64, w_channel=64, out_token=70)
GOOD_LINEAR = dict(dtype=0, num_tokens=5, num_requests=3, heads=4, kv_heads=2, dim=64, num_slots=6, scale=0.1, pad=0,
                   d_q=P, d_k=P, d_v=P, d_out=P, d_state=P, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128,
                   v_head=64, out_token=256, out_head=64, state_slot=8192, state_head=4096, d_log_decay=P,
                   d_row_start=P, d_read=P, d_write=0, d_status=0)
INF, NAN = float("inf"), float("nan")


def _pack(record, fields, good, change):
    d = dict(good, struct_size=record.size)
    d.update(change)
    return bytes(record.pack(*[d[f] for f in fields]))


def norm(**kw):
    return _pack(L.NORM_RECORD, NORM, GOOD_NORM, kw)


def product(**kw):
    return _pack(L.PRODUCT_RECORD, PRODUCT, GOOD_PRODUCT, kw)


def linear(**kw):
    return _pack(L.LINEAR_RECORD, LINEAR, GOOD_LINEAR, kw)


def test_records_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    kinds = (("kvr_norm", NORM, L.NORM_RECORD), ("kvr_product", PRODUCT, L.PRODUCT_RECORD),
             ("kvr_linear", LINEAR, L.LINEAR_RECORD))
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "kvr.h"', "int main(void) {"]
    for name, fields, _ in kinds:
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        lines += [f'  printf("%zu %zu\\n", offsetof({name}, {f}), sizeof((({name}*)0)->{f}));' for f in fields]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([cc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = iter(subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n"))
    for name, fields, record in kinds:
        assert int(next(out)) == record.size, name
        codes, count = [], ""
        for c in record.format.lstrip("<"):
            if c.isdigit():
                count += c
            else:
                codes += [c] * int(count or 1)
                count = ""
        assert len(codes) == len(fields)
        at = 0
        for f, c in zip(fields, codes):
            size = {"I": 4, "i": 4, "f": 4, "q": 8, "Q": 8}[c]
            assert [int(x) for x in next(out).split()] == [at, size], (name, f)
            at += size


def _names(cases):
    return ["-".join(f"{k}={v}" for k, v in c.items()) for c in cases]


def _refused(call, status=K.KVR_EINVAL):
    with pytest.raises(K.KvrError) as ei:
        call()
    assert ei.value.status == status and K.kvr_last_error()


BAD_NORMS = [dict(struct_size=8), dict(dtype=2), dict(dtype=3), dict(dtype=4), dict(out_dtype=1), dict(out_dtype=2),
             dict(out_dtype=4), dict(num_tokens=-1), dict(dim=0), dict(dim=65537), dict(activation=-1),
             dict(activation=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=INF), dict(eps=NAN), dict(residual_scale=INF),
             dict(residual_scale=NAN), dict(d_residual_out=0), dict(d_residual=0), dict(residual_dtype=1),
             dict(residual_dtype=3), dict(out_dtype=3), dict(d_out_scale=P), dict(d_x=0), dict(d_out=0), dict(d_x=P + 1),
             dict(d_after=P + 1), dict(d_gate=P + 1), dict(d_before=P + 1), dict(d_residual=P + 1),
             dict(residual_dtype=4, d_residual=P + 2), dict(d_residual_out=P + 1), dict(d_out=P + 1),
             dict(out_dtype=3, d_out_scale=P + 2)]


@pytest.mark.parametrize("bad", BAD_NORMS, ids=_names(BAD_NORMS))
def test_norms_refused(bad):
    _refused(lambda: K.kvr_block_norm(norm(**bad)))


BAD_PRODUCTS = [dict(struct_size=8), dict(dtype=2), dict(dtype=4), dict(out_dtype=2), dict(out_dtype=3),
                dict(num_tokens=-1), dict(dim=0), dict(dim=8), dict(dim=72), dict(dim=65552), dict(channels=0),
                dict(channels=(1 << 24) + 1), dict(num_tokens=1 << 20, channels=1 << 20), dict(d_x_scale=0),
                dict(dtype=0)]
BAD_PRODUCT_BUFFERS = [dict(d_x=0), dict(d_w=0), dict(d_out=0), dict(d_w_scale=0), dict(d_x=P + 8), dict(d_w=P + 8),
                       dict(x_token=72), dict(w_channel=72), dict(d_out=P + 1), dict(out_dtype=4, d_out=P + 2),
                       dict(d_x_scale=P + 2), dict(d_w_scale=P + 2), dict(d_bias=P + 2),
                       dict(dtype=0, d_x_scale=0, d_x=P + 1)]


@pytest.mark.parametrize("bad", BAD_PRODUCTS, ids=_names(BAD_PRODUCTS))
def test_products_refused(bad):
    _refused(lambda: K.kvr_product_workspace(product(**bad)))
    _refused(lambda: K.kvr_integer_product(product(**bad), P, 1 << 30))


@pytest.mark.parametrize("bad", BAD_PRODUCT_BUFFERS, ids=_names(BAD_PRODUCT_BUFFERS))
def test_product_buffers_refused(bad):
    _refused(lambda: K.kvr_integer_product(product(**bad), P, 1 << 30))


BAD_LINEARS = [dict(struct_size=8), dict(dtype=2), dict(dtype=4), dict(num_tokens=-1), dict(num_requests=0),
               dict(num_requests=(1 << 20) + 1), dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(kv_heads=1025),
               dict(dim=32), dict(dim=96), dict(dim=256), dict(num_tokens=1 << 29), dict(num_slots=0), dict(scale=INF),
               dict(scale=NAN), dict(d_row_start=0), dict(num_requests=1 << 20, kv_heads=16, heads=16)]
BAD_LINEAR_BUFFERS = [dict(d_q=0), dict(d_k=0), dict(d_v=0), dict(d_out=0), dict(d_state=0), dict(d_log_decay=0),
                      dict(d_read=0), dict(d_q=P + 8), dict(d_k=P + 8), dict(d_v=P + 8), dict(d_out=P + 4),
                      dict(d_state=P + 8), dict(q_token=260), dict(q_head=68), dict(k_head=68), dict(v_token=132),
                      dict(out_head=66), dict(state_slot=8194), dict(state_head=4098), dict(d_read=P + 2)]


@pytest.mark.parametrize("bad", BAD_LINEARS, ids=_names(BAD_LINEARS))
def test_linears_refused(bad):
    _refused(lambda: K.kvr_linear_workspace(linear(**bad)))
    _refused(lambda: K.kvr_linear_attention(linear(**bad), P, 1 << 40))


@pytest.mark.parametrize("bad", BAD_LINEAR_BUFFERS, ids=_names(BAD_LINEAR_BUFFERS))
def test_linear_buffers_refused(bad):
    _refused(lambda: K.kvr_linear_attention(linear(**bad), P, 1 << 40))


def test_small_or_missing_workspaces_refused():
    halves = dict(dtype=0, d_x_scale=0, num_tokens=2000)
    assert K.kvr_product_workspace(product()) == 0
    assert K.kvr_product_workspace(product(**halves)) >= 2000 * 64 + 8000
    # few tokens are brought to integers by every workgroup: as long as there is one round of these
    few = dict(halves, num_tokens=64)
    assert K.kvr_product_workspace(product(**few, dim=1024, channels=8192)) == 0
    assert K.kvr_product_workspace(product(**few, dim=1040, channels=8192)) >= 64 * 1040 + 256
    assert K.kvr_product_workspace(product(**few, dim=1024, channels=8193)) >= 64 * 1024 + 256
    assert K.kvr_product_workspace(product(**dict(few, num_tokens=16), dim=4096, channels=1 << 20)) == 0
    _refused(lambda: K.kvr_integer_product(product(**halves), 0, 1 << 20))
    _refused(lambda: K.kvr_integer_product(product(**halves), P + 8, 1 << 20))
    _refused(lambda: K.kvr_integer_product(product(**halves), P, 64), K.KVR_ENOMEM)
    # few requests that are not cut take no workspace
    assert K.kvr_linear_workspace(linear()) == 0 and K.kvr_linear_workspace(linear(num_requests=256)) == 0
    assert K.kvr_linear_workspace(linear(num_requests=257)) > 0
    # (three requests, two heads to a state: cut from 64 tokens each on, as the device would be half empty)
    assert K.kvr_linear_workspace(linear(num_tokens=192)) == 0
    # (short ones are not, while they are few tokens in all)
    assert K.kvr_linear_workspace(linear(num_tokens=512, num_requests=32)) == 0
    assert K.kvr_linear_workspace(linear(num_tokens=512, num_requests=31)) > 0
    cut = dict(num_tokens=193)
    assert K.kvr_linear_workspace(linear(**cut)) >= 2 * 2 * 64 * 64 * 4
    _refused(lambda: K.kvr_linear_attention(linear(**cut), 0, 1 << 40))
    _refused(lambda: K.kvr_linear_attention(linear(**cut), P + 16, 1 << 40))
    _refused(lambda: K.kvr_linear_attention(linear(**cut), P, 16), K.KVR_ENOMEM)


def test_nothing_to_do_is_no_error_and_no_launch():
    K.kvr_block_norm(norm(num_tokens=0))
    K.kvr_integer_product(product(num_tokens=0))


def test_null_structs_refused():
    lib = K.load_library()
    assert lib.kvr_block_norm(None, None) == K.KVR_EINVAL
    assert lib.kvr_integer_product(None, P, 1 << 20, None) == K.KVR_EINVAL
    assert lib.kvr_product_workspace(product(), None) == K.KVR_EINVAL
    assert lib.kvr_linear_attention(None, P, 1 << 20, None) == K.KVR_EINVAL
    assert lib.kvr_linear_workspace(linear(), None) == K.KVR_EINVAL


def test_overlapping_pieces():
    # a lattice of pieces of three elements; those that lie between each other without touching are refused too
    def touch(n, step, m, each):
        seen = [i * step + j * each + e for i in range(n) for j in range(m) for e in range(3)]
        return len(seen) != len(set(seen))

    for n in range(4):
        for m in range(4):
            for step in range(14):
                for each in range(14):
                    said = L._overlap(n, step, m, each, 3)
                    assert said or not touch(n, step, m, each), (n, step, m, each)
                    if n <= 1 or m <= 1 or step >= m * each or each >= n * step:
                        assert said == touch(n, step, m, each), (n, step, m, each)


def test_tensors_on_the_cpu_refused():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    w = torch.zeros((8, 64), dtype=torch.int8)
    _refused(lambda: K.block_norm(x))
    _refused(lambda: K.integer_product(x, w, torch.ones(8)))
    q = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    at = torch.zeros(1, dtype=torch.int32)
    _refused(lambda: K.linear_attention(q, q, q, torch.zeros(1, 2, 64, 64), torch.zeros(2), at))

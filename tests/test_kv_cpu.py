"""Host-side checks of the paged KV cache that need no GPU: null contexts are
refused, the binding's structs have the header's fields, and the documented
layout is a permutation that the measured cases' plain form undoes."""
import re

import numpy as np
import pytest
import torch

import kv_oracle as ko
from perf import operators
from paper_2606_00946_amd import lodestar
from test_abi_cpu import HEADER


def test_null_context_is_refused():
    lib = lodestar.library()
    assert lib.ls_kv_append(None, None, None, None, None, 0, None, 0, None, 0, 1, None, 0, None) == lodestar.LS_ERR_INVALID
    assert lib.ls_kv_attention(None, None, None, None, 0, 1, 1.0, 0, 0, None, 0, None) == lodestar.LS_ERR_INVALID
    assert lib.ls_kv_read(None, None, None, None, None, None) == lodestar.LS_ERR_INVALID


@pytest.mark.parametrize("struct", [lodestar.ls_kv_cache, lodestar.ls_kv_batch, lodestar.ls_rope])
def test_structs_follow_the_header(struct):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + struct.__name__ + ";", text).group(1)
    names = [n.strip(" *\n") for line in body.split(";") for n in re.sub(r"^\s*(const )?\w+\s", "", line).split(",")]
    assert [n for n in names if n] == [f[0] for f in struct._fields_]


@pytest.mark.parametrize("page,D", [(16, 64), (16, 128), (64, 128), (128, 256)])
@pytest.mark.parametrize("values", [False, True])
def test_layout(page, D, values):
    at = ko.offsets(page, D, values)
    assert sorted(at.ravel()) == list(range(page * D))
    x = torch.randint(0, 256, (3, page, D), dtype=torch.uint8)
    laid = operators._laid_out(x, values).reshape(3, -1)
    assert torch.equal(laid[:, torch.from_numpy(at)], x)
    assert torch.equal(operators._natural(laid.reshape(3, page // 16, D // 64, 1024), values), x)


def test_e4m3_values():
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), ko.E4M3)

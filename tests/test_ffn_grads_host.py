"""Gated blocks and norms of gradients without a GPU: mirrors of the C structures, null arguments, the binding's own checks."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2311_14898_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CLIENT = r"""
#include <stddef.h>
#include <stdio.h>
#include "hongtu.h"
int main(void) {
  printf("%d %d %d %d %d %d\n", (int)sizeof(ht_ffn_desc), (int)offsetof(ht_ffn_desc, act), (int)offsetof(ht_ffn_desc, accumulate_dW), HT_FFN_MAX_WIDTH, HT_GATE_SILU,
         HT_GATE_SIGMOID);
  /* without a context nothing is looked at */
  if (ht_ffn_fwd(NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL) != HT_EINVAL) return 1;
  if (ht_ffn_bwd(NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL) != HT_EINVAL) return 2;
  if (ht_grad_norm(NULL, 1, NULL, NULL) != HT_EINVAL) return 3;
  if (ht_grad_clip(NULL, 1, NULL, 1.0, 1.0, 0, NULL, NULL) != HT_EINVAL) return 4;
  return 0;
}
"""


def test_a_c99_program_sees_the_same_structures(tmp_path):
    B.load()
    libdir = os.path.join(ROOT, "paper_2311_14898_amd")
    src, exe = tmp_path / "client.c", tmp_path / "client"
    src.write_text(CLIENT)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe), "-L", libdir, "-lhongtu",
                    f"-Wl,-rpath,{libdir}", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    out = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [C.sizeof(B.ht_ffn_desc), B.ht_ffn_desc.act.offset, B.ht_ffn_desc.accumulate_dW.offset, B.HT_FFN_MAX_WIDTH, B.HT_GATE_SILU, B.HT_GATE_SIGMOID]


def test_tensors_on_the_host_are_refused_by_the_binding():
    m, one = torch.zeros(4, 8), torch.zeros(1)
    with pytest.raises(AssertionError):
        B.ht_ffn_fwd(None, 8, 8, 8, m, m, m, m, m, sync=False)
    with pytest.raises(AssertionError):
        B.ht_ffn_bwd(None, 8, 8, 8, m, m, m, m, m, sync=False)
    with pytest.raises(AssertionError):
        B.ht_grad_norm(None, [m], one, sync=False)
    with pytest.raises(AssertionError):
        B.ht_grad_clip(None, [m], 1.0, sync=False)

"""The calls of models over ids without a GPU: mirrors of the C structures, null arguments, the binding's own checks."""
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
  printf("%d %d %d %d %d %d\n", (int)sizeof(ht_head_desc), (int)offsetof(ht_head_desc, accumulate_dW), (int)sizeof(ht_distill_desc),
         (int)offsetof(ht_distill_desc, temperature), HT_HEAD_MAX_CLASSES, HT_DISTILL_MAX_K);
  /* without a context nothing is looked at */
  if (ht_embed_fwd(NULL, NULL, NULL, 1.0f, NULL) != HT_EINVAL) return 1;
  if (ht_embed_bwd(NULL, NULL, NULL, 1.0f, 0, NULL) != HT_EINVAL) return 2;
  if (ht_head_loss(NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL) != HT_EINVAL) return 3;
  if (ht_distill_loss(NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL) != HT_EINVAL) return 4;
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
    assert out == [C.sizeof(B.ht_head_desc), B.ht_head_desc.accumulate_dW.offset, C.sizeof(B.ht_distill_desc), B.ht_distill_desc.temperature.offset,
                   B.HT_HEAD_MAX_CLASSES, B.HT_DISTILL_MAX_K]


def test_tensors_on_the_host_are_refused_by_the_binding():
    m, ids, one = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(1)
    with pytest.raises(AssertionError):
        B.ht_embed_fwd(None, 8, m, ids, m, sync=False)
    with pytest.raises(AssertionError):
        B.ht_embed_bwd(None, 8, m, ids, m, sync=False)
    with pytest.raises(AssertionError):
        B.ht_head_loss(None, 8, 4, m, m, ids, one, w_form=B.HT_W_OUT_IN, sync=False)
    with pytest.raises(AssertionError):
        B.ht_distill_loss(None, 8, m, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), one, sync=False)

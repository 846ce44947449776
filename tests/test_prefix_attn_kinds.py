"""The calls of prefix_attn_kinds.py go to the kernels they are there for, and no kernel is without one (host only: nothing is launched)."""
import re
import subprocess

import pytest

from paper_2511_11641_amd import binding as B
from paper_2511_11641_amd import build as bld
from prefix_attn_kinds import CASES, chosen


@pytest.fixture(scope="module")
def lib():
    return B.load()


def descriptor(Bn, L, h, h_kv, e, f, P, own_max):
    cap = own_max + 3
    return B.Cache(B.BF16, Bn, h, h_kv, e, f, cap, own_max, P, 0.125, 4096, 8192, h_kv * cap * e, cap * e, e, h_kv * cap * f, cap * f, f,
                   16384, 32768, P * e, e, P * f, f, 65536)


def test_the_calls_go_where_they_say(lib):
    wrong = [(kernel, form, shape, chosen(lib, descriptor(*shape), shape[1])) for kernel, form, shape in CASES
             if chosen(lib, descriptor(*shape), shape[1]) != (kernel, form)]
    assert not wrong, wrong[:5]


def test_every_kernel_has_a_call(lib):
    names = subprocess.run(["nm", "-D", "--defined-only", bld.LIB], check=True, capture_output=True, text=True).stdout
    built = {tuple(map(int, m)) for m in re.findall(r"prefix_attn_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)EEv", names)}
    assert len(built) > 60 and {kernel for kernel, _, _ in CASES} == built

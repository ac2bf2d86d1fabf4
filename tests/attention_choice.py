"""The library's choice among its kernels of attention under a rule (csrc/attention_choice.h), compiled for the host and asked through
ctypes."""
import ctypes
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2102_03161_amd", "csrc")

SOURCE = r"""
#include "attention_choice.h"
using namespace pt;
extern "C" int share(int what, int nb, int Sq, int Sk, int H, int Hkv, int dh, int ordered, int documents) {
  const RuleShape s{nb, Sq, Sk, H, Hkv, dh, ordered != 0, documents != 0};
  switch (what) {
    case 0: return rule_share_fwd(s);
    case 1: return rule_share_dq(s);
    case 2: return rule_share_dkv(s);
    case 3: return rule_share_f32_fwd(s);
    case 4: return rule_share_f32_dq(s);
    default: return rule_share_f32_dkv(s);
  }
}
"""

_lib = None


def shares(nb, Sq, Sk, H, Hkv, dh, ordered=False, documents=False, bf16=True):
    """Waves that share the rows of a wave: (forward, dq, dk and dv)."""
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            so = os.path.join(d, "choice.so")
            subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", CSRC, "-x", "c++", "-", "-o", so],
                           input=SOURCE.encode(), check=True)
            _lib = ctypes.CDLL(so)
    return tuple(_lib.share(what, nb, Sq, Sk, H, Hkv, dh, int(ordered), int(documents)) for what in ((0, 1, 2) if bf16 else (3, 4, 5)))

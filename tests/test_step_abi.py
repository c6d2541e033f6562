"""CPU-side checks of the calls at the end of a fine-tuning step: the header is plain C, the layouts
that the binding packs are the header's, and a null context is refused."""
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import binding
from paper_2305_19982_b200 import build as adama_build

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def lib():
    adama_build.build()
    return adama.load_library()


def test_layouts_are_those_of_the_header(tmp_path):
    """Field by field: values packed by the binding are read back by C code that includes adama.h."""
    src = tmp_path / "layout.c"
    src.write_text(r'''
#include <stdio.h>
#include <string.h>
#include "adama.h"
_Static_assert(sizeof(adama_state8) == 32, "four pointers");
_Static_assert(sizeof(adama_grad_norm) == 16, "two floats and a double");
_Static_assert(ADAMA_STATE8_BLOCK == %d && ADAMA_WORKSPACE_BYTES == %d, "constants of the binding");
int main(void) {
    adama_policy_args a;
    if (fread(&a, 1, sizeof(a) + 1, stdin) != sizeof(a)) return 1;
    printf("%%p %%p %%d %%d %%lld %%lld %%lld %%lld %%p %%p %%p %%p %%p %%g %%g %%g %%g %%p %%p %%p\n", a.logits, a.dlogits,
           a.logits_dtype, a.dlogits_dtype, (long long)a.rows, (long long)a.vocab, (long long)a.ld_logits,
           (long long)a.ld_dlogits, (void *)a.targets, (void *)a.old_logp, (void *)a.ref_logp, (void *)a.advantages,
           (void *)a.weights, a.logit_scale, a.clip_low, a.clip_high, a.kl_coef, (void *)a.logp, (void *)a.stats, a.workspace);
    return 0;
}
''' % (binding.STATE8_BLOCK, binding.WORKSPACE_BYTES))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", str(ROOT / "include"), str(src), "-o", str(exe)], check=True)
    values = [1, 2, 0, 1, 5, 6, 7, 8, 9, 10, 11, 12, 13, 1.25, 0.2, 0.3, 0.05, 14, 15, 16]
    out = subprocess.run([str(exe)], input=binding._POLICY_ARGS.pack(*values), capture_output=True, check=True).stdout.split()
    got = [float(int(x, 16)) if b"0x" in x else float(x) for x in out]
    assert got == [float(v) for v in values]


def test_null_contexts_are_refused(lib):
    bad = adama.Status.ERR_INVALID_ARG
    assert lib.adama_fold_apply_multi(None, None, 0, None, None, None, None, None, 0, 1e-3, None, None) == bad
    assert lib.adama_fold_apply8_multi(None, None, 0, None, None, None, None, 0, 1e-3, None, None) == bad
    assert lib.adama_state8_pack_multi(None, None, None, None, None, 0, None) == bad
    assert lib.adama_state8_unpack_multi(None, None, None, None, None, 0, None) == bad
    assert lib.adama_grad_norm_multi(None, None, 0, None, 0, 1.0, 0, None, None, None) == bad
    assert lib.adama_token_logprobs(None, None, 0, 0, 1, 1, None, 1.0, None, None, None, None) == bad
    assert lib.adama_policy_loss(None, None, None) == bad


def test_states_are_refused_off_the_device():
    with pytest.raises(TypeError):
        adama.State8.zeros(300, device="cpu")
    with pytest.raises(ValueError):   # one scale for 256 elements
        adama.State8(torch.zeros(300, dtype=torch.float8_e4m3fn), torch.zeros(1), torch.zeros(300, dtype=torch.uint8), torch.zeros(1))


"""The kernels on rows of logits load through functions of their own.  Read off the sources, no GPU: which device functions load from global memory, found from the loads themselves and from who calls
them, and that no kernel calls one before its dependency wait, but for the tiles of W (a constant of the stream) by TMA."""
import os
import re

import pytest

from test_dependency_loads import CSRC, KERNELS, _strip

FILES = ("logits.cu", "linear_logprobs.cu")
PRIMITIVE = r"ld\.global|cp\.async\.cg|\bdep_load\w*\s*\(|\bload16\w*\s*\(|\btma_load\w*\s*\(|__ldcs|__ldcg"


def _kernel(file, name, params, body):
    if name == "__cluster_dims__":                         # (the first word before a parenthesis)
        name, params = re.search(r"__cluster_dims__\([^)]*\)\s*__launch_bounds__\([^)]*\)\s*(\w+)\(([^)]*)\)", _strip(open(os.path.join(CSRC, file)).read())).groups()
    return file, name, params, body


HERE = [_kernel(*k) for k in KERNELS if k[0] in FILES]


def _functions(text):
    """name -> bodies of every function that is no kernel (members too)."""
    out = {}
    for m in re.finditer(r"__device__ __forceinline__ (?:explicit )?(?:static )?[\w:<>,&* ]*?(\w+|operator\(\))\s*\(", text):
        i, depth = m.end(), 1
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        j = text.find("{", i)
        if j < 0 or ";" in text[i:j]:
            continue
        if ":" in text[i:j]:                               # (a constructor's list may hold braces)
            j = i + re.search(r"\{(?![^{}]*\}\s*[,{])", text[i:]).start()
        k, depth = j + 1, 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[k], 0)
            k += 1
        out.setdefault(m.group(1), []).append(text[i:k])
    return out


def _loaders(file):
    functions = _functions(_strip(open(os.path.join(CSRC, "logits.cuh")).read()) + _strip(open(os.path.join(CSRC, file)).read()))
    loading = set()
    while True:
        calls = "|".join(sorted(loading)) or r"\b\B"
        more = {n for n, bodies in functions.items() if n not in loading and any(re.search(PRIMITIVE + r"|\b(?:" + calls + r")(?:<[^;()]*>)?\s*\(", b) for b in bodies)}
        if not more:
            return loading
        loading |= more


def test_the_kernels_and_their_loads_are_found():
    assert {k[1] for k in HERE} == {"token_logprobs_kernel", "distill_kernel", "distill_loss_kernel", "token_logprobs_grad_kernel", "distill_grad_kernel", "linear_logprobs_kernel", "linear_finish_kernel"}
    assert {"load16_once", "cp_async16", "load", "fetch", "build", "each", "partial", "warp_select", "far_part"} <= _loaders("logits.cu")
    assert "load_bf16" in _loaders("linear_logprobs.cu")


def _early(body, loaders):
    """Loads in front of the wait of each warp role (a body without roles is one)."""
    calls = PRIMITIVE + r"|\b(?:" + "|".join(sorted(loaders)) + r")(?:<[^;()]*>)?\s*\("
    found = []
    for role in re.split(r"\belse\s+if\s*\(warp == 1\)|\belse\s*\{\s*(?=pdl_wait)", body):
        head = role[:role.index("pdl_wait()")]
        found += [head[m.start():head.index(";", m.start())] for m in re.finditer(calls, head)]
    return found


@pytest.mark.parametrize("file,name,params,body", HERE, ids=[k[1] for k in HERE])
def test_nothing_is_loaded_before_the_wait(file, name, params, body):
    assert body.index("pdl_trigger()") < body.index("pdl_wait()")
    early = _early(body, _loaders(file))
    if name == "linear_logprobs_kernel":
        assert body.count("pdl_wait()") == 3               # producer, product, epilogue
        assert len(early) == 1 and early[0].startswith("tma_load_2d_pair(") and "&tmB" in early[0]
        early = []
    assert not early
    assert "__ldg" not in body and not re.search(r"\bconst\s+\w+\s*\*\s*__restrict__", params)


@pytest.mark.parametrize("file,name,params,body", HERE, ids=[k[1] for k in HERE])
def test_a_planted_load_is_seen(file, name, params, body):
    loaders = _loaders(file)
    plain = len(_early(body, loaders))
    for load in ["dep_load(p.ids)"] + (["sg.load(x)", "Elem<T>::load(xrow)", "sl.fetch()", "cp_async16(0, xrow)", "load16_once(xrow)"] if file == "logits.cu" else ["load_bf16(p.bias)"]):
        assert len(_early(body.replace("pdl_trigger();", "pdl_trigger(); " + load + ";", 1), loaders)) == plain + 1, load

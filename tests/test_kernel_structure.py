"""What the order of a few calls inside the kernels has to be, read off the sources: a kernel that breaks one of these would hang or
race on the GPU, so nothing here runs one."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_04127_b200", "csrc")


def _kernels():
    """(file, name, body) of every __global__ function, comments removed."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        with open(path) as f:
            src = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
        for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\([^)]*\)\s+)?(\w+)\s*\(", src):
            start = src.index("{", m.end())
            depth, i = 0, start
            while True:
                depth += {"{": 1, "}": -1}.get(src[i], 0)
                if depth == 0:
                    break
                i += 1
            out.append((os.path.basename(path), m.group(1), src[start:i + 1]))
    return out


KERNELS = _kernels()
TENSOR_MEMORY = [k for k in KERNELS if "tmem_alloc(" in k[2]]


def test_the_kernels_are_found():
    assert {"split_gemm_kernel", "tc_fwd_causal_kernel", "tc_bwd_nc_kernel", "tc_bwd_k_kernel"} <= {k[1] for k in TENSOR_MEMORY}


@pytest.mark.parametrize("file,name,body", TENSOR_MEMORY, ids=[k[1] for k in TENSOR_MEMORY])
def test_tensor_memory_is_taken_before_dependents_may_start(file, name, body):
    """A dependent kernel holds all of an SM's tensor memory while it waits for this kernel's end; a block of this kernel that had
    yet to take its own would wait for it, for good."""
    trigger = re.search(r"pdl_wait\w*\(\)|griddepcontrol\.launch_dependents", body)
    if trigger:
        assert re.search(r"tmem_alloc\(.*__syncthreads\(\)", body[:trigger.start()], re.S), f"{file}: {name}"


@pytest.mark.parametrize("file,name,body", TENSOR_MEMORY, ids=[k[1] for k in TENSOR_MEMORY])
def test_a_kernel_that_gave_up_waits_for_its_copies(file, name, body):
    """After a wait ran into its limit, loads into the block's shared memory may still be in flight: it sleeps before it ends."""
    assert re.search(r"__nanosleep\(200000\);(?!.*\bmbar_).*tmem_dealloc\(", body, re.S), f"{file}: {name}"


TMA = [k for k in KERNELS if re.search(r"tma_load_\w+\(|bulk_load\(", k[2])]


@pytest.mark.parametrize("file,name,body", TMA, ids=[k[1] for k in TMA])
def test_tma_reads_behind_a_proxy_fence(file, name, body):
    """What a kernel before wrote with ordinary stores is read by TMA only behind the fence that goes with the early start."""
    wait = re.search(r"pdl_wait_tma\(\)", body)
    assert wait and wait.start() < re.search(r"tma_load_\w+\(|bulk_load\(", body).start(), f"{file}: {name}"
    assert not re.search(r"pdl_wait\(\)|griddepcontrol", body), f"{file}: {name}"


@pytest.mark.parametrize("file,name,body", TENSOR_MEMORY, ids=[k[1] for k in TENSOR_MEMORY])
def test_a_wait_has_one_answer_before_tensor_memory_is_read(file, name, body):
    """Tensor-memory loads and stores are instructions of a whole warp: where the lanes of a warp could leave a wait with different
    answers, half of it would enter one. The warp votes in between."""
    for wait in re.finditer(r"(?<!__all_sync\(0xffffffffu, )\b(?:wait_or_abort|mbar_wait)\(", body):
        access = re.search(r"\btmem_(?:ld|st|row_to_tile)\w*\(", body[wait.end():])
        if access:
            between = body[wait.end():wait.end() + access.start()]
            assert "__all_sync(" in between or "warp_wait(" in between, f"{file}: {name}: {body[wait.start():wait.start() + 60]}"


def _functions(src):
    """(name, body) of every function of a source without comments."""
    for m in re.finditer(r"(\w+)\s*\([^;{}()]*(?:\([^;{}()]*\)[^;{}()]*)*\)\s*\{", src):
        depth, i = 0, m.end() - 1
        while True:
            depth += {"{": 1, "}": -1}.get(src[i], 0)
            if depth == 0:
                break
            i += 1
        yield m.group(1), src[m.end() - 1:i + 1]


def _sources():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        with open(path) as f:
            yield os.path.basename(path), re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


def test_every_loop_over_tries_is_limited_and_in_the_self_test():
    """A loop over tries of a barrier ends by the clock or by their number; the self-test lets it run out, by itself or in a wait made of it."""
    bodies = {name: body for _, src in _sources() for name, body in _functions(src)}
    loops = {name for name, body in bodies.items() if re.search(r"\bmbar_try_wait\(", body) and re.search(r"\b(?:for|while)\b", body)}
    loops |= {name for name, body in bodies.items() if "mbarrier.try_wait" in body and re.search(r"\bbra\b|\bfor\b|\bwhile\b", body)}
    assert loops == {"mbar_wait_limited", "warp_wait_tries"}
    assert "kWaitLimitNs" in bodies["mbar_wait_limited"]
    assert re.search(r"mov\.u32 n, \d+;.*sub\.u32 n, n, 1;.*setp\.ne\.u32 q, n, 0;.*@q bra", bodies["warp_wait_tries"], re.S)
    assert "mbar_wait_limited(" in bodies["wait_or_abort"]
    selftest = dict(_sources())["selftest.cu"]
    assert "warp_wait_tries(" in selftest and "wait_or_abort(" in selftest


@pytest.mark.parametrize("file,name,body", TENSOR_MEMORY, ids=[k[1] for k in TENSOR_MEMORY])
def test_the_waits_of_tensor_memory_kernels_are_known(file, name, body):
    """Those that a lane answers by itself are looked at above; the others vote."""
    waits = set(re.findall(r"\b(\w*wait\w*)\(", body)) - {"pdl_wait_tma", "tmem_wait_ld", "tmem_wait_st", "tma_store_wait_read", "tma_store_wait_all"}
    waits -= set(re.findall(r"auto (\w+) = \[&\]", body))         # made of the others
    voting = {"warp_wait", "warp_wait_tries"}
    assert waits and waits <= voting | {"wait_or_abort", "mbar_wait"}, f"{file}: {name}: {waits}"
    common = dict(_functions(dict(_sources())["tc_common.cuh"]))
    assert all("__all_sync(" in common[w] for w in voting)

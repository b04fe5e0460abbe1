"""The operators around the 4-bit key/value cache (include/moe_kv.h) against plain implementations (kv_reference.py).

Integers and stored bytes have to be equal.  Bounds of computed numbers:
  rope        each output is two products and a sum in fp32: at most 3 half-ulps of |u| + |w|, plus the output's rounding
  attention   with A = sum_j w_j |v_j| of an output and X = c max_j sum_d |q_d k_jd| of its row (natural exponents):
              weights are off by e = the rounding of a weight (2^-11 in f16; 2^-21 as two f16 parts) + 2^-21 (ex2.approx
              and the fp32 exponent's own rounding, which is 2^-23 of at most 2^4 near the largest weight and matters
              less below) + X * W * 2^-23 (fp32 sums of exact products, one step per product at worst);
              numerator and denominator both carry e, sums over n keys n * 2^-23 (at worst),
              so |error| <= A (2 e + n 2^-22) + the output's rounding.
"""
import ctypes
import math
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

import kv_reference as ref
from paper_2509_02753_b200 import binding as B
from paper_2509_02753_b200 import build
from paper_2509_02753_b200 import decoder
from paper_2509_02753_b200 import kv_cache as K
from paper_2509_02753_b200 import synth

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
gpu = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
UNIT = {t: torch.finfo(t).eps for t in (BF16, F32)}       # spacing of a type next to 1: 2^-7 and 2^-23


def plan_for(heads=4, kv=2, dim=64, page=16, dtype=F32, requests=16, tokens=4096):
    return K.KVPlan(n_heads=heads, n_kv_heads=kv, head_dim=dim, page_size=page, dtype=dtype, max_requests=requests, max_tokens=tokens)


def dev(a, dtype=None):
    t = torch.as_tensor(np.asarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def i32(a):
    return dev(np.asarray(a, np.int32))


def host(t):
    return t.float().cpu().numpy() if t.dtype == BF16 else t.cpu().numpy()


# ------------------------------------------------------------------------------------------ no device needed

def test_every_declared_entry_point_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "moe_kv.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", text))
    assert names == set(K.EXPORTS)
    lib = K.load_library()
    for n in names:
        assert hasattr(lib, n)
    K.load_native()


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(K.moe_kv_config_t) == 28
    assert ctypes.sizeof(K.moe_kv_rows_t) == 24
    assert ctypes.sizeof(K.moe_rope_config_t) == 56


@pytest.mark.parametrize("bad, status", [
    ((4, 3, 64, 16, 1, 1, 1), -1), ((0, 1, 64, 16, 1, 1, 1), -1), ((4, 0, 64, 16, 1, 1, 1), -1), ((4, 2, 64, 16, 0, 1, 1), -1),
    ((4, 2, 64, 16, 1, 0, 1), -1), ((4, 2, 64, 16, 1, 1, 2), -1), ((4, 2, 60, 16, 1, 1, 1), -2), ((4, 2, 264, 16, 1, 1, 1), -2),
    ((4, 2, 0, 16, 1, 1, 1), -2), ((4, 2, 64, 24, 1, 1, 1), -2), ((4, 2, 64, 256, 1, 1, 1), -2), ((4, 2, 64, 16, 4097, 1, 1), -2),
    ((2048, 2, 64, 16, 1, 1, 1), -2)])
def test_plan_create_refuses_bad_configurations(bad, status):
    lib, out = K.load_library(), ctypes.c_void_p()
    cfg = K.moe_kv_config_t(*bad)
    assert lib.moe_kv_plan_create(ctypes.byref(cfg), ctypes.byref(out)) == status and out.value is None
    assert lib.moe_kv_page_bytes(ctypes.byref(cfg)) == 0


def test_null_arguments():
    lib = K.load_library()
    assert lib.moe_kv_plan_create(None, None) == -1
    assert lib.moe_kv_plan_destroy(None) == 0
    assert lib.moe_kv_plan_workspace_bytes(None) == 0
    assert lib.moe_kv_device_status(None, None, None) == -1
    assert lib.moe_kv_attention(None, None, 0, None, None, 0, 0, None, 0, None, 0, 1.0, 1.0, 1.0, 0, 0, None, None) == -1
    assert lib.moe_kv_read(None, None, 0, None, 0, 1.0, 1.0, None, None, None) == -1


@pytest.mark.parametrize("dim, page, kv", [(64, 16, 1), (80, 32, 3), (128, 64, 8), (136, 128, 2), (256, 16, 5)])
def test_page_bytes(dim, page, kv):
    cfg = K.moe_kv_config_t(kv, kv, dim, page, 1, 1, 1)
    assert K.load_library().moe_kv_page_bytes(ctypes.byref(cfg)) == kv * (page // 16) * ref.block_bytes(dim)


def test_status_word_and_caches_are_the_plans_device(monkeypatch):
    """Two devices, the first current, the plan on the second: the status word is read behind the second's stream."""
    current, seen = [0], []

    class On:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            current.append(self.index)

        def __exit__(self, *exc):
            current.pop()

    class Stream:
        def __init__(self, cuda_stream):
            self.cuda_stream = cuda_stream

    class Lib:
        def moe_kv_device_status(self, handle, bits, stream):
            seen.append((current[-1], stream))
            return 0

        def moe_kv_page_bytes(self, cfg):
            return K.load_library().moe_kv_page_bytes(cfg)

        def moe_kv_plan_destroy(self, handle):
            return 0

    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(1000 + (current[-1] if device is None else device)))
    monkeypatch.setattr(torch, "zeros", lambda size, **more: seen.append(more["device"]))
    plan = K.KVPlan.__new__(K.KVPlan)
    plan.cfg = K.moe_kv_config_t(4, 2, 64, 16, 1, 1, B.MOE_F32)
    plan.n_kv_heads, plan.page_size, plan.handle, plan.device, plan._lib = 2, 16, 1, 1, Lib()
    assert plan.device_status() == (0, 0) and plan.device_status(Stream(7)) == (0, 0)
    plan.new_cache(3)
    assert seen == [(1, 1001), (1, 7), torch.device("cuda", 1)]


def test_every_workload_has_heads_that_a_plan_takes():
    known = {"qwen15": (16, 4), "olmoe": (16, 4), "dsv2lite": (16, 4), "mixtral": (32, 8), "minicpm": (18, 3), "dsvl2tiny": (10, 2), "tiny": (2, 1)}
    for name, wl in synth.WORKLOADS.items():
        attn = decoder.attention_of(wl)
        assert (attn.n_heads, attn.n_kv_heads) == known.get(name, (attn.n_heads, attn.n_kv_heads)), name
        cfg = K.moe_kv_config_t(attn.n_heads, attn.n_kv_heads, attn.head_dim, 64, 1, 1, B.MOE_BF16)
        assert K.load_library().moe_kv_page_bytes(ctypes.byref(cfg)) > 0, name


def test_the_native_module_is_built_for_the_torch_there_is(monkeypatch, tmp_path):
    """Built again for another torch though no source changed; without torch left out, and the library is built all the same."""
    monkeypatch.setattr(build, "NATIVE", str(tmp_path / "native.so"))
    monkeypatch.setattr(build, "OBJ_DIR", str(tmp_path))
    ran = []

    def run(cmd):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    build.build_native(run, [], False)
    build.build_native(run, [], False)
    assert len(ran) == 1
    monkeypatch.setattr(torch, "__version__", "0.0")
    build.build_native(run, [], False)
    assert len(ran) == 2
    monkeypatch.setitem(sys.modules, "torch", None)          # import raises
    build.build_native(run, [], True)
    assert len(ran) == 2


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-device path")
def test_no_device_means_an_error():
    with pytest.raises(B.MoEError) as e:
        plan_for()
    assert e.value.status == -5


RING = r"""
#include <cstdio>
#include <cstdlib>
#include "kv_ring.cuh"

// ring PIECES [steps, number of the wait that runs out or -1]...: prints every wait (stage, parity) and every step that was used
int main(int argc, char **argv) {
    lexi::kv::RingWaits<2> ring;
    int waits = 0, bad = atoi(argv[1]);
    for (int i = 2; i < argc; ++i) {
        const int steps = atoi(argv[i]);
        for (int k = 0; k < steps; ++k) {
            const bool there = ring.arrived(k, steps, [&](int stage, uint32_t parity) {
                printf("w%d%u ", stage, parity);
                return waits++ != bad;
            });
            if (!there) break;
            printf("u%d ", k);
        }
        printf("| ");
    }
    printf("%s", ring.dead ? "dead" : "alive");
}
"""


@pytest.mark.parametrize("bad, pieces, want", [
    (-1, (3, 1, 2), "w00 u0 w10 u1 w01 u2 | w00 u0 | w01 u0 w11 u1 | alive"),          # parities go on from piece to piece
    (2, (5, 2), "w00 u0 w10 u1 w01 w01 w11 | | dead"),          # two were under way: once more each; nothing of the next piece
    (4, (5, 2, 1), "w00 u0 w10 u1 w01 u2 w11 u3 w00 w00 | | | dead"),          # the last step: one
    (0, (1, 1), "w00 w00 | | dead")])
def test_a_ring_whose_wait_ran_out_is_not_used_again(bad, pieces, want, tmp_path):
    """A copy that arrives after its wait ran out would pass for one of the next piece."""
    (tmp_path / "ring.cpp").write_text(RING)
    subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2509_02753_b200", "csrc"), str(tmp_path / "ring.cpp"), "-o", str(tmp_path / "ring")], check=True)
    got = subprocess.run([str(tmp_path / "ring"), str(bad), *map(str, pieces)], check=True, capture_output=True, text=True).stdout
    assert got.split() == want.split()


# ------------------------------------------------------------------------------------------ tables

def check_tables(ctx, new, free, table, page, capacity, bits):
    with plan_for(page=page, requests=max(1, len(ctx)), tokens=max(1, capacity)) as plan:
        t = i32(table)
        got = plan.tables(i32(ctx), i32(new), i32(free), t, capacity)
        want = ref.tables(ctx, new, free, np.asarray(table, np.int64), page, capacity)
        for name, g, w in zip(("table", "kv_len", "cu", "positions", "slots"), (t,) + got[:4], want):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w)), name
        assert int(got[4]) == want[5]
        assert plan.device_status() == ((0, 0) if bits == 0 else (-8, bits))
        assert plan.device_status() == (0, 0)


@gpu
@pytest.mark.parametrize("n", [1, 2, 31, 33, 255, 256, 257, 700])
@pytest.mark.parametrize("page", [16, 128])
def test_tables(n, page):
    rng = np.random.default_rng(n + page)
    ctx = rng.integers(0, 300, n) * rng.integers(0, 2, n)
    new = rng.integers(0, 40, n) * rng.integers(0, 2, n)
    ctx[0], new[n // 2] = page, page + 1
    width = int((ctx + new).max() + page - 1) // page + 1
    pool = rng.permutation(20 * n * width)
    table = np.full((n, width), -7)
    for i in range(n):
        held = -(-ctx[i] // page)
        table[i, :held], pool = pool[:held], pool[held:]
    check_tables(ctx, new, pool[: 60 * n], table, page, int(new.sum()) + n % 3, 0)


@gpu
def test_tables_of_nothing():
    check_tables([], [], [3, 4], np.zeros((0, 4)), 16, 5, 0)
    check_tables([0, 5], [0, 0], [3], np.full((2, 2), -1), 16, 0, 0)
    check_tables([0, 5], [0, 0], [], np.full((2, 2), 1), 16, 3, 0)


@gpu
def test_tables_that_do_not_fit():
    check_tables([0, 16, 30], [20, 17, 3], [5, 9], [[-1, -1], [8, -1], [1, 2]], 16, 40, K.STATUS_NO_PAGES | 0)        # too few free pages
    check_tables([0, 16], [40, 1], [5, 9, 6, 4], [[-1, -1], [8, -1]], 16, 41, K.STATUS_NO_PAGES)                     # the row is too short
    check_tables([0, -3], [4, 2], [5, 9], [[-1], [-1]], 16, 6, K.STATUS_BAD_INDEX)                                  # a negative length
    check_tables([0, 3], [4, 2], [5, 9], [[-1], [7]], 16, 4, K.STATUS_BAD_INDEX)                                    # more tokens than room


@gpu
def test_new_tokens_whose_page_is_no_page():
    """A negative entry that a new token needs, of the table or of the free list, loses the token and says so."""
    check_tables([20, 3], [2, 1], [5, 9], [[4, -1], [7, -1]], 16, 3, K.STATUS_BAD_INDEX)
    check_tables([16, 3], [2, 1], [-1, 9], [[4, -1], [7, -1]], 16, 3, K.STATUS_BAD_INDEX)
    check_tables([20, 3], [0, 1], [5, 9], [[4, -1], [7, -1]], 16, 1, 0)          # nothing new there


@gpu
def test_tables_of_lengths_that_pass_32_bits():
    with plan_for(requests=300, tokens=8) as plan:
        n = 300
        new = np.full(n, 2 ** 31 - 1)
        new[0] = 3
        t = i32(np.full((n, 1), -7))
        kv_len, cu, position, slot, taken = plan.tables(i32(np.full(n, 2 ** 31 - 1) * (np.arange(n) > 0)), i32(new), i32([4]), t, 8)
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX | K.STATUS_NO_PAGES)
        assert position[:3].tolist() == [0, 1, 2] and slot.tolist() == [64, 65, 66] + [-1] * 5
        assert cu[:3].tolist() == [0, 3, 2 ** 31 - 1] and int(cu[-1]) == int(kv_len[-1]) == int(taken) == 2 ** 31 - 1
        assert t.flatten().tolist() == [4] + [-7] * (n - 1)


# ------------------------------------------------------------------------------------------ rope

def plain_angles(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2) / rot)


@gpu
@pytest.mark.parametrize("scaling, more", [("plain", {}), ("linear", {"factor": 4.0}), ("base", {"factor": 8.0}),
                                           ("parts", {"factor": 16.0, "low": 1.0, "high": 32.0, "original_context": 4096.0}),
                                           ("bands", {"factor": 8.0, "low": 1.0, "high": 4.0, "original_context": 8192.0}),
                                           ("parts", {"factor": 2.5, "low": 2.0, "high": 3.0, "original_context": 100.0, "magnitude": 0.7})])
@pytest.mark.parametrize("rot", [2, 20, 128])
def test_rope_table(scaling, more, rot):
    n, base = 70000 if rot == 20 else 3000, 10000.0
    theta = plain_angles(rot, base)
    f, mag = more.get("factor", 1.0), more.get("magnitude", 1.0)
    if scaling == "linear":
        theta = theta / f
    elif scaling == "base" and rot > 2:
        theta = plain_angles(rot, base * f ** (rot / (rot - 2)))
    elif scaling == "parts":
        at = [rot * math.log(more["original_context"] / (2 * math.pi * t)) / (2 * math.log(base)) for t in (more["high"], more["low"])]
        a, b = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        ramp = np.clip((np.arange(rot // 2) - a) / max(b - a, 1e-3), 0, 1)
        theta = theta * (1 - ramp) + theta / f * ramp
        mag = more.get("magnitude", 0.1 * math.log(f) + 1)
    elif scaling == "bands":
        keep = np.clip((more["original_context"] * theta / (2 * math.pi) - more["low"]) / (more["high"] - more["low"]), 0, 1)
        theta = theta * keep + theta / f * (1 - keep)
    got = K.rope_table(rot, n, base=base, scaling=scaling, **more).cpu().numpy()
    angle = np.arange(n)[:, None] * theta[None]
    want = np.stack((np.cos(angle), np.sin(angle)), -1) * mag
    # one rounding to fp32 of numbers up to mag; angles in 64 bits differ by a few units of 2^-53 * n
    assert np.abs(got - want).max() <= mag * (2.0 ** -24 + 8 * n * 2.0 ** -53)


def test_rope_table_refusals():
    lib = K.load_library()
    good = dict(rope_dim=64, scaling=0, base=1e4, factor=1.0, low=1.0, high=32.0, original_context=4096.0, magnitude=0.0)
    for change in ({"rope_dim": 0}, {"rope_dim": 7}, {"rope_dim": 258}, {"scaling": 5}, {"scaling": -1}, {"base": 0.0}, {"factor": 0.5}, {"magnitude": -1.0},
                   {"scaling": 3, "low": 0.0}, {"scaling": 4, "high": 1.0}, {"scaling": 3, "original_context": 0.0}, {"base": float("nan")}):
        cfg = K.moe_rope_config_t(*[{**good, **change}[f] for f, _ in K.moe_rope_config_t._fields_])
        assert lib.moe_rope_table(ctypes.byref(cfg), 4, 16, None) == -1, change
    cfg = K.moe_rope_config_t(*[good[f] for f, _ in K.moe_rope_config_t._fields_])
    assert lib.moe_rope_table(ctypes.byref(cfg), 4, None, None) == -1
    assert lib.moe_rope_table(ctypes.byref(cfg), 4, 12, None) == -3


@gpu
def test_angles_on_another_stream_are_that_streams_memory():
    """What the call allocates belongs to the stream that fills it: a block of the current stream may still be in use there."""
    side = torch.cuda.Stream()
    turns = K.rope_table(64, 5000, stream=side)
    at = turns.data_ptr()
    own = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]
    assert own == [side.cuda_stream]
    side.synchronize()
    assert torch.equal(turns, K.rope_table(64, 5000))


def strided(rng, tokens, heads, dim, dtype, pad):
    """Rows of a wider tensor, `pad` elements in front and behind."""
    wide = torch.from_numpy(rng.standard_normal((tokens, heads * dim + 2 * pad)).astype(np.float32)).to(dtype).cuda()
    return wide[:, pad: pad + heads * dim].unflatten(1, (heads, dim))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("tokens, heads, dim, rot, pad", [(1, 1, 8, 2, 0), (1, 5, 64, 64, 0), (3, 4, 80, 20, 8), (7, 3, 96, 48, 3), (5, 2, 128, 128, 64),
                                                          (17, 8, 128, 32, 1), (2, 2, 256, 256, 0), (4, 1, 256, 18, 0), (300, 6, 72, 72, 0)])
def test_rope(tokens, heads, dim, rot, layout, dtype, pad):
    rng = np.random.default_rng(dim + rot)
    x = strided(rng, tokens, heads, dim, dtype, pad)
    pos = rng.integers(0, 900, tokens).astype(np.int32)
    turns = K.rope_table(rot, 900)
    with plan_for(dim=dim, dtype=dtype) as plan:
        for inverse in (False, True):
            want = ref.rotate(host(x).astype(np.float64), pos, turns.cpu().numpy(), rot, layout, inverse)
            got = plan.rope(x, i32(pos), turns, layout=layout, inverse=inverse)
            size = np.abs(host(x)).max()
            assert np.abs(host(got) - want).max() <= 2 * size * 3 * 2.0 ** -24 + UNIT[dtype] / 2 * 2 * size
            one_by_one = ref.rotate(host(x).astype(np.float32), pos, turns.cpu().numpy(), rot, layout, inverse)
            assert torch.equal(got.cpu(), torch.from_numpy(one_by_one).to(dtype))
            inplace = strided(np.random.default_rng(1), tokens, heads, dim, dtype, pad)
            around = inplace._base.clone()
            inplace.copy_(x)
            assert plan.rope(inplace, i32(pos), turns, layout=layout, inverse=inverse, out=inplace) is inplace
            assert torch.equal(inplace, got)
            if pad:
                assert torch.equal(inplace._base[:, :pad], around[:, :pad]) and torch.equal(inplace._base[:, -pad:], around[:, -pad:])
        assert plan.device_status() == (0, 0)


@gpu
def test_rope_backward_is_the_gradient():
    """y = R x is linear: <g, R(x + h e) - R x> / h = (R^-1 g)_e for a rotation, and <g, R x> = <R^-1 g, x>."""
    rng = np.random.default_rng(3)
    turns, pos = K.rope_table(20, 64), i32(rng.integers(0, 64, 6))
    x, g = (torch.from_numpy(rng.standard_normal((6, 3, 40)).astype(np.float32)).cuda() for _ in range(2))
    for layout in ("half", "pairs"):
        with plan_for(dim=40) as plan:
            dx = plan.rope(g, pos, turns, layout=layout, inverse=True)
            y = plan.rope(x, pos, turns, layout=layout)
            a, b = float((g.double() * y.double()).sum()), float((dx.double() * x.double()).sum())
            # each side: 720 terms of size about 1, each off by at most 6 half-ulps
            assert abs(a - b) <= 720 * 6 * 2.0 ** -24 * 16
            for e in ((0, 0, 0), (2, 1, 9), (2, 1, 10), (3, 2, 19), (5, 0, 39)):
                moved = x.clone()
                moved[e] += 1.0
                diff = float((g.double() * (plan.rope(moved, pos, turns, layout=layout).double() - y.double())).sum())
                assert abs(diff - float(dx[e])) <= 8 * 6 * 2.0 ** -24 * 8


@gpu
def test_rope_outside_the_table():
    x = torch.randn(4, 2, 64, device="cuda")
    turns = K.rope_table(64, 10)
    with plan_for() as plan:
        y = plan.rope(x, i32([3, 10, -1, 9]), turns)
        assert torch.equal(y[1:3], x[1:3]) and not torch.equal(y[0], x[0])
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dim, rot, pad", [(96, 24, 0), (96, 24, 1), (80, 20, 8), (80, 20, 3), (40, 2, 0), (128, 64, 0), (128, 34, 8)])
def test_numbers_that_are_not_finite_keep_to_their_pair(dim, rot, pad, layout, dtype):
    """An infinity or a NaN reaches what it turns with and nothing else; what lies behind rope_dim passes, a -0 too, in every walk."""
    rng = np.random.default_rng(dim + rot)
    x = strided(rng, 6, 4, dim, dtype, pad)
    x[0, :, rot], x[1, :, rot + 1], x[2, :, rot + 2], x[3, :, rot:] = float("inf"), float("-inf"), float("nan"), -0.0
    x[4, :, 0], x[5, :, rot - 1] = float("inf"), float("nan")
    pos = np.array([3, 0, 7, 4, 9, 8], np.int32)
    turns = K.rope_table(rot, 10)
    with plan_for(4, 1, dim, dtype=dtype, page=16) as plan, np.errstate(invalid="ignore"):
        for inverse in (False, True):
            want = torch.from_numpy(ref.rotate(host(x).astype(np.float32), pos, turns.cpu().numpy(), rot, layout, inverse)).to(dtype)
            y = [plan.rope(x, i32(pos), turns, layout=layout, inverse=inverse), plan.rope(x, i32(pos), turns, layout=layout, inverse=inverse, out=x.clone())]
            there = torch.zeros_like(x).copy_(x)
            y.append(plan.rope(there, i32(pos), turns, layout=layout, inverse=inverse, out=there))
            if not inverse:
                k = torch.zeros(6, 1, dim, dtype=dtype, device="cuda")
                y.append(plan.append(x, k, k, dev(np.arange(6)), plan.new_cache(1), positions=i32(pos), turns=turns, layout=layout))
            for got in y:
                got = got.cpu()
                assert torch.equal(torch.isnan(got), torch.isnan(want))
                assert torch.equal(torch.nan_to_num(got, nan=0.0, posinf=9.0, neginf=-9.0), torch.nan_to_num(want, nan=0.0, posinf=9.0, neginf=-9.0))
                assert torch.equal(torch.signbit(got)[~torch.isnan(want)], torch.signbit(want)[~torch.isnan(want)])
        assert plan.device_status() == (0, 0)


# ------------------------------------------------------------------------------------------ append and read

@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim, kv, page, rot, layout, tokens, pad", [(64, 1, 16, 64, "half", 1, 0), (64, 2, 32, 20, "pairs", 37, 0), (80, 3, 16, 80, "half", 5, 8),
                                                                     (128, 2, 64, 128, "half", 100, 0), (128, 1, 128, 32, "pairs", 19, 5), (8, 2, 16, 0, "half", 9, 0),
                                                                     (136, 2, 16, 34, "half", 18, 0), (256, 2, 32, 256, "pairs", 33, 0), (256, 1, 16, 64, "half", 3, 1)])
def test_append_and_read(dim, kv, page, rot, layout, tokens, dtype, pad):
    rng = np.random.default_rng(dim * 7 + tokens)
    heads, ks, vs = 3 * kv, 0.03125, 0.75
    wide = strided(rng, tokens, heads + 2 * kv, dim, dtype, pad)
    wide[:, ::2, dim // 2] *= 40        # a loud dimension
    wide[0, heads] = 0                  # a key of zeros
    if tokens > 2:
        wide[2, -1] *= 2.0 ** -30       # a value whose scale rounds to 0
    q, k, v = wide[:, :heads], wide[:, heads: heads + kv], wide[:, heads + kv:]
    n_pages = tokens // page + 5
    slots = rng.permutation(n_pages * page)[:tokens].astype(np.int64) if tokens < 30 else np.arange(tokens, dtype=np.int64) + 5
    if tokens > 4:
        slots[3] = -1
    pos = rng.integers(0, 500, tokens).astype(np.int32)
    more = {"positions": i32(pos), "turns": K.rope_table(rot, 500), "layout": layout} if rot else {}
    with plan_for(heads, kv, dim, page, dtype) as plan:
        cache = torch.from_numpy(rng.integers(0, 256, (n_pages, kv, page // 16, ref.block_bytes(dim)), dtype=np.uint8)).cuda()
        want = cache.cpu().numpy().copy()
        got_q = plan.append(q, k, v, dev(slots), cache, k_scale=ks, v_scale=vs, **more)
        turned = [host(x).astype(np.float32) for x in (q, k)]
        if rot:
            turned = [ref.rotate(x, pos, more["turns"].cpu().numpy(), rot, layout) for x in turned]
        assert torch.equal(got_q.cpu(), torch.from_numpy(turned[0]).to(dtype))
        ref.store(want, turned[1], host(v).astype(np.float32), slots, page, ks, vs)
        assert np.array_equal(cache.cpu().numpy(), want)
        rk, rv = plan.read(cache, dev(slots), k_scale=ks, v_scale=vs)
        for t in range(tokens):
            a, b = ref.load(want, slots[t], page, dim) if slots[t] >= 0 else (np.zeros((kv, dim)),) * 2
            for g, w, s in ((rk, a, ks), (rv, b, vs)):
                assert torch.equal(g[t].cpu(), (torch.from_numpy(w).float() * s).to(dtype))
        assert plan.append(None, k, v, dev(slots), cache, k_scale=ks, v_scale=vs, **more) is None
        assert np.array_equal(cache.cpu().numpy(), want)
        if not pad and rot:
            dense = q.contiguous()
            assert plan.append(dense, k, v, dev(slots), cache, k_scale=ks, v_scale=vs, q_out=dense, **more) is dense and torch.equal(dense, got_q)
        assert plan.device_status() == (0, 0)


@gpu
def test_stored_numbers_are_near():
    """A stored number is off by at most half a step: 1/6 of the group's largest number at worst between the codes 4 and 6,
    times the scale's own rounding (2^-4 relative)."""
    x = torch.randn(64, 2, 128, device="cuda")
    with plan_for(2, 2, 128) as plan:
        cache = plan.new_cache(4)
        plan.append(None, x, x * 3, torch.arange(64, device="cuda"), cache, k_scale=0.01, v_scale=0.05)
        for got, want in zip(plan.read(cache, torch.arange(64, device="cuda"), k_scale=0.01, v_scale=0.05), (x, x * 3)):
            top = want.unflatten(-1, (8, 16)).abs().amax(-1, keepdim=True)
            assert bool(((got - want).unflatten(-1, (8, 16)).abs() <= top / 6 * (1 + 2 ** -4)).all())


@gpu
def test_numbers_that_are_not_finite():
    k = torch.randn(3, 1, 64, device="cuda")
    v = torch.randn(3, 1, 64, device="cuda")
    with plan_for(1, 1, 64) as plan:
        cache = plan.new_cache(1)
        k[0, 0, 5], v[1, 0, 40], v[2, 0, 0] = float("nan"), float("inf"), float("-inf")
        want = cache.cpu().numpy()
        ref.store(want, k.cpu().numpy(), v.cpu().numpy(), [0, 1, 2], 16, 1.0, 1.0)
        plan.append(None, k, v, torch.arange(3, device="cuda"), cache)
        assert np.array_equal(cache.cpu().numpy(), want)
        rk, rv = plan.read(cache, torch.arange(3, device="cuda"))
        assert float(rk[0, 0, 5]) == 0.0 and float(rv[1, 0, 40]) == 2688.0 and float(rv[2, 0, 0]) == -2688.0
        assert bool(torch.isfinite(rk).all()) and bool(torch.isfinite(rv).all())
        assert plan.device_status() == (-8, K.STATUS_NONFINITE)


@gpu
def test_layers_of_the_smallest_scales():
    """A group's scale times the layer's below 2^-128, whose reciprocal is no fp32 number: zeros stay zeros, and what is stored is as near
    as elsewhere.  Not above that: products of numbers below 2^-126 are rounded to multiples of 2^-149 besides."""
    x = torch.zeros(4, 1, 64, device="cuda")
    x[0, 0, 3], x[0, 0, 20], x[1, 0, 1:16], x[2] = 1e-38, -2e-39, 3e-38, torch.randn(1, 64, device="cuda") * 2e-38
    with plan_for(1, 1, 64) as plan:
        for scale in (1e-37, 2.0 ** -126, 1e-36, 1e-30):
            cache = plan.new_cache(1)
            plan.append(None, x, x, torch.arange(4, device="cuda"), cache, k_scale=scale, v_scale=scale)
            for got in plan.read(cache, torch.arange(4, device="cuda"), k_scale=scale, v_scale=scale):
                assert bool((got[x == 0] == 0).all())
                if scale <= 1e-36:
                    top = x.double().unflatten(-1, (4, 16)).abs().amax(-1, keepdim=True)
                    # half a step of the largest code; the scale's own rounding (relative 2^-4, or 2^-10 of the smallest); 64 steps of 2^-149
                    limit = top / 6 * (1 + 2 ** -4) + 6 * scale * 2.0 ** -10 + 64 * 2.0 ** -149
                    assert bool(((got.double() - x.double()).unflatten(-1, (4, 16)).abs() <= limit).all())
        for scale in (2.0 ** -127, 1e-45):          # not normal numbers
            k = x[:1]
            for call in (lambda: plan.append(None, k, k, torch.arange(1, device="cuda"), cache, k_scale=scale), lambda: plan.read(cache, torch.arange(1, device="cuda"), v_scale=scale)):
                with pytest.raises(B.MoEError) as e:
                    call()
                assert e.value.status == -1


@gpu
def test_slots_outside_the_cache():
    k = torch.randn(4, 2, 64, device="cuda")
    with plan_for() as plan:
        cache = plan.new_cache(2)
        slots = dev(np.array([31, 32, -2, 1 << 40], np.int64))
        plan.append(None, k, k, slots, cache)
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX)
        rk, rv = plan.read(cache, slots)
        assert bool((rk[1:] == 0).all()) and bool((rv[1:] == 0).all()) and bool((rk[0] != 0).any())
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX)


# ------------------------------------------------------------------------------------------ attention

def attend_case(seed, lens, new, heads, kv, dim, page, dtype, window=0, sinks=0, pad=0, max_new=None, loud=1.0, extra_rows=0, absent=(), columns=0):
    """Runs one call on a cache whose unused bytes are NaN scales and whose unused table entries are no pages; `absent`:
    entries (request, column) that name no page although their tokens count; `columns`: the table's, at least."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    held = [-(-x // page) for x in lens]
    n_pages, width = sum(held) + 2, max(max(held + [1]) + 1, columns)
    order = rng.permutation(n_pages)
    table = np.full((n, width), 1 << 30)
    at = 0
    for i in range(n):
        table[i, : held[i]] = order[at: at + held[i]]
        at += held[i]
    cache = np.full((n_pages, kv, page // 16, ref.block_bytes(dim)), 0x7F, np.uint8)
    for i in range(n):
        if lens[i]:
            x = rng.standard_normal((2, lens[i], kv, dim)).astype(np.float32)
            x[0, :, :, dim // 3] *= 6 * loud
            slots = [int(table[i, j // page]) * page + j % page for j in range(lens[i])]
            ref.store(cache, x[0], x[1], slots, page, 0.05, 0.02)
    for k, (i, col) in enumerate(absent):
        table[i, col] = (-1, n_pages, 1 << 30)[k % 3]
    cu = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    q = strided(rng, int(cu[-1]) + extra_rows, heads, dim, dtype, pad)
    scale = 1.0 / math.sqrt(dim)
    with plan_for(heads, kv, dim, page, dtype, requests=n, tokens=max(1, q.shape[0])) as plan:
        args = (q, dev(cu), i32(lens), i32(table), torch.from_numpy(cache).cuda())
        more = dict(max_new=max(new) if max_new is None else max_new, window=window, sinks=sinks, k_scale=0.05, v_scale=0.02)
        out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
        got = plan.attention(*args, out=out, **more)
        again = plan.attention(*args, **more)
        assert plan.device_status() == ((-8, K.STATUS_BAD_INDEX) if absent else (0, 0))
    assert bool((got[cu[-1]:] == 7).all())
    got, again = got[: cu[-1]], again[: cu[-1]]
    assert torch.equal(got, again), "equal calls give equal bits"
    want, spread, exponent, count = ref.attention(host(q)[: cu[-1]], cu, lens, table, cache, page, window, sinks, scale,
                                                  float(np.float32(0.05)), float(np.float32(0.02)))
    e = (2.0 ** -11 if dtype == BF16 else 2.0 ** -21) + 2.0 ** -21 + exponent * ref.width(dim) * 2.0 ** -23
    limit = spread * (2 * e + count * 2.0 ** -22) + np.abs(want) * UNIT[dtype] / 2 + 1e-30
    err = np.abs(host(got) - want)
    assert np.isfinite(host(got)).all()
    assert (err <= limit).all(), f"{(err / limit).max()} of the bound"
    return got


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256, 8, 80, 96, 200])
@pytest.mark.parametrize("lens", [[1], [16, 0, 17], [15, 33, 2, 160]])
def test_single_tokens(lens, dim, dtype):
    attend_case(dim, lens, [1] * len(lens), 4, 2, dim, 16, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads, kv", [(1, 1), (3, 3), (7, 1), (8, 1), (9, 1), (14, 2), (16, 1), (17, 1), (40, 1), (64, 2), (15, 5)])
def test_head_layouts(heads, kv, dtype):
    attend_case(heads, [40, 5], [1, 1], heads, kv, 64, 32, dtype, pad=3)
    attend_case(heads, [21], [1], heads, kv, 128, 16, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_pages_and_several_tokens(page, dtype):
    attend_case(page, [130, 7, 64, 65], [3, 7, 1, 0], 4, 2, 64, page, dtype)
    attend_case(page, [129, 40], [5, 2], 6, 2, 128, page, dtype, max_new=0)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (16, 4), (17, 16), (31, 33), (100, 0), (1000, 5), (2, 300), (48, 15)])
@pytest.mark.parametrize("new", [1, 4])
def test_windows_and_first_tokens(window, sinks, new, dtype):
    attend_case(window, [200, 16, 61], [new, new, 1], 4, 2, 64, 16, dtype, window=window, sinks=sinks)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing(dtype):
    got = attend_case(5, [0, 3, 20], [2, 5, 1], 4, 2, 64, 16, dtype)
    assert bool((got[:4] == 0).all()) and bool((got[4:] != 0).any())       # nothing cached; two tokens more than cached


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_contexts_are_split(dtype):
    attend_case(1, [9000], [1], 2, 1, 64, 64, dtype)
    attend_case(2, [3000, 10, 700, 1500], [1, 1, 1, 1], 8, 2, 128, 16, dtype)
    attend_case(3, [2500, 1200], [2, 1], 4, 1, 256, 32, dtype)


@gpu
def test_many_requests():
    rng = np.random.default_rng(0)
    attend_case(4, [int(x) for x in rng.integers(0, 60, 300)], [1] * 300, 2, 2, 64, 16, BF16)
    attend_case(5, [int(x) for x in rng.integers(1, 60, 130)] + [1800], [1] * 131, 16, 8, 64, 16, BF16)      # one long among short ones


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_prompts(dim, dtype):
    attend_case(6, [70, 40], [70, 33], 4, 2, dim, 16, dtype)
    attend_case(7, [300], [45], 6, 2, dim, 64, dtype, window=50, sinks=4, extra_rows=3)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts_and_tokens_in_one_call(dtype):
    """Requests of many and of few rows, none, and hints of the largest that are unknown or wrong: kernels differ, results do not."""
    lens, new = [400, 30, 0, 100, 7], [300, 1, 0, 40, 2]
    a = attend_case(11, lens, new, 4, 2, 64, 16, dtype)
    for hint in (0, 1, 40, 1000):
        b = attend_case(11, lens, new, 4, 2, 64, 16, dtype, max_new=hint)
        assert (a.float() - b.float()).abs().max() <= 2 * UNIT[dtype] * a.float().abs().max() + 2.0 ** -11
    attend_case(12, [200, 200], [60, 20], 8, 1, 128, 32, dtype, max_new=40)          # as many tokens as two of 40, but not alike
    attend_case(13, [64, 64, 64], [20, 20, 20], 8, 2, 80, 16, dtype, pad=1)         # alike, rows on odd addresses


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompts_on_long_contexts_are_split(dim, dtype):
    attend_case(14, [2600], [40], 4, 1, dim, 64, dtype)
    attend_case(15, [1500, 129], [17, 128], 3, 1, dim, 16, dtype, window=700, sinks=5)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts_longer_than_what_is_cached(dtype):
    got = attend_case(16, [100, 0, 200], [150, 50, 20], 4, 1, 64, 16, dtype)
    assert bool((got[:50] == 0).all()) and bool((got[150:200] == 0).all()) and bool((got[50:150] != 0).any())


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_absent_pages(dim, dtype):
    attend_case(17, [300, 90], [1, 1], 2, 1, dim, 16, dtype, absent=[(0, 3), (1, 0), (0, 18)])
    attend_case(18, [300, 90], [200, 80], 2, 1, dim, 16, dtype, absent=[(0, 3), (1, 2), (0, 9), (0, 10)])
    attend_case(19, [300, 260], [100, 100], 2, 1, dim, 128, dtype, absent=[(0, 1), (1, 0)])


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompt_rows_that_are_not_finite_stay_alone(dtype):
    with plan_for(2, 1, 64, 16, dtype, requests=1) as plan:
        cache = plan.new_cache(10)
        x = torch.randn(150, 1, 64, device="cuda").to(dtype)
        plan.append(None, x, x, torch.arange(150, device="cuda"), cache)
        q = torch.randn(150, 2, 64, device="cuda").to(dtype)
        args = (i32([0, 150]), i32([150]), i32([list(range(10))]), cache)
        fine = plan.attention(q, *args)
        q[70, 1, 3], q[20, 0, 60], q[90, 0, 0] = float("nan"), float("inf"), float("-inf")
        got = plan.attention(q, *args)
        odd = torch.zeros(150, 2, dtype=torch.bool, device="cuda")
        odd[70, 1] = odd[20, 0] = odd[90, 0] = True
        assert bool(torch.isnan(got[odd]).all()) and torch.equal(got[~odd], fine[~odd])


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_softmax_scales_of_any_sign(dtype, scale):
    """Scale 0 is the mean of the values; a negative one is the positive one of the negative queries."""
    with plan_for(2, 1, 64, 16, dtype, requests=1) as plan:
        cache = plan.new_cache(10)
        x = torch.randn(150, 1, 64, device="cuda").to(dtype)
        plan.append(None, x, x, torch.arange(150, device="cuda"), cache)
        for n in (1, 100):
            q = torch.randn(n, 2, 64, device="cuda").to(dtype)
            args = (i32([0, n]), i32([150]), i32([list(range(10))]), cache)
            got = plan.attention(q, *args, softmax_scale=scale)
            if scale:
                assert torch.equal(got, plan.attention(-q, *args, softmax_scale=-scale))
            else:
                v = plan.read(cache, torch.arange(150, device="cuda"))[1].double()[:, 0]
                want = (v.cumsum(0) / torch.arange(1, 151, device="cuda").view(-1, 1))[150 - n:].unsqueeze(1)
                assert ((got.double() - want).abs() <= v.abs().mean() * 2.0 ** -10 + want.abs() * UNIT[dtype] / 2).all()


# A table with room for a long context takes prompts to tiles of 128 rows, however short they are.
LONG = 5000


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 136, 256])
def test_prompts_in_tiles(dim, dtype):
    attend_case(31, [70, 40], [70, 33], 4, 2, dim, 16, dtype, columns=LONG)
    attend_case(32, [300], [45], 6, 2, dim, 64, dtype, window=50, sinks=4, extra_rows=3, columns=LONG)
    attend_case(33, [129, 0, 257], [65, 60, 130], 2, 1, dim, 16, dtype, pad=1, columns=LONG)
    attend_case(34, [100, 200], [150, 80], 3, 1, dim, 128, dtype, window=1, columns=LONG)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompts_in_tiles_on_long_contexts(dim, dtype):
    attend_case(35, [2600], [40], 4, 1, dim, 64, dtype, columns=LONG)
    attend_case(36, [1500, 129], [37, 128], 3, 1, dim, 16, dtype, window=700, sinks=5, columns=LONG)
    attend_case(37, [640, 33, 900], [300, 1, 70], 2, 2, dim, 32, dtype, sinks=200, window=300, columns=LONG)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts_in_tiles_of_many_requests(dtype):
    """More requests than the threads that line them up at once, some with nothing."""
    rng = np.random.default_rng(41)
    lens = [int(x) for x in rng.integers(9, 13, 530) * (rng.random(530) < 0.9)]
    attend_case(41, lens, lens, 4, 1, 64, 16, dtype, columns=LONG)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_absent_pages_under_tiles(dim, dtype):
    attend_case(38, [300, 90], [200, 80], 2, 1, dim, 16, dtype, absent=[(0, 3), (1, 2), (0, 9), (0, 10)], columns=LONG)
    attend_case(39, [600, 260], [100, 100], 2, 1, dim, 128, dtype, absent=[(0, 1), (1, 0)], columns=LONG)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page, columns", [(16, 0), (16, LONG), (64, LONG), (128, LONG)])
def test_pages_behind_the_window_may_be_gone(page, columns, dim, dtype):
    """A serving loop gives back the pages that no row sees any more: neither the outputs nor the status word tell."""
    rng = np.random.default_rng(page + dim)
    lens, new = [700, 1000, 300], [40, 70, 1]
    width = max(-(-max(lens) // page) + 1, columns)
    for window, sinks in ((100, 0), (57, 4), (1, 0), (300, 129)):
        pages = rng.permutation(sum(-(-n // page) for n in lens))
        table, gone, at = np.full((3, width), -1), np.full((3, width), -1), 0
        for i, n in enumerate(lens):
            held = -(-n // page)
            table[i, :held] = pages[at: at + held]
            at += held
            first = max(n - new[i] - window + 1, 0)          # what the first new row sees
            for col in range(held):
                if (col + 1) * page > first or col * page < sinks:
                    gone[i, col] = table[i, col]
        assert (gone != table).any()
        with plan_for(4, 2, dim, page, dtype, requests=3) as plan:
            cache = plan.new_cache(len(pages))
            for i, n in enumerate(lens):
                x = torch.from_numpy(rng.standard_normal((2, n, 2, dim)).astype(np.float32)).to(dtype).cuda()
                plan.append(None, x[0], x[1], dev(np.array([table[i, j // page] * page + j % page for j in range(n)], np.int64)), cache, k_scale=0.05, v_scale=0.05)
            q = torch.from_numpy(rng.standard_normal((sum(new), 4, dim)).astype(np.float32)).to(dtype).cuda()
            args = (q, i32(np.cumsum([0] + new)), i32(lens))
            more = dict(max_new=max(new), window=window, sinks=sinks, k_scale=0.05, v_scale=0.05)
            want = plan.attention(*args, i32(table), cache, **more)
            assert plan.device_status() == (0, 0)
            got = plan.attention(*args, i32(gone), cache, **more)
            assert plan.device_status() == (0, 0)
            assert torch.equal(got, want) and bool(torch.isfinite(got).all())


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_requests_of_many_and_few_rows_in_tiles(dtype):
    lens, new = [400, 30, 0, 100, 7], [300, 1, 0, 40, 2]
    for hint in (300, 0, 1):
        attend_case(40, lens, new, 4, 2, 128, 16, dtype, max_new=hint, columns=LONG)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_in_tiles_that_are_not_finite_and_scales_of_any_sign(dim, dtype):
    with plan_for(2, 1, dim, 16, dtype, requests=1) as plan:
        cache = plan.new_cache(10)
        x = torch.randn(150, 1, dim, device="cuda").to(dtype)
        plan.append(None, x, x, torch.arange(150, device="cuda"), cache)
        q = torch.randn(150, 2, dim, device="cuda").to(dtype)
        args = (i32([0, 150]), i32([150]), i32([list(range(10)) + [0] * LONG]), cache)
        assert torch.equal(plan.attention(q, *args, softmax_scale=-0.3), plan.attention(-q, *args, softmax_scale=0.3))
        v = plan.read(cache, torch.arange(150, device="cuda"))[1].double()[:, 0]
        want = (v.cumsum(0) / torch.arange(1, 151, device="cuda").view(-1, 1)).unsqueeze(1)
        got = plan.attention(q, *args, softmax_scale=0.0).double()
        assert ((got - want).abs() <= v.abs().mean() * 2.0 ** -10 + want.abs() * UNIT[dtype] / 2).all()
        fine = plan.attention(q, *args)
        q[70, 1, 3], q[20, 0, dim - 4], q[90, 0, 0] = float("nan"), float("inf"), float("-inf")
        got = plan.attention(q, *args)
        odd = torch.zeros(150, 2, dtype=torch.bool, device="cuda")
        odd[70, 1] = odd[20, 0] = odd[90, 0] = True
        assert bool(torch.isnan(got[odd]).all()) and torch.equal(got[~odd], fine[~odd])


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_peaked_and_flat_weights(dtype):
    attend_case(8, [400], [1], 2, 1, 64, 16, dtype, loud=30.0)      # one key takes nearly all: scores in the hundreds
    attend_case(9, [400], [1], 2, 1, 64, 16, dtype, loud=0.0)


@gpu
def test_queries_of_zero_and_not_finite():
    with plan_for(2, 1, 64, 16, F32) as plan:
        cache = plan.new_cache(2)
        x = torch.randn(20, 1, 64, device="cuda")
        plan.append(None, x, x, torch.arange(20, device="cuda"), cache)
        q = torch.zeros(1, 2, 64, device="cuda")
        args = (i32([0, 1]), i32([20]), i32([[0, 1]]), cache)
        out = plan.attention(q, *args, max_new=1)
        v = plan.read(cache, torch.arange(20, device="cuda"))[1]
        assert bool(((out[0] - v[:, 0].mean(0)).abs() <= 2.0 ** -18 * v.abs().mean()).all())
        q[0, 1, 3] = float("nan")
        out = plan.attention(q, *args, max_new=1)
        assert bool(torch.isfinite(out[0, 0]).all()) and bool(torch.isnan(out[0, 1]).all())      # its own row only


@gpu
def test_pages_outside_the_cache_count_as_absent():
    with plan_for(2, 1, 64, 16, F32) as plan:
        cache = plan.new_cache(3)
        x = torch.randn(48, 1, 64, device="cuda")
        plan.append(None, x, x, torch.arange(48, device="cuda"), cache)
        q = torch.randn(1, 2, 64, device="cuda")
        full = plan.attention(q, i32([0, 1]), i32([16]), i32([[0]]), cache, max_new=1)
        got = plan.attention(q, i32([0, 1]), i32([48]), i32([[0, 3, -1]]), cache, max_new=1)
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX)
        assert torch.equal(got, full)
        plan.attention(q, i32([0, 1]), i32([49]), i32([[0, 1, 2]]), cache, max_new=1)            # longer than the table's row
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX)
        out = torch.full_like(q, 3.0)
        plan.attention(q, i32([0, 2]), i32([16]), i32([[0]]), cache, max_new=1, out=out)         # tokens behind the call's
        assert plan.device_status() == (-8, K.STATUS_BAD_INDEX) and bool((out == 3.0).all())


@gpu
def test_offsets_past_32_bits():
    """The last pages of a cache of 5 GiB."""
    with plan_for(2, 1, 128, 128, BF16) as plan:
        n = 5 * 2 ** 30 // plan.page_bytes
        cache = torch.empty((n, 1, 8, ref.block_bytes(128)), dtype=torch.uint8, device="cuda")
        x = torch.randn(200, 1, 128, device="cuda").to(BF16)
        pages = [n - 1, n - 2]
        slots = torch.tensor([pages[j // 128] * 128 + j % 128 for j in range(200)], device="cuda")
        plan.append(None, x, x, slots, cache)
        small = plan.new_cache(2)
        plan.append(None, x, x, torch.arange(200, device="cuda"), small)
        assert torch.equal(plan.read(cache, slots)[0], plan.read(small, torch.arange(200, device="cuda"))[0])
        q = torch.randn(1, 2, 128, device="cuda").to(BF16)
        a = plan.attention(q, i32([0, 1]), i32([200]), i32([pages]), cache, max_new=1)
        assert torch.equal(a, plan.attention(q, i32([0, 1]), i32([200]), i32([[0, 1]]), small, max_new=1))
        assert plan.device_status() == (0, 0)


@gpu
def test_another_stream():
    x = torch.randn(40, 2, 64, device="cuda")
    with plan_for() as plan:
        cache, q = plan.new_cache(3), torch.randn(1, 4, 64, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        args = (q, i32([0, 1]), i32([40]), i32([[0, 1, 2]]), cache)
        torch.cuda.synchronize()
        plan.append(None, x, x, torch.arange(40, device="cuda"), cache, stream=side)
        out = plan.attention(*args, max_new=1, stream=side)
        assert plan.device_status(side) == (0, 0)
        with torch.cuda.stream(side):
            assert torch.equal(plan.attention(*args, max_new=1), out)
        torch.cuda.synchronize()
        assert torch.equal(plan.attention(*args, max_new=1), out)


@gpu
def test_calls_in_a_graph():
    """A captured step sees the lengths that are on the device when it is replayed."""
    with plan_for(4, 2, 64, 16, F32, requests=2) as plan:
        cache, table = plan.new_cache(40), torch.full((2, 20), -1, dtype=torch.int32, device="cuda")
        free, ctx, new = i32(range(40)), i32([0, 0]), i32([0, 0])
        q, k, v = torch.randn(6, 4, 64, device="cuda"), torch.randn(6, 2, 64, device="cuda"), torch.randn(6, 2, 64, device="cuda")
        turns, out = K.rope_table(64, 100), torch.zeros(6, 4, 64, device="cuda")

        def step():
            kv_len, cu, pos, slots, _ = plan.tables(ctx, new, free, table, 6)
            turned = plan.append(q, k, v, slots, cache, positions=pos, turns=turns)
            return plan.attention(turned, cu, kv_len, table, cache, out=out)

        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for lens in ([4, 2], [1, 5], [0, 6]):
            new.copy_(i32(lens))
            table.fill_(-1)
            graph.replay()
            got = out.clone()
            table.fill_(-1)
            assert torch.equal(step(), got)
        assert plan.device_status() == (0, 0)


@gpu
def test_calls_of_nothing():
    with plan_for() as plan:
        cache = plan.new_cache(1)
        before = plan.launch_count
        none = torch.zeros(0, 2, 64, device="cuda")
        q = torch.zeros(0, 4, 64, device="cuda")
        slots = torch.zeros(0, dtype=torch.int64, device="cuda")
        assert plan.append(q, none, none, slots, cache).shape == (0, 4, 64)
        assert plan.read(cache, slots)[0].shape == (0, 2, 64)
        assert plan.rope(q, i32([]), K.rope_table(64, 4)).shape == (0, 4, 64)
        assert plan.attention(q, i32([0, 0]), i32([5]), i32([[0]]), cache).shape == (0, 4, 64)
        assert plan.launch_count == before


# ------------------------------------------------------------------------------------------ refusals

@gpu
def test_refusals():
    f = torch.zeros
    with plan_for(4, 2, 64, 16, F32, requests=2, tokens=8) as plan:
        cache, turns = plan.new_cache(2), K.rope_table(64, 8)
        q, k, slots, pos = f(2, 4, 64, device="cuda"), f(2, 2, 64, device="cuda"), f(2, dtype=torch.int64, device="cuda"), i32([0, 1])
        many = f(9, 4, 64, device="cuda")
        cu, lens, table = i32([0, 1, 2]), i32([1, 1]), i32([[0], [1]])
        for call in (lambda: plan.rope(many, i32(range(9)), K.rope_table(64, 9)),                      # more tokens than the plan's
                     lambda: plan.append(None, k, k, slots, cache, k_scale=0.0),
                     lambda: plan.append(None, k, k, slots, cache, v_scale=float("inf")),
                     lambda: plan.append(None, k, k, slots, cache, k_scale=-1.0),
                     lambda: plan.read(cache, slots, k_scale=float("nan")),
                     lambda: plan.attention(q, cu, lens, table, cache, softmax_scale=float("nan")),
                     lambda: plan.attention(q, cu, lens, table, cache, window=-1),
                     lambda: plan.attention(q, cu, lens, table, cache, sinks=-1),
                     lambda: plan.attention(q, i32([0, 1, 1, 2]), i32([1, 1, 1]), i32([[0], [1], [0]]), cache),      # more requests than the plan's
                     lambda: plan.tables(i32([0, 0, 0]), i32([1, 1, 1]), i32([0]), i32([[0], [0], [0]]), 3),
                     lambda: plan.tables(i32([0]), i32([1]), i32([0]), i32([[0]]), 9)):
            with pytest.raises(B.MoEError) as e:
                call()
            assert e.value.status == -1
        with pytest.raises(B.MoEError) as e:
            plan.rope(q, pos, K.rope_table(128, 8))          # more dimensions than the head's
        assert e.value.status == -2
        for call in (lambda: plan.rope(q.half(), pos, turns), lambda: plan.rope(q.bfloat16(), pos, turns), lambda: plan.rope(q[..., :32], pos, turns),
                     lambda: plan.rope(q, pos.long(), turns), lambda: plan.rope(q, pos[:1], turns), lambda: plan.rope(q, pos, turns.double()),
                     lambda: plan.rope(q.transpose(0, 2), pos, turns), lambda: plan.append(q, k, k, slots.int(), cache),
                     lambda: plan.append(q[:1], k, k, slots, cache), lambda: plan.append(k, k, k, slots, cache), lambda: plan.append(q, q, k, slots, cache),
                     lambda: plan.append(q, k, k, slots, cache[:, :1]), lambda: plan.append(q, k, k, slots, cache[..., :64].contiguous()),
                     lambda: plan.append(q.cpu(), k, k, slots, cache), lambda: plan.attention(q, cu[:2], lens, table, cache),
                     lambda: plan.attention(q, cu, lens, table[:1], cache), lambda: plan.attention(q, cu.long(), lens, table, cache),
                     lambda: plan.attention(q, cu, lens, table, cache, out=q[:1]), lambda: plan.tables(lens, lens, lens, table[:1], 2),
                     lambda: plan.attention(None, cu, lens, table, cache)):
            with pytest.raises(AssertionError):
                call()
        with pytest.raises(KeyError):
            plan.rope(q, pos, turns, layout="thirds")
        assert plan.device_status() == (0, 0)
    with pytest.raises(AssertionError):
        plan.rope(q, pos, turns)             # closed


@gpu
def test_alignment_refusals():
    lib = K.load_library()
    with plan_for(4, 2, 64, 16, BF16) as plan:
        mem = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        p = mem.data_ptr()
        rows = lambda at: ctypes.byref(K.moe_kv_rows_t(at, 256, 64))  # noqa: E731
        att = lambda q, out, cache: lib.moe_kv_attention(plan.handle, rows(q), 1, p, p, 1, 1, p, 1, cache, 1, 1.0, 1.0, 1.0, 0, 0, out, None)  # noqa: E731
        assert att(p + 1, p, p) == -3 and att(p, p + 2, p) == -3 and att(p, p, p + 8) == -3
        assert att(p, None, p) == -1 and att(None, p, p) == -1
        app = lambda k, cache, q_out: lib.moe_kv_append(plan.handle, rows(p), rows(k), rows(p), 1, None, None, 0, 0, 0, p, 1.0, 1.0, q_out, cache, 1, None)  # noqa: E731
        assert app(p + 1, p, p) == -3 and app(p, p + 8, p) == -3 and app(p, p, p + 1) == -3 and app(p, None, p) == -1 and app(p, p, None) == -1
        assert lib.moe_kv_read(plan.handle, p, 1, p, 1, 1.0, 1.0, p + 8, None, None) == -3
        assert lib.moe_rope(plan.handle, rows(p), 1, 4, p, p + 4, 4, 64, 0, 0, p, 256, 64, None) == -3
        assert lib.moe_rope(plan.handle, rows(p), 1, 4, p, p, 4, 63, 0, 0, p, 256, 64, None) == -2
        assert lib.moe_rope(plan.handle, rows(p), 1, 4, p, p, 4, 64, 2, 0, p, 256, 64, None) == -1
        assert lib.moe_rope(plan.handle, rows(p), 1, 4, p, p, 4, 64, 0, 2, p, 256, 64, None) == -1
        assert plan.device_status() == (0, 0)


@gpu
def test_integer_arrays_off_their_alignment_are_refused():
    lib = K.load_library()
    with plan_for(4, 2, 64, 16, BF16) as plan:
        mem = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        p, before = mem.data_ptr(), plan.launch_count
        rows = ctypes.byref(K.moe_kv_rows_t(p, 256, 64))
        calls = {
            "tables": (lib.moe_kv_tables, [plan.handle, p, p, 1, p, 1, p, 1, 1, p, p, p, p, p, None], {1: 2, 2: 2, 4: 2, 6: 2, 9: 2, 10: 2, 11: 2, 12: 4, 13: 2}),
            "rope": (lib.moe_rope, [plan.handle, rows, 1, 4, p, p, 4, 64, 0, 0, p, 256, 64, None], {4: 2}),
            "append": (lib.moe_kv_append, [plan.handle, rows, rows, rows, 1, p, p, 4, 64, 0, p, 1.0, 1.0, p, p, 1, None], {5: 2, 10: 4}),
            "read": (lib.moe_kv_read, [plan.handle, p, 1, p, 1, 1.0, 1.0, p, p, None], {3: 4}),
            "attention": (lib.moe_kv_attention, [plan.handle, rows, 1, p, p, 1, 1, p, 1, p, 1, 1.0, 1.0, 1.0, 0, 0, p, None], {3: 2, 4: 2, 7: 2})}
        for name, (f, args, off) in calls.items():
            for at, by in off.items():
                assert f(*[a + by if i == at else a for i, a in enumerate(args)]) == -3, (name, at)
        assert plan.launch_count == before and plan.device_status() == (0, 0)

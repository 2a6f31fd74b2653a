"""The example service: its tasks run on the four attention calls together, and its records go through the profile and the gap fill."""
import math

import numpy as np
import pytest
import torch

import oracle
import serve_model as model
from paper_2311_10359_amd import binding, service, traces

pytestmark = pytest.mark.gpu
SIZES = service.Sizes(layers=2, q_heads=8, kv_heads=2, dim=64, block=16, blocks=400, vocabulary=512)


def test_steps_see_what_prompts_and_steps_have_put_into_the_cache():
    """One layer, a few requests: the attention of the third step against 64 bits on the cache's values, and these against the keys
    that went in (an E4M3 code is within 2^-4 of a value that is not below the smallest normal code, 2^-6 of the block's scale)."""
    sizes = SIZES._replace(layers=1)
    s = service.Service(sizes, 3, 80, seed=3)
    lengths = [5, 40, 17]
    seen = []

    def record(name, _, f, *args, **more):
        got = f(*args, **more)
        if name == "append":
            seen.append((args[4].double().cpu(), args[5].double().cpu()))
        if name == "cache attention":
            seen.append((args[0].double().cpu(), got.out.double().cpu()))
        return got
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    x = torch.randn((62, sizes.hidden), generator=gen, device="cuda:0").to(torch.bfloat16)
    s.prompts(record, x, lengths)
    for _ in range(3):
        s.step(record, torch.randn((3, sizes.hidden), generator=gen, device="cuda:0").to(torch.bfloat16))
    assert s.lengths.tolist() == [n + 3 for n in lengths]
    keys, values = seen[0]
    q, out = seen[-1]
    table = s.table.cpu()
    codes = [c.view(torch.uint8).cpu() for c in s.caches[0]]
    at = 0
    for r, n in enumerate(lengths):
        k, v = (torch.cat([t[0][at:at + n] if i == 0 else t[1][at:at + n]] + [(seen[j][0] if i == 0 else seen[j][1])[r:r + 1] for j in (1, 3, 5)])
                for i, t in enumerate((seen[0], seen[0])))
        held = [model.cache_values(codes[i], codes[2 + i], table[r], n + 3, sizes.block) for i in (0, 1)]
        for given, kept in zip((k, v), held):
            block_most = given.abs().max()
            assert bool(((given - kept).abs() <= given.abs() / 16 + block_most * 2.0 ** -9).all())
        want = model.Rows(q[r:r + 1], *held, 1 / math.sqrt(sizes.dim), [n + 3], torch.bfloat16)
        assert model.near(out[r:r + 1], want.out, want.bound)
        at += n


def test_records_go_through_the_profile_and_the_gap_fill():
    (decode, names), (prompts, _), got, s = service.measure(SIZES, requests=5, longest_prompt=60, steps=4, host_ms=0.2)
    assert torch.isfinite(got["step"]).all() and torch.isfinite(got["prompts"]).all() and int(s.status) == 0
    assert decode.size == 4 * (2 + 2 * 4) and prompts.size == 1 + 2 * 4 and set(names) == {"plan", "append", "cache attention", "back",
                                                                                          "to queries, keys, values", "to tokens"}
    assert (decode["end_ns"] >= decode["start_ns"]).all() and (np.diff(decode["start_ns"]) >= 0).all()
    decode["run"] = 0
    rec = np.concatenate([decode, prompts])
    off = np.array([0, decode.size, rec.size], dtype=np.uint64)
    ids, rows, tro = oracle.profile(rec, off)
    hp, lp = np.array([0], dtype=np.uint32), np.array([1], dtype=np.uint32)
    go = traces.gap_offsets(off, hp)
    want = oracle.gapfill(ids, off, rows, tro, hp, lp, 500, 0, go)
    dev = "cuda:0"
    profile, fill = binding.fikit_profile_gapfill(binding.to_device_records(rec, dev), binding.to_device_u64(off, dev), binding.to_device_u32(hp, dev),
                                                  binding.to_device_u32(lp, dev), binding.to_device_u64(go, dev), margin_ns=500, min_gap_ns=0)
    assert binding.rows_to_numpy(profile.rows).tobytes() == rows.tobytes()
    assert np.array_equal(binding.u32_to_numpy(fill.fill_count), want[0]) and np.array_equal(fill.filled_ns.cpu().numpy(), want[1])

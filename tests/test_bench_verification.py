"""What `bench.py --verify` times: paths that move tokens, reserves that hand pages out."""
import numpy as np
import pytest
import torch

import bench
import workloads as W


def test_the_path_goes_from_the_root_to_the_last_node():
    # 0 and 1 below the root, 2 and 3 below 1, 4 below 2; a tree of its root alone; a chain
    assert bench.deepest_paths([[-1, -1, 1, 1, 2], [-1] * 5, [-1, 0, 1, 7, 7]], [5, 0, 3]) == [[0, 2, 3, 5], [0], [0, 1, 2, 3]]


@pytest.mark.gpu
def test_the_calls_that_are_timed_do_their_work():
    from _harness import make_gpu
    cfg = dict(idx=93, B=3, V=1009, dtype="bf16", D=3, F=6, K=4, h=6, beta=0.0, N=15, zipf_s=1.2, sigma=(0.5, 1.5), spike_frac=0.0, desc="verification")
    ctx = make_gpu(cfg, W.classifier(cfg, 2))
    ctx.reset()
    for l in range(cfg["D"]):
        ctx.expand_layer(torch.nn.functional.pad(W.logits_layer(cfg, l, device="cuda"), (0, -cfg["V"] % 8)))
    got = bench.time_verification(torch, np, cfg, ctx.finalize_tree(), torch.device("cuda:0"), 100, 2)
    assert set(got["us"]) == {"truncate_and_reserve", "write", "attention", "adjust", "truncate_and_commit"}
    assert got["moved_tokens"] > 0 and got["new_pages"] > 0

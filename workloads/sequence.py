"""A net of gated sequence blocks and attention blocks with random weights, and an
example that serves it: a batch of prompts, then tokens one by one.

    python -m workloads.sequence [--dim 2048 --heads 64 --blocks 4 --prompt 1024 --tokens 32 --seqs 2
                                  --attention 0 --store same]

``--attention n`` makes every n-th block an attention block, ``--store i8`` keeps
their caches in 8 bits.
"""

import argparse
import time

import numpy as np


def sequence_config(dim=256, heads=8, head_dim=64, groups=1, state=64, conv=4, group=64):
    return {"dim": dim, "heads": heads, "head_dim": head_dim, "groups": groups, "state": state, "conv": conv, "group": group}


def attention_config(dim=256, heads=4, kv_heads=2, head_dim=64, rot=None, base=10000.0, window=0, page=64, store="same", group=64):
    return {"kind": "attention", "dim": dim, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot": head_dim if rot is None else rot, "base": base, "window": window, "page": page, "store": store, "group": group}


def sequence_weights(config, blocks=2, seed=0, zero=True):
    """Random weights (``np.random.default_rng(seed)``) in the form that
    ``SequenceNet`` takes: He-like projections quantised to 4 bits, step sizes of
    0.001 to 0.1 at the bias, decay rates of 1 to 16.  ``config``: of all ``blocks``
    blocks, or a list with one for each."""
    from paper_2110_06037_amd import quantize4
    r = np.random.default_rng(seed)
    configs = list(config) if isinstance(config, (list, tuple)) else [config] * blocks
    blocks = len(configs)
    f32 = lambda v: np.asarray(v, np.float32)

    def projection(c, rows, cols):
        return quantize4(r.standard_normal((rows, cols)) / np.sqrt(cols), c["group"], zero)

    def attention(c):
        heads, kv, n = c["heads"], c["kv_heads"], c["head_dim"]
        return {"config": c,
                "in_proj": projection(c, (heads + 2 * kv) * n, c["dim"]),
                "out_proj": projection(c, c["dim"], heads * n),
                "q_norm": f32(r.uniform(0.5, 1.5, n)),
                "k_norm": f32(r.uniform(0.5, 1.5, n)),
                "scale": 1 / np.sqrt(2 * blocks),
                "norm": f32(r.uniform(0.5, 1.5, c["dim"]))}

    def block(c):
        if c.get("kind") == "attention":
            return attention(c)
        inner = c["heads"] * c["head_dim"]
        chans = inner + 2 * c["groups"] * c["state"]
        step = np.exp(r.uniform(np.log(1e-3), np.log(1e-1), c["heads"]))
        return {"config": c,
                "in_proj": projection(c, inner + chans + c["heads"], c["dim"]),
                "out_proj": projection(c, c["dim"], inner),
                "conv_w": f32(r.uniform(-1, 1, (chans, c["conv"])) / np.sqrt(c["conv"])),
                "conv_b": f32(r.uniform(-0.1, 0.1, chans)),
                "a": f32(-r.uniform(1, 16, c["heads"])),
                "d": f32(r.uniform(0.5, 1.5, c["heads"])),
                "dt_bias": f32(step + np.log(-np.expm1(-step))),
                "gate_norm": f32(r.uniform(0.5, 1.5, inner)),
                "scale": 1 / np.sqrt(2 * blocks),
                "norm": f32(r.uniform(0.5, 1.5, c["dim"]))}

    return {"norm": f32(r.uniform(0.5, 1.5, configs[0]["dim"])), "blocks": [block(c) for c in configs]}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("dim", 2048), ("heads", 64), ("blocks", 4), ("prompt", 1024), ("tokens", 32), ("seqs", 2),
                        ("attention", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--store", choices=("same", "i8"), default="same")
    a = ap.parse_args()
    import torch
    from paper_2110_06037_amd import SequenceNet
    c = sequence_config(a.dim, a.heads, 2 * a.dim // a.heads, 1, 128, 4, 128)
    attend = attention_config(a.dim, a.dim // 64, max(1, a.dim // 256), 128, store=a.store, group=128)
    configs = [attend if a.attention and i % a.attention == a.attention - 1 else c for i in range(a.blocks)]
    net = SequenceNet("bf16", sequence_weights(configs), max_seqs=a.seqs, max_tokens=a.seqs * a.prompt)
    positions = a.prompt + a.tokens + 1
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(a.seqs * a.prompt, a.dim, generator=g, device="cuda").bfloat16()
    net.run(x, net.new_state(a.seqs, positions))  # the first run also loads the kernels

    def timed(f, n):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(n):
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - t) / n

    state = net.new_state(a.seqs, positions)
    prompt = timed(lambda: net.run(x, state), 1)
    token, out, replay = net.capture_step(state)

    def one():
        # stands in for what a sampler would feed back
        token.copy_(torch.nn.functional.normalize(out.float(), dim=1).mul(a.dim ** 0.5))
        replay()

    one()
    step = timed(one, a.tokens)
    print(f"{a.blocks} blocks of {a.dim}, {a.seqs} sequences: prompt of {a.prompt} tokens {prompt * 1e3:.2f} ms "
          f"({a.seqs * a.prompt / prompt:.0f} tokens/s), {a.tokens} tokens at {step * 1e6:.0f} us a step; "
          f"outputs finite: {bool(torch.isfinite(out).all())}")
    net.close()


if __name__ == "__main__":
    main()

"""Sizes at which the operators' kernels go round their loops; test_operators_choose.py says by the library's own rules that they do, test_gpu_operators_long.py
checks the values."""

# block norms: every kind of team with several rows each in both passes, the last slab cut short
BLOCK = [dict(P=P, rows=rows, d=d, post=post, pre=pre, gate=gate, act=act, dtype=dtype, res=res) for P, rows, d, post, pre, gate, act, dtype, res in (
    (2, 70001, 40, "rms", "layer", "rows", "sigmoid", "bf16", "fp32"),
    (2, 70001, 40, "layer", "rms", "vector", "none", "fp32", "bf16"),
    (2, 60011, 5, "layer", "layer", "vector", "tanh", "bf16", "bf16"),        # rows that are read one by one
    (1, 60001, 100, "layer", "layer", "rows", "silu", "bf16", "bf16"),
    (3, 12001, 200, "rms", "rms", "vector", "sigmoid", "fp32", "fp32"),
    (3, 4099, 512, "rms", "layer", "vector", "none", "bf16", "bf16"),
    (3, 4099, 400, "layer", "none", "rows", "none", "bf16", "fp32"),
    (1, 5003, 1500, "none", "layer", "rows", "tanh", "bf16", "bf16"),
    (1, 8203, 519, "layer", "rms", "vector", "none", "bf16", "fp32"),         # the last wavefront reads its few elements one by one
    (1, 1031, 5001, "rms", "layer", "vector", "none", "bf16", "bf16"),
    (2, 601, 7000, "layer", "layer", "none", "none", "bf16", "bf16"),
    (2, 601, 7000, "rms", "rms", "none", "none", "bf16", "bf16"),             # the widest rows' kernel for gains alone
)]


def block_params(c):
    """Names of a case's parameters: no biases where both norms are divisions by the root mean square."""
    biases = "layer" in (c["post"], c["pre"])
    return [k + part for k in ("post", "pre") if c[k] != "none" for part in (["_gain", "_bias"] if biases else ["_gain"])] + (["gate"] if c["gate"] == "vector" else [])


# rotary: rows, heads of the groups, width, rot, in place or apart
ROTARY = [dict(rows=rows, heads=heads, width=width, rot=rot, apart=apart) for rows, heads, width, rot, apart in (
    (20011, (5,), 84, 42, True), (20011, (5,), 84, 42, False), (20011, (16,), 64, 64, True), (20011, (1,), 128, 128, True), (20011, (3,), 20, 18, False),
    (20011, (12, 2), 64, 48, False), (20011, (7, 1, 2, 1), 24, 16, True), (1500, (600,), 64, 64, True), (1500, (600, 9), 64, 40, False))]

# clipping: P, sizes, types (one for all, or by turns)
CLIP = [
    (70, [40003], "bf16"), (70, [30001, 77, 9000, 1, 26000], "fp32"), (64, [64 * 1000 + 8, 513], "mixed"),          # eight units a thread
    (5, [2001, 8, 0, 77, 513, 1, 9000], "mixed"),                                                                    # four
    (3, [100003, 77, 135201, 1, 499999, 513], "mixed"), (3, [101] * 40 + [30007], "mixed"),                          # ranges: tensor by tensor, unit by unit
    (4, [300 + 17 * k for k in range(150)], "mixed"),                                                                # three tables
    (3, [160001 + 317 * k for k in range(70)], "bf16"), (3, [130003 + 101 * k for k in range(66)], "mixed"),         # past the caches, two tables
    (1024, [601 + k % 7 for k in range(70)], "bf16"),
]


def clip_dtypes(sizes, kind):
    return [kind if kind != "mixed" else ("fp32", "bf16", "bf16")[k % 3] for k in range(len(sizes))]

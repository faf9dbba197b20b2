"""Shapes of the calls on 8-bit blocks that large tiles take, by the kind of tile and by whether its sums are split."""
F32, BF16 = 0, 2

# (call, type of the result, m, n, k): (kind, whether it is split)
KINDS = {
    ("product", BF16, 1316, 4457, 66): ("tiles_8bit", False),
    ("product", BF16, 72, 4359, 4739): ("tiles_8bit", True),
    ("product", F32, 1316, 4457, 66): ("tiles_128", False),
    ("product", F32, 132, 5637, 4311): ("tiles_128", True),
    ("product", F32, 4208, 5227, 260): ("tiles_256", False),
    ("product", F32, 4273, 265, 4714): ("tiles_256", True),
    ("gated", BF16, 1316, 4457, 66): ("tiles_8bit", False),
    ("gated", BF16, 132, 5637, 4311): ("tiles_8bit", True),
    ("gated", F32, 1316, 4457, 66): ("tiles_256", False),
    ("gated", F32, 132, 5637, 4311): ("tiles_256", True),
    ("gated_to_blocks", BF16, 1316, 4457, 66): ("tiles_8bit", False),
    ("gated_to_blocks", BF16, 132, 5637, 4311): ("tiles_8bit", True),
    ("gated_kept", BF16, 1316, 4457, 66): ("tiles_256", False),
    ("gated_kept", BF16, 132, 5637, 4311): ("tiles_256", True),
    ("input_grad", F32, 5626, 66, 522): ("tiles_128", False),
    ("input_grad", F32, 65, 4352, 4100): ("tiles_128", True),
    ("input_grad", F32, 4273, 265, 4714): ("tiles_256", False),
    ("input_grad", F32, 4208, 5227, 260): ("tiles_256", True),
    ("weight_grad", F32, 333, 3001, 2100): ("tiles_128", False),
    ("weight_grad", F32, 4273, 265, 4714): ("tiles_128", True),
    ("weight_grad", F32, 65, 4352, 4100): ("tiles_256", False),
    ("weight_grad", F32, 5502, 4242, 258): ("tiles_256", True),
    ("gated_input_grad", BF16, 5626, 66, 522): ("tiles_128", False),
    ("gated_input_grad", BF16, 65, 4352, 4100): ("tiles_128", True),
    ("gated_input_grad", F32, 65, 4352, 4100): ("tiles_128", True),
    ("gated_input_grad", BF16, 4273, 265, 4714): ("tiles_256", False),
    ("gated_input_grad", F32, 4273, 265, 4714): ("tiles_256", False),
    ("gated_input_grad", BF16, 132, 5637, 4311): ("tiles_256", True),
    ("gated_input_grad", F32, 132, 5637, 4311): ("tiles_256", True),
    ("gated_weight_grads", BF16, 1000, 2100, 1200): ("tiles_128", False),
    ("gated_weight_grads", F32, 1000, 2100, 1200): ("tiles_128", False),
    ("gated_weight_grads", BF16, 4273, 265, 4714): ("tiles_128", True),
    ("gated_weight_grads", F32, 4273, 265, 4714): ("tiles_128", True),
    ("gated_weight_grads", BF16, 65, 4352, 4100): ("tiles_256", False),
    ("gated_weight_grads", F32, 65, 4352, 4100): ("tiles_256", False),
    ("gated_weight_grads", BF16, 4208, 5227, 260): ("tiles_256", True),
    ("gated_weight_grads", F32, 4208, 5227, 260): ("tiles_256", True),
}


def shapes_of(*calls):
    """The shapes at which one of these calls is in the list."""
    return sorted({key[2:] for key in KINDS if key[0] in calls})

"""Sizes of the gate's products whose loops run in their steady state, by the tiles they take."""

# rows, hidden, experts, and (tiles, parts) of logits, dx and dwg
GATE = [
    # a training step's batch: logits by an undivided ring of 64 stages, 64 strips and 128 stages in each part of the gradients
    (32771, 4096, 128, dict(logits=("ring", 1), dx=("strips", 8), dwg=("ring", 4))),
    (32771, 1024, 100, dict(logits=("ring", 1), dx=("strips", 32), dwg=("ring", 16))),
    # the depth of the logits in parts
    (8195, 8192, 60, dict(logits=("ring", 2), dx=("strips", 4), dwg=("ring", 2))),
    (4099, 4096, 200, dict(logits=("ring", 2), dx=("strips", 8), dwg=("ring", 2))),
    # strips of every width, beside both kinds of rings
    (20011, 1024, 60, dict(logits=("few4", 1), dx=("strips", 32), dwg=("ring", 16))),
    (20011, 1024, 190, dict(logits=("small", 1), dx=("strips", 32), dwg=("ring", 8))),
    (20011, 2048, 190, dict(logits=("small", 1), dx=("strips", 16), dwg=("broad", 8))),
    (20011, 1024, 256, dict(logits=("small", 1), dx=("strips", 32), dwg=("ring", 8))),
    (20011, 2048, 256, dict(logits=("small", 1), dx=("strips", 16), dwg=("broad", 8))),
    # and before wide tiles
    (32771, 4096, 256, dict(logits=("small", 1), dx=("strips", 16), dwg=("wide", 16))),
    # more experts than strips take
    (8195, 4096, 300, dict(logits=("ring", 1), dx=("small", 1), dwg=("ring", 2))),
    (20011, 4096, 300, dict(logits=("small", 1), dx=("wide", 1), dwg=("wide", 8))),
]

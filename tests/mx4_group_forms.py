"""Sizes of more experts than a wave has lanes that lead to every form of tiles, for the test that runs them and the one that looks at the plan."""
# (mx4 X, experts, rows, outputs, contraction): form
MX4_GROUP_FORMS = {
    (False, 130, 5000, 40, 256): "ring64",
    (False, 130, 5000, 96, 128): "ring32",
    (False, 130, 5000, 300, 256): "ring64w",
    (False, 130, 9000, 150, 128): "big",
    (False, 130, 16000, 96, 256): "mid",
    (True, 200, 5000, 96, 256): "ring32",
    (True, 130, 5000, 40, 256): "ring64",
    (True, 130, 5000, 300, 256): "ring64w",
    (True, 130, 16000, 96, 256): "mid",
    (True, 130, 30000, 150, 256): "big",
}

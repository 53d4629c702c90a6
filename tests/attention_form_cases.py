"""Batches that reach uniprefill_attention's work-groups of 256 rows, with the keys whole and cut into pieces, for every
type and head dimension.  The CPU test checks that each batch does get its form, the GPU tests run the same batches against
the oracle."""

# lengths, earlier tokens, query heads, kv heads, whether the keys are cut
FORMS = [([520], [129], 256, 16, False), ([500, 40], [0, 6000], 256, 16, True)]
TYPES = [(64, False), (128, False), (256, False), (64, True), (128, True)]      # head dimension, float operands

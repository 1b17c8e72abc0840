"""Blocks (T, d) of rows of more than 8192 values, on sixteen waves with two to four chunks of 512 values each: more rows than the gradient's workgroups, and more
than the forward pass's (test_training_sizes_cpu.py)."""
WIDE = [(3, 10240), (300, 16384), (260, 16392), (300, 20000), (2, 24576), (270, 32768)]
WIDE_MANY = [(4100, 16384), (4099, 20000), (4100, 24584)]

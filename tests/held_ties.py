"""Groups whose (max - min) / (2^b - 1) lies half-way between two fp16 numbers, to a step of binary32."""

# by bits: (largest value, smallest value, bits of the scale that a held pool gives the group).  That scale is
# fp16((max - min) * c) with c the binary32 number next to 1 / (2^b - 1), which lies above it at 4 and at 8 bits: the upper neighbour.
# A swap record's is fp16 of the quotient, which goes to the even neighbour, here the lower one
TIES = {
    4: [(8.5703125, -0.002685546875, 0x3893), (8.59375, 0.006103515625, 0x3895), (8.609375, 0.007080078125, 0x3897)],
    8: [(8.96875, 1.52587890625e-05, 0x2881), (8.984375, 7.62939453125e-05, 0x2883), (9.0, 0.0001373291015625, 0x2885)],
}
